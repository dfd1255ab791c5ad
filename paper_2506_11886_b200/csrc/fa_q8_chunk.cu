// fa_q8_attention with many query columns to a KV head (a chunk of a prompt): scores and outputs on the 5th-generation
// tensor cores (tcgen05.mma, halves in, fp32 accumulators in tensor memory).
//
// A CTA takes 256 rows, a row being one (query, query head) of a KV head, as two tiles of 128, over blocks of 128 tokens.  Per block and tile:
// S = Q K^T (accumulators), the weights P of the softmax rounded to halves in the place of S, O += P V with P read from
// tensor memory.  The two tiles take turns: the tensor cores work for one while the other's weights are formed.
//   warps 0-3, 4-7   a tile each, a thread a row: the row's maximum, exponentials, sums; O is rescaled in tensor memory only when
//                    a maximum has grown by more than 8 (powers of two: exactly)
//   warps 8-11       8-bit values to halves (exactly) in shared memory, K and V in turn, the other one's bytes under way; two stages for each
//   warp 12          issues the MMAs (13-15 idle)
// Scales, the tail and the weights are as in fa_q8_attn.cu with 2^7 in the place of 2^15, which leaves the maxima room to grow.  The blocks of all
// tiles stand in a line that is cut into equal parts, one for each SM; the parts of a tile that is cut meet in the workspace, and a second kernel
// joins them, spread over all SMs.
// The loops of the roles share the instruction cache: what is unrolled (a row of scores in registers) is written once, the rest kept small.
// Bound by the exponentials (16 a clock and SM: 2048 clocks for a block and 256 rows of any head dim) and, at 128 dims, by as many clocks of the tensor cores.
#include "fa_q8.cuh"
#include "fa_umma.cuh"

namespace fa {
namespace {

using namespace umma;

constexpr int kRows = 256, kTok = 128;
constexpr int kConv = 8, kMma = 12;                        // first converting warp, the issuing warp
constexpr int kChunkThreads = 16 * 32;                     // (four warps have the same registers: three of the last four idle)
// Registers of a thread of the four groups of warps; together those that the launch has (4 x 128): the weights keep a row of 128 scores.
constexpr int kRegsRow = 176, kRegsConv = 104, kRegsMma = 56;
static_assert(2 * kRegsRow + kRegsConv + kRegsMma == 4 * 128, "");
constexpr int kScSlots = 4;                                // scales of blocks: a slot is free when the weights of the block two in front are done

struct ChunkArgs {
    Q8Dims s;
    Q8Cache c;
    const __nv_bfloat16* q;
    int64_t sb, si, sg;
    __nv_bfloat16* out;
    int n_q, n_ct;                                         // column tiles of a KV head
    int ctas;
    float* part;                                           // [2 * CTAs][256][D + 4]
};

__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }       // -126 <= e <= 127
__device__ __forceinline__ float pow2_down(float a, float b) {
    const float e = fmaxf(a - b, -127.f);
    return e <= -127.f ? 0.f : pow2i((int)e);
}
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t half2_of(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ int exponent_of(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }

// Tokens of row b that the cache holds; those that column tile ct sees, in blocks of 128.
__device__ __forceinline__ int row_len(const ChunkArgs& a, int b) {
    const int len = a.c.state[b * kQ8State];
    return len < 0 || len > (a.s.nb << a.s.lb) ? 0 : len;
}
__device__ __forceinline__ int blocks_of(const ChunkArgs& a, int len, int ct) {
    const int last = min(a.n_q - 1, (ct * kRows + kRows - 1) / a.s.G);
    const int seen = len - a.n_q + 1 + last;
    return seen > 0 ? (seen + kTok - 1) / kTok : 0;
}

// The line of blocks: row b, column tile ct, KV head h, block, the last fastest.  A CTA's part of it as segments of one tile.
struct Seg {
    int b, ct, h, len, i0, i1, n;                          // blocks i0 .. i1 of the tile's n
    unsigned u;                                            // the tile's first block in the line
};
struct Line {
    unsigned total, per, u0, u1;
    unsigned base;                                         // in front of tile k of all heads
    int k;                                                 // b * n_ct + ct
    __device__ __forceinline__ unsigned blocks_at(const ChunkArgs& a, int k) const {
        return k < a.s.B * a.n_ct ? (unsigned)blocks_of(a, row_len(a, k / a.n_ct), k % a.n_ct) * (unsigned)a.s.H : 0u;
    }
    // Whole warps.
    __device__ __forceinline__ void measure(const ChunkArgs& a, int lane) {
        total = 0;
        for (int k0 = 0; k0 < a.s.B * a.n_ct; k0 += 32) total += __reduce_add_sync(0xffffffffu, blocks_at(a, k0 + lane));
        per = max((total + a.ctas - 1) / (unsigned)a.ctas, 2u);
    }
    __device__ __forceinline__ void seek(const ChunkArgs& a, int lane, unsigned from) {
        unsigned before = 0;
        k = a.s.B * a.n_ct;
        for (int k0 = 0; k0 < a.s.B * a.n_ct; k0 += 32) {
            const unsigned n = blocks_at(a, k0 + lane);
            unsigned v = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const unsigned w = __shfl_up_sync(0xffffffffu, v, d);
                if (lane >= d) v += w;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, before + v > from);
            if (hit) {
                const int src = __ffs(hit) - 1;
                k = k0 + src;
                base = before + __shfl_sync(0xffffffffu, v - n, src);
                return;
            }
            before += __shfl_sync(0xffffffffu, v, 31);
        }
    }
    __device__ __forceinline__ void begin(const ChunkArgs& a, int lane, int cta) {
        measure(a, lane);
        u0 = min(per * (unsigned)cta, total);
        u1 = min(u0 + per, total);
        if (u0 < u1) seek(a, lane, u0);
    }
    __device__ __forceinline__ bool next(const ChunkArgs& a, Seg& g) {
        if (u0 >= u1) return false;
        while (u0 >= base + blocks_at(a, k)) base += blocks_at(a, k++);
        g.b = k / a.n_ct;
        g.ct = k % a.n_ct;
        g.len = row_len(a, g.b);
        g.n = blocks_of(a, g.len, g.ct);
        g.h = (int)((u0 - base) / (unsigned)g.n);
        g.u = base + (unsigned)g.h * (unsigned)g.n;
        g.i0 = (int)(u0 - g.u);
        g.i1 = (int)min(u1 - g.u, (unsigned)g.n);
        u0 = g.u + g.i1;
        return true;
    }
};

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
                 "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\ntcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
// 32 columns without waiting for them.
__device__ __forceinline__ void tmem_ld32_start(uint32_t taddr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Loads of read-only memory where `there` says so, zeros elsewhere, without a branch.
__device__ __forceinline__ uint4 ld_if16(const uint8_t* p, bool there) {
    uint4 r;
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %5, 0;\n mov.u32 %0, 0;\n mov.u32 %1, 0;\n mov.u32 %2, 0;\n mov.u32 %3, 0;\n @p ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];\n}\n"
        : "=&r"(r.x), "=&r"(r.y), "=&r"(r.z), "=&r"(r.w)
        : "l"(p), "r"((uint32_t)there));
    return r;
}
__device__ __forceinline__ float ld_if(const float* p, bool there) {
    float r;
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n mov.f32 %0, 0f00000000;\n @p ld.global.nc.f32 %0, [%1];\n}\n" : "=&f"(r) : "l"(p), "r"((uint32_t)there));
    return r;
}
// Two floats as one operand of the packed instructions.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D += A B with A (halves, two to a column) in tensor memory.
__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(tmem_d), "r"(tmem_a),
                 "l"(bdesc), "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Row r, 16-byte chunk c (8 dims) of a K-major or MN-major operand of D dims: 64 dims to a 128-byte row, chunks permuted by the row.
__device__ __forceinline__ int operand_offset(int r, int c) { return (c >> 3) * (kTok * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4); }

struct Bars {
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], q_full[2], s_full[2], p_full[2], o_done[2];
};

template <int FMT, int D>
__global__ void __launch_bounds__(kChunkThreads, 1) q8_chunk_kernel(const ChunkArgs a) {
    constexpr int kTile = kTok * D * 2;                    // bytes of an operand tile
    constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)(kTok >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    constexpr uint32_t kIdescO = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char *qs = smem, *ks = smem + 2 * kTile, *vs = smem + 4 * kTile;
    __shared__ Bars bar;
    __shared__ float2 sc[kScSlots][8];                     // K and V scale of 16 tokens each; a V scale below zero: they have no page
    __shared__ int sc_gone[kScSlots];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int fail;
    const Q8Dims& s = a.s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    asm volatile("griddepcontrol.launch_dependents;");
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar.k_full + i, 4); mbar_init(bar.k_empty + i, 1); mbar_init(bar.v_full + i, 4); mbar_init(bar.v_empty + i, 1);
            mbar_init(bar.q_full + i, 4); mbar_init(bar.s_full + i, 1); mbar_init(bar.p_full + i, 4); mbar_init(bar.o_done + i, 1);
        }
        fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMma) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t tmem = tmem_slot;
    const uint32_t tmem_s[2] = {tmem, tmem + 128}, tmem_o[2] = {tmem + 256, tmem + 256 + D};
    int32_t* status = a.c.status;

    Line line;
    line.begin(a, lane, (int)blockIdx.x);
    Seg g;
    auto two_tiles = [&](const Seg& g) { return g.ct * kRows + 128 < a.n_q * s.G; };
    uint32_t blk = 0;                                      // blocks so far: stages and phases
    bool ok = true;

    if (warp < kConv) {
        // ---- a tile's weights ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsRow));
        const int tile = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tmem_s[tile] + lanes, to = tmem_o[tile] + lanes;
        uint32_t n_s = 0, n_o = 0;                         // phases of s_full, o_done
        while (ok && line.next(a, g)) {
            if (tile == 1 && !two_tiles(g)) { blk += g.i1 - g.i0; continue; }
            const int col = g.ct * kRows + tile * 128 + row, qi = col / s.G;
            const bool there = qi < a.n_q;
            // q: scaled by a power of two to halves, into shared memory
            const int64_t qoff = (int64_t)g.b * a.sb + (int64_t)qi * a.si + (int64_t)(g.h * s.G + col % s.G) * a.sg;
            Vec16<__nv_bfloat16> v[D / 16];
            uint32_t mx = 0;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                if (there) v[c].load(a.q + qoff + 16 * c);
                else v[c].zero();
                mx = max(mx, v[c].amax_bits());
            }
            const int eq = max((int)(mx >> 23) - 127, -100);
            const float fq = pow2i(13 - eq), f = pow2i(eq - 13) * (s.scale * kLog2e);
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                uint4 w;
                const int e = 8 * (c & 1);
                w.x = half2_of(v[c >> 1].at(e) * fq, v[c >> 1].at(e + 1) * fq);
                w.y = half2_of(v[c >> 1].at(e + 2) * fq, v[c >> 1].at(e + 3) * fq);
                w.z = half2_of(v[c >> 1].at(e + 4) * fq, v[c >> 1].at(e + 5) * fq);
                w.w = half2_of(v[c >> 1].at(e + 6) * fq, v[c >> 1].at(e + 7) * fq);
                *reinterpret_cast<uint4*>(qs + tile * kTile + operand_offset(row, c)) = w;
            }
            fence_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.q_full + tile);

            const int last = there ? g.len - a.n_q + qi : -1;            // the last token that the row sees
            // the first token that some row of the warp does not see
            const int sure = __reduce_min_sync(0xffffffffu, there ? last : 0x7fffffff);
            float m = kNegBig, mp = kNegBig;
            f32x2 l = pack2(0.f, 0.f);                     // of the even and the odd tokens
            for (int i = g.i0; i < g.i1; ++i, ++blk, ++n_s) {
                ok = mbar_wait(bar.s_full + tile, n_s & 1, &fail, status);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                fence_after();
                const float2* scale = sc[blk % kScSlots];
                const int t0 = i * kTok;
                const bool edge = t0 + kTok - 1 > sure || sc_gone[blk % kScSlots];
                if (edge) {                                // what is not seen becomes -infinity, in tensor memory
#pragma unroll 1
                    for (int u = 0; u < 8; ++u) {
                        const int n = scale[u].y < 0.f ? 0 : last + 1 - (t0 + 16 * u);     // tokens that are seen
                        uint32_t y[16];
                        tmem_ld16(ts + 16 * u, y);
#pragma unroll
                        for (int j = 0; j < 16; ++j) y[j] = j < n ? y[j] : 0xff800000u;
                        tmem_st16(ts + 16 * u, y);
                    }
                    tmem_st_wait();
                }
                float x[kTok];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32_start(ts + 32 * c, x + 32 * c);
                float kf[8], sv[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const float2 k = scale[u];
                    kf[u] = k.x * f;
                    sv[u] = k.y;
                    if (edge) {                            // (0 x -infinity; a scale that is NaN in tokens that the row does not see)
                        const bool none = k.y < 0.f || t0 + 16 * u > last;
                        kf[u] = none || kf[u] == 0.f ? 1.f : kf[u];
                        sv[u] = none ? 0.f : sv[u];
                    }
                }
                tmem_ld_wait();
                // maxima of scores and of score + exponent of V's scale
                float bm = kNegBig, bp = kNegBig;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    float top = x[16 * u];
#pragma unroll
                    for (int j = 1; j < 15; j += 2) top = fmaxf(top, fmaxf(x[16 * u + j], x[16 * u + j + 1]));
                    top = fmaxf(top, x[16 * u + 15]) * kf[u];
                    bm = fmaxf(bm, top);
                    bp = fmaxf(bp, top + (float)(exponent_of(sv[u]) + 1));
                }
                const bool grow = bm > m + 8.f || bp > mp + 8.f;
                if (__any_sync(0xffffffffu, grow)) {
                    const float m2 = grow ? fmaxf(m, ceilf(bm)) : m, p2 = grow ? fmaxf(mp, ceilf(bp)) : mp;
                    const float rl = pow2_down(m, m2), r = pow2_down(mp, p2);
                    l = mul2(l, pack2(rl, rl));
                    m = m2;
                    mp = p2;
                    if (i > g.i0) {
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(to + c, o);
#pragma unroll
                            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * r);
                            tmem_st16(to + c, o);
                        }
                    }
                }
                // weights: w = p sv 2^(m - m' + 7)
                const float d = fmaxf(m - mp + 7.f, -250.f);
                const f32x2 neg = pack2(-m, -m);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int hlf = 0; hlf < 2; ++hlf) {
                        const int u = 2 * c + hlf;
                        const int e = (int)fminf(d, (float)min(126, 125 - exponent_of(sv[u])));
                        const float cw = sv[u] * pow2i(e / 2) * pow2i(e - e / 2);
                        const f32x2 k2 = pack2(kf[u], kf[u]), c2 = pack2(cw, cw);
#pragma unroll
                        for (int j = 0; j < 16; j += 2) {
                            float y0, y1;
                            unpack2(fma2(pack2(x[16 * u + j], x[16 * u + j + 1]), k2, neg), y0, y1);
                            const f32x2 p = pack2(ex2(y0), ex2(y1));
                            l = add2(l, p);
                            unpack2(mul2(p, c2), y0, y1);
                            w[8 * hlf + (j >> 1)] = half2_of(y0, y1);
                        }
                    }
                    tmem_st16(ts + 16 * c, w);
                }
                tmem_st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.p_full + tile);
            }
            ok = ok && mbar_wait(bar.o_done + tile, n_o & 1, &fail, status);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            ++n_o;
            fence_after();
            float l0, l1;
            unpack2(l, l0, l1);
            l0 += l1;
            if (g.i0 == 0 && g.i1 == g.n) {
                const int e = (int)fminf(fmaxf(mp - m - 7.f, -250.f), 250.f);
                const float f1 = pow2i(e / 2), f2 = pow2i(e - e / 2), r = l0 == 0.f ? 0.f : 1.f / l0;
                __nv_bfloat16* o = a.out + (((size_t)g.b * a.n_q + qi) * s.Hq + g.h * s.G + col % s.G) * D;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    float x[32];
                    tmem_ld32(to + c, x);
                    if (there) {
#pragma unroll
                        for (int j = 0; j < 32; j += 8) {
                            uint32_t w[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const __nv_bfloat162 h = __floats2bfloat162_rn(x[j + 2 * k] * r * f1 * f2, x[j + 2 * k + 1] * r * f1 * f2);
                                w[k] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                            *reinterpret_cast<uint4*>(o + c + j) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                    __syncwarp();
                }
            } else {
                // parts of a tile lie one behind the other from 2 x its first CTA + 1 on (as in fa_q8_attn.cu)
                const unsigned cta0 = g.u / line.per;
                float* o = a.part + ((size_t)(cta0 + 1 + blockIdx.x) * kRows + tile * 128 + row) * (D + 4);
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    float x[32];
                    tmem_ld32(to + c, x);
#pragma unroll
                    for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(o + c + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
                }
                *reinterpret_cast<float4*>(o + D) = make_float4(m, mp, l0, 0.f);
            }
            fence_before();                                // the next segment's MMAs come behind its first p_full
        }
    } else if (warp < kMma) {
        // ---- 8-bit values to halves ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsConv));
        constexpr int kChunks = D / 16, kPass = 128 / kChunks, kPasses = kTok / kPass;       // 16-value chunks of a row; rows of a pass
        const int t = tid - kConv * 32, ch = t % kChunks, r0 = t / kChunks;
        uint4 raw[kPasses];                                // of the step that comes: K of a block, then V
        const unsigned char* tails[2] = {static_cast<const unsigned char*>(a.c.k_tail), static_cast<const unsigned char*>(a.c.v_tail)};
        auto paged_of = [&](const Seg& g) { return g.len >> s.lb << s.lb; };
        // Lanes 0-7: where 16 tokens of block i lie each, counted in 16 rows of the pages; kGone where no page is, kTail in the tail and
        // behind the row's last token.
        constexpr uint32_t kGone = 0xffffffffu, kTail = 0xfffffffeu;
        auto pages_of = [&](const Seg& g, int i) {
            const int tok = i * kTok + 16 * (lane & 7);
            if (tok >= paged_of(g)) return kTail;
            const int page = __ldg(a.c.table + (size_t)g.b * s.nb + (tok >> s.lb));
            if (page < 0 || page >= s.n_pages) return kGone;
            return (uint32_t)((((size_t)page * s.H + g.h) * (size_t)s.blk + (tok & (s.blk - 1))) >> 4);
        };
        auto scales_of = [&](const Seg& g, int i, uint32_t at) {
            const size_t ph = at >> (s.lb - 4);
            float2 k = make_float2(ld_if(a.c.k_scale + ph, at < kTail), ld_if(a.c.v_scale + ph, at < kTail));
            if (at == kGone) k.y = -1.f;
            if (at == kTail && i * kTok + 16 * (lane & 7) < g.len) {
                const float* am = a.c.tail_amax + ((size_t)g.b * s.H + g.h) * 2;
                const uint32_t km = __float_as_uint(am[0]), vm = __float_as_uint(am[1]);
                k.x = km >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : pow2i(max((int)(km >> 23) - 127, -100) - 13);
                k.y = vm >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : pow2i(max((int)(vm >> 23) - 127, -100) - 13);
            }
            return k;
        };
        const uint32_t lane_at = (uint32_t)((r0 & 15) * D + 16 * ch);
        auto in_pages = [&](const Seg& g, int i) { return (i + 1) * kTok <= paged_of(g); };      // the block, as a whole (others are read when they are converted)
        auto fetch = [&](int p, const uint8_t* side, uint32_t pages, bool there) {
            const uint32_t at = __shfl_sync(0xffffffffu, pages, (p * kPass + r0) >> 4);
            raw[p] = ld_if16(side + (size_t)at * (16 * D) + lane_at, there && at < kTail);
        };
        // (the upper half of the lanes of a row stores its second chunk first: no two meet in a bank)
        const bool swap = kChunks == 8 && ch >= 4;
        auto put = [&](unsigned char* dst, int r, const uint32_t (&h)[8]) {
            const uint4 lo = make_uint4(h[0], h[1], h[2], h[3]), hi = make_uint4(h[4], h[5], h[6], h[7]);
            *reinterpret_cast<uint4*>(dst + operand_offset(r, 2 * ch + (swap ? 1 : 0))) = swap ? hi : lo;
            *reinterpret_cast<uint4*>(dst + operand_offset(r, 2 * ch + (swap ? 0 : 1))) = swap ? lo : hi;
        };
        auto halves = [&](const uint4& x, uint32_t (&h)[8]) {
            const uint32_t w[4] = {q8_flip<FMT>(x.x), q8_flip<FMT>(x.y), q8_flip<FMT>(x.z), q8_flip<FMT>(x.w)};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                h[2 * k] = q8_halves<FMT>(w[k], 0);
                h[2 * k + 1] = q8_halves<FMT>(w[k], 1);
            }
        };
        bool more = line.next(a, g);
        uint32_t pages = kTail;
        float2 scale = make_float2(0.f, 0.f);
        if (more) {
            pages = pages_of(g, g.i0);
            scale = scales_of(g, g.i0, pages);
#pragma unroll
            for (int p = 0; p < kPasses; ++p) fetch(p, a.c.k_pages, pages, in_pages(g, g.i0));
        }
        while (ok && more) {
            Seg nx = g;
            for (int i = g.i0; i < g.i1; ++i, ++blk) {
                const uint32_t st = blk & 1, ph = (blk >> 1) & 1;
                const bool inside = in_pages(g, i);
                if (i + 1 == g.i1) more = line.next(a, nx);
                const bool go = i + 1 < g.i1 || more;
                const int ni = i + 1 < g.i1 ? i + 1 : nx.i0;                // (nx is g within the segment)
                const uint32_t npages = go ? pages_of(nx, ni) : kTail;
                const bool ninside = go && in_pages(nx, ni);
                float2 nscale = make_float2(0.f, 0.f);
#pragma unroll 1
                for (int side = 0; side < 2; ++side) {
                    if (blk >= 2) ok = mbar_wait((side ? bar.v_empty : bar.k_empty) + st, ph ^ 1, &fail, status);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    if (side == 0 && warp == kConv) {
                        const unsigned gone = __ballot_sync(0xffffffffu, pages == kGone);
                        if (lane < 8) sc[blk % kScSlots][lane] = scale;
                        if (lane == 0) {
                            sc_gone[blk % kScSlots] = gone != 0;
                            if (gone) q8_report(status, FA_ERR_INDEX);
                        }
                    }
                    if (side == 0) nscale = scales_of(nx, ni, go ? npages : kGone);
                    unsigned char* dst = (side ? vs : ks) + st * kTile;
                    const uint8_t* next_side = side ? a.c.k_pages : a.c.v_pages;
                    const uint32_t next_pages = side ? npages : pages;
                    const bool next_inside = side ? ninside : inside;
                    if (inside) {
#pragma unroll
                        for (int p = 0; p < kPasses; ++p) {
                            uint32_t h[8];
                            halves(raw[p], h);
                            fetch(p, next_side, next_pages, next_inside);
                            put(dst, p * kPass + r0, h);
                        }
                    } else {
#pragma unroll 1
                        for (int p = 0; p < kPasses; ++p) {
                            const int r = p * kPass + r0, tok = i * kTok + r;
                            const uint32_t at = __shfl_sync(0xffffffffu, pages, r >> 4);
                            uint32_t h[8];
                            if (at == kTail && tok < g.len) {      // the tail: scaled by the power of two above its largest magnitude
                                const uint32_t mx = __float_as_uint(a.c.tail_amax[((size_t)g.b * s.H + g.h) * 2 + side]);
                                Vec16<__nv_bfloat16> v;
                                if (mx < 0x7f800000u)
                                    v.load(reinterpret_cast<const __nv_bfloat16*>(tails[side]) +
                                           (((size_t)g.b * s.H + g.h) * (size_t)s.blk + (tok - paged_of(g))) * D + 16 * ch);
                                else v.zero();
                                const float f = pow2i(13 - max((int)(mx >> 23) - 127, -100));
#pragma unroll
                                for (int k = 0; k < 8; ++k) h[k] = half2_of(v.at(2 * k) * f, v.at(2 * k + 1) * f);
                            } else if (at < kTail) {
                                halves(ld_if16((side ? a.c.v_pages : a.c.k_pages) + (size_t)at * (16 * D) + lane_at, true), h);
                            } else {
#pragma unroll
                                for (int k = 0; k < 8; ++k) h[k] = 0u;
                            }
                            put(dst, r, h);
                        }
#pragma unroll
                        for (int p = 0; p < kPasses; ++p) fetch(p, next_side, next_pages, next_inside);
                    }
                    fence_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive((side ? bar.v_full : bar.k_full) + st);
                }
                if (!ok) break;
                pages = npages;
                scale = nscale;
            }
            g = nx;
        }
    } else {
        // ---- the MMAs ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsMma));
        // operands: K-major with 64 dims to a row of 128 bytes, the next 64 a box further; V the same read along the tokens (MN-major)
        const uint64_t qd0 = umma_desc(smem_u32(qs), 1, 1024 >> 4), kd0 = umma_desc(smem_u32(ks), 1, 1024 >> 4);
        const uint64_t vd0 = umma_desc(smem_u32(vs), (kTok * 128) >> 4, 1024 >> 4);
        uint32_t n_p[2] = {0, 0}, n_q[2] = {0, 0};         // phases of p_full, q_full
        while (warp == kMma && ok && line.next(a, g)) {
            const int tiles = two_tiles(g) ? 2 : 1;
            const int n = g.i1 - g.i0;
            for (int t = 0; t < tiles && ok; ++t) ok = mbar_wait(bar.q_full + t, n_q[t]++ & 1, &fail, status);
            // step i: the outputs of block i - 1, then the scores of block i, for each tile
#pragma unroll 1
            for (int i = 0; i <= n && ok; ++i) {
                const uint32_t bk = blk + i, bv = bk - 1;
                if (i < n) ok = mbar_wait(bar.k_full + (bk & 1), (bk >> 1) & 1, &fail, status);
                if (ok && i > 0) ok = mbar_wait(bar.v_full + (bv & 1), (bv >> 1) & 1, &fail, status);
                const uint64_t kd = kd0 + (uint64_t)((bk & 1) * kTile >> 4), vd = vd0 + (uint64_t)((bv & 1) * kTile >> 4);
#pragma unroll 1
                for (int t = 0; t < tiles && ok; ++t) {
                    if (i > 0) {
                        if (!(ok = mbar_wait(bar.p_full + t, n_p[t]++ & 1, &fail, status))) break;
                        fence_after();
                        if (lane == 0) {
                            const uint32_t p = tmem + 128 * t, o = tmem + 256 + D * t;
#pragma unroll
                            for (int k = 0; k < kTok / 16; ++k) umma_ts(o, p + 8 * k, vd + (uint64_t)(k * 2048 >> 4), kIdescO, i > 1 || k > 0);
                            if (i == n) umma_commit(bar.o_done + t);
                        }
                        __syncwarp();
                    }
                    if (i < n) {
                        fence_after();
                        if (lane == 0) {
                            const uint64_t qd = qd0 + (uint64_t)(t * kTile >> 4);
#pragma unroll
                            for (int k = 0; k < D / 16; ++k) {
                                const uint64_t off = (uint64_t)(((k >> 2) * (kTok * 128) + (k & 3) * 32) >> 4);
                                umma_bf16(tmem + 128 * t, qd + off, kd + off, kIdescS, k > 0);
                            }
                            umma_commit(bar.s_full + t);
                        }
                        __syncwarp();
                    }
                }
                if (ok && lane == 0) {
                    if (i > 0) umma_commit(bar.v_empty + (bv & 1));
                    if (i < n) umma_commit(bar.k_empty + (bk & 1));
                }
                __syncwarp();
            }
            blk += n;
        }
    }
    fence_before();
    __syncthreads();
    if (warp == kMma) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
    }
}

// Joins the parts of tiles that were cut, in the order of the tokens; zeros for tiles that see nothing.  A CTA takes 32 rows of a tile.
template <int D>
__global__ void __launch_bounds__(256) q8_chunk_join_kernel(const ChunkArgs a) {
    const Q8Dims& s = a.s;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int k = (int)(blockIdx.x / (unsigned)s.H), h = (int)(blockIdx.x % (unsigned)s.H);
    const int b = k / a.n_ct, ct = k % a.n_ct;
    const int n = blocks_of(a, row_len(a, b), ct);
    Line line;
    unsigned u = 0, cta0 = 0, parts = 0;
    if (n > 0) {
        line.measure(a, lane);
        unsigned before = 0;
        for (int k0 = 0; k0 < k; k0 += 32) before += __reduce_add_sync(0xffffffffu, k0 + lane < k ? line.blocks_at(a, k0 + lane) : 0u);
        u = before + (unsigned)h * (unsigned)n;
        cta0 = u / line.per;
        parts = (u + n - 1) / line.per - cta0 + 1;
        if (parts == 1) return;
    }
    constexpr int kPitch = D + 4, kVec = D / 32;           // floats of a lane
    for (int r = blockIdx.y * 32 + warp; r < (int)blockIdx.y * 32 + 32; r += 8) {
        const int col = ct * kRows + r, qi = col / s.G;
        if (qi >= a.n_q) return;
        const float* p = a.part + ((size_t)(2 * cta0 + 1) * kRows + r) * kPitch;
        float m = kNegBig, mp = kNegBig, l = 0.f, o[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) o[i] = 0.f;
#pragma unroll 4
        for (unsigned j = 0; j < parts; ++j) {
            const float* pj = p + (size_t)j * kRows * kPitch;
            const float4 hd = __ldcg(reinterpret_cast<const float4*>(pj + D));
            float x[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) x[i] = __ldcg(pj + lane + 32 * i);
            const float m2 = fmaxf(m, hd.x), p2 = fmaxf(mp, hd.y);
            l = fmaf(l, pow2_down(m, m2), hd.z * pow2_down(hd.x, m2));
            const float f0 = pow2_down(mp, p2), f1 = pow2_down(hd.y, p2);
#pragma unroll
            for (int i = 0; i < kVec; ++i) o[i] = fmaf(o[i], f0, x[i] * f1);
            m = m2;
            mp = p2;
        }
        const int e = (int)fminf(fmaxf(mp - m - 7.f, -250.f), 250.f);
        const float f1 = pow2i(e / 2), f2 = pow2i(e - e / 2), inv = l == 0.f ? 0.f : 1.f / l;
        __nv_bfloat16* out = a.out + (((size_t)b * a.n_q + qi) * s.Hq + h * s.G + col % s.G) * D;
#pragma unroll
        for (int i = 0; i < kVec; ++i) out[lane + 32 * i] = __float2bfloat16_rn(parts ? o[i] * inv * f1 * f2 : 0.f);
    }
}

int chunk_tiles(const Q8Dims& s, int n_q) { return (int)(((long long)n_q * s.G + kRows - 1) / kRows); }
int chunk_ctas() { return sm_count() < kQ8MaxCtas ? sm_count() : kQ8MaxCtas; }

template <int FMT, int D>
cudaError_t chunk_of(const ChunkArgs& a, cudaStream_t stream) {
    const size_t smem = (size_t)6 * kTok * D * 2 + 1024;
    cudaError_t e = ensure_dynamic_smem(q8_chunk_kernel<FMT, D>, smem);
    if (e == cudaSuccess) e = launch_behind(q8_chunk_kernel<FMT, D>, dim3((unsigned)a.ctas), kChunkThreads, smem, stream, a);
    if (e == cudaSuccess) e = launch_behind(q8_chunk_join_kernel<D>, dim3((unsigned)(a.s.B * a.n_ct * a.s.H), kRows / 32), 256, 0, stream, a);
    return e;
}

}  // namespace

bool q8_chunk_takes(const Q8Dims& s, int dtype, int n_q) {
    if (dtype != FA_BF16 || s.d > 128 || (long long)n_q * s.G < 64) return false;
    const long long tiles = (long long)s.B * chunk_tiles(s, n_q);
    return tiles * s.H * (((long long)s.nb * s.blk + kTok - 1) / kTok) <= 0x7fffffff && tiles * s.H <= 0x7fffffff;
}
size_t q8_chunk_ws_bytes(const Q8Dims& s) { return 4096 + (size_t)2 * chunk_ctas() * kRows * (s.d + 4) * sizeof(float); }

cudaError_t launch_q8_chunk(const Q8Dims& s, const Q8Cache& c, int fmt, const void* q, int64_t sb, int64_t si, int64_t sg, void* out, int n_q, char* ws,
                            cudaStream_t stream) {
    const ChunkArgs a = {s, c, static_cast<const __nv_bfloat16*>(q), sb, si, sg, static_cast<__nv_bfloat16*>(out), n_q, chunk_tiles(s, n_q), chunk_ctas(),
                         reinterpret_cast<float*>(ws + 4096)};
    if (s.d == 64) return fmt == FA_Q8_INT8 ? chunk_of<FA_Q8_INT8, 64>(a, stream) : chunk_of<FA_Q8_E4M3, 64>(a, stream);
    return fmt == FA_Q8_INT8 ? chunk_of<FA_Q8_INT8, 128>(a, stream) : chunk_of<FA_Q8_E4M3, 128>(a, stream);
}

}  // namespace fa
