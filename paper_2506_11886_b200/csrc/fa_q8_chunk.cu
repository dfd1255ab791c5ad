// fa_q8_attention with many query columns to a KV head (a chunk of a prompt): scores and outputs on the 5th-generation
// tensor cores (tcgen05.mma, halves in, fp32 accumulators in tensor memory).
//
// A CTA takes 256 rows, a row being one (query, query head) of a KV head, as two tiles of 128, over blocks of 128 tokens.  Per block and tile:
// S = Q K^T (accumulators), the weights P of the softmax rounded to halves in the place of S, O += P V with P read from
// tensor memory.  The two tiles take turns: the tensor cores work for one while the other's weights are formed.
//   warps 0-7, 8-15  a tile each, two threads to a row with 64 of the block's tokens each: the row's maximum (exchanged), exponentials,
//                    sums; O is rescaled in tensor memory only when a maximum has grown by more than 8 (powers of two: exactly).  (One thread to a row, its 128
//                    scores in registers, took 6000 clocks a block: two warps to a scheduler do not cover their own latencies.)
//   warps 16-19, 21-23  8-bit values to halves (exactly) in shared memory, K and V in turn, the other one's bytes under way; two stages for each
//   warp 20          issues the MMAs
// Scales, the tail and the weights are as in fa_q8_attn.cu with 2^7 in the place of 2^15, which leaves the maxima room to grow; a weight is one exponential, of
// score + log2 of V's scale - m' + 7, and 16 tokens' sum of weights becomes their sum of p by one factor.  int8 K values are taken as q + 128 in the place of
// a half's last bits (that is (q + 128) 2^-24, exactly): two instructions less a value; 128 times the sum of the row's q is subtracted from the scores.  The blocks of all
// tiles stand in a line that is cut into equal parts, one for each SM; the parts of a tile that is cut meet in the workspace, and a second kernel
// joins them, spread over all SMs.
// The loops of the roles share the instruction cache: what is unrolled (a row of scores in registers) is written once, the rest kept small.
// The exponentials (16 a clock and SM) take 2048 clocks for a block and 256 rows of any head dim, the tensor cores as many at 128 dims; it is bound by the chain of a tile
// (scores, maximum, exponentials, products), 5300 clocks, of which two run at a time: 2048 queries of 32/8 heads of 128 over 16384 tokens 650 us (793 TFLOP/s; e4m3
// 669).  Registers are bounded at 80 a thread: 60 to 124 bytes are spilled.
#include <type_traits>

#include "fa_q8.cuh"
#include "fa_umma.cuh"

namespace fa {
namespace {

using namespace umma;

constexpr int kRows = 256, kTok = 128;
constexpr int kConv = 16, kMma = 20, kConvWarps = 7;       // first converting warp, the issuing warp, converting warps (16-19, 21-23)
constexpr int kChunkThreads = 24 * 32;
// Blocks whose outputs one accumulator takes, a power of two.  The MMAs' sums are cut off, not rounded: over 8192 blocks of V of one sign the outputs
// came out 4.2e-3 of themselves too small.  After a run its sums go to the workspace, where they are added with rounding: 4e-4, which is no more
// than the halves and the output lose.  Tiles below 32768 tokens to a CTA are one run; they pay 1 % for the branch (639 -> 645 us).  The sums of p are kept in
// the same runs: one sum over 2^24 tokens, rounded at every addition, was 0.8 % too small where all p were alike.
constexpr int kRun = 256;
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

__device__ __forceinline__ bool is_length(const ChunkArgs& a, int len) { return len >= 0 && len <= (a.s.nb << a.s.lb); }
// Tokens of row b that the cache holds (none if its state is no length: the joining kernel reports that); those that column tile ct sees, in blocks of 128.
__device__ __forceinline__ int row_len(const ChunkArgs& a, int b) {
    const int len = a.c.state[b * kQ8State];
    return is_length(a, len) ? len : 0;
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

// Row r, dims 8 c .. 8 c + 7 of an operand of D dims: 64 dims to a 128-byte row, its 16-byte chunks permuted by the row.  With 128 dims the even c come first,
// then the odd ones, in q, K and V alike (and so in the columns of O): the lanes that store a row's chunks then meet all banks.
template <int D>
__device__ __forceinline__ int operand_offset(int r, int c) {
    const int at = D == 128 ? (c >> 1) + 8 * (c & 1) : c;
    return (at >> 3) * (kTok * 128) + r * 128 + (((at & 7) ^ (r & 7)) << 4);
}
// First of the 8 dims that columns 8 at .. 8 at + 7 of O are.
template <int D>
__device__ __forceinline__ int dim_of(int at) { return D == 128 ? 16 * (at & 7) + 8 * (at >> 3) : 8 * at; }

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
    __shared__ float2 sc[kScSlots][8];                     // K scale (NaN if V's is) and log2 of V's scale of 16 tokens each
    __shared__ int sc_marks[kScSlots];                     // bit u: 16 tokens that have no page; bit 8 + u: in the tail
    __shared__ float2 meet[2][2][2][128];                  // what the two threads of a row tell each other: [turn][tile][half][row]
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int fail;
    const Q8Dims& s = a.s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar.k_full + i, kConvWarps); mbar_init(bar.k_empty + i, 1); mbar_init(bar.v_full + i, kConvWarps); mbar_init(bar.v_empty + i, 1);
            mbar_init(bar.q_full + i, 8); mbar_init(bar.s_full + i, 1); mbar_init(bar.p_full + i, 8); mbar_init(bar.o_done + i, 1);
        }
        fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // Tensor memory is taken when the kernel in front has ended, and the one behind comes when this one has its own: none holds what another waits for.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == kMma) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    asm volatile("griddepcontrol.launch_dependents;");
    const uint32_t tmem = tmem_slot;
    const uint32_t tmem_s[2] = {tmem, tmem + 128}, tmem_o[2] = {tmem + 256, tmem + 256 + D};
    int32_t* status = a.c.status;

    Line line;
    line.begin(a, lane, (int)blockIdx.x);
    Seg g;
    auto two_tiles = [&](const Seg& g) { return g.ct * kRows + 128 < a.n_q * s.G; };
    uint32_t blk = 0;                                      // blocks so far: stages and phases
    bool ok = true;

    if (warp < 16) {
        // ---- a tile's weights ----
        const int tile = warp >> 3, half = (warp >> 2) & 1, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        // this thread's scores, whose place its weights take (two to a column), and its half of the columns of O
        const uint32_t ts = tmem_s[tile] + lanes + 64 * half, to = tmem_o[tile] + lanes + (D / 2) * half;
        uint32_t n_s = 0, n_o = 0, turn = 0;               // phases of s_full, o_done; turns of `meet`
        // Both threads of a row: what the other one says.  (Two turns' places: a place is written again when both are past the turn between.)
        auto tell = [&](float2 v) {
            meet[turn & 1][tile][half][row] = v;
            asm volatile("bar.sync %0, 64;" ::"r"(1 + tile * 4 + (warp & 3)) : "memory");
            v = meet[turn & 1][tile][half ^ 1][row];
            ++turn;
            return v;
        };
        // A wait that gave up (recorded by mbar_wait, which then returns at once everywhere) does not end these loops: the two threads of a row meet at
        // barriers that know no limit, so both go through all of them, whatever the numbers are.
        while (line.next(a, g)) {
            if (tile == 1 && !two_tiles(g)) { blk += g.i1 - g.i0; continue; }
            const int col = g.ct * kRows + tile * 128 + row, qi = col / s.G;
            const bool there = qi < a.n_q;
            // q: scaled by a power of two to halves, into shared memory; a thread has half of the dims
            float f, shift;
            {
                const __nv_bfloat16* qp = a.q + (int64_t)g.b * a.sb + (int64_t)qi * a.si + (int64_t)(g.h * s.G + col % s.G) * a.sg + (D / 2) * half;
                Vec16<__nv_bfloat16> v[D / 32];
                uint32_t mx = 0;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    if (there) v[c].load(qp + 16 * c);
                    else v[c].zero();
                    mx = max(mx, v[c].amax_bits());
                }
                mx = max(mx, __float_as_uint(tell(make_float2(__uint_as_float(mx), 0.f)).x));
                const int eq = max((int)(mx >> 23) - 127, -100);
                const float fq = pow2i(13 - eq);
                f = pow2i(eq - 13) * (s.scale * kLog2e);
                float sum = 0.f;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        y[k] = v[c >> 1].at(8 * (c & 1) + k) * fq;
                        sum += y[k];                       // (as the halves have it, but for values below 2^-29 of the largest)
                    }
                    *reinterpret_cast<uint4*>(qs + tile * kTile + operand_offset<D>(row, half * (D / 16) + c)) =
                        make_uint4(half2_of(y[0], y[1]), half2_of(y[2], y[3]), half2_of(y[4], y[5]), half2_of(y[6], y[7]));
                }
                const float other = tell(make_float2(sum, 0.f)).x;
                sum = half ? other + sum : sum + other;    // (the same bits in both)
                // a product of int8 K is (q + 128) 2^-24 times q: score = (product - shift) x scale
                shift = FMT == FA_Q8_INT8 ? 128.f * sum : 0.f;
            }
            constexpr float grain = FMT == FA_Q8_INT8 ? 0x1p24f : 1.f;
            fence_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.q_full + tile);

            const int last = there ? g.len - a.n_q + qi : -1;            // the last token that the row sees
            // the first token that some row of the warp does not see
            const int sure = __reduce_min_sync(0xffffffffu, there ? last : 0x7fffffff);
            float m = kNegBig, mp = kNegBig;
            float l = 0.f, l_runs = 0.f;                   // of this half's tokens: of the present run, of those before
            // The weights of block i.  edge: some row of the warp does not see all of its tokens, or some of them are in the tail.
            auto weights = [&](auto edge_of, const float2* scale, int marks, int i) {
                constexpr bool edge = decltype(edge_of)::value;
                const int t0 = i * kTok + 64 * half;
                if constexpr (edge) {                      // what is not seen becomes -infinity, in tensor memory
#pragma unroll 1
                    for (int u = 0; u < 4; ++u) {
                        const int n = marks >> u & 1 ? 0 : last + 1 - (t0 + 16 * u);       // tokens that are seen
                        uint32_t y[16];
                        tmem_ld16(ts + 16 * u, y);
#pragma unroll
                        for (int j = 0; j < 16; ++j) y[j] = j < n ? y[j] : 0xff800000u;
                        tmem_st16(ts + 16 * u, y);
                    }
                    tmem_st_wait();
                }
                // Of 16 tokens: score = product x kf + off; log2 of V's scale.
                float kf[4], off[4], lv[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float2 k = scale[u];
                    float kk = k.x * f;
                    kf[u] = kk * grain;
                    off[u] = -kk * shift;
                    if constexpr (edge) {                  // tokens that are not seen, in whatever scale; 0 x -infinity; the tail's products have no shift
                        const bool none = (marks >> u & 1) || t0 + 16 * u > last, tail = marks >> (8 + u) & 1;
                        kk = none ? 1.f : kk == 0.f ? 0x1p-100f : kk;
                        kf[u] = tail ? kk : kk * grain;
                        off[u] = none || tail ? 0.f : -kk * shift;
                    }
                    lv[u] = k.y;
                }
                // maxima of scores and of score + log2 of V's scale
                float bm = kNegBig, bp = kNegBig;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float x[32], top[2];
                    tmem_ld32(ts + 32 * c, x);
#pragma unroll
                    for (int h2 = 0; h2 < 2; ++h2) {
                        const float* y = x + 16 * h2;
                        const float p = fmaxf(fmaxf(y[0], y[1]), y[2]), q = fmaxf(fmaxf(y[3], y[4]), y[5]), r = fmaxf(fmaxf(y[6], y[7]), y[8]);
                        const float w = fmaxf(fmaxf(y[9], y[10]), y[11]), v = fmaxf(fmaxf(y[12], y[13]), y[14]);
                        top[h2] = fmaxf(fmaxf(fmaxf(p, q), fmaxf(r, w)), fmaxf(v, y[15]));
                    }
#pragma unroll
                    for (int h2 = 0; h2 < 2; ++h2) {
                        const float y = fmaf(top[h2], kf[2 * c + h2], off[2 * c + h2]);
                        bm = fmaxf(bm, y);
                        bp = fmaxf(bp, y + lv[2 * c + h2]);
                    }
                }
                const float2 other = tell(make_float2(bm, bp));
                bm = fmaxf(bm, other.x);
                bp = fmaxf(bp, other.y);
                const bool grow = bm > m + 8.f || bp > mp + 8.f;
                if (__any_sync(0xffffffffu, grow)) {
                    const float m2 = grow ? fmaxf(m, ceilf(bm)) : m, p2 = grow ? fmaxf(mp, ceilf(bp)) : mp;
                    const float rl = pow2_down(m, m2), r = pow2_down(mp, p2);
                    l *= rl;
                    l_runs *= rl;
                    m = m2;
                    mp = p2;
                    if (i > g.i0) {
#pragma unroll 1
                        for (int c = 0; c < D / 2; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(to + c, o);
#pragma unroll
                            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * r);
                            tmem_st16(to + c, o);
                        }
                    }
                }
                // weights: w = p sv 2^(m - m' + 7); below 2^-100 p they are none, and p is what the sum needs
                const float d = m - mp + 7.f;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t w[16];
                    float x[32];
                    tmem_ld32(ts + 32 * c, x);                       // (again: they would not all stay in registers)
#pragma unroll
                    for (int h2 = 0; h2 < 2; ++h2) {
                        const int u = 2 * c + h2;
                        const float e = fmaxf(lv[u] + d, -100.f), back = ex2(-e), z = off[u] + (e - m);
                        const f32x2 k2 = pack2(kf[u], kf[u]), z2 = pack2(z, z);
                        f32x2 sum = pack2(0.f, 0.f);
#pragma unroll
                        for (int j = 0; j < 16; j += 2) {
                            float y0, y1;
                            unpack2(fma2(pack2(x[16 * h2 + j], x[16 * h2 + j + 1]), k2, z2), y0, y1);
                            y0 = ex2(y0);
                            y1 = ex2(y1);
                            sum = add2(sum, pack2(y0, y1));
                            w[8 * h2 + (j >> 1)] = half2_of(y0, y1);
                        }
                        float s0, s1;
                        unpack2(sum, s0, s1);
                        l = fmaf(s0 + s1, back, l);
                    }
                    tmem_st16(ts + 16 * c, w);
                }
            };
            // Parts of a tile lie one behind the other from 2 x its first CTA + 1 on (as in fa_q8_attn.cu); a tile that is not cut has a place there too.
            // (Found anew where it is needed: registers are short in between.)
            auto place = [&] {
                unsigned cta;
                asm volatile("mov.u32 %0, %%ctaid.x;" : "=r"(cta));
                return a.part + ((size_t)(g.u / line.per + 1 + cta) * kRows + tile * 128 + row) * (D + 4);
            };
            for (int i = g.i0; i < g.i1; ++i, ++blk, ++n_s) {
                mbar_wait(bar.s_full + tile, n_s & 1, &fail, status);
                __syncwarp();
                fence_after();
                if (i > g.i0 && ((i - g.i0) & (kRun - 1)) == 0) {      // (the MMAs of the block before are done, those of this one start from zero)
                    float* part = place();
                    const bool more = i - g.i0 > kRun;
                    const float r = more ? pow2_down(part[D + half], mp) : 0.f;            // (the m' of what stands there)
                    __syncwarp();
#pragma unroll 1
                    for (int c = 0; c < D / 2; c += 16) {
                        uint32_t x[16];
                        tmem_ld16(to + c, x);
                        const int at = ((D / 2) * half + c) >> 3;
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            float4* p = reinterpret_cast<float4*>(part + dim_of<D>(at + (j >> 3)) + (j & 4));
                            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (more) y = *p;
                            *p = make_float4(fmaf(y.x, r, __uint_as_float(x[j])), fmaf(y.y, r, __uint_as_float(x[j + 1])),
                                             fmaf(y.z, r, __uint_as_float(x[j + 2])), fmaf(y.w, r, __uint_as_float(x[j + 3])));
                        }
                        __syncwarp();
                    }
                    part[D + half] = mp;
                    l_runs += l;
                    l = 0.f;
                }
                const int marks = sc_marks[blk % kScSlots] >> (4 * half);           // (bits 0-3 and 8-11 are this half's)
                if (i * kTok + 64 * half + 63 > sure || (marks & 0xf0f)) weights(std::true_type(), sc[blk % kScSlots] + 4 * half, marks, i);
                else weights(std::false_type(), sc[blk % kScSlots] + 4 * half, marks, i);
                tmem_st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.p_full + tile);
            }
            mbar_wait(bar.o_done + tile, n_o & 1, &fail, status);
            __syncwarp();
            ++n_o;
            fence_after();
            l += l_runs;
            float* part = place();
            const bool runs = g.i1 - g.i0 > kRun;          // sums of the runs before stand in `part`
            const float rh = runs ? pow2_down(part[D + half], mp) : 0.f;           // (read in front of the turn: the other thread writes here at the end)
            const float l_other = tell(make_float2(l, 0.f)).x;
            l = half ? l_other + l : l + l_other;
            const int e = (int)fminf(fmaxf(mp - m - 7.f, -250.f), 250.f);
            const float f1 = pow2i(e / 2), f2 = pow2i(e - e / 2), r = l == 0.f ? 0.f : 1.f / l;
            const bool lone = g.i0 == 0 && g.i1 == g.n;
            __nv_bfloat16* o = a.out + (((size_t)g.b * a.n_q + qi) * s.Hq + g.h * s.G + col % s.G) * D;
#pragma unroll 1
            for (int c = 0; c < D / 2; c += 16) {
                uint32_t x[16];
                tmem_ld16(to + c, x);
                const int at = ((D / 2) * half + c) >> 3;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = __uint_as_float(x[8 * j + k]);
                    const int dim = dim_of<D>(at + j);
                    if (runs) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] = fmaf(part[dim + k], rh, y[k]);
                    }
                    if (lone && there) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * k] * r * f1 * f2, y[2 * k + 1] * r * f1 * f2);
                            w[k] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                        *reinterpret_cast<uint4*>(o + dim) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    if (!lone) {
                        *reinterpret_cast<float4*>(part + dim) = make_float4(y[0], y[1], y[2], y[3]);
                        *reinterpret_cast<float4*>(part + dim + 4) = make_float4(y[4], y[5], y[6], y[7]);
                    }
                }
                __syncwarp();
            }
            if (!lone && half == 0) *reinterpret_cast<float4*>(part + D) = make_float4(m, mp, l, 0.f);
            fence_before();                                // the next segment's MMAs come behind its first p_full
        }
    } else if (warp != kMma) {
        // ---- 8-bit values to halves ----
        constexpr int kChunks = D / 16, kRowsOf = 32 / kChunks, kItems = kTok / kRowsOf;      // 16-value chunks of a row; rows of a warp's load; loads of a side
        constexpr int kMine = (kItems + kConvWarps - 1) / kConvWarps;                         // ... of a warp
        const int w0 = warp < kMma ? warp - kConv : warp - kConv - 1, ch = lane % kChunks, r0 = lane / kChunks;
        uint4 raw[kMine];                                  // of the step that comes: K of a block, then V
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
        auto scales_of = [&](const Seg& g, int i, uint32_t at) {     // K's and V's
            const size_t ph = at >> (s.lb - 4);
            float2 k = make_float2(0.f, 0.f);
            if (at < kTail) k = make_float2(__ldg(a.c.k_scale + ph), __ldg(a.c.v_scale + ph));
            if (at == kTail && i * kTok + 16 * (lane & 7) < g.len) {
                const float* am = a.c.tail_amax + ((size_t)g.b * s.H + g.h) * 2;
                const uint32_t km = __float_as_uint(am[0]), vm = __float_as_uint(am[1]);
                k.x = km >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : pow2i(max((int)(km >> 23) - 127, -100) - 13);
                k.y = vm >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : pow2i(max((int)(vm >> 23) - 127, -100) - 13);
            }
            return k;
        };
        // A block that lies in pages as a whole is loaded a step ahead; others are read when they are converted.
        auto in_pages = [&](uint32_t pages) { return !__any_sync(0xffffffffu, pages >= kTail); };
        auto fetch = [&](int p, const uint8_t* side, uint32_t pages) {
            const int it = w0 + p * kConvWarps;
            if (it < kItems) {                             // (the whole warp)
                const int r = it * kRowsOf + r0;
                const uint32_t at = __shfl_sync(0xffffffffu, pages, r >> 4);
                raw[p] = __ldg(reinterpret_cast<const uint4*>(side + (size_t)at * (16 * D) + (uint32_t)((r & 15) * D + 16 * ch)));
            }
        };
        auto put = [&](unsigned char* dst, int r, const uint32_t (&h)[8]) {
            *reinterpret_cast<uint4*>(dst + operand_offset<D>(r, 2 * ch)) = make_uint4(h[0], h[1], h[2], h[3]);
            *reinterpret_cast<uint4*>(dst + operand_offset<D>(r, 2 * ch + 1)) = make_uint4(h[4], h[5], h[6], h[7]);
        };
        auto halves = [&](const uint4& x, bool low, uint32_t (&h)[8]) {           // low: q + 128 as the last bits
            const uint32_t w[4] = {q8_flip<FMT>(x.x), q8_flip<FMT>(x.y), q8_flip<FMT>(x.z), q8_flip<FMT>(x.w)};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (FMT == FA_Q8_INT8 && low) {
                    h[2 * k] = __byte_perm(w[k], 0u, 0x4140);
                    h[2 * k + 1] = __byte_perm(w[k], 0u, 0x4342);
                } else {
                    h[2 * k] = q8_halves<FMT>(w[k], 0);
                    h[2 * k + 1] = q8_halves<FMT>(w[k], 1);
                }
            }
        };
        bool more = line.next(a, g);
        uint32_t pages = kTail;
        float2 scale = make_float2(0.f, 0.f);
        bool inside = false;
        if (more) {
            pages = pages_of(g, g.i0);
            scale = scales_of(g, g.i0, pages);
            inside = in_pages(pages);
            if (inside)
#pragma unroll
                for (int p = 0; p < kMine; ++p) fetch(p, a.c.k_pages, pages);
        }
        while (ok && more) {
            Seg nx = g;
            for (int i = g.i0; i < g.i1; ++i, ++blk) {
                const uint32_t st = blk & 1, ph = (blk >> 1) & 1;
                if (i + 1 == g.i1) more = line.next(a, nx);
                const int ni = i + 1 < g.i1 ? i + 1 : nx.i0;                // (nx is g within the segment)
                const uint32_t npages = i + 1 < g.i1 || more ? pages_of(nx, ni) : kTail;
                const bool ninside = in_pages(npages);
                float2 nscale = make_float2(0.f, 0.f);
#pragma unroll 1
                for (int side = 0; side < 2; ++side) {
                    if (blk >= 2) ok = mbar_wait((side ? bar.v_empty : bar.k_empty) + st, ph ^ 1, &fail, status);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    if (side == 0) {
                        if (warp == kConv) {
                            const unsigned gone = __ballot_sync(0xffffffffu, pages == kGone) & 0xffu, tail = __ballot_sync(0xffffffffu, pages == kTail) & 0xffu;
                            if (lane < 8) sc[blk % kScSlots][lane] = make_float2(scale.y != scale.y ? scale.y : scale.x, log2f(scale.y));
                            if (lane == 0) {
                                sc_marks[blk % kScSlots] = (int)(gone | tail << 8);
                                if (gone) q8_report(status, FA_ERR_INDEX);
                            }
                        }
                        if (i + 1 < g.i1 || more) nscale = scales_of(nx, ni, npages);
                    }
                    unsigned char* dst = (side ? vs : ks) + st * kTile;
                    const uint8_t* next_side = side ? a.c.k_pages : a.c.v_pages;
                    const uint32_t next_pages = side ? npages : pages;
                    const bool next_inside = side ? ninside : inside;
                    if (inside && next_inside) {
#pragma unroll
                        for (int p = 0; p < kMine; ++p) {
                            uint32_t h[8];
                            halves(raw[p], side == 0, h);
                            fetch(p, next_side, next_pages);
                            if (w0 + p * kConvWarps < kItems) put(dst, (w0 + p * kConvWarps) * kRowsOf + r0, h);
                        }
                    } else {
                        if (inside) {                      // its last step: nothing to be loaded ahead
#pragma unroll
                            for (int p = 0; p < kMine; ++p) {
                                uint32_t h[8];
                                halves(raw[p], side == 0, h);
                                if (w0 + p * kConvWarps < kItems) put(dst, (w0 + p * kConvWarps) * kRowsOf + r0, h);
                            }
                        } else {
#pragma unroll 1
                            for (int it = w0; it < kItems; it += kConvWarps) {
                                const int r = it * kRowsOf + r0, tok = i * kTok + r;
                                const uint32_t at = __shfl_sync(0xffffffffu, pages, r >> 4);
                                uint32_t h[8];
                                if (at == kTail && tok < g.len) {  // the tail: scaled by the power of two above its largest magnitude
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
                                    halves(__ldg(reinterpret_cast<const uint4*>((side ? a.c.v_pages : a.c.k_pages) + (size_t)at * (16 * D) + (uint32_t)((r & 15) * D + 16 * ch))),
                                           side == 0, h);
                                } else {
#pragma unroll
                                    for (int k = 0; k < 8; ++k) h[k] = 0u;
                                }
                                put(dst, r, h);
                            }
                        }
                        if (next_inside)
#pragma unroll
                            for (int p = 0; p < kMine; ++p) fetch(p, next_side, next_pages);
                    }
                    fence_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive((side ? bar.v_full : bar.k_full) + st);
                }
                if (!ok) break;
                pages = npages;
                scale = nscale;
                inside = ninside;
            }
            g = nx;
        }
    } else {
        // ---- the MMAs ----
        // operands: K-major with 64 dims to a row of 128 bytes, the next 64 a box further; V the same read along the tokens (MN-major)
        const uint64_t qd0 = umma_desc(smem_u32(qs), 1, 1024 >> 4), kd0 = umma_desc(smem_u32(ks), 1, 1024 >> 4);
        const uint64_t vd0 = umma_desc(smem_u32(vs), (kTok * 128) >> 4, 1024 >> 4);
        uint32_t n_p[2] = {0, 0}, n_q[2] = {0, 0};         // phases of p_full, q_full
        while (ok && line.next(a, g)) {
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
                            for (int k = 0; k < kTok / 16; ++k) umma_ts(o, p + 8 * k + 32 * (k >> 2), vd + (uint64_t)(k * 2048 >> 4), kIdescO, ((i - 1) & (kRun - 1)) != 0 || k > 0);
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

// Joins the parts of tiles that were cut, in the order of the tokens; zeros for tiles that see nothing; rows whose state is no length are reported.  A warp
// takes a row.
template <int D>
__global__ void __launch_bounds__(256) q8_chunk_join_kernel(const ChunkArgs a) {
    const Q8Dims& s = a.s;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int k = (int)(blockIdx.x / (unsigned)s.H), h = (int)(blockIdx.x % (unsigned)s.H);
    const int b = k / a.n_ct, ct = k % a.n_ct;
    if (ct == 0 && h == 0 && blockIdx.y == 0 && threadIdx.x == 0 && !is_length(a, a.c.state[b * kQ8State])) q8_report(a.c.status, FA_ERR_CAPACITY);
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
    {
        const int r = (int)blockIdx.y * 8 + warp, col = ct * kRows + r, qi = col / s.G;
        if (qi >= a.n_q) return;
        const float* p = a.part + ((size_t)(2 * cta0 + 1) * kRows + r) * kPitch;
        float m = kNegBig, mp = kNegBig, l = 0.f, o[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) o[i] = 0.f;
#pragma unroll 8
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
    if (e == cudaSuccess) e = launch_behind(q8_chunk_join_kernel<D>, dim3((unsigned)(a.s.B * a.n_ct * a.s.H), kRows / 8), 256, 0, stream, a);
    return e;
}

}  // namespace

bool q8_chunk_takes(const Q8Dims& s, int dtype, int n_q) {
    // Over 64 columns to a KV head: one row of 16384 tokens, 32/8 heads of 128, us here / by tiles of 16 columns: 64 columns 55 / 49, 128 56 / 86,
    // 256 68 / 155; of 1000 tokens 128 columns 24 / 17, 512 30 / 40; eight rows of 4000 tokens 64 columns 68 / 87.  The rows' lengths, by which this would
    // go as well, are on the device: columns alone decide, which costs the short rows of these 7 us and the eight rows 19.
    if (dtype != FA_BF16 || s.d > 128 || (long long)n_q * s.G <= 64) return false;
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
