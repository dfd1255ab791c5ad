// fa_q8_attention and fa_q8_step: softmax attention over the dense cache in 8 bits, few query columns to a KV head.
//
// A column is one (query, query head) of a KV head; a pass over the head's tokens serves 8 or 16 columns.  Scores and
// outputs are formed transposed, S^T = K Q^T and O^T = V^T P^T (mma.sync m16n8k16, halves in, fp32 sums): the 16 rows are tokens,
// then head dims, and no row is lost to padding of the few columns.  The contraction over head dims may take them in any order as long as
// q follows it, and the rows of O^T may be any dims: a lane reads its operand rows as 16 consecutive bytes of a token row.
// 8-bit values are halves exactly; q is scaled by a power of two per column, which makes its bf16 values halves exactly (fp32 q: a high
// and a low half, two products).  With bf16 q, int8 K is taken as q8 + 128 in a half's last bits, that is (q8 + 128) 2^-24, exactly: a subtraction less for two
// values; 128 times the sum of the column's q goes off the scores in the multiplication by the scale.
//
// Scales: a score is multiplied by its block's K scale.  The weight of a token in O is w = p sv 2^(m - m' + 15), sv its block's
// V scale, m the column's running maximum of the scores, m' that of score + exponent of sv, both rounded up to whole numbers (of log2), so
// that rescaling is exact: w is at most 2^15 and its rounding to a half is relative to 2^-24 of the largest weight
// or better; the sum of the p runs beside it in fp32.  The exponent of sv counts as -111 at least, which keeps 2^(m - m' + 15) a number: where all of V is
// smaller, the weights are p sv 2^126 and use less of the range.  The tail is the same with the power of two above its largest magnitude
// in the place of the scale.
//
// Work: a (row, head, column tile) pair has one unit for every 16 tokens in pages and one for the tail.  As long as there are fewer pairs than CTAs,
// the pairs are cut into parts, as many in all as there are CTAs, no part over the end of a pair; with more pairs the units of
// all pairs stand in a line that is cut into equal parts, whatever the rows' lengths.  In a part each of 8 warps takes every 8th
// unit by itself, through a ring of its own in shared memory (cp.async, 16-byte chunks permuted so that the operand reads meet all banks);
// the warps join in shared memory, the parts of a pair in the workspace, by the last CTA to finish, in the order of the tokens.
// Bound by HBM for long rows, by the chain lengths - page - values - join for short ones.  32/8 heads of 128, one row of 128 / 1003 / 8192 / 32001 / 131000 tokens:
// 6.4 / 9.5 / 12.2 / 23.1 / 56 us (int8), four rows of 131000 190 us (e4m3, 5.65 TB/s, back to back, at the clocks of the power cap); from one GPU to another up to 6 % apart.
#include "fa_q8.cuh"

namespace fa {
namespace {

constexpr int kUnit = 16;            // tokens
constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kFlat = 40;            // parts that one CTA joins in one go
// Units whose sums a warp keeps in registers.  The MMAs' sums are cut off, not rounded, and rounded ones of equal addends err one way too: over 131072 units
// outputs of one sign came out 1.2e-2 too small, fp32 ones 5e-5.  After a run the sums go to the workspace, where they are added with rounding.  Rows below
// 131072 tokens to a CTA are one run; they pay up to 2 % for the loop around (32001 tokens 22.7 -> 23.1 us).
constexpr int kRun = 1024;
__host__ __device__ constexpr int run_floats(int d, int nt) { return nt * (d / 4 + 6); }         // of a lane: outputs; m, m', sum of p of its two columns
constexpr float kMinExp = -111.f;    // V scales count as 2^-112 at least in m'
constexpr int kTailExp = -113;       // a tail's largest magnitude as this power of two at least: 2^(13 - kTailExp) is a number

struct AttnArgs {
    Q8Dims s;
    Q8Cache c;
    const void* q;
    int64_t sb, si, sg;
    void* out;
    int n_q, n_ct;                   // queries a row, column tiles of a KV head
    int share;                       // CTAs to a (head, column tile) if there is one row, 0 if there are more of these than CTAs
    const void *k_new, *v_new;       // a step
    unsigned* tickets;
    float* part;                     // [2 * CTAs][cols][D + 4]
    float* runs;                     // [CTAs][warps][run_floats][32]; none where no warp can have more than kRun units
};

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix_t(uint32_t a) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }       // -126 <= e <= 127
// 2^(a - b) for whole a <= b.
__device__ __forceinline__ float pow2_down(float a, float b) {
    const float e = fmaxf(a - b, -127.f);
    return e <= -127.f ? 0.f : pow2i((int)e);
}
__device__ __forceinline__ uint32_t half2_of(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// What the rounding to halves left, as halves.
__device__ __forceinline__ uint32_t half2_rest(float a, float b, uint32_t hi) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    return half2_of(a - f.x, b - f.y);
}
__device__ __forceinline__ int exponent_of(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there = true) {      // zeros if not there
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a) : "memory");
    return r;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a) : "memory");
    return r;
}
__device__ __forceinline__ float lds4(uint32_t a) {
    float r;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(r) : "r"(a) : "memory");
    return r;
}

// Ring of a warp.  A stage holds a unit (16 tokens) of pages: K rows, V rows, the two scales.  The tail's unit, in T, takes
// kTail stages before the first unit of pages comes (none: fp32 rows of 256 dims, read from global memory instead).
template <typename T, int D>
struct Ring {
    static constexpr int kBytes = 32 * D + 16;
    static constexpr int kTail = sizeof(T) == 4 && D == 256 ? 0 : (int)sizeof(T);
    static constexpr int kStages = kTail == 4 ? 5 : 3;
    static constexpr int kFirst = kStages == 5 ? 4 : 2;              // stage of a part's first unit
    static_assert(kTail * 32 * D >= (kTail ? 32 * D * (int)sizeof(T) : 0), "the tail's unit fits");
};
// Chunk (16 bytes) `c` of row `r` of a unit: the chunks of a 128-byte line are permuted by a key that differs between the rows that a read meets.
template <int D>
__device__ __forceinline__ int unit_offset(int r, int c) {
    if constexpr (D == 64) return (r >> 1) * 128 + (((((r & 1) << 2) | c) ^ (r & 6)) << 4);
    else return r * D + (((c & ~7) | ((c ^ r) & 7)) << 4);
}
// First dim of the 16 that lane t of a quad takes of a K row (and of q) as its `c`-th piece.
template <int D>
__device__ __forceinline__ int k_dim(int c, int t) { return D == 64 ? 16 * t : 128 * (c >> 1) + 32 * t + 16 * (c & 1); }

template <int D>
__device__ __forceinline__ void issue_unit(uint32_t stage, const uint8_t* kp, const uint8_t* vp, const float* scale, int lane) {   // scale: lane 0 K's, lane 1 V's
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const int l = i * 32 + lane, off = unit_offset<D>(l / (D / 16), l % (D / 16));
        cp16(stage + off, kp + 16 * l);
        cp16(stage + 16 * D + off, vp + 16 * l);
    }
    if (lane < 2) cp4(stage + 32 * D + 4 * lane, scale);
}

// The columns of a segment as a warp holds them.
template <typename T, int D, int NT>
struct Columns {
    static constexpr int kMt = D / 16;
    uint32_t q[NT][kMt][2];          // column g: dims in the order of the lanes' K bytes
    uint32_t ql[sizeof(T) == 4 ? NT : 1][sizeof(T) == 4 ? kMt : 1][2];
    static constexpr bool kF32 = sizeof(T) == 4;
    float f[NT][2];                  // columns 2 t, 2 t + 1: logits (base 2) per product
    float shift[kF32 ? 1 : NT][2];   // 128 times the sum of their q (as halves)
    int last[NT][2];                 // the last token they see
    float m[NT][2], mp[NT][2], l[NT][2];
    float g[NT][2];                  // 2^(m - m' + 15)
    float o[NT][kMt][4];

    __device__ __forceinline__ void mma_s(float (&s)[NT][4], int kt, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) const {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mma16816(s[nt], a0, a1, a2, a3, q[nt][kt][0], q[nt][kt][1]);
            if constexpr (kF32) mma16816(s[nt], a0, a1, a2, a3, ql[nt][kt][0], ql[nt][kt][1]);
        }
    }
    // The factor between p and the weights of V of scale 1.  m' <= m + 128 and m' >= m - 111 (kMinExp): the exponent is in range (the bounds are for maxima
    // of 2^24 and more, where m + exponent of sv is rounded).
    __device__ __forceinline__ void factor(int nt, int k) { g[nt][k] = pow2i((int)fminf(fmaxf(m[nt][k] - mp[nt][k] + 15.f, -126.f), 126.f)); }
    // Scores of a unit (as products) to weights; tok: the token of row g (masks only if `edge`).
    // low: products of q8 + 128 in the last bits.
    template <bool LOW>
    __device__ __forceinline__ void weights(float (&s)[NT][4], float ks, float vs, int tok, bool edge, uint32_t (&w)[NT][2], uint32_t (&wl)[NT][2]) {
        const float ev = fmaxf((float)(exponent_of(vs) + 1), kMinExp);
        ks = fmaf(vs, 0.f, ks);      // (a V scale that is NaN makes the scores so)
        const float vf = fminf(vs, 0x1.fffffep127f);       // (finite: what is not seen is 0 x vf)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float f0 = f[nt][0] * ks, f1 = f[nt][1] * ks;
            float (&x)[4] = s[nt];
            if constexpr (LOW) {
                const float g0 = f0 * 0x1p24f, g1 = f1 * 0x1p24f, o0 = -f0 * shift[nt][0], o1 = -f1 * shift[nt][1];
                x[0] = fmaf(x[0], g0, o0); x[1] = fmaf(x[1], g1, o1); x[2] = fmaf(x[2], g0, o0); x[3] = fmaf(x[3], g1, o1);
            } else {
                x[0] *= f0; x[1] *= f1; x[2] *= f0; x[3] *= f1;
            }
            if (edge) {              // (p and w are 0: the factors are finite)
                x[0] = tok > last[nt][0] ? -INFINITY : x[0];
                x[1] = tok > last[nt][1] ? -INFINITY : x[1];
                x[2] = tok + 8 > last[nt][0] ? -INFINITY : x[2];
                x[3] = tok + 8 > last[nt][1] ? -INFINITY : x[3];
            }
            const float b0 = fmaxf(x[0], x[2]), b1 = fmaxf(x[1], x[3]);
            const bool up = b0 > m[nt][0] || b1 > m[nt][1] || b0 + ev > mp[nt][0] || b1 + ev > mp[nt][1];
            if (__any_sync(0xffffffffu, up)) {
                float c0 = b0, c1 = b1;
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    c0 = fmaxf(c0, __shfl_xor_sync(0xffffffffu, c0, d));
                    c1 = fmaxf(c1, __shfl_xor_sync(0xffffffffu, c1, d));
                }
                c0 = ceilf(c0); c1 = ceilf(c1);
                const float m0 = fmaxf(m[nt][0], c0), m1 = fmaxf(m[nt][1], c1);
                const float p0 = fmaxf(mp[nt][0], c0 + ev), p1 = fmaxf(mp[nt][1], c1 + ev);
                l[nt][0] *= pow2_down(m[nt][0], m0);
                l[nt][1] *= pow2_down(m[nt][1], m1);
                const float r0 = pow2_down(mp[nt][0], p0), r1 = pow2_down(mp[nt][1], p1);
#pragma unroll
                for (int i = 0; i < kMt; ++i) { o[nt][i][0] *= r0; o[nt][i][1] *= r1; o[nt][i][2] *= r0; o[nt][i][3] *= r1; }
                m[nt][0] = m0; m[nt][1] = m1; mp[nt][0] = p0; mp[nt][1] = p1;
                factor(nt, 0);
                factor(nt, 1);
            }
            const float p0 = ex2(x[0] - m[nt][0]), p1 = ex2(x[1] - m[nt][1]), p2 = ex2(x[2] - m[nt][0]), p3 = ex2(x[3] - m[nt][1]);
            l[nt][0] += p0 + p2;
            l[nt][1] += p1 + p3;
            // w = p g sv, in this order: sv may be as many powers of two above the others as p is below one, and g sv beyond the range
            float w0, w1, w2, w3;
            if constexpr (kF32) {
                w0 = p0 * g[nt][0] * vf; w1 = p1 * g[nt][1] * vf; w2 = p2 * g[nt][0] * vf; w3 = p3 * g[nt][1] * vf;
            } else {                 // (packed 2 % faster with many pairs; of fp32, 10 % slower)
                const Q8Two<float> g2 = Q8Two<float>::of(g[nt][0], g[nt][1]), v2 = Q8Two<float>::of(vf, vf);
                Q8Two<float>::of(p0, p1).times(g2).times(v2).get(w0, w1);
                Q8Two<float>::of(p2, p3).times(g2).times(v2).get(w2, w3);
            }
            const uint32_t u0 = half2_of(w0, w1), u1 = half2_of(w2, w3);
            w[nt][0] = movmatrix_t(u0);
            w[nt][1] = movmatrix_t(u1);
            if constexpr (kF32) {
                wl[nt][0] = movmatrix_t(half2_rest(w0, w1, u0));
                wl[nt][1] = movmatrix_t(half2_rest(w2, w3, u1));
            }
        }
    }
    // Adds what the lane's places p, p + 32, ... hold of the runs before (if `more`); PUT: leaves the sums there and starts anew.
    template <bool PUT>
    __device__ __forceinline__ void join_runs(float* p, bool more) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float r[2];
#pragma unroll
            for (int k = 0; k < 2; ++k, p += 96) {
                r[k] = more ? pow2_down(p[32], mp[nt][k]) : 0.f;
                if (more) l[nt][k] = fmaf(p[64], pow2_down(p[0], m[nt][k]), l[nt][k]);
                if constexpr (PUT) { p[0] = m[nt][k]; p[32] = mp[nt][k]; p[64] = l[nt][k]; l[nt][k] = 0.f; }
            }
#pragma unroll
            for (int i = 0; i < kMt; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k, p += 32) {
                    float& x = o[nt][i][k];
                    if (more) x = fmaf(p[0], r[k & 1], x);
                    if constexpr (PUT) { p[0] = x; x = 0.f; }
                }
        }
    }
    __device__ __forceinline__ void mma_o(int mt, const uint32_t (&w)[NT][2], const uint32_t (&wl)[NT][2], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if constexpr (kF32) {    // (the MMA's own sums are cut off, not rounded: over many units that would add up)
                float c[4] = {0.f, 0.f, 0.f, 0.f};
                mma16816(c, a0, a1, a2, a3, wl[nt][0], wl[nt][1]);
                mma16816(c, a0, a1, a2, a3, w[nt][0], w[nt][1]);
#pragma unroll
                for (int k = 0; k < 4; ++k) o[nt][mt][k] += c[k];
            } else {
                mma16816(o[nt][mt], a0, a1, a2, a3, w[nt][0], w[nt][1]);
            }
        }
    }
};

template <typename T, int FMT, int D, int NT>
__device__ __forceinline__ void unit_of_page(Columns<T, D, NT>& C, uint32_t stage, int tok, bool edge, int lane) {
    const int g = lane >> 2, t = lane & 3;
    constexpr bool kLow = FMT == FA_Q8_INT8 && sizeof(T) == 2;
    auto half_k = [](uint32_t w, int hi) { return kLow ? __byte_perm(w, 0u, hi ? 0x4342 : 0x4140) : q8_halves<FMT>(w, hi); };
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
        const uint4 x4 = lds16(stage + unit_offset<D>(g, k_dim<D>(c, t) >> 4)), y4 = lds16(stage + unit_offset<D>(g + 8, k_dim<D>(c, t) >> 4));
        const uint32_t xw[4] = {x4.x, x4.y, x4.z, x4.w}, yw[4] = {y4.x, y4.y, y4.z, y4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = q8_flip<FMT>(xw[j]), y = q8_flip<FMT>(yw[j]);
            C.mma_s(s, 4 * c + j, half_k(x, 0), half_k(y, 0), half_k(x, 1), half_k(y, 1));
        }
    }
    uint32_t w[NT][2], wl[NT][2];
    C.template weights<kLow>(s, lds4(stage + 32 * D), lds4(stage + 32 * D + 4), tok, edge, w, wl);
    const uint32_t vst = stage + 16 * D;
#pragma unroll
    for (int c = 0; c < (D == 64 ? 1 : D / 128); ++c) {
        constexpr int kW = D == 64 ? 2 : 4;
        uint32_t v[4][kW];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 2 * t + (r & 1) + (r >> 1) * 8;
            if constexpr (D == 64) {
                const uint2 x = lds8(vst + unit_offset<D>(row, g >> 1) + 8 * (g & 1));
                v[r][0] = x.x; v[r][1] = x.y;
            } else {
                const uint4 x = lds16(vst + unit_offset<D>(row, 8 * c + g));
                v[r][0] = x.x; v[r][1] = x.y; v[r][2] = x.z; v[r][3] = x.w;
            }
        }
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            const uint32_t p = q8_flip<FMT>(v[0][i]), q = q8_flip<FMT>(v[1][i]), r = q8_flip<FMT>(v[2][i]), u = q8_flip<FMT>(v[3][i]);
            const uint32_t ab0 = __byte_perm(p, q, 0x5140), ab1 = __byte_perm(p, q, 0x7362), cd0 = __byte_perm(r, u, 0x5140), cd1 = __byte_perm(r, u, 0x7362);
            const int mt = 2 * kW * c + 2 * i;
            C.mma_o(mt, w, wl, q8_halves<FMT>(ab0, 0), q8_halves<FMT>(ab0, 1), q8_halves<FMT>(cd0, 0), q8_halves<FMT>(cd0, 1));
            C.mma_o(mt + 1, w, wl, q8_halves<FMT>(ab1, 0), q8_halves<FMT>(ab1, 1), q8_halves<FMT>(cd1, 0), q8_halves<FMT>(cd1, 1));
        }
    }
}

// Two neighbouring elements of 16 as halves, scaled by f; `rest`: what that left of fp32 elements.
template <typename T>
__device__ __forceinline__ uint32_t pair_of(const Vec16<T>& v, int i, float f, bool rest) {
    const float a = v.at(i) * f, b = v.at(i + 1) * f;
    const uint32_t h = half2_of(a, b);
    return rest ? half2_rest(a, b, h) : h;
}
template <typename T>
__device__ __forceinline__ uint32_t pair_of2(const Vec16<T>& u, const Vec16<T>& v, int i, float f, bool rest) {
    const float a = u.at(i) * f, b = v.at(i) * f;
    const uint32_t h = half2_of(a, b);
    return rest ? half2_rest(a, b, h) : h;
}
// The tail of a KV head as a warp meets it.  `fresh`: the row that a step pushes comes from k_new / v_new (another warp may be writing it).
template <typename T>
struct Tail {
    const T *k, *v, *k_new, *v_new;
    int here, fresh;                 // tokens in the tail; the row that is pushed, -1 without one
    uint32_t kmax, vmax;
    __device__ __forceinline__ const T* row(int side, int r, int D) const { return r == fresh ? (side ? v_new : k_new) : (side ? v : k) + (size_t)r * D; }
};
template <typename T, int D>
__device__ __forceinline__ void issue_tail(uint32_t ring, const Tail<T>& tl, int sub, int lane) {
    constexpr int kChunks = D * (int)sizeof(T) / 16;      // of a row
#pragma unroll
    for (int i = 0; i < 16 * kChunks / 32; ++i) {
        const int l = i * 32 + lane, r = sub * kUnit + l / kChunks, e = (l % kChunks) * (16 / (int)sizeof(T));
        const bool there = r < tl.here;
        cp16(ring + 16 * l, tl.row(0, there ? r : 0, D) + e, there);
        cp16(ring + 16 * (l + 16 * kChunks), tl.row(1, there ? r : 0, D) + e, there);
    }
}

// Unit `sub` of the tail, which starts at token `first` of the row; from the ring, or from global memory.
template <typename T, int D, int NT>
__device__ __forceinline__ void unit_of_tail(Columns<T, D, NT>& C, const Tail<T>& tl, uint32_t ring, int sub, int first, int lane) {
    constexpr bool kF32 = sizeof(T) == 4, kRing = Ring<T, D>::kTail != 0;
    const int g = lane >> 2, t = lane & 3, row0 = sub * kUnit;
    // the power of two that brings the largest magnitude to 2^13 .. 2^14, where halves hold the values next to it in full
    const bool kbad = tl.kmax >= 0x7f800000u, vbad = tl.vmax >= 0x7f800000u;
    const int ek = max((int)(tl.kmax >> 23) - 127, kTailExp), evt = max((int)(tl.vmax >> 23) - 127, kTailExp);
    const float kf = pow2i(13 - ek), vf = pow2i(13 - evt);
    const float ks = kbad ? __uint_as_float(0x7fc00000u) : pow2i(ek - 13), vs = vbad ? __uint_as_float(0x7fc00000u) : pow2i(evt - 13);
    auto get = [&](Vec16<T>& x, int side, int r, int e) {            // 16 elements of row r of the unit; zeros behind the row's last token
        if ((side ? vbad : kbad) || row0 + r >= tl.here) { x.zero(); return; }
        if constexpr (kRing) {
            uint4 w[sizeof(T)];
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) w[i] = lds16(ring + (16 * side + r) * D * (int)sizeof(T) + e * (int)sizeof(T) + 16 * i);
            memcpy(&x, w, sizeof(x));
        } else {
            x.load(tl.row(side, row0 + r, D) + e);
        }
    };
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
        Vec16<T> x, y;
        get(x, 0, g, k_dim<D>(c, t));
        get(y, 0, g + 8, k_dim<D>(c, t));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            C.mma_s(s, 4 * c + j, pair_of(x, 4 * j, kf, false), pair_of(y, 4 * j, kf, false), pair_of(x, 4 * j + 2, kf, false), pair_of(y, 4 * j + 2, kf, false));
            if constexpr (kF32)
                C.mma_s(s, 4 * c + j, pair_of(x, 4 * j, kf, true), pair_of(y, 4 * j, kf, true), pair_of(x, 4 * j + 2, kf, true), pair_of(y, 4 * j + 2, kf, true));
        }
    }
    uint32_t w[NT][2], wl[NT][2];
    C.template weights<false>(s, ks, vs, first + row0 + g, true, w, wl);
#pragma unroll
    for (int c = 0; c < (D == 64 ? 1 : D / 128); ++c) {
        Vec16<T> v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) get(v[r], 1, 2 * t + (r & 1) + (r >> 1) * 8, D == 64 ? (g >> 1) * 16 : 128 * c + 16 * g);
#pragma unroll
        for (int i = 0; i < (D == 64 ? 4 : 8); ++i) {
            // (D = 64: a lane's 8 dims are one half of its 16)
            auto two = [&](int r, int k, bool rest) {
                if constexpr (D == 64) {
                    const uint32_t lo = pair_of2(v[r], v[r + 1], 2 * i + k, vf, rest), hi = pair_of2(v[r], v[r + 1], 8 + 2 * i + k, vf, rest);
                    return (g & 1) ? hi : lo;
                } else {
                    return pair_of2(v[r], v[r + 1], 2 * i + k, vf, rest);
                }
            };
            C.mma_o(8 * c + i, w, wl, two(0, 0, false), two(0, 1, false), two(2, 0, false), two(2, 1, false));
            if constexpr (kF32) C.mma_o(8 * c + i, w, wl, two(0, 0, true), two(0, 1, true), two(2, 0, true), two(2, 1, true));
        }
    }
}

struct RowPlan {
    int len;                         // tokens that are attended to (a step: with the pushed one)
    int first;                       // the first token of the tail unit
    int units;
    bool push;                       // a step: the push goes ahead
};
template <bool STEP>
__device__ __forceinline__ RowPlan row_plan(const AttnArgs& a, int b, bool tell) {
    const Q8Dims& s = a.s;
    RowPlan r;
    int len = a.c.state[b * kQ8State];
    const int cap = s.nb << s.lb;
    if (len < 0 || len > cap) {
        if (tell) q8_report(a.c.status, FA_ERR_CAPACITY);
        r.len = 0; r.first = 0; r.units = 0; r.push = false;
        return r;
    }
    r.push = false;
    if constexpr (STEP) {
        r.push = len < cap;
        int err = r.push ? FA_OK : FA_ERR_CAPACITY;
        if (r.push && ((len + 1) & (s.blk - 1)) == 0) {
            const int page = a.c.table[(size_t)b * s.nb + (len >> s.lb)];
            if (page < 0 || page >= s.n_pages) { r.push = false; err = FA_ERR_INDEX; }
        }
        if (err != FA_OK && tell) q8_report(a.c.status, err);
    }
    r.first = len >> s.lb << s.lb;
    r.len = len + (r.push ? 1 : 0);
    r.units = r.first / kUnit + (r.len > r.first ? 1 : 0);
    return r;
}

// The push of a step for one KV head, by the CTA that has the tail unit.  Largest magnitudes with the pushed token, by every warp for itself:
template <typename T, int D>
__device__ __forceinline__ void push_amax(const AttnArgs& a, int b, int h, int r, int lane, uint32_t& km, uint32_t& vm) {
    const size_t bh = (size_t)b * a.s.H + h;
    uint32_t m = 0;
    if ((lane & 15) < D / 16) {                            // K by lanes 0 .., V by lanes 16 ..
        Vec16<T> v;
        v.load(reinterpret_cast<const T*>(lane < 16 ? a.k_new : a.v_new) + bh * D + 16 * (lane & 15));
        m = v.amax_bits();
    }
    if (r > 0 && (lane & 15) == 0) m = max(m, __float_as_uint(a.c.tail_amax[bh * 2 + (lane >> 4)]));
    km = __reduce_max_sync(0xffffffffu, lane < 16 ? m : 0u);
    vm = __reduce_max_sync(0xffffffffu, lane < 16 ? 0u : m);
}
// ... the token's rows, by one warp (its magnitudes are written when all warps have read the old ones) ...
template <typename T, int D>
__device__ __forceinline__ void push_rows(const AttnArgs& a, int b, int h, int r, T* kt, T* vt, int lane) {
    if ((lane & 15) >= D / 16) return;
    Vec16<T> v;
    v.load(reinterpret_cast<const T*>(lane < 16 ? a.k_new : a.v_new) + ((size_t)b * a.s.H + h) * D + 16 * (lane & 15));
    v.store((lane < 16 ? kt : vt) + (size_t)r * D + 16 * (lane & 15));
}
// ... and the block's page, if the token completes it, by the whole CTA (the rows are written, all threads are past a barrier).
template <typename T, int FMT, int D>
__device__ __forceinline__ void push_page(const AttnArgs& a, size_t ph, const T* kt, const T* vt, uint32_t km, uint32_t vm) {
    const int nvec = a.s.blk * (D / 16);
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        const uint32_t m = side ? vm : km;
        const Q8Round<FMT, T> to(m);
        uint8_t* out = (side ? a.c.v_pages : a.c.k_pages) + ph * (size_t)(a.s.blk * D);
#pragma unroll 1
        for (int i = threadIdx.x; i < nvec; i += kThreads) {
            Vec16<T> v;
            v.load((side ? vt : kt) + (size_t)i * 16);
            uint4 o;
            o.x = to.pack(v.at(0), v.at(1), v.at(2), v.at(3));
            o.y = to.pack(v.at(4), v.at(5), v.at(6), v.at(7));
            o.z = to.pack(v.at(8), v.at(9), v.at(10), v.at(11));
            o.w = to.pack(v.at(12), v.at(13), v.at(14), v.at(15));
            *reinterpret_cast<uint4*>(out + (size_t)i * 16) = o;
        }
        if (threadIdx.x == 0) (side ? a.c.v_scale : a.c.k_scale)[ph] = Q8Round<FMT, T>::scale(m);
    }
}

// o 2^(m' - m - 15) / l, the power of two in two factors; a column that saw nothing is zero.
__device__ __forceinline__ float2 finish(float2 o, float m, float mp, float l) {
    const int e = (int)fminf(fmaxf(mp - m - 15.f, -250.f), 250.f), e0 = e / 2;
    const float f = pow2i(e0), f2 = pow2i(e - e0), r = l == 0.f ? 0.f : 1.f / l;
    return make_float2(o.x * r * f * f2, o.y * r * f * f2);
}

// The n <= kFlat parts at p, p + step, ... of a pair to one, in that order: sums go to out(column, dim, two sums, m, m', l).  The first
// loads are in flight while a warp for each column finds the maxima and the parts' factors.  (Code that runs once costs by its length, its
// instructions come from L2: few of them, in loops.)
template <int D, int kCols, typename Out>
__device__ __forceinline__ void join_parts(const float* p, size_t step, int n, int n_col, float* fac, float (*ml)[kWarps][kCols], const Out& out) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kFly = 20, kPitch = D + 4;
    float2 x[kFly];
#pragma unroll 1
    for (int i0 = 0; i0 < n_col * (D / 2); i0 += kThreads) {
        const int i = i0 + tid, col = min(i / (D / 2), n_col - 1), e = i % (D / 2) * 2;
        float2 o = make_float2(0.f, 0.f);
#pragma unroll 1
        for (int k0 = 0; k0 < n; k0 += kFly) {
            const float* q = p + step * k0 + col * kPitch + e;
#pragma unroll
            for (int k = 0; k < kFly; ++k) {
                if (k0 + k < n) x[k] = __ldcg(reinterpret_cast<const float2*>(q));
                else x[k] = make_float2(0.f, 0.f);
                q += step;
            }
            if (i0 == 0 && k0 == 0) {
#pragma unroll 1
                for (int c = warp; c < n_col; c += kWarps) {
                    static_assert(kFlat <= 64, "two parts to a lane");
                    const float4 none = make_float4(kNegBig, kNegBig, 0.f, 0.f);
                    const float* hd = p + step * lane + c * kPitch + D;
                    const float4 u = lane < n ? __ldcg(reinterpret_cast<const float4*>(hd)) : none;
                    const float4 v = lane + 32 < n ? __ldcg(reinterpret_cast<const float4*>(hd + 32 * step)) : none;
                    const float m = warp_max(fmaxf(u.x, v.x)), mp = warp_max(fmaxf(u.y, v.y));
                    const float l = warp_sum(fmaf(u.z, pow2_down(u.x, m), v.z * pow2_down(v.x, m)));
                    fac[c * 64 + lane] = pow2_down(u.y, mp);
                    fac[c * 64 + lane + 32] = pow2_down(v.y, mp);
                    if (lane == 0) { ml[0][0][c] = m; ml[1][0][c] = mp; ml[2][0][c] = l; }
                }
                __syncthreads();
            }
#pragma unroll
            for (int k = 0; k < kFly; ++k) {
                const float f = fac[col * 64 + min(k0 + k, 63)];
                o.x = fmaf(x[k].x, f, o.x);
                o.y = fmaf(x[k].y, f, o.y);
            }
        }
        if (i < n_col * (D / 2)) out(col, e, o, ml[0][0][col], ml[1][0][col], ml[2][0][col]);
    }
}
// One arrival of the CTA, whose writes are done, on a ticket of n; true for the last one, which sees the others' writes.
__device__ __forceinline__ bool arrive_last(unsigned* ticket, int n, int* flag) {
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        *flag = atomicInc(ticket, (unsigned)(n - 1)) == (unsigned)(n - 1) ? 1 : 0;
        __threadfence();
    }
    __syncthreads();
    return *flag != 0;
}

template <typename T, int FMT, int D, int NT, bool STEP>
__global__ void __launch_bounds__(kThreads, NT == 1 && D <= 128 && sizeof(T) == 2 ? 2 : 1) q8_attn_kernel(const AttnArgs a) {
    constexpr bool kF32 = sizeof(T) == 4;
    constexpr int kCols = 8 * NT, kMt = D / 16, kPitch = D + 4;
    using R = Ring<T, D>;
    extern __shared__ float4 smem4[];
    float* osm = reinterpret_cast<float*>(smem4);          // the rings; then [warps][columns][pitch]; then a join's factors and shares
    __shared__ float ml[3][kWarps][kCols], wf[kCols][kWarps];
    __shared__ int last_s;
    const Q8Dims& s = a.s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const unsigned per_row = (unsigned)(s.H * a.n_ct), ctas = gridDim.x;
    const uint32_t ring = smem_addr(smem4) + (uint32_t)(warp * R::kStages * R::kBytes);

    asm volatile("griddepcontrol.launch_dependents;");       // the next call's CTAs may come; this one's wait for what is in front of it
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // ---- this CTA's part, found by every warp for itself; lanes hold 32 rows at a time ----
    RowPlan mine = {0, 0, 0, false};
    auto rows_from = [&](int b0, bool tell) {              // (up to 32 rows are loaded once)
        if (s.B <= 32 && !tell) return;
        mine = RowPlan{0, 0, 0, false};
        if (b0 + lane < s.B) mine = row_plan<STEP>(a, b0 + lane, tell && blockIdx.x == 0 && warp == 0);
    };
    bool line = false;
    unsigned per = kWarps, u0 = blockIdx.x, u1 = blockIdx.x + 1;     // units of a part; this CTA's: of the line, or the number of its part
    unsigned base = 0;                                               // units (parts) in front of row b
    int b = 0;
    RowPlan row = {0, 0, 0, false};
    auto of_row = [&](int units) { return (line ? (unsigned)units : ((unsigned)units + per - 1) / per) * per_row; };
    if (s.B == 1) {                                                  // (a.share: CTAs to a pair)
        row = row_plan<STEP>(a, 0, blockIdx.x == 0 && tid == 0);
        if (a.share > 0) per = max(((unsigned)row.units + a.share - 1) / (unsigned)a.share, (unsigned)kWarps);
    }
    if (s.B > 1 || a.share == 0) {
        unsigned total = 0, pairs = 0, most = 0;
        for (int b0 = 0; b0 < s.B; b0 += 32) {
            rows_from(b0, true);
            total += __reduce_add_sync(0xffffffffu, (unsigned)mine.units * per_row);
            pairs += (unsigned)__popc(__ballot_sync(0xffffffffu, mine.units > 0)) * per_row;
            most = max(most, __reduce_max_sync(0xffffffffu, (unsigned)mine.units));
        }
        // Fewer pairs than CTAs: the smallest parts (of a unit for each warp at least) that are no more than the CTAs.
        // Each lane tries a size, 2^(1/10) apart from total / CTAs on, the last one that of the longest pair.
        line = pairs > ctas;
        per = max((total + ctas - 1) / ctas, (unsigned)kWarps);
        if (!line) {
            const unsigned size = lane == 31 ? max(most, per) : (unsigned)ceilf((float)per * exp2f(0.1f * (float)lane));
            unsigned parts = 0;
            for (int b0 = 0; b0 < s.B; b0 += 32) {
                rows_from(b0, false);
                for (int i = 0; i < min(32, s.B - b0); ++i) parts += ((unsigned)__shfl_sync(0xffffffffu, mine.units, i) + size - 1) / size * per_row;
            }
            per = __shfl_sync(0xffffffffu, size, __ffs(__ballot_sync(0xffffffffu, parts <= ctas)) - 1);
        }
        if (line) {
            u0 = min(per * blockIdx.x, total);
            u1 = min(u0 + per, total);
        }
        {
            bool found = false;
            unsigned before = 0;
            for (int b0 = 0; b0 < s.B && !found; b0 += 32) {
                rows_from(b0, false);
                const unsigned n = of_row(mine.units);
                unsigned v = n;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const unsigned w = __shfl_up_sync(0xffffffffu, v, d);
                    if (lane >= d) v += w;
                }
                const unsigned hit = __ballot_sync(0xffffffffu, before + v > u0);
                if (hit) {
                    const int src = __ffs(hit) - 1;
                    b = b0 + src;
                    base = before + __shfl_sync(0xffffffffu, v - n, src);
                    row.len = __shfl_sync(0xffffffffu, mine.len, src);
                    row.first = __shfl_sync(0xffffffffu, mine.first, src);
                    row.units = __shfl_sync(0xffffffffu, mine.units, src);
                    row.push = __shfl_sync(0xffffffffu, (int)mine.push, src);
                    found = true;
                }
                before += __shfl_sync(0xffffffffu, v, 31);
            }
            if (!found) u0 = u1;
        }
    }
    if (u0 >= u1 || (s.B == 1 && u0 >= of_row(row.units))) u0 = u1;      // nothing left for this CTA

    while (u0 < u1) {
        if (u0 >= base + of_row(row.units)) {              // (a line only)
            base += of_row(row.units);
            row = row_plan<STEP>(a, ++b, false);
            continue;
        }
        int pair, s0, s1, cta0, n_seg;
        if (line) {
            pair = (int)((u0 - base) / (unsigned)row.units);
            const unsigned pair0 = base + (unsigned)pair * (unsigned)row.units;
            s0 = (int)(u0 - pair0);
            s1 = (int)min(u1 - pair0, (unsigned)row.units);
            u0 = pair0 + s1;
            cta0 = (int)(pair0 / per);
            n_seg = (int)((pair0 + row.units - 1) / per) - cta0 + 1;
        } else {
            n_seg = (int)(((unsigned)row.units + per - 1) / per);
            pair = (int)((u0 - base) / (unsigned)n_seg);
            const int j = (int)(u0 - base) - pair * n_seg, even = (row.units + n_seg - 1) / n_seg;
            s0 = min(j * even, row.units);
            s1 = min(s0 + even, row.units);
            cta0 = (int)u0 - j;
            ++u0;
        }
        const int h = pair / a.n_ct, ct = pair % a.n_ct;
        const int paged = row.first / kUnit;
        T* kt = reinterpret_cast<T*>(a.c.k_tail) + ((size_t)b * s.H + h) * (size_t)s.blk * D;
        T* vt = reinterpret_cast<T*>(a.c.v_tail) + ((size_t)b * s.H + h) * (size_t)s.blk * D;
        const int32_t* table = a.c.table + (size_t)b * s.nb;
        const int lu = s.lb - 4;                           // units of a block
        const int seen = row.len - a.n_q + 1 + min(a.n_q - 1, (ct * kCols + kCols - 1) / s.G);   // tokens that some column of the tile sees
        const int sure = row.len - a.n_q + 1 + ct * kCols / s.G;                                 // ... that all columns see
        const int stop = min(min(s1, paged), (seen + kUnit - 1) / kUnit);

        // ---- loads: q, the tail's unit, the first unit in pages ----
        Vec16<T> qv[NT][D / 64];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int col = ct * kCols + nt * 8 + g, qi = s.G == 1 ? col : col / s.G, gq = col - qi * s.G;
            const T* qp = reinterpret_cast<const T*>(a.q) + (int64_t)b * a.sb + (int64_t)qi * a.si + (int64_t)(h * s.G + gq) * a.sg;
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                if (qi < a.n_q) qv[nt][c].load(qp + k_dim<D>(c, t));
                else qv[nt][c].zero();
            }
        }
        const float* scales = lane ? a.c.v_scale : a.c.k_scale;
        auto page_of = [&](int u) { return u < stop ? __ldg(table + (u >> lu)) : -1; };
        auto checked = [&](int u, int p) {                 // -1 for a page that is not there
            if ((unsigned)p < (unsigned)s.n_pages) return p;
            if (u < stop && lane == 0) q8_report(a.c.status, FA_ERR_INDEX);
            return -1;
        };
        auto issue = [&](int stage, int u, int page) {
            if (page >= 0) {
                const uint32_t ph = (uint32_t)page * (uint32_t)s.H + (uint32_t)h, at = (ph << lu) + (uint32_t)(u & ((1 << lu) - 1));         // (counted in units)
                issue_unit<D>(ring + (uint32_t)(stage * R::kBytes), a.c.k_pages + (size_t)at * (kUnit * D), a.c.v_pages + (size_t)at * (kUnit * D), scales + ph, lane);
            }
            cp_commit();
        };
        constexpr int kAhead = R::kStages - 1;
        int u = s0 + warp, pages[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) pages[i] = checked(u + i * kWarps, page_of(u + i * kWarps));
        Tail<T> tl = {kt, vt, nullptr, nullptr, row.len - row.first, -1, 0u, 0u};
        bool tail = s1 > paged && row.first + warp * kUnit < min(row.len, seen);       // this warp has a unit of the tail
        bool whole = false;                                                             // which a step has just completed
        if (s1 > paged) {
            const size_t bh = (size_t)b * s.H + h;
            if (STEP && row.push) {
                push_amax<T, D>(a, b, h, tl.here - 1, lane, tl.kmax, tl.vmax);
                if (warp == kWarps - 1) push_rows<T, D>(a, b, h, tl.here - 1, kt, vt, lane);
                tl.fresh = tl.here - 1;
                tl.k_new = reinterpret_cast<const T*>(a.k_new) + bh * D;
                tl.v_new = reinterpret_cast<const T*>(a.v_new) + bh * D;
                __syncthreads();
                if (tid < 2) a.c.tail_amax[bh * 2 + tid] = __uint_as_float(tid ? tl.vmax : tl.kmax);
                if (tl.here == s.blk) {
                    const size_t ph = (size_t)table[row.first >> s.lb] * s.H + h;       // (in range: row_plan)
                    push_page<T, FMT, D>(a, ph, kt, vt, tl.kmax, tl.vmax);
                    __threadfence();
                    __syncthreads();
                    whole = true;
                    if (tail) {
                        const size_t at = (ph * (size_t)s.blk + (size_t)warp * kUnit) * D;
                        issue_unit<D>(ring, a.c.k_pages + at, a.c.v_pages + at, scales + ph, lane);
                    }
                }
            } else {
                tl.kmax = __float_as_uint(a.c.tail_amax[bh * 2]);
                tl.vmax = __float_as_uint(a.c.tail_amax[bh * 2 + 1]);
            }
            if (tail && !whole && R::kTail) issue_tail<T, D>(ring, tl, warp, lane);
        }
        cp_commit();
        issue(R::kFirst, u, pages[0]);

        // ---- columns ----
        Columns<T, D, NT> C;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int qi = (ct * kCols + nt * 8 + g) / s.G;
            uint32_t mxq = 0;
#pragma unroll
            for (int c = 0; c < D / 64; ++c) mxq = max(mxq, qv[nt][c].amax_bits());
            mxq = max(mxq, __shfl_xor_sync(0xffffffffu, mxq, 1));
            mxq = max(mxq, __shfl_xor_sync(0xffffffffu, mxq, 2));
            const int e = max((int)(mxq >> 23) - 127, -100);            // (an infinity or NaN stays one in the product)
            const float f = pow2i(13 - e);
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        C.q[nt][4 * c + j][k] = pair_of(qv[nt][c], 4 * j + 2 * k, f, false);
                        if constexpr (kF32) C.ql[nt][4 * c + j][k] = pair_of(qv[nt][c], 4 * j + 2 * k, f, true);
                    }
            const float fcol = pow2i(e - 13) * (s.scale * kLog2e);
            float sum = 0.f;
            if constexpr (!kF32) {
#pragma unroll
                for (int c = 0; c < D / 64; ++c)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum += qv[nt][c].at(j) * f;
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                sum *= 128.f;
            }
            const int lastq = qi < a.n_q ? row.len - a.n_q + qi : -1;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                C.f[nt][k] = __shfl_sync(0xffffffffu, fcol, (2 * t + k) * 4);
                if constexpr (!kF32) C.shift[nt][k] = __shfl_sync(0xffffffffu, sum, (2 * t + k) * 4);
                C.last[nt][k] = __shfl_sync(0xffffffffu, lastq, (2 * t + k) * 4);
                C.m[nt][k] = C.mp[nt][k] = kNegBig;
                C.l[nt][k] = 0.f;
                C.factor(nt, k);
            }
#pragma unroll
            for (int i = 0; i < kMt; ++i) C.o[nt][i][0] = C.o[nt][i][1] = C.o[nt][i][2] = C.o[nt][i][3] = 0.f;
        }
        // ---- the tail ----
        if (tail) {
            cp_wait<1>();
            __syncwarp();
            if (STEP && whole) unit_of_page<T, FMT, D, NT>(C, ring, row.first + warp * kUnit + g, true, lane);
            else unit_of_tail<T, D, NT>(C, tl, ring, warp, row.first, lane);
            __syncwarp();
        }
        // ---- units in pages ----
#pragma unroll
        for (int i = 1; i < kAhead; ++i) issue((R::kFirst + i) % R::kStages, u + i * kWarps, pages[i]);
        int stage = R::kFirst, page1 = page_of(u + kAhead * kWarps);
        auto runs = [&] { return a.runs + ((size_t)blockIdx.x * kWarps + warp) * (run_floats(D, NT) * 32) + lane; };
        bool more = false;                                 // sums of runs are in the workspace
#pragma unroll 1
        for (int run_stop = min(stop, u + kRun * kWarps);;) {
#pragma unroll 1
            for (; u < run_stop; u += kWarps) {
                cp_wait<kAhead - 1>();
                __syncwarp();
                const int page2 = page_of(u + (kAhead + 1) * kWarps);
                page1 = checked(u + kAhead * kWarps, page1);
                issue(stage == 0 ? R::kStages - 1 : stage - 1, u + kAhead * kWarps, page1);          // (the stage read last)
                if (pages[0] >= 0) unit_of_page<T, FMT, D, NT>(C, ring + (uint32_t)(stage * R::kBytes), u * kUnit + g, u * kUnit + kUnit > sure, lane);
#pragma unroll
                for (int i = 0; i + 1 < kAhead; ++i) pages[i] = pages[i + 1];
                pages[kAhead - 1] = page1;
                page1 = page2;
                if (++stage == R::kStages) stage = 0;
                __syncwarp();
            }
            if (u >= stop) break;
            C.template join_runs<true>(runs(), more);
            more = true;
            run_stop = min(stop, u + kRun * kWarps);
        }
        if (more) C.template join_runs<false>(runs(), true);
        cp_wait<0>();
        __syncthreads();                                   // the rings give way to the sums
        // ---- join the warps ----
        const int n_col = min(kCols, a.n_q * s.G - ct * kCols);      // columns of the tile that are there
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int col = nt * 8 + 2 * t + k;
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) C.l[nt][k] += __shfl_xor_sync(0xffffffffu, C.l[nt][k], d);
                if (g == 0) { ml[0][warp][col] = C.m[nt][k]; ml[1][warp][col] = C.mp[nt][k]; ml[2][warp][col] = C.l[nt][k]; }
                if (col < n_col) {
                    float* dst = osm + ((size_t)warp * kCols + col) * kPitch;
#pragma unroll
                    for (int i = 0; i < kMt; ++i) {
                        const int d = D == 64 ? 8 * g + 2 * i : 128 * (i >> 3) + 16 * g + 2 * (i & 7);
                        *reinterpret_cast<float2*>(dst + d) = make_float2(C.o[nt][i][k], C.o[nt][i][2 + k]);
                    }
                }
            }
        __syncthreads();
        auto store = [&](int col, int e, float2 o, float m, float mp, float l) {
            const int c = ct * kCols + col, qi = c / s.G;
            T* p = reinterpret_cast<T*>(a.out) + (((size_t)b * a.n_q + qi) * s.Hq + h * s.G + c - qi * s.G) * D + e;
            const float2 r = finish(o, m, mp, l);
            if constexpr (kF32) *reinterpret_cast<float2*>(p) = r;
            else *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(r.x, r.y);
        };
        // Parts of a pair lie one behind the other from 2 x its first CTA + 1 on: in a line a CTA can be the last of one pair and the first
        // of the next (those in between have no other part), and the next pair's places then start past this one's.
        constexpr size_t kPart = (size_t)kCols * kPitch;
        float* parts = a.part + (size_t)(2 * cta0 + 1) * kPart;
        auto keep = [&](int j) {
            return [=](int col, int e, float2 o, float m, float mp, float l) {
                float* p = parts + (size_t)j * kPart + col * kPitch;
                *reinterpret_cast<float2*>(p + e) = o;
                if (e == 0) *reinterpret_cast<float4*>(p + D) = make_float4(m, mp, l, 0.f);
            };
        };
        const int mine_j = (int)blockIdx.x - cta0;                   // this part's place in the pair
        const auto keep_mine = keep(mine_j);
        if (tid < n_col * kWarps) {                                  // the warps' factors, in the places of their maxima
            const int col = tid / kWarps, w = tid % kWarps;
            float m = ml[0][w][col], mp = ml[1][w][col], l = ml[2][w][col];
            const unsigned group = 0xffu << (lane & 24);
#pragma unroll
            for (int d = 1; d < kWarps; d <<= 1) { m = fmaxf(m, __shfl_xor_sync(group, m, d)); mp = fmaxf(mp, __shfl_xor_sync(group, mp, d)); }
            l *= pow2_down(ml[0][w][col], m);
#pragma unroll
            for (int d = 1; d < kWarps; d <<= 1) l += __shfl_xor_sync(group, l, d);
            wf[col][w] = pow2_down(ml[1][w][col], mp);
            if (w == 0) { ml[0][0][col] = m; ml[1][0][col] = mp; ml[2][0][col] = l; }
        }
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < n_col * (D / 2); i += kThreads) {
            const int col = i / (D / 2), e = i % (D / 2) * 2;
            float2 o = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float2 x = *reinterpret_cast<const float2*>(osm + ((size_t)w * kCols + col) * kPitch + e);
                o.x = fmaf(x.x, wf[col][w], o.x);
                o.y = fmaf(x.y, wf[col][w], o.y);
            }
            if (n_seg == 1) store(col, e, o, ml[0][0][col], ml[1][0][col], ml[2][0][col]);
            else keep_mine(col, e, o, ml[0][0][col], ml[1][0][col], ml[2][0][col]);
        }
        // ---- join the parts; many of them by groups, each by its last part to finish, then the groups by the last of those ----
        if (n_seg > 1) {
            int size = n_seg;
            if (n_seg > kFlat) {
                size = 7;
                while (size * size < n_seg) ++size;                  // (n_seg <= 500: 23 at most)
                const int j0 = mine_j / size * size, n = min(size, n_seg - j0);
                if (n == 1 || arrive_last(a.tickets + cta0 + j0, n, &last_s)) {
                    if (n > 1) join_parts<D, kCols>(parts + j0 * kPart, kPart, n, n_col, osm, ml, keep(j0));
                    if (arrive_last(a.tickets + kQ8GroupTickets + cta0, (n_seg + size - 1) / size, &last_s))
                        join_parts<D, kCols>(parts, size * kPart, (n_seg + size - 1) / size, n_col, osm, ml, store);
                }
            } else if (arrive_last(a.tickets + cta0, n_seg, &last_s)) {
                join_parts<D, kCols>(parts, kPart, n_seg, n_col, osm, ml, store);
            }
        }
        __syncthreads();
    }
    // rows without a token: zeros
    for (int i = blockIdx.x; i < s.B; i += gridDim.x)
        if (row_plan<STEP>(a, i, false).units == 0) {
            const size_t n16 = (size_t)a.n_q * s.Hq * D * sizeof(T) / 16;
            uint4* o = reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.out) + (size_t)i * a.n_q * s.Hq * D);
            for (size_t k = tid; k < n16; k += kThreads) o[k] = make_uint4(0u, 0u, 0u, 0u);
        }
    if constexpr (STEP) {                                  // the lengths grow when every CTA is past reading them
        if (arrive_last(a.tickets + kQ8StepTicket, (int)gridDim.x, &last_s))
            for (int i = tid; i < s.B; i += kThreads)
                if (row_plan<true>(a, i, false).push) a.c.state[i * kQ8State] += 1;
    }
}

struct Q8Plan {
    int nt, n_ct, ctas;
    long long units;                 // of all pairs, at most
    size_t smem, part, runs;
};
Q8Plan plan_q8(const Q8Dims& s, int n_q, int elt) {
    Q8Plan p;
    const long long cols = (long long)n_q * s.G;
    p.nt = cols <= 8 ? 1 : 2;
    const int per = 8 * p.nt;
    p.n_ct = (int)((cols + per - 1) / per);
    p.units = (long long)s.B * s.H * p.n_ct * ((long long)s.nb * s.blk / kUnit + 1);
    const long long most = (long long)sm_count() * (p.nt == 1 && s.d <= 128 && elt == 2 ? 2 : 1);
    const long long pairs = (long long)s.B * s.H * p.n_ct, parts = (p.units + kWarps - 1) / kWarps, need = parts > pairs ? parts : pairs;
    p.ctas = (int)(need < most ? need : most);
    if (p.ctas > kQ8MaxCtas) p.ctas = kQ8MaxCtas;
    // the rings; the warps' sums; the factors of the parts that are joined
    const size_t stage = 32 * (size_t)s.d + 16, rings = kWarps * stage * (elt == 4 && s.d < 256 ? 5 : 3);
    const size_t sums = (size_t)kWarps * per * (s.d + 4) * sizeof(float), heads = 64 * (size_t)per * sizeof(float);
    p.smem = rings > sums ? rings : sums;
    if (heads > p.smem) p.smem = heads;
    p.part = (size_t)2 * p.ctas * per * (s.d + 4) * sizeof(float);
    p.runs = (long long)s.nb * s.blk > (long long)kRun * kWarps * kUnit ? (size_t)p.ctas * kWarps * run_floats(s.d, p.nt) * 32 * sizeof(float) : 0;
    return p;
}

template <typename T, int FMT, int D, int NT>
cudaError_t attn_of(const AttnArgs& a, const Q8Plan& p, cudaStream_t stream) {
    const auto kernel = a.k_new ? q8_attn_kernel<T, FMT, D, NT, true> : q8_attn_kernel<T, FMT, D, NT, false>;
    const cudaError_t e = ensure_dynamic_smem(kernel, p.smem);
    if (e != cudaSuccess) return e;
    return launch_behind(kernel, dim3((unsigned)p.ctas), kThreads, p.smem, stream, a);
}
template <typename T, int FMT>
cudaError_t attn_dims(const AttnArgs& a, const Q8Plan& p, cudaStream_t stream) {
    switch (a.s.d) {
        case 64: return p.nt == 1 ? attn_of<T, FMT, 64, 1>(a, p, stream) : attn_of<T, FMT, 64, 2>(a, p, stream);
        case 128: return p.nt == 1 ? attn_of<T, FMT, 128, 1>(a, p, stream) : attn_of<T, FMT, 128, 2>(a, p, stream);
        default: return p.nt == 1 ? attn_of<T, FMT, 256, 1>(a, p, stream) : attn_of<T, FMT, 256, 2>(a, p, stream);
    }
}

}  // namespace

size_t q8_attention_ws_bytes(const Q8Dims& s, int n_q) {
    const Q8Plan p = plan_q8(s, n_q, 2), p4 = plan_q8(s, n_q, 4);
    const size_t a = 4096 + p.part + p.runs, b = 4096 + p4.part + p4.runs, c = q8_chunk_takes(s, FA_BF16, n_q) ? q8_chunk_ws_bytes(s) : 0;
    return a > b ? (a > c ? a : c) : (b > c ? b : c);
}

bool q8_attention_fits(const Q8Dims& s, int n_q) { return plan_q8(s, n_q, 2).units <= 0x7fffffff; }

cudaError_t launch_q8_attention(const Q8Dims& s, const Q8Cache& c, int fmt, int dtype, const void* q, int64_t sb, int64_t si, int64_t sg, void* out, int n_q,
                                const void* k_new, const void* v_new, char* ws, cudaStream_t stream) {
    if (!k_new && q8_chunk_takes(s, dtype, n_q)) return launch_q8_chunk(s, c, fmt, q, sb, si, sg, out, n_q, ws, stream);
    const Q8Plan p = plan_q8(s, n_q, dtype == FA_BF16 ? 2 : 4);
    const AttnArgs a = {s, c, q, sb, si, sg, out, n_q, p.n_ct, (int)(p.ctas / ((long long)s.H * p.n_ct)), k_new, v_new, reinterpret_cast<unsigned*>(ws), reinterpret_cast<float*>(ws + 4096),
                        p.runs ? reinterpret_cast<float*>(ws + 4096 + p.part) : nullptr};
    if (dtype == FA_BF16) return fmt == FA_Q8_INT8 ? attn_dims<__nv_bfloat16, FA_Q8_INT8>(a, p, stream) : attn_dims<__nv_bfloat16, FA_Q8_E4M3>(a, p, stream);
    return fmt == FA_Q8_INT8 ? attn_dims<float, FA_Q8_INT8>(a, p, stream) : attn_dims<float, FA_Q8_E4M3>(a, p, stream);
}

}  // namespace fa
