// fa_q8_attention and fa_q8_step: softmax attention over the dense cache in 8 bits, few query columns to a KV head.
//
// A column is one (query, query head) of a KV head; a pass over the head's tokens serves 8 or 16 columns.  Scores and
// outputs are formed transposed, S^T = K Q^T and O^T = V^T P^T (mma.sync m16n8k16, halves in, fp32 sums): the 16 rows are tokens,
// then head dims, and no row is lost to padding of the few columns.  Both operands from the cache go straight from HBM to registers in
// 16-byte pieces of token rows: the contraction over head dims may take them in any order as long as q follows it, and the rows
// of O^T may be any dims, so that a lane's bytes are its own operand rows.  8-bit values are halves exactly; q is scaled by a
// power of two per column, which makes its bf16 values halves exactly (fp32 q: a high and a low half, two products).
//
// Scales: a score is multiplied by its block's K scale.  The weight of a token in O is w = p sv 2^(m - m' + 15), sv its block's
// V scale, m the column's running maximum of the scores, m' that of score + exponent of sv, both rounded up to whole numbers (of log2), so
// that rescaling is exact: w is at most 2^15 and its rounding to a half is relative to 2^-24 of the largest weight
// or better; the sum of the p runs beside it in fp32.  The tail is the same with the power of two above its largest magnitude
// in the place of the scale.
//
// Work: the (row, head, column tile) pairs have one unit for every 16 tokens in pages and one for the tail; the units of all pairs in a
// line are cut into equal parts, one for each CTA, whatever the rows' lengths.  In a part, each of 8 warps takes every
// 8th unit by itself with its loads one unit ahead; the warps join in shared memory, parts of one pair in the workspace, by the last CTA to finish, in a fixed order.
// Bound by HBM for long rows, by the chain lengths - page - values - join for short ones.
#include "fa_q8.cuh"

namespace fa {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kUnit = 16;            // tokens

struct AttnArgs {
    Q8Dims s;
    Q8Cache c;
    const void* q;
    int64_t sb, si, sg;
    void* out;
    int n_q, n_ct;                   // queries a row, column tiles of a KV head
    const void *k_new, *v_new;       // a step
    unsigned* tickets;
    float* part;                     // [2 * CTAs][cols][D + 4]
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


template <bool OWN>
__device__ __forceinline__ uint4 ld16(const uint8_t* p) {
    uint4 r;
    if constexpr (OWN)                                     // written by this CTA
        asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    else
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// The bytes of one unit (16 tokens of a page) that a lane (g, t) = (lane / 4, lane % 4) holds.
template <int D, bool OWN = false>
struct Raw {
    static constexpr int kC = D / 64, kV = D == 64 ? 2 : D / 32;      // K chunks of 64 dims; words of a V row that a lane has
    uint32_t k[kC][2][4];            // dims 64 c + 16 t .. + 15 of tokens g and g + 8
    uint32_t v[4][kV];               // tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9: dims 128 c + 16 g .. + 15 (D = 64: 8 g .. + 7)
    float ks, vs;
    __device__ __forceinline__ void load(const uint8_t* kp, const uint8_t* vp, int lane) {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const uint4 x = ld16<OWN>(kp + (g + 8 * r) * D + 64 * c + 16 * t);
                k[c][r][0] = x.x; k[c][r][1] = x.y; k[c][r][2] = x.z; k[c][r][3] = x.w;
            }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint8_t* p = vp + (2 * t + (r & 1) + (r >> 1) * 8) * D;
            if constexpr (D == 64) {
                asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(v[r][0]), "=r"(v[r][1]) : "l"(p + 8 * g) : "memory");
            } else {
#pragma unroll
                for (int c = 0; c < D / 128; ++c) {
                    const uint4 x = ld16<OWN>(p + 128 * c + 16 * g);
                    v[r][4 * c] = x.x; v[r][4 * c + 1] = x.y; v[r][4 * c + 2] = x.z; v[r][4 * c + 3] = x.w;
                }
            }
        }
    }
};

// The columns of a segment as a warp holds them.
template <typename T, int D, int NT>
struct Columns {
    static constexpr bool kF32 = sizeof(T) == 4;
    static constexpr int kMt = D / 16;
    uint32_t q[NT][kMt][2];          // column g: dims in the order of the lanes' K bytes
    uint32_t ql[kF32 ? NT : 1][kF32 ? kMt : 1][2];
    float f[NT][2];                  // columns 2 t, 2 t + 1: logits (base 2) per product
    int last[NT][2];                 // the last token they see
    float m[NT][2], mp[NT][2], l[NT][2];
    float o[NT][kMt][4];

    __device__ __forceinline__ void mma_s(float (&s)[NT][4], int kt, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) const {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mma16816(s[nt], a0, a1, a2, a3, q[nt][kt][0], q[nt][kt][1]);
            if constexpr (kF32) mma16816(s[nt], a0, a1, a2, a3, ql[nt][kt][0], ql[nt][kt][1]);
        }
    }
    // Scores of a unit (as products) to weights; tok: the token of row g; stop: tokens of the row (masks only if `edge`).
    __device__ __forceinline__ void weights(float (&s)[NT][4], float ks, float vs, int tok, bool edge, uint32_t (&w)[NT][2], uint32_t (&wl)[NT][2]) {
        const int ev = exponent_of(vs) + 1;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float f0 = f[nt][0] * ks, f1 = f[nt][1] * ks;
            float (&x)[4] = s[nt];
            x[0] *= f0; x[1] *= f1; x[2] *= f0; x[3] *= f1;
            bool h0 = false, h1 = false, h2 = false, h3 = false;
            if (edge) {
                h0 = tok > last[nt][0]; h1 = tok > last[nt][1]; h2 = tok + 8 > last[nt][0]; h3 = tok + 8 > last[nt][1];
                x[0] = h0 ? -INFINITY : x[0]; x[1] = h1 ? -INFINITY : x[1]; x[2] = h2 ? -INFINITY : x[2]; x[3] = h3 ? -INFINITY : x[3];
            }
            const float b0 = fmaxf(x[0], x[2]), b1 = fmaxf(x[1], x[3]);
            const bool up = b0 > m[nt][0] || b1 > m[nt][1] || b0 + (float)ev > mp[nt][0] || b1 + (float)ev > mp[nt][1];
            if (__any_sync(0xffffffffu, up)) {
                float c0 = b0, c1 = b1;
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    c0 = fmaxf(c0, __shfl_xor_sync(0xffffffffu, c0, d));
                    c1 = fmaxf(c1, __shfl_xor_sync(0xffffffffu, c1, d));
                }
                c0 = ceilf(c0); c1 = ceilf(c1);
                const float m0 = fmaxf(m[nt][0], c0), m1 = fmaxf(m[nt][1], c1);
                const float p0 = fmaxf(mp[nt][0], c0 + (float)ev), p1 = fmaxf(mp[nt][1], c1 + (float)ev);
                l[nt][0] *= pow2_down(m[nt][0], m0);
                l[nt][1] *= pow2_down(m[nt][1], m1);
                const float r0 = pow2_down(mp[nt][0], p0), r1 = pow2_down(mp[nt][1], p1);
#pragma unroll
                for (int i = 0; i < kMt; ++i) { o[nt][i][0] *= r0; o[nt][i][1] *= r1; o[nt][i][2] *= r0; o[nt][i][3] *= r1; }
                m[nt][0] = m0; m[nt][1] = m1; mp[nt][0] = p0; mp[nt][1] = p1;
            }
            const float p0 = ex2(x[0] - m[nt][0]), p1 = ex2(x[1] - m[nt][1]), p2 = ex2(x[2] - m[nt][0]), p3 = ex2(x[3] - m[nt][1]);
            l[nt][0] += p0 + p2;
            l[nt][1] += p1 + p3;
            // m' <= m + 128 and m' >= m - 126: only the upper end can leave the range, for a V scale below 2^-111, where the weights then use less of it
            const float most = (float)min(126, 126 - ev);
            const float c0 = vs * pow2i((int)fminf(fmaxf(m[nt][0] - mp[nt][0] + 15.f, -126.f), most));
            const float c1 = vs * pow2i((int)fminf(fmaxf(m[nt][1] - mp[nt][1] + 15.f, -126.f), most));
            const float w0 = h0 ? 0.f : p0 * c0, w1 = h1 ? 0.f : p1 * c1, w2 = h2 ? 0.f : p2 * c0, w3 = h3 ? 0.f : p3 * c1;
            const uint32_t u0 = half2_of(w0, w1), u1 = half2_of(w2, w3);
            w[nt][0] = movmatrix_t(u0);
            w[nt][1] = movmatrix_t(u1);
            if constexpr (kF32) {
                wl[nt][0] = movmatrix_t(half2_rest(w0, w1, u0));
                wl[nt][1] = movmatrix_t(half2_rest(w2, w3, u1));
            }
        }
    }
    __device__ __forceinline__ void mma_o(int mt, const uint32_t (&w)[NT][2], const uint32_t (&wl)[NT][2], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mma16816(o[nt][mt], a0, a1, a2, a3, w[nt][0], w[nt][1]);
            if constexpr (kF32) mma16816(o[nt][mt], a0, a1, a2, a3, wl[nt][0], wl[nt][1]);
        }
    }
};

template <typename T, int FMT, int D, int NT, bool OWN>
__device__ __forceinline__ void unit_of_page(Columns<T, D, NT>& C, const Raw<D, OWN>& r, int tok, bool edge) {
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = q8_flip<FMT>(r.k[c][0][j]), y = q8_flip<FMT>(r.k[c][1][j]);
            C.mma_s(s, 4 * c + j, q8_halves<FMT>(x, 0), q8_halves<FMT>(y, 0), q8_halves<FMT>(x, 1), q8_halves<FMT>(y, 1));
        }
    uint32_t w[NT][2], wl[NT][2];
    C.weights(s, r.ks, r.vs, tok, edge, w, wl);
#pragma unroll
    for (int i = 0; i < Raw<D>::kV; ++i) {
        const uint32_t a = q8_flip<FMT>(r.v[0][i]), b = q8_flip<FMT>(r.v[1][i]), c = q8_flip<FMT>(r.v[2][i]), d = q8_flip<FMT>(r.v[3][i]);
        const uint32_t ab0 = __byte_perm(a, b, 0x5140), ab1 = __byte_perm(a, b, 0x7362), cd0 = __byte_perm(c, d, 0x5140), cd1 = __byte_perm(c, d, 0x7362);
        C.mma_o(2 * i, w, wl, q8_halves<FMT>(ab0, 0), q8_halves<FMT>(ab0, 1), q8_halves<FMT>(cd0, 0), q8_halves<FMT>(cd0, 1));
        C.mma_o(2 * i + 1, w, wl, q8_halves<FMT>(ab1, 0), q8_halves<FMT>(ab1, 1), q8_halves<FMT>(cd1, 0), q8_halves<FMT>(cd1, 1));
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
// Sixteen elements of the tail that this kernel may have written; nothing behind the row's last token is read.
template <typename T>
__device__ __forceinline__ void load_own16(Vec16<T>& v, const T* p, bool there) {
    if (!there) { v.zero(); return; }
    uint4 x[sizeof(T)];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) x[i] = ld16<true>(reinterpret_cast<const uint8_t*>(p) + 16 * i);
    memcpy(&v, x, sizeof(v));
}

// Unit `sub` of the tail: `here` tokens of the row are in the tail, which starts at token `first`.
template <typename T, int D, int NT>
__device__ __forceinline__ void unit_of_tail(Columns<T, D, NT>& C, const T* kt, const T* vt, uint32_t kmax, uint32_t vmax, int sub, int here, int first,
                                             int lane) {
    constexpr bool kF32 = sizeof(T) == 4;
    const int g = lane >> 2, t = lane & 3, row0 = sub * kUnit;
    // the power of two that brings the largest magnitude to 2^13 .. 2^14, where halves hold the values next to it in full
    const bool kbad = kmax >= 0x7f800000u, vbad = vmax >= 0x7f800000u;
    const int ek = max((int)(kmax >> 23) - 127, -100), evt = max((int)(vmax >> 23) - 127, -100);
    const float kf = kbad ? 0.f : pow2i(13 - ek), vf = vbad ? 0.f : pow2i(13 - evt);
    const float ks = kbad ? __uint_as_float(0x7fc00000u) : pow2i(ek - 13), vs = vbad ? __uint_as_float(0x7fc00000u) : pow2i(evt - 13);
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
        Vec16<T> x, y;
        load_own16(x, kt + (size_t)(row0 + g) * D + 64 * c + 16 * t, row0 + g < here && !kbad);
        load_own16(y, kt + (size_t)(row0 + g + 8) * D + 64 * c + 16 * t, row0 + g + 8 < here && !kbad);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            C.mma_s(s, 4 * c + j, pair_of(x, 4 * j, kf, false), pair_of(y, 4 * j, kf, false), pair_of(x, 4 * j + 2, kf, false), pair_of(y, 4 * j + 2, kf, false));
            if constexpr (kF32)
                C.mma_s(s, 4 * c + j, pair_of(x, 4 * j, kf, true), pair_of(y, 4 * j, kf, true), pair_of(x, 4 * j + 2, kf, true), pair_of(y, 4 * j + 2, kf, true));
        }
    }
    uint32_t w[NT][2], wl[NT][2];
    C.weights(s, ks, vs, first + row0 + g, true, w, wl);
#pragma unroll
    for (int c = 0; c < (D == 64 ? 1 : D / 128); ++c) {
        Vec16<T> v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = row0 + 2 * t + (r & 1) + (r >> 1) * 8;
            const int e = D == 64 ? (g >> 1) * 16 : 128 * c + 16 * g;
            load_own16(v[r], vt + (size_t)row * D + e, row < here && !vbad);
        }
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

// The push of a step for one KV head, by the CTA that has the tail unit: the token into the tail; if that completes the
// block, its page.  mx: largest magnitudes of the tail's K and V (as bits) for all threads.
template <typename T, int FMT, int D>
__device__ __forceinline__ void push_token(const AttnArgs& a, int b, int h, int len, T* kt, T* vt, uint32_t* mx) {
    const Q8Dims& s = a.s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = len & (s.blk - 1);
    float* amax = a.c.tail_amax + ((size_t)b * s.H + h) * 2;
    if (warp < 2) {                                        // K by warp 0, V by warp 1
        const T* src = reinterpret_cast<const T*>(warp ? a.v_new : a.k_new) + ((size_t)b * s.H + h) * D;
        T* dst = (warp ? vt : kt) + (size_t)r * D;
        uint32_t m = 0;
        if (lane < D / 16) {
            Vec16<T> v;
            v.load(src + 16 * lane);
            v.store(dst + 16 * lane);
            m = v.amax_bits();
        }
        m = __reduce_max_sync(0xffffffffu, m);
        if (lane == 0) {
            if (r > 0) m = max(m, __float_as_uint(amax[warp]));
            amax[warp] = __uint_as_float(m);
            mx[warp] = m;
        }
    }
    __syncthreads();
    if (r + 1 < s.blk) return;
    const int page = a.c.table[(size_t)b * s.nb + (len >> s.lb)];      // (in range: row_plan)
    const size_t ph = (size_t)page * s.H + h;
    const int nvec = s.blk * (D / 16);
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        const Q8Round<FMT, T> to(mx[side]);
        uint8_t* out = (side ? a.c.v_pages : a.c.k_pages) + ph * (size_t)(s.blk * D);
        for (int i = tid; i < nvec; i += kThreads) {
            Vec16<T> v;
            load_own16(v, (side ? vt : kt) + (size_t)i * 16, true);
            uint4 o;
            o.x = to.pack(v.at(0), v.at(1), v.at(2), v.at(3));
            o.y = to.pack(v.at(4), v.at(5), v.at(6), v.at(7));
            o.z = to.pack(v.at(8), v.at(9), v.at(10), v.at(11));
            o.w = to.pack(v.at(12), v.at(13), v.at(14), v.at(15));
            *reinterpret_cast<uint4*>(out + (size_t)i * 16) = o;
        }
        if (tid == 0) (side ? a.c.v_scale : a.c.k_scale)[ph] = Q8Round<FMT, T>::scale(mx[side]);
    }
    __syncthreads();
}

template <typename T>
__device__ __forceinline__ void st4(T* p, float4 v) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = v;
    } else {
        const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
        uint2 u;
        u.x = *reinterpret_cast<const uint32_t*>(&a);
        u.y = *reinterpret_cast<const uint32_t*>(&b);
        *reinterpret_cast<uint2*>(p) = u;
    }
}
// o 2^(m' - m - 15) / l, the power of two in two factors; a column that saw nothing is zero.
__device__ __forceinline__ float4 finish(float4 o, float m, float mp, float l) {
    const int e = (int)fminf(fmaxf(mp - m - 15.f, -250.f), 250.f), e0 = e / 2;
    const float f = pow2i(e0), f2 = pow2i(e - e0), r = l == 0.f ? 0.f : 1.f / l;
    return make_float4(o.x * r * f * f2, o.y * r * f * f2, o.z * r * f * f2, o.w * r * f * f2);
}

template <typename T, int FMT, int D, int NT, bool STEP>
__global__ void __launch_bounds__(kThreads, NT == 1 && D <= 128 && sizeof(T) == 2 ? 2 : 1) q8_attn_kernel(const AttnArgs a) {
    constexpr bool kF32 = sizeof(T) == 4;
    constexpr int kCols = 8 * NT, kMt = D / 16, kPitch = D + 4;
    extern __shared__ float4 smem4[];
    float* osm = reinterpret_cast<float*>(smem4);          // [warps][columns][pitch]
    __shared__ float ml[3][kWarps][kCols];
    __shared__ long long plan_s[3];                        // units of all pairs; the first row of this CTA's part, its units before
    __shared__ uint32_t mx[2];
    __shared__ int last_s;
    const Q8Dims& s = a.s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int per_row = s.H * a.n_ct;

    // ---- the part of the line of units that is this CTA's ----
    if (warp == 0) {
        long long total = 0;
        for (int b0 = 0; b0 < s.B; b0 += 32) {
            int u = b0 + lane < s.B ? row_plan<STEP>(a, b0 + lane, blockIdx.x == 0).units : 0;
            long long v = (long long)u * per_row;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
            total += v;
        }
        if (lane == 0) plan_s[0] = total;
    }
    __syncthreads();
    const long long total = plan_s[0];
    long long per = (total + gridDim.x - 1) / gridDim.x;
    if (per < kWarps) per = kWarps;                        // a unit for each warp at least
    long long u0 = per * blockIdx.x;
    const long long u1 = u0 + per < total ? u0 + per : total;
    if (warp == 0) {
        long long before = 0;
        for (int b0 = 0; b0 < s.B; b0 += 32) {
            int u = b0 + lane < s.B ? row_plan<STEP>(a, b0 + lane, false).units : 0;
            const long long mine = (long long)u * per_row;
            long long v = mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long w = __shfl_up_sync(0xffffffffu, v, d);
                if (lane >= d) v += w;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, before + v > u0);
            if (hit) {
                const int src = __ffs(hit) - 1;
                const long long row_before = before + __shfl_sync(0xffffffffu, v - mine, src);
                if (lane == 0) { plan_s[1] = b0 + src; plan_s[2] = row_before; }
                break;
            }
            before += __shfl_sync(0xffffffffu, v, 31);
        }
    }
    // rows without a token: zeros
    for (int b = blockIdx.x; b < s.B; b += gridDim.x)
        if (row_plan<STEP>(a, b, false).units == 0) {
            const int n4 = a.n_q * s.Hq * D / 4;
            T* o = reinterpret_cast<T*>(a.out) + (size_t)b * a.n_q * s.Hq * D;
            for (int i = tid; i < n4; i += kThreads) st4(o + (size_t)i * 4, make_float4(0.f, 0.f, 0.f, 0.f));
        }
    __syncthreads();
    int b = (int)plan_s[1];
    long long base = plan_s[2];
    while (u0 < u1) {
        RowPlan row = row_plan<STEP>(a, b, false);
        const long long row_units = (long long)row.units * per_row;
        if (u0 >= base + row_units) { base += row_units; ++b; continue; }
        const int pair = (int)((u0 - base) / row.units);
        const int h = pair / a.n_ct, ct = pair % a.n_ct;
        const long long pair0 = base + (long long)pair * row.units;
        const int s0 = (int)(u0 - pair0), s1 = (int)(u1 - pair0 < row.units ? u1 - pair0 : row.units);
        u0 = pair0 + s1;
        const int paged = row.first / kUnit;
        T* kt = reinterpret_cast<T*>(a.c.k_tail) + ((size_t)b * s.H + h) * (size_t)s.blk * D;
        T* vt = reinterpret_cast<T*>(a.c.v_tail) + ((size_t)b * s.H + h) * (size_t)s.blk * D;

        // ---- columns ----
        Columns<T, D, NT> C;
        int seen = 0;                                      // tokens that some column of the tile sees
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int col = ct * kCols + nt * 8 + g, qi = col / s.G, gq = col % s.G;
            const bool there = qi < a.n_q;
            const T* qp = reinterpret_cast<const T*>(a.q) + (int64_t)b * a.sb + (int64_t)qi * a.si + (int64_t)(h * s.G + gq) * a.sg;
            Vec16<T> v[D / 64];
            uint32_t mxq = 0;
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                if (there) v[c].load(qp + 64 * c + 16 * t);
                else v[c].zero();
                mxq = max(mxq, v[c].amax_bits());
            }
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
                        C.q[nt][4 * c + j][k] = pair_of(v[c], 4 * j + 2 * k, f, false);
                        if constexpr (kF32) C.ql[nt][4 * c + j][k] = pair_of(v[c], 4 * j + 2 * k, f, true);
                    }
            const float fcol = pow2i(e - 13) * (s.scale * kLog2e);
            const int lastq = there ? row.len - a.n_q + qi : -1;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                C.f[nt][k] = __shfl_sync(0xffffffffu, fcol, (2 * t + k) * 4);
                C.last[nt][k] = __shfl_sync(0xffffffffu, lastq, (2 * t + k) * 4);
                C.m[nt][k] = C.mp[nt][k] = kNegBig;
                C.l[nt][k] = 0.f;
            }
            seen = max(seen, __reduce_max_sync(0xffffffffu, lastq) + 1);
#pragma unroll
            for (int i = 0; i < kMt; ++i) C.o[nt][i][0] = C.o[nt][i][1] = C.o[nt][i][2] = C.o[nt][i][3] = 0.f;
        }
        int sure = row.len - a.n_q + 1 + ct * kCols / s.G;  // tokens that all columns of the tile see
        // ---- units in pages ----
        {
            const int32_t* table = a.c.table + (size_t)b * s.nb;
            const int stop = min(min(s1, paged), (seen + kUnit - 1) / kUnit);
            const int lu = s.lb - 4;                        // units of a block
            auto page_of = [&](int u) {
                if (u >= stop) return -1;
                const int p = table[u >> lu];
                if (p >= 0 && p < s.n_pages) return p;
                if (lane == 0) q8_report(a.c.status, FA_ERR_INDEX);
                return -1;
            };
            auto fetch = [&](Raw<D>& r, int u, int page) {
                if (page < 0) return;
                const size_t ph = (size_t)page * s.H + h;
                const size_t at = (ph * (size_t)s.blk + (size_t)(u & ((1 << lu) - 1)) * kUnit) * D;
                r.load(a.c.k_pages + at, a.c.v_pages + at, lane);
                r.ks = __ldg(a.c.k_scale + ph);
                r.vs = __ldg(a.c.v_scale + ph);
            };
            int u = s0 + warp;
            int page = page_of(u), page1 = page_of(u + kWarps);
            Raw<D> cur, nxt;
            fetch(cur, u, page);
            for (; u < stop; u += kWarps) {
                const int page2 = page_of(u + 2 * kWarps);
                fetch(nxt, u + kWarps, page1);
                if (page >= 0) unit_of_page<T, FMT, D, NT, false>(C, cur, u * kUnit + g, u * kUnit + kUnit > sure);
                cur = nxt;
                page = page1;
                page1 = page2;
            }
        }
        // ---- the tail ----
        if (s1 > paged) {
            const int here = row.len - row.first;
            uint32_t km, vm;
            if constexpr (STEP) {
                if (row.push) push_token<T, FMT, D>(a, b, h, row.len - 1, kt, vt, mx);
            }
            if (STEP && row.push) {
                km = mx[0];
                vm = mx[1];
            } else {
                const float* am = a.c.tail_amax + ((size_t)b * s.H + h) * 2;
                km = __float_as_uint(am[0]);
                vm = __float_as_uint(am[1]);
            }
            if (warp * kUnit < here && row.first + warp * kUnit < seen) {
                if (STEP && here == s.blk) {               // complete with this token
                    const int page = a.c.table[(size_t)b * s.nb + (row.first >> s.lb)];
                    const size_t ph = (size_t)page * s.H + h, at = (ph * (size_t)s.blk + (size_t)warp * kUnit) * D;
                    Raw<D, true> r;
                    r.load(a.c.k_pages + at, a.c.v_pages + at, lane);
                    r.ks = Q8Round<FMT, T>::scale(km);
                    r.vs = Q8Round<FMT, T>::scale(vm);
                    unit_of_page<T, FMT, D, NT, true>(C, r, row.first + warp * kUnit + g, true);
                } else {
                    unit_of_tail<T, D, NT>(C, kt, vt, km, vm, warp, here, row.first, lane);
                }
            }
        }
        // ---- join the warps ----
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) C.l[nt][k] += __shfl_xor_sync(0xffffffffu, C.l[nt][k], d);
                if (g == 0) {
                    ml[0][warp][nt * 8 + 2 * t + k] = C.m[nt][k];
                    ml[1][warp][nt * 8 + 2 * t + k] = C.mp[nt][k];
                    ml[2][warp][nt * 8 + 2 * t + k] = C.l[nt][k];
                }
            }
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int col = nt * 8 + 2 * t + k;
                float mp = kNegBig;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) mp = fmaxf(mp, ml[1][w][col]);
                const float f = pow2_down(C.mp[nt][k], mp);
                float* dst = osm + ((size_t)warp * kCols + col) * kPitch;
#pragma unroll
                for (int i = 0; i < kMt; ++i) {
                    const int d = D == 64 ? 8 * g + 2 * i : 128 * (i >> 3) + 16 * g + 2 * (i & 7);
                    *reinterpret_cast<float2*>(dst + d) = make_float2(C.o[nt][i][k] * f, C.o[nt][i][2 + k] * f);
                }
            }
        __syncthreads();
        const bool lone = s0 == 0 && s1 == row.units;
        const int cta0 = (int)(pair0 / per), n_seg = (int)((pair0 + row.units - 1) / per) - cta0 + 1;
        float* mine = a.part + ((size_t)2 * blockIdx.x + (s0 == 0 ? 1 : 0)) * kCols * kPitch;
        auto store = [&](int col, int e, float4 o, float m, float mp, float l) {
            const int c = ct * kCols + col, qi = c / s.G;
            if (qi >= a.n_q) return;
            st4(reinterpret_cast<T*>(a.out) + (((size_t)b * a.n_q + qi) * s.Hq + h * s.G + c % s.G) * D + e, finish(o, m, mp, l));
        };
        for (int i = tid; i < kCols * (D / 4); i += kThreads) {
            const int col = i / (D / 4), e = (i % (D / 4)) * 4;
            float m = kNegBig, mp = kNegBig, l = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) { m = fmaxf(m, ml[0][w][col]); mp = fmaxf(mp, ml[1][w][col]); }
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                l += ml[2][w][col] * pow2_down(ml[0][w][col], m);
                const float4 x = *reinterpret_cast<const float4*>(osm + ((size_t)w * kCols + col) * kPitch + e);
                o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
            }
            if (lone) {
                store(col, e, o, m, mp, l);
            } else {
                *reinterpret_cast<float4*>(mine + col * kPitch + e) = o;
                if (e == 0) *reinterpret_cast<float4*>(mine + col * kPitch + D) = make_float4(m, mp, l, 0.f);
            }
        }
        if (!lone) {
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                last_s = atomicInc(a.tickets + cta0, n_seg - 1) == (unsigned)(n_seg - 1) ? 1 : 0;
                __threadfence();
            }
            __syncthreads();
            if (last_s) {
                for (int i = tid; i < kCols * (D / 4); i += kThreads) {
                    const int col = i / (D / 4), e = (i % (D / 4)) * 4;
                    float m = kNegBig, mp = kNegBig, l = 0.f;
                    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int j = 0; j < n_seg; ++j) {      // in the order of the tokens
                        const float* p = a.part + ((size_t)2 * (cta0 + j) + (j == 0 ? 1 : 0)) * kCols * kPitch + col * kPitch;
                        const float4 hd = __ldcg(reinterpret_cast<const float4*>(p + D));
                        const float4 x = __ldcg(reinterpret_cast<const float4*>(p + e));
                        const float mn = fmaxf(m, hd.x), pn = fmaxf(mp, hd.y);
                        l = l * pow2_down(m, mn) + hd.z * pow2_down(hd.x, mn);
                        const float f0 = pow2_down(mp, pn), f1 = pow2_down(hd.y, pn);
                        o.x = o.x * f0 + x.x * f1; o.y = o.y * f0 + x.y * f1; o.z = o.z * f0 + x.z * f1; o.w = o.w * f0 + x.w * f1;
                        m = mn;
                        mp = pn;
                    }
                    store(col, e, o, m, mp, l);
                }
            }
        }
        __syncthreads();
    }
    if constexpr (STEP) {                                  // the lengths grow when every CTA is past reading them
        if (tid == 0) {
            last_s = atomicInc(a.tickets + kQ8StepTicket, gridDim.x - 1) == gridDim.x - 1 ? 1 : 0;
            __threadfence();
        }
        __syncthreads();
        if (last_s)
            for (int i = tid; i < s.B; i += kThreads)
                if (row_plan<true>(a, i, false).push) a.c.state[i * kQ8State] += 1;
    }
}

struct Q8Plan {
    int nt, n_ct, ctas;
    size_t smem, part;
};
Q8Plan plan_q8(const Q8Dims& s, int n_q, int elt) {
    Q8Plan p;
    const long long cols = (long long)n_q * s.G;
    p.nt = cols <= 8 ? 1 : 2;
    const int per = 8 * p.nt;
    p.n_ct = (int)((cols + per - 1) / per);
    const long long units = (long long)s.B * s.H * p.n_ct * ((long long)s.nb * s.blk / kUnit + 1);
    const long long most = (long long)sm_count() * (p.nt == 1 && s.d <= 128 && elt == 2 ? 2 : 1), need = (units + kWarps - 1) / kWarps;
    p.ctas = (int)(need < most ? need : most);
    if (p.ctas > kQ8MaxCtas) p.ctas = kQ8MaxCtas;
    p.smem = (size_t)kWarps * per * (s.d + 4) * sizeof(float);
    p.part = (size_t)2 * p.ctas * per * (s.d + 4) * sizeof(float);
    return p;
}

template <typename T, int FMT, int D, int NT>
cudaError_t attn_of(const AttnArgs& a, const Q8Plan& p, cudaStream_t stream) {
    if (a.k_new) {
        cudaError_t e = ensure_dynamic_smem(q8_attn_kernel<T, FMT, D, NT, true>, p.smem);
        if (e != cudaSuccess) return e;
        q8_attn_kernel<T, FMT, D, NT, true><<<p.ctas, kThreads, p.smem, stream>>>(a);
    } else {
        cudaError_t e = ensure_dynamic_smem(q8_attn_kernel<T, FMT, D, NT, false>, p.smem);
        if (e != cudaSuccess) return e;
        q8_attn_kernel<T, FMT, D, NT, false><<<p.ctas, kThreads, p.smem, stream>>>(a);
    }
    return cudaGetLastError();
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
    // the fp32 and the bf16 plan differ in CTAs only
    return 4096 + plan_q8(s, n_q, 2).part;
}

cudaError_t launch_q8_attention(const Q8Dims& s, const Q8Cache& c, int fmt, int dtype, const void* q, int64_t sb, int64_t si, int64_t sg, void* out, int n_q,
                                const void* k_new, const void* v_new, char* ws, cudaStream_t stream) {
    const Q8Plan p = plan_q8(s, n_q, dtype == FA_BF16 ? 2 : 4);
    const AttnArgs a = {s, c, q, sb, si, sg, out, n_q, p.n_ct, k_new, v_new, reinterpret_cast<unsigned*>(ws), reinterpret_cast<float*>(ws + 4096)};
    if (dtype == FA_BF16) return fmt == FA_Q8_INT8 ? attn_dims<__nv_bfloat16, FA_Q8_INT8>(a, p, stream) : attn_dims<__nv_bfloat16, FA_Q8_E4M3>(a, p, stream);
    return fmt == FA_Q8_INT8 ? attn_dims<float, FA_Q8_INT8>(a, p, stream) : attn_dims<float, FA_Q8_E4M3>(a, p, stream);
}

}  // namespace fa
