// Shared parts of the kernels on the dense cache in 8 bits: its numbers, the rounding of a block, the conversion of
// its bytes to the 16-bit operands of the tensor cores.
#pragma once

#include <cuda_fp16.h>

#include "fa_common.cuh"

namespace fa {

constexpr int kQ8State = 4;          // int32 words of state per row: tokens, 3 spare
constexpr int kQ8MaxCtas = 500;      // CTAs of an attention launch; tickets in the first 4 KiB of the workspace: of groups of parts from 0, of
constexpr int kQ8GroupTickets = 512; // pairs of many groups from here on, and
constexpr int kQ8StepTicket = 1023;  // of the CTAs of a step which have read the lengths

struct Q8Dims {
    int B, Hq, H, G, d;
    int blk, lb;                     // tokens of a block and their log2
    int nb, n_pages;
    float scale;
};
inline Q8Dims make_q8_dims(const fa_q8_layout& l) {
    Q8Dims s;
    s.B = l.batch; s.Hq = l.n_q_heads; s.H = l.n_kv_heads; s.G = l.n_q_heads / l.n_kv_heads; s.d = l.head_dim;
    s.blk = l.block; s.lb = l.block == 16 ? 4 : l.block == 32 ? 5 : l.block == 64 ? 6 : 7;
    s.nb = l.max_blocks; s.n_pages = l.n_pages; s.scale = l.softmax_scale;
    return s;
}
struct Q8Cache {
    uint8_t *k_pages, *v_pages;
    float *k_scale, *v_scale;
    void *k_tail, *v_tail;
    float* tail_amax;
    const int32_t* table;
    int32_t *state, *status;
};
inline Q8Cache make_q8_cache(const fa_q8_cache& c) {
    return {c.k_pages, c.v_pages, c.k_scale, c.v_scale, c.k_tail, c.v_tail, c.tail_amax, c.block_table, c.state, c.status};
}

// Launchers.  fmt: fa_q8_format, dtype: fa_dtype.
cudaError_t launch_q8_reset(const Q8Dims&, const Q8Cache&, cudaStream_t);
cudaError_t launch_q8_store(const Q8Dims&, const Q8Cache&, int fmt, int dtype, const void* K, const void* V, int64_t sb, int64_t st, int64_t sh, int n,
                            const int32_t* n_row, bool append, cudaStream_t);
cudaError_t launch_q8_read(const Q8Dims&, const Q8Cache&, int fmt, int dtype, void* K, void* V, int64_t sb, int64_t st, int64_t sh, int t0, int n,
                           cudaStream_t);
// k_new / v_new non-null: a step (n_q = 1).
size_t q8_attention_ws_bytes(const Q8Dims&, int n_q);
bool q8_attention_fits(const Q8Dims&, int n_q);      // the units of work are counted in 32 bits (of calls that q8_chunk_takes does not take)
cudaError_t launch_q8_attention(const Q8Dims&, const Q8Cache&, int fmt, int dtype, const void* q, int64_t sb, int64_t si, int64_t sg, void* out, int n_q,
                                const void* k_new, const void* v_new, char* ws, cudaStream_t);
// The same for many query columns to a KV head, as far as their blocks are counted in 32 bits (fa_q8_chunk.cu).
bool q8_chunk_takes(const Q8Dims&, int dtype, int n_q);
size_t q8_chunk_ws_bytes(const Q8Dims&);
cudaError_t launch_q8_chunk(const Q8Dims&, const Q8Cache&, int fmt, const void* q, int64_t sb, int64_t si, int64_t sg, void* out, int n_q, char* ws,
                            cudaStream_t);

#ifdef __CUDACC__
// A launch whose CTAs may be scheduled under the tail of the kernel in front (they wait for its end before their first read).
template <typename... P, typename... A>
inline cudaError_t launch_behind(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, const A&... args) {
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = dim3((unsigned)threads);
    c.dynamicSmemBytes = smem;
    c.stream = stream;
    c.attrs = at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, kernel, args...);
}
__device__ __forceinline__ void q8_report(int32_t* status, int err) { atomicCAS(status, (int)FA_OK, err); }

// What a block's values are multiplied by.  A quotient x * top / amax is rounded twice at most (to 32 or 64 bits, then to
// the 8-bit number), so it has to be exact wherever it lies half way between two 8-bit numbers.  y = (x top) (1 / amax) is off by
// an ulp or two; the remainder x * top - y * amax is exact (x * top and the products have few bits), and y + remainder / amax
// rounds to the nearest number, which is the quotient itself where that is representable, as half-way points are.
// Elsewhere the quotient is further from a half-way point than the rounding: 2 x top and (an odd number) x amax are whole multiples of one unit, so
// 2^-16 relative for 8-bit significands and 2^-32 for 24 (in 64 bits).  p, a power of two, keeps all of it normal; values below 2^-60 amax become zero either way.
template <typename T>
struct Q8Real { using type = float; };
template <>
struct Q8Real<float> { using type = double; };

// Two of them as one operand of the packed fp32 instructions; of 64 bits, two.
template <typename R>
struct Q8Two;
template <>
struct Q8Two<float> {
    unsigned long long v;
    static __device__ __forceinline__ Q8Two of(float a, float b) {
        Q8Two r;
        asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
        return r;
    }
    __device__ __forceinline__ Q8Two times(Q8Two b) const {
        Q8Two r;
        asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(v), "l"(b.v));
        return r;
    }
    __device__ __forceinline__ Q8Two times_plus(Q8Two b, Q8Two c) const {
        Q8Two r;
        asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(v), "l"(b.v), "l"(c.v));
        return r;
    }
    __device__ __forceinline__ Q8Two plus(Q8Two b) const {
        Q8Two r;
        asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(v), "l"(b.v));
        return r;
    }
    __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
template <>
struct Q8Two<double> {
    double a, b;
    static __device__ __forceinline__ Q8Two of(double x, double y) { return {x, y}; }
    __device__ __forceinline__ Q8Two times(Q8Two o) const { return {a * o.a, b * o.b}; }
    __device__ __forceinline__ Q8Two times_plus(Q8Two o, Q8Two c) const { return {fma(a, o.a, c.a), fma(b, o.b, c.b)}; }
    __device__ __forceinline__ Q8Two plus(Q8Two o) const { return {a + o.a, b + o.b}; }
    __device__ __forceinline__ void get(double& x, double& y) const { x = a; y = b; }
};

template <int FMT, typename T>
struct Q8Round {
    using R = typename Q8Real<T>::type;
    using Two = Q8Two<R>;
    static constexpr float kTop = FMT == FA_Q8_INT8 ? 127.f : 448.f;
    R top, minus, inv;               // p top, -p amax, 1 / (p amax)
    uint32_t keep;                   // all bits if some value is not zero and all are finite; else the bytes are zero
    __device__ __forceinline__ explicit Q8Round(uint32_t amax_bits) {
        const bool live = amax_bits != 0 && amax_bits < 0x7f800000u;
        keep = live ? 0xffffffffu : 0u;
        const float p = amax_bits < 0x21800000u ? 0x1p64f : amax_bits > 0x5d800000u ? 0x1p-64f : 1.f;
        const float as = __uint_as_float(amax_bits) * p;
        top = (R)(kTop * p);
        minus = (R)-as;
        inv = live ? (R)1 / (R)as : (R)0;
    }
    __device__ __forceinline__ Two quotient(float x0, float x1) const {
        const Two i2 = Two::of(inv, inv);
        const Two xt = Two::of((R)x0, (R)x1).times(Two::of(top, top)), y = xt.times(i2);
        return y.times_plus(Two::of(minus, minus), xt).times_plus(i2, y);
    }
    // Four values to four bytes.
    __device__ __forceinline__ uint32_t pack(float a, float b, float c, float d) const {
        Two q0 = quotient(a, b), q1 = quotient(c, d);
        R r0, r1, r2, r3;
        uint32_t r;
        if constexpr (FMT == FA_Q8_INT8) {
            // 1.5 2^23 (2^52) behind it, a sum's last bits are the quotient rounded to a whole number, half to even
            constexpr R kBehind = sizeof(R) == 8 ? (R)6755399441055744.0 : (R)12582912.0f;
            q0 = q0.plus(Two::of(kBehind, kBehind));
            q1 = q1.plus(Two::of(kBehind, kBehind));
            q0.get(r0, r1);
            q1.get(r2, r3);
            r = __byte_perm(__byte_perm(last_word(r0), last_word(r1), 0x0040), __byte_perm(last_word(r2), last_word(r3), 0x0040), 0x5410);
        } else {
            q0.get(r0, r1);
            q1.get(r2, r3);
            asm("{\n .reg .b16 lo, hi;\n cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n mov.b32 %0, {lo, hi};\n}\n"
                : "=r"(r)
                : "f"(narrow(r0)), "f"(narrow(r1)), "f"(narrow(r2)), "f"(narrow(r3)));
        }
        return r & keep;
    }
    static __device__ __forceinline__ uint32_t last_word(float x) { return __float_as_uint(x); }
    static __device__ __forceinline__ uint32_t last_word(double x) { return (uint32_t)__double2loint(x); }
    // 64 to 32 bits by rounding to odd: the second rounding, to 4 bits, then comes out as one from 64 bits would.
    static __device__ __forceinline__ float narrow(float y) { return y; }
    static __device__ __forceinline__ float narrow(double y) {
        const float f = __double2float_rz(y);
        return (double)f == y ? f : __uint_as_float(__float_as_uint(f) | 1u);
    }
    static __device__ __forceinline__ float scale(uint32_t amax_bits) {
        if (amax_bits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
        const float a = __uint_as_float(amax_bits), r = __fdiv_rn(a, kTop);
        return r * kTop > 0x1.fffffep127f ? __fdiv_rz(a, kTop) : r;          // (the largest numbers: top x scale must not overflow)
    }
};

// Sixteen consecutive elements.
template <typename T>
struct Vec16;
template <>
struct Vec16<__nv_bfloat16> {
    uint4 a, b;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        a = *reinterpret_cast<const uint4*>(p);
        b = *(reinterpret_cast<const uint4*>(p) + 1);
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const {
        *reinterpret_cast<uint4*>(p) = a;
        *(reinterpret_cast<uint4*>(p) + 1) = b;
    }
    __device__ __forceinline__ void zero() { a = b = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ uint32_t word(int i) const { return i < 4 ? (i == 0 ? a.x : i == 1 ? a.y : i == 2 ? a.z : a.w) : (i == 4 ? b.x : i == 5 ? b.y : i == 6 ? b.z : b.w); }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? word(i >> 1) & 0xffff0000u : word(i >> 1) << 16); }
    // Largest magnitude as a bit pattern of a float: NaN above infinity above all numbers.
    __device__ __forceinline__ uint32_t amax_bits() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = __vmaxu2(m, word(i) & 0x7fff7fffu);
        return max(m << 16, m & 0xffff0000u);
    }
};
template <>
struct Vec16<float> {
    float4 v[4];
    __device__ __forceinline__ void load(const float* p) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *(reinterpret_cast<const float4*>(p) + i);
    }
    __device__ __forceinline__ void store(float* p) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) *(reinterpret_cast<float4*>(p) + i) = v[i];
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __device__ __forceinline__ float at(int i) const { const float4& f = v[i >> 2]; return (i & 3) == 0 ? f.x : (i & 3) == 1 ? f.y : (i & 3) == 2 ? f.z : f.w; }
    __device__ __forceinline__ uint32_t amax_bits() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(at(i)) & 0x7fffffffu);
        return m;
    }
};

// Two 8-bit values (in the low 16 bits of w) as two halves, exactly.  int8 words arrive with their sign bits flipped (q + 128).
template <int FMT>
__device__ __forceinline__ uint32_t q8_halves(uint32_t w, int hi) {
    uint32_t r;
    if constexpr (FMT == FA_Q8_INT8) {
        const uint32_t u = hi ? __byte_perm(w, 0x64646464u, 0x4342) : __byte_perm(w, 0x64646464u, 0x4140);   // halves of 1024 + 128 + q
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(u), "r"(0x64806480u));
    } else {
        if (hi) asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %1;\n cvt.rn.f16x2.e4m3x2 %0, b;\n}\n" : "=r"(r) : "r"(w));
        else asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %1;\n cvt.rn.f16x2.e4m3x2 %0, a;\n}\n" : "=r"(r) : "r"(w));
    }
    return r;
}
template <int FMT>
__device__ __forceinline__ uint32_t q8_flip(uint32_t w) { return FMT == FA_Q8_INT8 ? w ^ 0x80808080u : w; }
// Four of them times f, each with one rounding.
template <int FMT>
__device__ __forceinline__ void q8_floats(uint32_t w, float f, float (&x)[4]) {
    Q8Two<float> lo, hi;
    if constexpr (FMT == FA_Q8_INT8) {
        const uint32_t u = q8_flip<FMT>(w);                // q + 128 as the last bits of 2^23 + 128 + q
        const Q8Two<float> less = Q8Two<float>::of(-8388736.f, -8388736.f);
        lo = Q8Two<float>::of(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441))).plus(less);
        hi = Q8Two<float>::of(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7442)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7443))).plus(less);
    } else {
        const uint32_t a = q8_halves<FMT>(w, 0), b = q8_halves<FMT>(w, 1);
        const float2 fa = __half22float2(*reinterpret_cast<const __half2*>(&a)), fb = __half22float2(*reinterpret_cast<const __half2*>(&b));
        lo = Q8Two<float>::of(fa.x, fa.y);
        hi = Q8Two<float>::of(fb.x, fb.y);
    }
    const Q8Two<float> ff = Q8Two<float>::of(f, f);
    lo.times(ff).get(x[0], x[1]);
    hi.times(ff).get(x[2], x[3]);
}
#endif  // __CUDACC__

}  // namespace fa
