// fa_q8_write, fa_q8_append, fa_q8_read: tokens into the dense cache in 8 bits and back.
//
// A CTA owns one block of one KV head and side (K or V).  A block that the call completes is rounded: its tokens, those
// that the tail holds already and the new ones, go to registers once, the CTA finds their largest magnitude, and 16 bytes
// a thread leave as a page.  The block that stays incomplete is copied to the tail, with the running largest magnitude.  The
// first block of a row that has a tail is read from it, and the last one of the call written to it: where these are
// two blocks, one CTA does both in that order.  The last CTA to take the ticket sets the rows' lengths, which the others have read by then.
// Bound by HBM: 2 (or 4) bytes in and 1 out per value, whole sectors on both sides.
#include "fa_q8.cuh"

namespace fa {
namespace {

template <typename T>
struct StoreArgs {
    Q8Dims s;
    Q8Cache c;
    const T *K, *V;
    int64_t sb, st, sh;
    int n;
    const int32_t* n_row;
    int append;
};

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(1024, 1) q8_store_kernel(const StoreArgs<T> a) {
    const Q8Dims& s = a.s;
    __shared__ uint32_t red[32];
    __shared__ int bad_s;
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5;
    const int h2 = (int)(blockIdx.x % (unsigned)(2 * s.H)), x = (int)(blockIdx.x / (unsigned)(2 * s.H)), b = blockIdx.y;
    const int h = h2 >> 1, side = h2 & 1;
    const int held = a.append ? a.c.state[b * kQ8State] : 0;
    const int cap = s.nb << s.lb;
    int n = a.n_row ? a.n_row[b] : a.n;
    n = n < 0 ? 0 : n > a.n ? a.n : n;
    const bool fits = held >= 0 && held <= cap && n <= cap - held;
    const int total = held + n;
    const int first = held >> s.lb, r = held & (s.blk - 1);          // the first block that gets tokens, what the tail has of it
    const int whole = total >> s.lb;                                 // complete blocks behind the call
    const int blk = first + x;
    const int32_t* table = a.c.table + (size_t)b * s.nb;

    const bool two = r > 0 && whole > first;                         // the tail is read and written
    const bool completes = fits && n > 0 && blk < whole;
    const bool fills = fits && n > 0 && (total & (s.blk - 1)) != 0 && (two ? x == 0 : blk == whole);
    if (tid == 0) bad_s = !fits;
    __syncthreads();
    if (fills) {                                                     // the tail stays as it is if any block of the row has no page
        for (int i = first + tid; i < whole; i += nt) {
            const int page = table[i];
            if (page < 0 || page >= s.n_pages) bad_s = 1;
        }
    }

    T* tail = reinterpret_cast<T*>(side ? a.c.v_tail : a.c.k_tail) + ((size_t)b * s.H + h) * (size_t)s.blk * D;
    const T* src = (side ? a.V : a.K) + (int64_t)b * a.sb + (int64_t)h * a.sh;
    float* amax_out = a.c.tail_amax + ((size_t)b * s.H + h) * 2 + side;
    const int nvec = s.blk * (D / 16);                               // two to a thread (nt = nvec / 2)
    auto block_max = [&](uint32_t m) {
        m = __reduce_max_sync(0xffffffffu, m);
        __syncthreads();
        if (lane == 0) red[warp] = m;
        __syncthreads();
        const uint32_t v = lane < (nt >> 5) ? red[lane] : 0u;
        return __reduce_max_sync(0xffffffffu, v);
    };
    if (completes) {
        const int page = table[blk];
        const bool good = page >= 0 && page < s.n_pages;
        if (!good && tid == 0) {
            q8_report(a.c.status, FA_ERR_INDEX);
            atomicExch(a.c.state + b * kQ8State + 1, 1);
        }
        Vec16<T> v[2];
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = tid + k * nt, t = i / (D / 16), e = (i % (D / 16)) * 16;
            const int at = (blk << s.lb) + t;                        // the token's place in the row
            if (i < nvec) v[k].load(at < held ? tail + (size_t)t * D + e : src + (int64_t)(at - held) * a.st + e);
            else v[k].zero();
            m = max(m, v[k].amax_bits());
        }
        m = block_max(m);
        if (good) {
            const Q8Round<FMT, T> to(m);
            const size_t ph = (size_t)page * s.H + h;
            uint8_t* out = (side ? a.c.v_pages : a.c.k_pages) + ph * (size_t)(s.blk * D);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int i = tid + k * nt;
                if (i >= nvec) break;
                uint4 o;
                o.x = to.pack(v[k].at(0), v[k].at(1), v[k].at(2), v[k].at(3));
                o.y = to.pack(v[k].at(4), v[k].at(5), v[k].at(6), v[k].at(7));
                o.z = to.pack(v[k].at(8), v[k].at(9), v[k].at(10), v[k].at(11));
                o.w = to.pack(v[k].at(12), v[k].at(13), v[k].at(14), v[k].at(15));
                *reinterpret_cast<uint4*>(out + (size_t)i * 16) = o;
            }
            if (tid == 0) (side ? a.c.v_scale : a.c.k_scale)[ph] = Q8Round<FMT, T>::scale(m);
        }
    }
    __syncthreads();
    if (fills && !bad_s) {
        // the row's new tokens from t0 on, behind the k0 that the tail has of this block
        const int t0 = max(held, whole << s.lb), k0 = whole > first ? 0 : r;
        const int nv = (total - t0) * (D / 16);
        uint32_t m = 0;
        for (int i = tid; i < nv; i += nt) {
            const int t = i / (D / 16), e = (i % (D / 16)) * 16;
            Vec16<T> v;
            v.load(src + (int64_t)(t0 - held + t) * a.st + e);
            v.store(tail + (size_t)(k0 + t) * D + e);
            m = max(m, v.amax_bits());
        }
        m = block_max(m);
        if (tid == 0) {
            const float before = k0 > 0 ? *amax_out : 0.f;
            *amax_out = __uint_as_float(max(m, __float_as_uint(before)));
        }
    }
    // the ticket
    __shared__ int last_s;
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        const unsigned all = gridDim.x * gridDim.y;
        last_s = atomicInc(reinterpret_cast<unsigned*>(a.c.status) + 1, all - 1) == all - 1;
        __threadfence();
    }
    __syncthreads();
    if (!last_s) return;
    for (int i = tid; i < s.B; i += nt) {
        int32_t* st = a.c.state + i * kQ8State;
        const int was = a.append ? st[0] : 0;
        int add = a.n_row ? a.n_row[i] : a.n;
        add = add < 0 ? 0 : add > a.n ? a.n : add;
        const bool bad = atomicExch(st + 1, 0) != 0;
        if (was < 0 || was > cap || add > cap - was) q8_report(a.c.status, FA_ERR_CAPACITY);
        else if (!bad) st[0] = was + add;
        else if (!a.append) st[0] = 0;                               // (pages of its blocks may have been written)
    }
}

// A CTA reads the same tokens of one head for K and V; a thread 16 values at a time.
template <typename T, int FMT, int D>
__global__ void __launch_bounds__(256) q8_read_kernel(Q8Dims s, Q8Cache c, T* __restrict__ K, T* __restrict__ V, int64_t sb, int64_t st, int64_t sh, int t0,
                                                      int n) {
    constexpr int kVecs = D / 16, kTok = 256 / kVecs;                // tokens that a pass of the CTA covers
    const int h = (int)(blockIdx.x % (unsigned)s.H), b = blockIdx.y;
    const int tile = (int)(blockIdx.x / (unsigned)s.H) * (2 * kTok);
    const int len = c.state[b * kQ8State];
    const int cap = s.nb << s.lb;
    const int e = (threadIdx.x % kVecs) * 16;
    if (len < 0 || len > cap) {
        if (threadIdx.x == 0) q8_report(c.status, FA_ERR_CAPACITY);
        return;
    }
    const int stop = min(len, t0 + n), paged = len >> s.lb << s.lb;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int t = t0 + tile + k * kTok + (int)threadIdx.x / kVecs;
        if (t >= stop) continue;
        const int64_t off = (int64_t)b * sb + (int64_t)(t - t0) * st + (int64_t)h * sh + e;
        if (t >= paged) {
            const size_t at = (((size_t)b * s.H + h) * (size_t)s.blk + (t - paged)) * D + e;
            Vec16<T> x;
            x.load(reinterpret_cast<const T*>(c.k_tail) + at);
            x.store(K + off);
            x.load(reinterpret_cast<const T*>(c.v_tail) + at);
            x.store(V + off);
            continue;
        }
        const int page = c.table[(size_t)b * s.nb + (t >> s.lb)];
        if (page < 0 || page >= s.n_pages) {
            q8_report(c.status, FA_ERR_INDEX);
            continue;
        }
        const size_t ph = (size_t)page * s.H + h, at = (ph * (size_t)s.blk + (t & (s.blk - 1))) * D + e;
        const uint4 kw = *reinterpret_cast<const uint4*>(c.k_pages + at), vw = *reinterpret_cast<const uint4*>(c.v_pages + at);
        const float ks = c.k_scale[ph], vs = c.v_scale[ph];
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const uint4 w = side ? vw : kw;
            const float f = side ? vs : ks;
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
            float x[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y[4];
                q8_floats<FMT>(ws[i], y);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[4 * i + j] = y[j] * f;
            }
            T* out = (side ? V : K) + off;
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i) *(reinterpret_cast<float4*>(out) + i) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
            } else {
                uint32_t o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                    o[i] = *reinterpret_cast<const uint32_t*>(&p);
                }
                *reinterpret_cast<uint4*>(out) = make_uint4(o[0], o[1], o[2], o[3]);
                *(reinterpret_cast<uint4*>(out) + 1) = make_uint4(o[4], o[5], o[6], o[7]);
            }
        }
    }
}

template <typename T, int FMT, int D>
cudaError_t store_of(const Q8Dims& s, const Q8Cache& c, const void* K, const void* V, int64_t sb, int64_t st, int64_t sh, int n, const int32_t* n_row,
                     bool append, cudaStream_t stream) {
    const StoreArgs<T> a = {s, c, static_cast<const T*>(K), static_cast<const T*>(V), sb, st, sh, n, n_row, append};
    // blocks that n tokens can touch behind a tail of blk - 1
    const int64_t touched = n == 0 ? 1 : ((int64_t)(append ? s.blk - 1 : 0) + n - 1) / s.blk + 1;
    q8_store_kernel<T, FMT, D><<<dim3((unsigned)(touched * 2 * s.H), (unsigned)s.B), s.blk * D / 32, 0, stream>>>(a);
    return cudaGetLastError();
}
template <typename T, int FMT, int D>
cudaError_t read_of(const Q8Dims& s, const Q8Cache& c, void* K, void* V, int64_t sb, int64_t st, int64_t sh, int t0, int n, cudaStream_t stream) {
    const int tok = 2 * 256 / (D / 16);
    const int64_t tiles = ((int64_t)n + tok - 1) / tok;
    q8_read_kernel<T, FMT, D><<<dim3((unsigned)(tiles * s.H), (unsigned)s.B), 256, 0, stream>>>(s, c, static_cast<T*>(K), static_cast<T*>(V), sb, st, sh, t0, n);
    return cudaGetLastError();
}

#define FA_Q8_DISPATCH(CALL)                                                                                               \
    do {                                                                                                                   \
        if (dtype == FA_BF16) {                                                                                            \
            if (fmt == FA_Q8_INT8) { FA_Q8_DIM(__nv_bfloat16, FA_Q8_INT8, CALL) } else { FA_Q8_DIM(__nv_bfloat16, FA_Q8_E4M3, CALL) } \
        } else {                                                                                                           \
            if (fmt == FA_Q8_INT8) { FA_Q8_DIM(float, FA_Q8_INT8, CALL) } else { FA_Q8_DIM(float, FA_Q8_E4M3, CALL) }        \
        }                                                                                                                  \
    } while (0)
#define FA_Q8_DIM(T, F, CALL)                                \
    switch (s.d) {                                           \
        case 64: return CALL(T, F, 64);                      \
        case 128: return CALL(T, F, 128);                    \
        default: return CALL(T, F, 256);                     \
    }

}  // namespace

cudaError_t launch_q8_store(const Q8Dims& s, const Q8Cache& c, int fmt, int dtype, const void* K, const void* V, int64_t sb, int64_t st, int64_t sh, int n,
                            const int32_t* n_row, bool append, cudaStream_t stream) {
#define FA_Q8_CALL(T, F, D) store_of<T, F, D>(s, c, K, V, sb, st, sh, n, n_row, append, stream)
    FA_Q8_DISPATCH(FA_Q8_CALL);
#undef FA_Q8_CALL
}
cudaError_t launch_q8_read(const Q8Dims& s, const Q8Cache& c, int fmt, int dtype, void* K, void* V, int64_t sb, int64_t st, int64_t sh, int t0, int n,
                           cudaStream_t stream) {
#define FA_Q8_CALL(T, F, D) read_of<T, F, D>(s, c, K, V, sb, st, sh, t0, n, stream)
    FA_Q8_DISPATCH(FA_Q8_CALL);
#undef FA_Q8_CALL
}

}  // namespace fa
