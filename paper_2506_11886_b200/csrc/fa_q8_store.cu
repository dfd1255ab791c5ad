// fa_q8_write, fa_q8_append, fa_q8_read: tokens into the dense cache in 8 bits and back.
//
// A group of threads takes a few blocks of one KV head and side (K or V) in turn, 32 values or more to a thread, the next block's loads under way.  A block that
// the call completes is rounded: its tokens, those that the tail holds already and the new ones, go to registers once, the group finds their largest magnitude,
// and 16 bytes a thread leave as a page.  The block that stays incomplete is copied to the tail, with the running largest magnitude.  The
// first block of a row that has a tail is read from it, and the last one of the call written to it: where these are
// two blocks, one group does both in that order.  Appending, each CTA takes a ticket once it has read its row's length; the last one sets all lengths.
// Bound by HBM and by instructions (13 a value and thread, 65 % of the issue slots): 2 (or 4) bytes in and 1 out per value, whole sectors on both sides.  32768 tokens of
// 8 heads of 128 in bf16: written in 44 us (4.6 TB/s), read in 37 (int8, 5.5 TB/s) or 33 (e4m3); one token of 8 heads appended 3.8 us.
#include <type_traits>

#include "fa_q8.cuh"

namespace fa {
namespace {

constexpr int kStoreThreads = 256;

template <typename T>
struct StoreArgs {
    Q8Dims s;
    Q8Cache c;
    const T *K, *V;
    int64_t sb, st, sh;
    int n;
    const int32_t* n_row;
    int append, run;                 // blocks that a group takes in turn
    int ld;                          // log2 of the head dim
};

// What the call does to row b.
struct StoreRow {
    int held, total, first, whole;   // tokens before and after; the first block that gets tokens, complete blocks after
    bool goes;                       // there are new tokens and they fit
};
template <typename T>
__device__ __forceinline__ StoreRow store_row(const StoreArgs<T>& a, int b, int held) {
    const int cap = a.s.nb << a.s.lb;
    int n = a.n_row ? a.n_row[b] : a.n;
    n = n < 0 ? 0 : n > a.n ? a.n : n;
    StoreRow r;
    r.held = held;
    r.goes = held >= 0 && held <= cap && n <= cap - held && n > 0;
    r.total = r.goes ? held + n : held;
    r.first = held >> a.s.lb;
    r.whole = r.total >> a.s.lb;
    return r;
}
// Whether every block that the call completes in row b has a page; by the threads i0, i0 + step, ...
template <typename T>
__device__ __forceinline__ bool pages_there(const StoreArgs<T>& a, int b, const StoreRow& r, int i0, int step) {
    bool ok = true;
    for (int i = r.first + i0; i < r.whole; i += step) {
        const int page = a.c.table[(size_t)b * a.s.nb + i];
        ok = ok && page >= 0 && page < a.s.n_pages;
    }
    return ok;
}

// NV vectors of 16 values to a thread.  Grid: runs of `run` blocks of each group, head and side, row.
template <typename T, int FMT, int NV>
__global__ void __launch_bounds__(kStoreThreads, NV * sizeof(T) == 4 ? 3 : NV * sizeof(T) == 8 ? 2 : 1) q8_store_kernel(const StoreArgs<T> a) {
    const Q8Dims& s = a.s;
    __shared__ uint32_t red[2][kStoreThreads / 32];
    __shared__ int last_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int lv = a.ld - 4;                                         // log2 of a row's vectors
    const int group = (s.blk << lv) / NV;                            // threads of a group: whole warps
    const int groups = kStoreThreads / group, gi = tid / group, gt = tid % group, gwarps = group >> 5;
    uint32_t turn = 0;
    auto group_max = [&](uint32_t m) {
        m = __reduce_max_sync(0xffffffffu, m);
        if (gwarps == 1) return m;
        uint32_t* place = red[turn++ & 1];
        if (lane == 0) place[warp] = m;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + gi), "r"(group) : "memory");
        const uint32_t v = lane < gwarps ? place[gi * gwarps + lane] : 0u;
        return __reduce_max_sync(0xffffffffu, v);
    };
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.z, h = blockIdx.y >> 1, side = blockIdx.y & 1;
    const int held = a.append ? a.c.state[b * kQ8State] : 0;
    if (a.append) {
        __syncthreads();                                             // (all threads have the length)
        if (tid == 0) {
            __threadfence();
            const unsigned all = gridDim.x * gridDim.y * gridDim.z;
            last_s = atomicInc(reinterpret_cast<unsigned*>(a.c.status) + 1, all - 1) == all - 1;
        }
    }
    const StoreRow r = store_row(a, b, held);
    const int x0 = (int)blockIdx.x * a.run * groups + gi;            // the group's blocks: x0, x0 + groups, ...
    const int k0 = r.held & (s.blk - 1);
    const bool two = k0 > 0 && r.whole > r.first;                    // the tail is read and written
    if (r.goes && r.first + (int)blockIdx.x * a.run * groups <= r.whole) {
        const int32_t* table = a.c.table + (size_t)b * s.nb;
        T* tail = reinterpret_cast<T*>(side ? a.c.v_tail : a.c.k_tail) + (((size_t)b * s.H + h) * (size_t)s.blk << a.ld);
        const T* src = (side ? a.V : a.K) + (int64_t)b * a.sb + (int64_t)h * a.sh;
        constexpr bool kAhead = NV * sizeof(T) <= 8;                 // (the next block's values in registers too)
        Vec16<T> v[NV], y[kAhead ? NV : 1];
        auto load = [&](Vec16<T>* to, int blk) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int i = gt + k * group, t = i >> lv, e = (i & ((1 << lv) - 1)) << 4;
                const int at = (blk << s.lb) + t;                    // the token's place in the row
                to[k].load(at < r.held ? tail + ((size_t)t << a.ld) + e : src + (int64_t)(at - r.held) * a.st + e);
            }
        };
        if (kAhead && r.first + x0 < r.whole) load(v, r.first + x0);
        for (int i = 0; i < a.run; ++i) {
            const int x = x0 + i * groups, blk = r.first + x;
            if (blk < r.whole) {                                     // completed by the call
                const int page = table[blk];
                if constexpr (kAhead) {
                    if (i + 1 < a.run && blk + groups < r.whole) load(y, blk + groups);
                } else {
                    load(v, blk);
                }
                uint32_t m = 0;
#pragma unroll
                for (int k = 0; k < NV; ++k) m = max(m, v[k].amax_bits());
                m = group_max(m);
                if (page >= 0 && page < s.n_pages) {
                    const Q8Round<FMT, T> to(m);
                    const size_t ph = (size_t)page * s.H + h;
                    uint8_t* out = (side ? a.c.v_pages : a.c.k_pages) + (ph * (size_t)s.blk << a.ld);
#pragma unroll
                    for (int k = 0; k < NV; ++k) {
                        uint4 o;
                        o.x = to.pack(v[k].at(0), v[k].at(1), v[k].at(2), v[k].at(3));
                        o.y = to.pack(v[k].at(4), v[k].at(5), v[k].at(6), v[k].at(7));
                        o.z = to.pack(v[k].at(8), v[k].at(9), v[k].at(10), v[k].at(11));
                        o.w = to.pack(v[k].at(12), v[k].at(13), v[k].at(14), v[k].at(15));
                        *reinterpret_cast<uint4*>(out + (size_t)(gt + k * group) * 16) = o;
                    }
                    if (gt == 0) (side ? a.c.v_scale : a.c.k_scale)[ph] = Q8Round<FMT, T>::scale(m);
                } else if (gt == 0) {
                    q8_report(a.c.status, FA_ERR_INDEX);
                }
                if constexpr (kAhead)
#pragma unroll
                    for (int k = 0; k < NV; ++k) v[k] = y[k];
            }
            if ((r.total & (s.blk - 1)) != 0 && (two ? x == 0 : blk == r.whole)) {
                // what stays incomplete; the tail stays as it is if any block of the row has no page (the group decides as one)
                if (group_max(pages_there(a, b, r, gt, group) ? 0u : 1u)) continue;
                // the row's new tokens from t0 on, behind the n0 that the tail has of this block
                const int t0 = max(r.held, r.whole << s.lb), n0 = r.whole > r.first ? 0 : k0;
                const int nv = (r.total - t0) << lv;
                uint32_t m = 0;
                for (int j = gt; j < nv; j += group) {
                    const int t = j >> lv, e = (j & ((1 << lv) - 1)) << 4;
                    Vec16<T> w;
                    w.load(src + (int64_t)(t0 - r.held + t) * a.st + e);
                    w.store(tail + ((size_t)(n0 + t) << a.ld) + e);
                    m = max(m, w.amax_bits());
                }
                m = group_max(m);
                if (gt == 0) {
                    float* amax = a.c.tail_amax + ((size_t)b * s.H + h) * 2 + side;
                    const float before = n0 > 0 ? *amax : 0.f;
                    *amax = __uint_as_float(max(m, __float_as_uint(before)));
                }
            }
        }
    }
    // ---- the rows' lengths: nobody reads them in a write ----
    __syncthreads();
    if (a.append ? !last_s : blockIdx.x + blockIdx.y + blockIdx.z != 0) return;
    const int cap = s.nb << s.lb;
    for (int i = warp; i < s.B; i += kStoreThreads / 32) {
        int32_t* st = a.c.state + i * kQ8State;
        const StoreRow q = store_row(a, i, a.append ? st[0] : 0);
        const bool there = __all_sync(0xffffffffu, pages_there(a, i, q, lane, 32));
        if (lane != 0) continue;
        const int n = a.n_row ? a.n_row[i] : a.n;
        if (q.held < 0 || q.held > cap || min(n, a.n) > cap - q.held) q8_report(a.c.status, FA_ERR_CAPACITY);
        else if (there) st[0] = q.total;
        else if (!a.append) st[0] = 0;                               // (pages of its blocks may have been written)
    }
}

// A CTA reads the same tokens of one head for K and V.  A thread's piece is 16 bytes of bf16 tensors' pages, two pieces for each side; neighbouring lanes exchange
// halves of what they write, so that a store covers whole sectors.  Of fp32 tensors it is what 16 written bytes take, four pieces.
template <typename T>
constexpr int kReadE = sizeof(T) == 2 ? 16 : 4;             // values of a piece
template <typename T>
constexpr int kReadPass = sizeof(T) == 2 ? 2 : 4;
template <typename T, int FMT, int D>
__global__ void __launch_bounds__(256) q8_read_kernel(Q8Dims s, Q8Cache c, T* __restrict__ K, T* __restrict__ V, int64_t sb, int64_t st, int64_t sh, int t0,
                                                      int n) {
    constexpr int kE = kReadE<T>, kPass = kReadPass<T>, kTok = 256 * kE / D;                 // tokens that a pass of the CTA covers
    using Bytes = typename std::conditional<kE == 16, uint4, uint32_t>::type;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int h = (int)(blockIdx.x % (unsigned)s.H), b = blockIdx.y;
    const int t1 = t0 + (int)(blockIdx.x / (unsigned)s.H) * (kPass * kTok) + (int)threadIdx.x / (D / kE), e = (threadIdx.x % (D / kE)) * kE;
    const int len = c.state[b * kQ8State];
    if (len < 0 || len > s.nb << s.lb) {
        if (threadIdx.x == 0) q8_report(c.status, FA_ERR_CAPACITY);
        return;
    }
    const int stop = min(len, t0 + n), paged = len >> s.lb << s.lb;
    T* const out[2] = {K + (int64_t)b * sb + (int64_t)h * sh + e, V + (int64_t)b * sb + (int64_t)h * sh + e};
    Bytes w[2][kPass];
    float f[2][kPass];
    bool there[kPass];
#pragma unroll
    for (int p = 0; p < kPass; ++p) {
        const int t = t1 + p * kTok;
        there[p] = t < stop && t < paged;
        if (there[p]) {
            const int page = c.table[(size_t)b * s.nb + (t >> s.lb)];
            if (page < 0 || page >= s.n_pages) {
                there[p] = false;
                q8_report(c.status, FA_ERR_INDEX);
            } else {
                const size_t ph = (size_t)page * s.H + h, at = (ph * (size_t)s.blk + (t & (s.blk - 1))) * D + e;
                w[0][p] = __ldg(reinterpret_cast<const Bytes*>(c.k_pages + at));
                w[1][p] = __ldg(reinterpret_cast<const Bytes*>(c.v_pages + at));
                f[0][p] = __ldg(c.k_scale + ph);
                f[1][p] = __ldg(c.v_scale + ph);
            }
        }
    }
#pragma unroll
    for (int p = 0; p < kPass; ++p) {
        const int t = t1 + p * kTok;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            T* to = out[side] + (int64_t)(t - t0) * st;
            if (there[p]) {                                          // (the lanes of a token agree)
                float x[4];
                if constexpr (kE == 16) {
                    const uint32_t ws[4] = {w[side][p].x, w[side][p].y, w[side][p].z, w[side][p].w};
                    uint32_t o[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        q8_floats<FMT>(ws[i], f[side][p], x);
                        const __nv_bfloat162 lo = __floats2bfloat162_rn(x[0], x[1]), hi = __floats2bfloat162_rn(x[2], x[3]);
                        o[2 * i] = *reinterpret_cast<const uint32_t*>(&lo);
                        o[2 * i + 1] = *reinterpret_cast<const uint32_t*>(&hi);
                    }
                    // the even lane gives its second 16 bytes for the odd lane's first: the first store is the even lane's 32 bytes, by both
                    const bool odd = threadIdx.x & 1;
                    const unsigned both = 3u << (threadIdx.x & 30);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t got = __shfl_xor_sync(both, odd ? o[i] : o[4 + i], 1);
                        if (odd) { o[i] = got; } else { o[4 + i] = got; }
                    }
                    *reinterpret_cast<uint4*>(to + (odd ? -8 : 0)) = make_uint4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<uint4*>(to + (odd ? 8 : 16)) = make_uint4(o[4], o[5], o[6], o[7]);
                } else {
                    q8_floats<FMT>(w[side][p], f[side][p], x);
                    *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
                }
            } else if (t >= paged && t < stop) {                     // the tail: as it is
                const T* tail = reinterpret_cast<const T*>(side ? c.v_tail : c.k_tail) + (((size_t)b * s.H + h) * (size_t)s.blk + (t - paged)) * D + e;
#pragma unroll
                for (int i = 0; i < kE * (int)sizeof(T) / 16; ++i) *(reinterpret_cast<uint4*>(to) + i) = *(reinterpret_cast<const uint4*>(tail) + i);
            }
        }
    }
}

__global__ void __launch_bounds__(256) q8_reset_kernel(int32_t* __restrict__ state, int n, int32_t* __restrict__ status) {
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) state[i] = 0;
    if (i < 4) status[i] = 0;
}

template <typename T, int FMT, int NV>
cudaError_t store_launch(StoreArgs<T> a, long long touched, cudaStream_t stream) {
    const int groups = kStoreThreads * NV * 16 / (a.s.blk * a.s.d);
    // runs of up to 8 blocks, as long as there are eight CTAs for each SM
    const long long ctas = (touched + groups - 1) / groups * 2 * a.s.H * a.s.B, run = ctas / (8 * sm_count());
    a.run = (int)(run < 1 ? 1 : run > 8 ? 8 : run);
    const long long per = (long long)a.run * groups;
    return launch_behind(q8_store_kernel<T, FMT, NV>, dim3((unsigned)((touched + per - 1) / per), (unsigned)(2 * a.s.H), (unsigned)a.s.B), kStoreThreads, 0, stream, a);
}
template <typename T, int FMT>
cudaError_t store_of(const Q8Dims& s, const Q8Cache& c, const void* K, const void* V, int64_t sb, int64_t st, int64_t sh, int n, const int32_t* n_row,
                     bool append, cudaStream_t stream) {
    // blocks that n tokens can touch behind a tail of blk - 1
    int64_t touched = n == 0 ? 1 : ((int64_t)(append ? s.blk - 1 : 0) + n - 1) / s.blk + 1;
    if (touched > s.nb + 1) touched = s.nb + 1;           // (rows that would need more are refused)
    const StoreArgs<T> a = {s, c, static_cast<const T*>(K), static_cast<const T*>(V), sb, st, sh, n, n_row, append, 1, s.d == 64 ? 6 : s.d == 128 ? 7 : 8};
    // 32 values to a thread, so that a block of the smallest size is a warp's; 64 or 128 where it is more than 256 threads'
    const int values = s.blk * s.d;
    return values <= 8192 ? store_launch<T, FMT, 2>(a, touched, stream)
                          : values <= 16384 ? store_launch<T, FMT, 4>(a, touched, stream) : store_launch<T, FMT, 8>(a, touched, stream);
}
template <typename T, int FMT, int D>
cudaError_t read_of(const Q8Dims& s, const Q8Cache& c, void* K, void* V, int64_t sb, int64_t st, int64_t sh, int t0, int n, cudaStream_t stream) {
    const int tok = kReadPass<T> * 256 * kReadE<T> / D;
    const int64_t tiles = ((int64_t)n + tok - 1) / tok;
    return launch_behind(q8_read_kernel<T, FMT, D>, dim3((unsigned)(tiles * s.H), (unsigned)s.B), 256, 0, stream, s, c, static_cast<T*>(K), static_cast<T*>(V), sb, st, sh, t0, n);
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

cudaError_t launch_q8_reset(const Q8Dims& s, const Q8Cache& c, cudaStream_t stream) {
    const int n = s.B * kQ8State;
    return launch_behind(q8_reset_kernel, dim3((unsigned)((n + 255) / 256)), 256, 0, stream, c.state, n, c.status);
}
cudaError_t launch_q8_store(const Q8Dims& s, const Q8Cache& c, int fmt, int dtype, const void* K, const void* V, int64_t sb, int64_t st, int64_t sh, int n,
                            const int32_t* n_row, bool append, cudaStream_t stream) {
    if (dtype == FA_BF16)
        return fmt == FA_Q8_INT8 ? store_of<__nv_bfloat16, FA_Q8_INT8>(s, c, K, V, sb, st, sh, n, n_row, append, stream)
                                 : store_of<__nv_bfloat16, FA_Q8_E4M3>(s, c, K, V, sb, st, sh, n, n_row, append, stream);
    return fmt == FA_Q8_INT8 ? store_of<float, FA_Q8_INT8>(s, c, K, V, sb, st, sh, n, n_row, append, stream)
                             : store_of<float, FA_Q8_E4M3>(s, c, K, V, sb, st, sh, n, n_row, append, stream);
}
cudaError_t launch_q8_read(const Q8Dims& s, const Q8Cache& c, int fmt, int dtype, void* K, void* V, int64_t sb, int64_t st, int64_t sh, int t0, int n,
                           cudaStream_t stream) {
#define FA_Q8_CALL(T, F, D) read_of<T, F, D>(s, c, K, V, sb, st, sh, t0, n, stream)
    FA_Q8_DISPATCH(FA_Q8_CALL);
#undef FA_Q8_CALL
}

}  // namespace fa
