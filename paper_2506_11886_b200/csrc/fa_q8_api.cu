// Host side of the dense cache in 8 bits: argument checks and launches of the fa_q8_* entry points of include/fa.h.
#include "fa_q8.cuh"

namespace fa {
namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

fa_status check_q8_layout(const fa_q8_layout* l) {
    if (!l) return FA_ERR_INVALID_ARG;
    if (l->batch < 1 || l->n_q_heads < 1 || l->n_kv_heads < 1 || l->head_dim < 1 || l->block < 1 || l->max_blocks < 1 || l->n_pages < 0) return FA_ERR_INVALID_ARG;
    if (l->n_q_heads % l->n_kv_heads != 0) return FA_ERR_INVALID_ARG;
    if (l->format != FA_Q8_INT8 && l->format != FA_Q8_E4M3) return FA_ERR_INVALID_ARG;
    if (l->kv_dtype != FA_F32 && l->kv_dtype != FA_BF16) return FA_ERR_INVALID_ARG;
    if (!(l->softmax_scale > 0.0f)) return FA_ERR_INVALID_ARG;
    if (l->head_dim != 64 && l->head_dim != 128 && l->head_dim != 256) return FA_ERR_UNSUPPORTED;
    if (l->block != 16 && l->block != 32 && l->block != 64 && l->block != 128) return FA_ERR_UNSUPPORTED;
    if (l->n_q_heads / l->n_kv_heads > 16) return FA_ERR_UNSUPPORTED;
    if (l->batch > 65535 || l->n_kv_heads > 4096) return FA_ERR_UNSUPPORTED;
    if ((int64_t)l->max_blocks * l->block > (1 << 30)) return FA_ERR_UNSUPPORTED;         // token counts are 32 bits
    if ((int64_t)l->n_pages * l->n_kv_heads * (l->block / 16) >= 0xfffffffell) return FA_ERR_UNSUPPORTED;      // 16 tokens of a head are counted in 32 bits
    return FA_OK;
}

fa_status check_q8_cache(const fa_q8_layout* l, const fa_q8_cache* c) {
    if (!c) return FA_ERR_INVALID_ARG;
    const void* always[] = {c->k_tail, c->v_tail, c->tail_amax, c->block_table, c->state, c->status};
    for (const void* p : always)
        if (!p || !aligned16(p)) return FA_ERR_INVALID_ARG;
    const void* paged[] = {c->k_pages, c->v_pages, c->k_scale, c->v_scale};
    for (const void* p : paged)
        if ((l->n_pages > 0 && !p) || !aligned16(p)) return FA_ERR_INVALID_ARG;
    return FA_OK;
}

fa_status check_tokens(const fa_q8_layout* l, const void* K, const void* V, int64_t sb, int64_t st, int64_t sh, int32_t n) {
    if (n < 0) return FA_ERR_INVALID_ARG;
    if (n == 0) return FA_OK;
    if (!K || !V || !aligned16(K) || !aligned16(V)) return FA_ERR_INVALID_ARG;
    if (sb < 0 || st < l->head_dim || sh < l->head_dim || ((sb | st | sh) & 7)) return FA_ERR_INVALID_ARG;
    // a launch's blocks of all rows and heads are counted in 32 bits
    const int64_t blocks = (int64_t)n / l->block + 2, most = (int64_t)l->max_blocks + 1;
    if ((blocks < most ? blocks : most) * 2 * l->n_kv_heads * l->batch > 0x7fffffff) return FA_ERR_UNSUPPORTED;
    return FA_OK;
}

fa_status store_call(const fa_q8_layout* layout, fa_q8_cache* cache, const void* K, const void* V, int64_t sb, int64_t st, int64_t sh, int32_t n,
                     const int32_t* n_row, bool append, void* stream) {
    fa_status e = check_q8_layout(layout);
    if (e == FA_OK) e = check_q8_cache(layout, cache);
    if (e == FA_OK) e = check_tokens(layout, K, V, sb, st, sh, n);
    if (e != FA_OK) return e;
    if (n == 0 && append) return FA_OK;
    return launch_q8_store(make_q8_dims(*layout), make_q8_cache(*cache), layout->format, layout->kv_dtype, K, V, sb, st, sh, n, n_row, append,
                           static_cast<cudaStream_t>(stream)) == cudaSuccess ? FA_OK : FA_ERR_CUDA;
}

fa_status attention_call(const fa_q8_layout* layout, const fa_q8_cache* cache, const void* q, int64_t sb, int64_t si, int64_t sg, void* out, int32_t n_q,
                         const void* k_new, const void* v_new, void* ws, size_t ws_bytes, void* stream) {
    if (!q || !out || !aligned16(q) || !aligned16(out)) return FA_ERR_INVALID_ARG;
    if (sb < 0 || si < layout->head_dim || sg < layout->head_dim || ((sb | si | sg) & 7)) return FA_ERR_INVALID_ARG;
    const Q8Dims s = make_q8_dims(*layout);
    if (!(k_new == nullptr && q8_chunk_takes(s, layout->kv_dtype, n_q)) && !q8_attention_fits(s, n_q)) return FA_ERR_UNSUPPORTED;
    if (!ws || !aligned16(ws) || ws_bytes < q8_attention_ws_bytes(s, n_q)) return FA_ERR_WORKSPACE;
    return launch_q8_attention(s, make_q8_cache(*cache), layout->format, layout->kv_dtype, q, sb, si, sg, out, n_q, k_new, v_new, static_cast<char*>(ws),
                               static_cast<cudaStream_t>(stream)) == cudaSuccess ? FA_OK : FA_ERR_CUDA;
}

}  // namespace
}  // namespace fa

using namespace fa;

extern "C" {

fa_status fa_q8_cache_sizes_of(const fa_q8_layout* l, fa_q8_cache_sizes* out) {
    const fa_status e = check_q8_layout(l);
    if (e != FA_OK) return e;
    if (!out) return FA_ERR_INVALID_ARG;
    const size_t eb = l->kv_dtype == FA_BF16 ? 2 : 4, heads = (size_t)l->n_kv_heads, blk = (size_t)l->block * l->head_dim;
    out->k_pages = out->v_pages = (size_t)l->n_pages * heads * blk;
    out->k_scale = out->v_scale = (size_t)l->n_pages * heads * 4;
    out->k_tail = out->v_tail = (size_t)l->batch * heads * blk * eb;
    out->tail_amax = (size_t)l->batch * heads * 2 * 4;
    out->block_table = (size_t)l->batch * l->max_blocks * 4;
    out->state = (size_t)l->batch * kQ8State * 4;
    out->status = 4 * 4;
    return FA_OK;
}

fa_status fa_q8_workspace_bytes(const fa_q8_layout* layout, int32_t n_q, size_t* out) {
    const fa_status e = check_q8_layout(layout);
    if (e != FA_OK) return e;
    if (!out || n_q < 1) return FA_ERR_INVALID_ARG;
    *out = q8_attention_ws_bytes(make_q8_dims(*layout), n_q);
    return FA_OK;
}

fa_status fa_q8_reset(const fa_q8_layout* layout, fa_q8_cache* cache, void* stream) {
    fa_status e = check_q8_layout(layout);
    if (e == FA_OK) e = check_q8_cache(layout, cache);
    if (e != FA_OK) return e;
    return launch_q8_reset(make_q8_dims(*layout), make_q8_cache(*cache), static_cast<cudaStream_t>(stream)) == cudaSuccess ? FA_OK : FA_ERR_CUDA;
}

fa_status fa_q8_write(const fa_q8_layout* layout, fa_q8_cache* cache, const void* K, const void* V, int64_t stride_b, int64_t stride_t, int64_t stride_h,
                      int32_t n, const int32_t* n_row, void* stream) {
    return store_call(layout, cache, K, V, stride_b, stride_t, stride_h, n, n_row, false, stream);
}

fa_status fa_q8_append(const fa_q8_layout* layout, fa_q8_cache* cache, const void* K, const void* V, int64_t stride_b, int64_t stride_t, int64_t stride_h,
                       int32_t n, const int32_t* n_row, void* stream) {
    return store_call(layout, cache, K, V, stride_b, stride_t, stride_h, n, n_row, true, stream);
}

fa_status fa_q8_read(const fa_q8_layout* layout, const fa_q8_cache* cache, void* K, void* V, int64_t stride_b, int64_t stride_t, int64_t stride_h, int32_t t0,
                     int32_t n, void* stream) {
    fa_status e = check_q8_layout(layout);
    if (e == FA_OK) e = check_q8_cache(layout, cache);
    if (e == FA_OK) e = check_tokens(layout, K, V, stride_b, stride_t, stride_h, n);
    if (e != FA_OK) return e;
    if (t0 < 0 || n > 0x7fffffff - t0) return FA_ERR_INVALID_ARG;
    const int32_t cap = layout->max_blocks * layout->block;
    if (t0 >= cap) return FA_OK;
    if (n > cap - t0) n = cap - t0;                        // (no row has more)
    if (n == 0) return FA_OK;
    return launch_q8_read(make_q8_dims(*layout), make_q8_cache(*cache), layout->format, layout->kv_dtype, K, V, stride_b, stride_t, stride_h, t0, n,
                          static_cast<cudaStream_t>(stream)) == cudaSuccess ? FA_OK : FA_ERR_CUDA;
}

fa_status fa_q8_attention(const fa_q8_layout* layout, const fa_q8_cache* cache, const void* q, int64_t stride_b, int64_t stride_i, int64_t stride_g, void* out,
                          int32_t n_q, void* ws, size_t ws_bytes, void* stream) {
    fa_status e = check_q8_layout(layout);
    if (e == FA_OK) e = check_q8_cache(layout, cache);
    if (e != FA_OK) return e;
    if (n_q < 0) return FA_ERR_INVALID_ARG;
    if (n_q == 0) return FA_OK;
    if ((int64_t)n_q * layout->n_q_heads > (1 << 26)) return FA_ERR_UNSUPPORTED;          // column tiles are 32 bits
    return attention_call(layout, cache, q, stride_b, stride_i, stride_g, out, n_q, nullptr, nullptr, ws, ws_bytes, stream);
}

fa_status fa_q8_step(const fa_q8_layout* layout, fa_q8_cache* cache, const void* q, const void* k_new, const void* v_new, void* out, void* ws,
                     size_t ws_bytes, void* stream) {
    fa_status e = check_q8_layout(layout);
    if (e == FA_OK) e = check_q8_cache(layout, cache);
    if (e != FA_OK) return e;
    if (!k_new || !v_new || !aligned16(k_new) || !aligned16(v_new)) return FA_ERR_INVALID_ARG;
    const int64_t row = (int64_t)layout->n_q_heads * layout->head_dim;
    return attention_call(layout, cache, q, row, row, layout->head_dim, out, 1, k_new, v_new, ws, ws_bytes, stream);
}

fa_status fa_q8_poll_status(const fa_q8_cache* cache, void* stream) {
    if (!cache || !cache->status) return FA_ERR_INVALID_ARG;
    fa_cache c = {};
    c.status = cache->status;
    return fa_poll_status(&c, stream);
}

}  // extern "C"
