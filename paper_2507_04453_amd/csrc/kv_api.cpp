// Host glue of the 4-bit key/value cache: argument checks and the launches behind the essa_kv_* entry points.
#include <new>

#include "kv_internal.h"

static bool sizes_valid(const essa_kv_desc& d) {
    const bool page = d.page_tokens >= 32 && d.page_tokens <= 1024 && (d.page_tokens & (d.page_tokens - 1)) == 0;
    return page && d.layers >= 1 && d.layers <= 1024 && d.n_kv_heads >= 1 && d.n_kv_heads <= 1024 && (d.head_dim == 64 || d.head_dim == 128) &&
           d.n_pages >= 1 && d.n_pages <= (1 << 18) && d.max_seqs >= 1 && d.max_seqs <= 4096 && d.max_pages >= 1 &&
           (int64_t)d.max_pages * d.page_tokens < ((int64_t)1 << 31);
}
static size_t page_bytes(const essa_kv_desc& d) {
    return (size_t)d.layers * d.n_kv_heads * (d.page_tokens / essa_k::kKvBlock) * essa_k::kv_block_bytes(d.head_dim);
}

extern "C" size_t essa_kv_pool_bytes(const essa_kv_desc* d) { return d && sizes_valid(*d) ? page_bytes(*d) * d->n_pages : 0; }

extern "C" void essa_kv_destroy(essa_kv* kv) {
    if (!kv) return;
    (void)hipSetDevice(kv->device);
    (void)hipDeviceSynchronize();
    if (kv->scratch) (void)hipFree(kv->scratch);
    delete kv;
}

extern "C" essa_status essa_kv_create(essa_ctx* ctx, const essa_kv_desc* d, essa_kv** out) {
    if (!ctx || !d || !out) return essa_fail(ESSA_ERR_INVALID_ARG, "essa_kv_create: NULL argument");
    *out = nullptr;
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim > 0)
        return essa_fail(ESSA_ERR_UNSUPPORTED, "essa_kv_create: head_dim=%d, built for 64 and 128", d->head_dim);
    if (!sizes_valid(*d))
        return essa_fail(ESSA_ERR_SHAPE, "essa_kv_create: layers=%d n_kv_heads=%d head_dim=%d page_tokens=%d n_pages=%d max_seqs=%d max_pages=%d", d->layers,
                         d->n_kv_heads, d->head_dim, d->page_tokens, d->n_pages, d->max_seqs, d->max_pages);
    if (!d->pool || !d->table || !d->len || !d->refs) return essa_fail(ESSA_ERR_INVALID_ARG, "essa_kv_create: NULL array");
    if ((uintptr_t)d->pool & 15) return essa_fail(ESSA_ERR_INVALID_ARG, "essa_kv_create: the pool must begin on 16 bytes");
    if (ctx->capturing) return essa_fail(ESSA_ERR_STATE, "essa_kv_create: not while a graph is being recorded");
    ESSA_HIP(hipSetDevice(ctx->device));
    essa_kv* kv = new (std::nothrow) essa_kv();
    if (!kv) return essa_fail(ESSA_ERR_OOM, "essa_kv_create: out of host memory");
    kv->ctx = ctx;
    kv->device = ctx->device;
    kv->d = *d;
    while ((essa_k::kKvBlock << kv->page_shift) < d->page_tokens) ++kv->page_shift;
    const size_t bytes = essa_k::kv_scratch_words(*d) * sizeof(int32_t);
    hipError_t e = hipMalloc((void**)&kv->scratch, bytes);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        delete kv;
        return essa_fail(ESSA_ERR_OOM, "essa_kv_create: hipMalloc of %zu bytes: %s", bytes, hipGetErrorString(e));
    }
    e = essa_k::kv_clear(ctx->stream, kv);
    if (e != hipSuccess) {
        essa_kv_destroy(kv);
        return essa_fail(ESSA_ERR_HIP, "essa_kv_create: %s", hipGetErrorString(e));
    }
    *out = kv;
    return ESSA_OK;
}

static essa_status check_kv(const essa_ctx* ctx, const essa_kv* kv, const char* who) {
    if (!ctx || !kv) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (kv->ctx != ctx) return essa_fail(ESSA_ERR_STATE, "%s: the cache belongs to another context", who);
    return ESSA_OK;
}
static essa_status check_entries(const essa_kv* kv, int n, const char* who) {
    if (n < 0 || n > kv->d.max_seqs) return essa_fail(ESSA_ERR_SHAPE, "%s: n=%d not in [0, max_seqs=%d]", who, n, kv->d.max_seqs);
    return ESSA_OK;
}

extern "C" essa_status essa_kv_extend(essa_ctx* ctx, essa_kv* kv, const int32_t* seqs, const int32_t* n_new, int n, int32_t* served) {
    ESSA_TRY(check_kv(ctx, kv, "essa_kv_extend"));
    ESSA_TRY(check_entries(kv, n, "essa_kv_extend"));
    if (n == 0) return ESSA_OK;
    if (!seqs || !n_new) return essa_fail(ESSA_ERR_INVALID_ARG, "essa_kv_extend: NULL argument");
    ESSA_HIP(hipSetDevice(ctx->device));
    ESSA_HIP(essa_k::kv_extend(ctx->stream, kv, seqs, n_new, n, served));
    return ESSA_OK;
}

extern "C" essa_status essa_kv_fork(essa_ctx* ctx, essa_kv* kv, const int32_t* src, const int32_t* dst, const int32_t* len, int n, int32_t* served) {
    ESSA_TRY(check_kv(ctx, kv, "essa_kv_fork"));
    ESSA_TRY(check_entries(kv, n, "essa_kv_fork"));
    if (n == 0) return ESSA_OK;
    if (!src || !dst) return essa_fail(ESSA_ERR_INVALID_ARG, "essa_kv_fork: NULL argument");
    ESSA_HIP(hipSetDevice(ctx->device));
    ESSA_HIP(essa_k::kv_fork(ctx->stream, kv, src, dst, len, n, served));
    return ESSA_OK;
}

extern "C" essa_status essa_kv_free(essa_ctx* ctx, essa_kv* kv, const int32_t* seqs, int n) {
    ESSA_TRY(check_kv(ctx, kv, "essa_kv_free"));
    ESSA_TRY(check_entries(kv, n, "essa_kv_free"));
    if (n == 0) return ESSA_OK;
    if (!seqs) return essa_fail(ESSA_ERR_INVALID_ARG, "essa_kv_free: NULL argument");
    ESSA_HIP(hipSetDevice(ctx->device));
    ESSA_HIP(essa_k::kv_fork(ctx->stream, kv, nullptr, seqs, nullptr, n, nullptr));
    return ESSA_OK;
}

extern "C" essa_status essa_kv_compact(essa_ctx* ctx, essa_kv* kv, int32_t* map_out, int32_t* used_out) {
    ESSA_TRY(check_kv(ctx, kv, "essa_kv_compact"));
    ESSA_HIP(hipSetDevice(ctx->device));
    ESSA_HIP(essa_k::kv_compact(ctx->stream, kv, map_out, used_out));
    return ESSA_OK;
}

// ---------------------------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------------------------
static essa_status check_rows(const essa_kv* kv, int layer, const essa_kv_batch* b, const char* who) {
    if (!b) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: NULL argument", who);
    ESSA_TRY(check_entries(kv, b->n, who));
    if (layer < 0 || layer >= kv->d.layers) return essa_fail(ESSA_ERR_SHAPE, "%s: layer=%d not in [0, %d)", who, layer, kv->d.layers);
    if (b->R < 0 || b->R > (1 << 24)) return essa_fail(ESSA_ERR_SHAPE, "%s: R=%d not in [0, 2^24]", who, b->R);
    if (!b->row_start && b->R != b->n) return essa_fail(ESSA_ERR_SHAPE, "%s: one row an entry, but R=%d and n=%d", who, b->R, b->n);
    if (b->n > 0 && !b->seqs) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: seqs is NULL", who);
    if (b->n == 0 && b->R > 0) return essa_fail(ESSA_ERR_SHAPE, "%s: R=%d rows and no entries", who, b->R);
    return ESSA_OK;
}
static essa_status make_tensor(essa_k::kv_tensor* t, const void* p, int64_t stride, int dtype, int64_t width, const char* name, const char* who) {
    if (!p) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
    if (dtype != ESSA_F32 && dtype != ESSA_BF16) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: %s has dtype %d", who, name, dtype);
    if (stride < width || stride > ((int64_t)1 << 32)) return essa_fail(ESSA_ERR_SHAPE, "%s: rows of %s are %lld values wide, %lld apart", who, name, (long long)width, (long long)stride);
    const size_t size = dtype == ESSA_F32 ? 4 : 2;
    if ((uintptr_t)p % size) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: %s is not aligned to its values", who, name);
    t->p = const_cast<void*>(p);
    t->stride = stride;
    t->dtype = dtype;
    t->aligned = ((uintptr_t)p % 16 == 0) && (stride * size % 16 == 0);
    return ESSA_OK;
}
static essa_k::kv_view view_of(const essa_kv* kv, int layer) {
    const essa_kv_desc& d = kv->d;
    essa_k::kv_view v;
    v.page_bytes = (long long)page_bytes(d);
    v.pool = (unsigned char*)d.pool + (size_t)layer * (page_bytes(d) / d.layers);
    v.table = d.table;
    v.len = d.len;
    v.heads = d.n_kv_heads;
    v.page_shift = kv->page_shift;
    v.n_pages = d.n_pages;
    v.max_seqs = d.max_seqs;
    v.max_pages = d.max_pages;
    v.max_len = essa_k::kv_max_len(d);
    return v;
}
static essa_k::kv_rows rows_of(const essa_kv_batch* b) { return {b->seqs, b->row_start, b->n, b->R}; }

extern "C" essa_status essa_kv_accept(essa_ctx* ctx, essa_kv* kv, const essa_kv_batch* batch, const int32_t* path, const int32_t* keep, int32_t* served) {
    ESSA_TRY(check_kv(ctx, kv, "essa_kv_accept"));
    ESSA_TRY(check_rows(kv, 0, batch, "essa_kv_accept"));
    if (batch->n == 0) return ESSA_OK;
    if (!keep || (batch->R > 0 && !path)) return essa_fail(ESSA_ERR_INVALID_ARG, "essa_kv_accept: NULL argument");
    ESSA_HIP(hipSetDevice(ctx->device));
    ESSA_HIP(essa_k::kv_accept(ctx->stream, kv, rows_of(batch), path, keep, served));
    return ESSA_OK;
}

extern "C" essa_status essa_kv_append(essa_ctx* ctx, essa_kv* kv, int layer, const void* K, int64_t k_stride, const void* V, int64_t v_stride, int x_dtype,
                                      const essa_kv_batch* batch) {
    ESSA_TRY(check_kv(ctx, kv, "essa_kv_append"));
    ESSA_TRY(check_rows(kv, layer, batch, "essa_kv_append"));
    if (batch->R == 0) return ESSA_OK;
    const int64_t width = (int64_t)kv->d.n_kv_heads * kv->d.head_dim;
    essa_k::kv_tensor k, v;
    ESSA_TRY(make_tensor(&k, K, k_stride, x_dtype, width, "K", "essa_kv_append"));
    ESSA_TRY(make_tensor(&v, V, v_stride, x_dtype, width, "V", "essa_kv_append"));
    ESSA_HIP(hipSetDevice(ctx->device));
    ESSA_HIP(essa_k::kv_append(ctx->stream, view_of(kv, layer), kv->d.head_dim, k, v, rows_of(batch)));
    return ESSA_OK;
}

extern "C" essa_status essa_kv_read(essa_ctx* ctx, const essa_kv* kv, int layer, void* K, int64_t k_stride, void* V, int64_t v_stride, int y_dtype,
                                    const essa_kv_batch* batch) {
    ESSA_TRY(check_kv(ctx, kv, "essa_kv_read"));
    ESSA_TRY(check_rows(kv, layer, batch, "essa_kv_read"));
    if (batch->R == 0) return ESSA_OK;
    const int64_t width = (int64_t)kv->d.n_kv_heads * kv->d.head_dim;
    essa_k::kv_tensor k, v;
    ESSA_TRY(make_tensor(&k, K, k_stride, y_dtype, width, "K", "essa_kv_read"));
    ESSA_TRY(make_tensor(&v, V, v_stride, y_dtype, width, "V", "essa_kv_read"));
    ESSA_HIP(hipSetDevice(ctx->device));
    ESSA_HIP(essa_k::kv_read(ctx->stream, view_of(kv, layer), kv->d.head_dim, k, v, rows_of(batch)));
    return ESSA_OK;
}

static essa_status attention(const char* who, essa_ctx* ctx, const essa_kv* kv, int layer, const void* Q, int64_t q_stride, int x_dtype, int n_q_heads,
                             const essa_kv_batch* batch, float scale, int window, uint32_t flags, const essa_k::kv_mask& mask, void* Y, int64_t y_stride, int y_dtype) {
    ESSA_TRY(check_kv(ctx, kv, who));
    ESSA_TRY(check_rows(kv, layer, batch, who));
    if (n_q_heads < 1 || n_q_heads > 32768 || n_q_heads % kv->d.n_kv_heads)
        return essa_fail(ESSA_ERR_SHAPE, "%s: %d query heads on %d key heads", who, n_q_heads, kv->d.n_kv_heads);
    if (flags & ~ESSA_KV_ALL) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: unknown flags 0x%x", who, flags);
    if (window < 0 || (window > 0 && (flags & ESSA_KV_ALL)))
        return essa_fail(ESSA_ERR_INVALID_ARG, "%s: window=%d%s", who, window, window < 0 ? "" : " together with ESSA_KV_ALL");
    const float scale2 = scale * essa_k::kLog2e;               // what the kernels take: exponents of 2
    if (!(scale2 - scale2 == 0.0f)) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: scale=%g, it and its product with log2(e) have to be finite", who, (double)scale);
    if (batch->R == 0) return ESSA_OK;
    const int64_t width = (int64_t)n_q_heads * kv->d.head_dim;
    if (batch->R * (int64_t)n_q_heads >= ((int64_t)1 << 31)) return essa_fail(ESSA_ERR_SHAPE, "%s: R=%d rows of %d heads", who, batch->R, n_q_heads);
    essa_k::kv_tensor q, y;
    ESSA_TRY(make_tensor(&q, Q, q_stride, x_dtype, width, "Q", who));
    ESSA_TRY(make_tensor(&y, Y, y_stride, y_dtype, width, "Y", who));
    ESSA_HIP(hipSetDevice(ctx->device));
    const essa_k::kv_view v = view_of(kv, layer);
    const essa_k::kv_rows rows = rows_of(batch);
    ESSA_TRY(essa_ws_reserve(ctx, essa_k::kv_attention_bytes(v, kv->d.head_dim, n_q_heads, rows, x_dtype)));
    ESSA_HIP(essa_k::kv_attention(ctx->stream, v, kv->d.head_dim, q, y, n_q_heads, rows, scale2, window, (flags & ESSA_KV_ALL) != 0,
                                  essa_k::kv_scratch_of(kv).done, ctx->ws, mask));
    return ESSA_OK;
}

extern "C" essa_status essa_kv_attention(essa_ctx* ctx, const essa_kv* kv, int layer, const void* Q, int64_t q_stride, int x_dtype, int n_q_heads,
                                         const essa_kv_batch* batch, float scale, int window, uint32_t flags, void* Y, int64_t y_stride, int y_dtype) {
    return attention("essa_kv_attention", ctx, kv, layer, Q, q_stride, x_dtype, n_q_heads, batch, scale, window, flags, {}, Y, y_stride, y_dtype);
}

extern "C" essa_status essa_kv_attention_masked(essa_ctx* ctx, const essa_kv* kv, int layer, const void* Q, int64_t q_stride, int x_dtype, int n_q_heads,
                                                const essa_kv_batch* batch, float scale, const essa_kv_mask* mask, void* Y, int64_t y_stride, int y_dtype) {
    const char* who = "essa_kv_attention_masked";
    if (!mask) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (mask->sinks < 0) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: sinks=%d", who, mask->sinks);
    if (mask->tree_words < 0 || mask->tree_words > ESSA_KV_TREE_WORDS)
        return essa_fail(ESSA_ERR_SHAPE, "%s: tree_words=%d not in [0, %d]", who, mask->tree_words, ESSA_KV_TREE_WORDS);
    if (mask->tree_words > 0 && batch && batch->R > 0 && !mask->tree) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: tree is NULL", who);
    if (mask->tree_words > 0 && (uintptr_t)mask->tree % 8) return essa_fail(ESSA_ERR_INVALID_ARG, "%s: tree is not aligned to its words", who);
    return attention(who, ctx, kv, layer, Q, q_stride, x_dtype, n_q_heads, batch, scale, mask->window, 0, {mask->sinks, mask->tree_words, mask->tree}, Y, y_stride, y_dtype);
}
