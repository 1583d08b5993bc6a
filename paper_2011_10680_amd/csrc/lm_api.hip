// C interface of the language-model operators: host-side argument validation and dispatch.  Nothing here touches device memory.
#include <algorithm>
#include <cmath>

#include "lm.h"

using namespace hawq;

namespace {

bool float16(int dt) { return dt == HAWQ_F16 || dt == HAWQ_BF16; }
bool at_multiple(int bytes, std::initializer_list<const void *> pointers) {
    uintptr_t any = 0;
    for (const void *p : pointers) any |= (uintptr_t)p;
    return (any & (uintptr_t)(bytes - 1)) == 0;
}

const int64_t kMostStride = (int64_t)1 << 40;
const int kMostKeys = INT32_MAX - 255;      // of a row: the kernels count them in 32 bits, whole tiles at a time

// strides of a tensor that is read: any that keep addresses inside 64 bits, 0 for a broadcast axis
bool strides_ok(int64_t token, int64_t head) { return token >= 0 && head >= 0 && token <= kMostStride && head <= kMostStride; }

// a number of rows times a stride, up to 2^71
typedef __int128 Extent;

// strides of a tensor [n][heads][dim] that is written: no two rows overlap, whichever of the two axes is the outer one
bool rows_apart(int64_t token, int64_t head, int64_t n, int64_t heads, int64_t dim) {
    if (!strides_ok(token, head) || (heads > 1 && head < dim) || (n > 1 && token < dim)) return false;
    return n <= 1 || heads <= 1 || token >= (Extent)(heads - 1) * head + dim || head >= (Extent)(n - 1) * token + dim;
}

hawq_status check_cache(const hawq_cache_desc &c, int dtype, const void *k, const void *v, const float *ks, const float *vs, bool pointers) {
    if (c.n_pages < 0 || c.page <= 0 || c.kv_heads <= 0 || c.head_dim <= 0 || c.head_dim > 256) return HAWQ_ERR_SHAPE;
    if (c.dtype != dtype && c.dtype != HAWQ_S8) return HAWQ_ERR_DTYPE;
    if (!rows_apart(c.token_stride, c.head_stride, c.page, c.kv_heads, c.head_dim)) return HAWQ_ERR_SHAPE;
    const Extent tokens = (Extent)(c.page - 1) * c.token_stride + c.head_dim, extent = tokens + (Extent)(c.kv_heads - 1) * c.head_stride;
    if (c.n_pages > 1 && (c.page_stride < c.head_dim || c.page_stride > kMostStride)) return HAWQ_ERR_SHAPE;
    // pages one behind the other (or the page axis inside the heads', each head's pages together)
    if (c.n_pages > 1 && c.page_stride < extent && !(c.kv_heads > 1 && c.head_stride >= (Extent)(c.n_pages - 1) * c.page_stride + tokens && c.page_stride >= tokens))
        return HAWQ_ERR_SHAPE;
    if (!pointers) return HAWQ_OK;
    if (c.n_pages > 0 && (!k || !v)) return HAWQ_ERR_NULL;
    if (c.dtype == HAWQ_S8) {
        if (c.n_pages > 0 && (!ks || !vs)) return HAWQ_ERR_NULL;
    } else if (ks || vs) return HAWQ_ERR_DTYPE;
    if (!at_multiple(c.dtype == HAWQ_S8 ? 1 : 2, {k, v}) || !at_multiple(4, {ks, vs})) return HAWQ_ERR_UNSUPPORTED;
    return HAWQ_OK;
}

CacheArgs cache_args(const hawq_cache_desc &c, const void *k, const void *v, const float *ks, const float *vs) {
    return {const_cast<void *>(k), const_cast<void *>(v), const_cast<float *>(ks), const_cast<float *>(vs), c.n_pages, c.page, c.dtype, fast_div((uint32_t)c.page),
            c.page_stride, c.token_stride, c.head_stride};
}

hawq_status tree_args(const hawq_attn_tree_desc *d, AttnTreeArgs &a) {
    if (!d) return HAWQ_ERR_NULL;
    const int kv = d->cache.kv_heads;
    if (d->n_seqs < 0 || d->total < 0 || d->max_drafts < 1 || d->max_drafts > 64 || d->max_cached < 0 || d->q_heads <= 0 || d->table_stride < 0) return HAWQ_ERR_SHAPE;
    if (!float16(d->dtype)) return HAWQ_ERR_DTYPE;
    const hawq_status st = check_cache(d->cache, d->dtype, nullptr, nullptr, nullptr, nullptr, false);
    if (st != HAWQ_OK) return st;
    if (d->q_heads % kv != 0) return HAWQ_ERR_SHAPE;
    if (!std::isfinite(d->scale)) return HAWQ_ERR_RANGE;
    if (!strides_ok(d->q_token, d->q_head) || !strides_ok(d->k_token, d->k_head) || !strides_ok(d->v_token, d->v_head) ||
        !rows_apart(d->y_token, d->y_head, d->total, d->q_heads, d->cache.head_dim))
        return HAWQ_ERR_SHAPE;
    if (d->n_seqs > 65535 || d->q_heads > 65535) return HAWQ_ERR_UNSUPPORTED;      // (a launch's workgroups along y and z)
    a = AttnTreeArgs{};
    a.cache = cache_args(d->cache, nullptr, nullptr, nullptr, nullptr);
    a.n_seqs = d->n_seqs; a.total = d->total; a.max_drafts = d->max_drafts; a.max_cached = d->max_cached; a.q_heads = d->q_heads;
    a.kv_heads = kv; a.head_dim = d->cache.head_dim; a.dtype = d->dtype; a.table_stride = d->table_stride; a.scale = d->scale;
    a.q_token = d->q_token; a.q_head = d->q_head; a.k_token = d->k_token; a.k_head = d->k_head;
    a.v_token = d->v_token; a.v_head = d->v_head; a.y_token = d->y_token; a.y_head = d->y_head;
    // no request sees more cached tokens than its row of the table has room for
    const int64_t room = (int64_t)a.table_stride * d->cache.page;
    if (a.max_cached > room) a.max_cached = (int32_t)room;
    a.max_cached = std::min(a.max_cached, kMostKeys - 64);
    if (a.cache.n_pages == 0) a.max_cached = 0;
    return HAWQ_OK;
}

}  // namespace

extern "C" {

hawq_status hawq_linear_w4(const hawq_linear_w4_desc *d, const void *x, const void *w, const void *scales, const uint8_t *zeros,
                           const void *bias, void *y, void *stream) {
    if (!d) return HAWQ_ERR_NULL;
    if (d->M < 0 || d->N <= 0 || d->K <= 0 || (d->K & 1) || d->group <= 0 || d->group % 32 != 0) return HAWQ_ERR_SHAPE;
    if ((d->x_stride < d->K && d->x_stride != 0) || d->y_stride < d->N) return HAWQ_ERR_SHAPE;      // (0: one row for all)
    if (!float16(d->x_dtype) || (d->w_dtype != HAWQ_S4 && d->w_dtype != HAWQ_U4)) return HAWQ_ERR_DTYPE;
    if (d->w_dtype == HAWQ_S4 && zeros) return HAWQ_ERR_DTYPE;
    if (d->M == 0) return HAWQ_OK;      // (an empty tensor has no address)
    if (!x || !w || !scales || !y || (d->w_dtype == HAWQ_U4 && !zeros)) return HAWQ_ERR_NULL;
    if (!at_multiple(2, {x, scales, bias, y}) || d->K > (1 << 25)) return HAWQ_ERR_UNSUPPORTED;
    LinearW4Args a{x, scales, bias, (const uint8_t *)w, zeros, y, d->M, d->N, d->K, d->group, (int32_t)(((int64_t)d->K + d->group - 1) / d->group),
                   d->x_stride, d->y_stride, d->x_dtype};
    return launch_linear_w4(a, (hipStream_t)stream);
}

hawq_status hawq_attn_prompt(const hawq_attn_prompt_desc *d, const void *q, const void *k, const void *v, const int32_t *starts,
                             void *y, void *stream) {
    if (!d) return HAWQ_ERR_NULL;
    if (d->n_seqs < 0 || d->total < 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->q_heads % d->kv_heads != 0 || d->head_dim <= 0 || d->head_dim > 256) return HAWQ_ERR_SHAPE;
    if (!float16(d->dtype)) return HAWQ_ERR_DTYPE;
    if (!std::isfinite(d->scale)) return HAWQ_ERR_RANGE;
    if (!strides_ok(d->q_token, d->q_head) || !strides_ok(d->k_token, d->k_head) || !strides_ok(d->v_token, d->v_head) ||
        !rows_apart(d->y_token, d->y_head, d->total, d->q_heads, d->head_dim))
        return HAWQ_ERR_SHAPE;
    if (d->n_seqs == 0 || d->total == 0) return HAWQ_OK;
    if (!q || !k || !v || !starts || !y) return HAWQ_ERR_NULL;
    if (d->total > kMostKeys || !at_multiple(2, {q, k, v, y}) || !at_multiple(4, {starts})) return HAWQ_ERR_UNSUPPORTED;
    AttnPromptArgs a{q, k, v, starts, y, d->n_seqs, d->total, d->q_heads, d->kv_heads, d->head_dim, d->dtype, d->scale,
                     d->q_token, d->q_head, d->k_token, d->k_head, d->v_token, d->v_head, d->y_token, d->y_head};
    return launch_attn_prompt(a, (hipStream_t)stream);
}

size_t hawq_attn_tree_workspace_bytes(const hawq_attn_tree_desc *desc) {
    AttnTreeArgs a;
    return tree_args(desc, a) == HAWQ_OK ? attn_tree_workspace(a) : 0;
}

hawq_status hawq_attn_tree(const hawq_attn_tree_desc *d, const void *q, const void *k, const void *v, const int32_t *starts,
                           const uint64_t *mask, const void *k_cache, const void *v_cache, const float *k_scales, const float *v_scales,
                           const int32_t *table, const int32_t *cached, void *y, void *workspace, size_t workspace_bytes, void *stream) {
    AttnTreeArgs a;
    hawq_status st = tree_args(d, a);
    if (st != HAWQ_OK || d->n_seqs == 0 || d->total == 0) return st;
    if (!q || !k || !v || !starts || (a.max_cached > 0 && !table) || !cached || !y) return HAWQ_ERR_NULL;      // (an empty table has no address)
    st = check_cache(d->cache, d->dtype, k_cache, v_cache, k_scales, v_scales, true);
    if (st != HAWQ_OK) return st;
    if (!at_multiple(2, {q, k, v, y}) || !at_multiple(4, {starts, table, cached}) || !at_multiple(8, {mask})) return HAWQ_ERR_UNSUPPORTED;
    const size_t need = attn_tree_workspace(a);
    if (need > 0 && (!workspace || workspace_bytes < need)) return workspace ? HAWQ_ERR_WORKSPACE : HAWQ_ERR_NULL;
    if (need > 0 && !at_multiple(16, {workspace})) return HAWQ_ERR_UNSUPPORTED;
    a.q = q; a.k = k; a.v = v; a.starts = starts; a.mask = mask; a.table = table; a.cached = cached; a.y = y; a.partial = (float *)workspace;
    a.cache.k = const_cast<void *>(k_cache); a.cache.v = const_cast<void *>(v_cache);
    a.cache.ks = const_cast<float *>(k_scales); a.cache.vs = const_cast<float *>(v_scales);
    return launch_attn_tree(a, (hipStream_t)stream);
}

hawq_status hawq_cache_plan(int32_t n_seqs, int32_t page, int32_t table_stride, int32_t n_free, int64_t n_slots, const int32_t *cached,
                            const int32_t *fresh, const int32_t *free_pages, int32_t *table, int32_t *starts, int64_t *slots,
                            int32_t *counts, void *stream) {
    if (!starts || !counts || (n_seqs > 0 && (!cached || !fresh || (table_stride > 0 && !table))) || (n_free > 0 && !free_pages) || (n_slots > 0 && !slots)) return HAWQ_ERR_NULL;
    if (n_seqs < 0 || page <= 0 || table_stride < 0 || n_free < 0 || n_slots < 0) return HAWQ_ERR_SHAPE;
    if (n_slots > INT32_MAX || (int64_t)n_seqs * std::max(table_stride, 1) > (1 << 30)) return HAWQ_ERR_UNSUPPORTED;      // (the pages taken are counted in 32 bits)
    if (!at_multiple(4, {cached, fresh, free_pages, table, starts, counts}) || !at_multiple(8, {slots})) return HAWQ_ERR_UNSUPPORTED;
    return launch_cache_plan({n_seqs, page, table_stride, n_free, n_slots, cached, fresh, free_pages, table, starts, slots, counts}, (hipStream_t)stream);
}

hawq_status hawq_cache_store(const hawq_cache_store_desc *d, const void *k, const void *v, const int64_t *slots, void *k_cache,
                             void *v_cache, float *k_scales, float *v_scales, void *stream) {
    if (!d) return HAWQ_ERR_NULL;
    if (d->total < 0 || !strides_ok(d->k_token, d->k_head) || !strides_ok(d->v_token, d->v_head)) return HAWQ_ERR_SHAPE;
    if (!float16(d->dtype)) return HAWQ_ERR_DTYPE;
    const bool any = d->total > 0 && d->cache.n_pages > 0;
    const hawq_status st = check_cache(d->cache, d->dtype, k_cache, v_cache, k_scales, v_scales, any);
    if (st != HAWQ_OK || !any) return st;
    if (!k || !v || !slots) return HAWQ_ERR_NULL;
    if (!at_multiple(2, {k, v}) || !at_multiple(8, {slots})) return HAWQ_ERR_UNSUPPORTED;
    CacheStoreArgs a{k, v, slots, cache_args(d->cache, k_cache, v_cache, k_scales, v_scales), d->total, d->cache.kv_heads, d->cache.head_dim, d->dtype,
                     d->k_token, d->k_head, d->v_token, d->v_head};
    return launch_cache_store(a, (hipStream_t)stream);
}

}  // extern "C"
