// Attention of drafted tokens over a paged cache and over one another.
#include "attn_any.h"

namespace hawq {

namespace {

template <class T>
__global__ __launch_bounds__(64) void attn_tree_any(AttnTreeArgs a) {
    typedef typename T::elem E;
    __shared__ float q_lds[256];
    const int b = blockIdx.z, h = blockIdx.y, hk = h / (a.q_heads / a.kv_heads);
    int from, to;
    sequence_rows(a.starts, b, a.total, from, to);
    const int drafts = min(to - from, a.max_drafts), t = blockIdx.x;
    if (t >= drafts) return;
    const int row = from + t, cached = min(max(a.cached[b], 0), a.max_cached);
    const uint64_t seen = a.mask ? a.mask[row] : t == 63 ? ~0ull : (2ull << t) - 1;
    const int32_t *table = a.table + (int64_t)b * a.table_stride;
    const bool codes = a.cache.dtype == HAWQ_S8;
    const int size = codes ? 1 : 2;
    auto key = [&](int j) -> KeyRow {
        if (j >= cached) {
            const int64_t r = from + j - cached;
            return {(const E *)a.k + r * a.k_token + hk * a.k_head, (const E *)a.v + r * a.v_token + hk * a.v_head, 1.f, 1.f, false};
        }
        const int i = (int)fdiv((uint32_t)j, a.cache.by_page), at = j - i * a.cache.page;
        const int64_t p = table[i], e = p * a.cache.page_stride + at * a.cache.token_stride + hk * a.cache.head_stride;
        const int64_t f = (p * a.cache.page + at) * a.kv_heads + hk;
        return {(const char *)a.cache.k + e * size, (const char *)a.cache.v + e * size, codes ? a.cache.ks[f] : 1.f, codes ? a.cache.vs[f] : 1.f, codes};
    };
    const auto visible = [&](int j) { return j < cached ? (uint32_t)table[fdiv((uint32_t)j, a.cache.by_page)] < (uint32_t)a.cache.n_pages : (seen >> (j - cached) & 1) != 0; };
    store_row<T>(attend_row<T>((const E *)a.q + row * a.q_token + h * a.q_head, a.head_dim, a.scale, 0, cached + drafts, q_lds, key, visible),
                 (E *)a.y + row * a.y_token + h * a.y_head, a.head_dim);
}

}  // namespace

size_t attn_tree_workspace(const AttnTreeArgs &) { return 0; }

hawq_status launch_attn_tree(const AttnTreeArgs &a, hipStream_t s) {
    if (a.q_heads > 65535 || a.n_seqs > 65535) return HAWQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)a.max_drafts, (unsigned)a.q_heads, (unsigned)a.n_seqs);
    if (a.dtype == HAWQ_F16) attn_tree_any<F16><<<grid, 64, 0, s>>>(a);
    else attn_tree_any<BF16><<<grid, 64, 0, s>>>(a);
    return check_launch();
}

}  // namespace hawq
