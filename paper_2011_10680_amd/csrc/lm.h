// Internal declarations of the language-model operators: element types, argument blocks, launchers (gfx950 only).
#pragma once
#include "common.h"
#include "fastdiv.h"

namespace hawq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

// The activations' type T: its name for the matrix instructions and how a float is rounded to it (nearest even).  lift: softmax weights
// are held as 2^lift times their own size, and no more than 2^8 times that.  A half goes down to 2^-24 and up to 2^16: with weights from
// 2^7 on, one that is 2^-31 of the largest is still there (from 1 on those below 2^-25 were lost, a thousandth of a result where 40000
// keys lay 17 nats below one).  bf16 has a float's range.
struct F16 {
    typedef _Float16 elem;
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    typedef _Float16 v4 __attribute__((ext_vector_type(4)));
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    static constexpr float lift = 7.f;
    static __device__ __forceinline__ v4f mfma16(v8 a, v8 b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ v16f mfma32(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
struct BF16 {
    typedef __bf16 elem;
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    typedef __bf16 v4 __attribute__((ext_vector_type(4)));
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    static constexpr float lift = 0.f;
    static __device__ __forceinline__ v4f mfma16(v8 a, v8 b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ v16f mfma32(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

struct LinearW4Args {
    const void *x, *scales, *bias;
    const uint8_t *w, *zeros;      // zeros == nullptr: signed weights
    void *y;
    int32_t M, N, K, group, groups;
    int64_t x_stride, y_stride;
    int32_t dtype;
    int32_t activation;            // of a gated pair: the rows of w, scales, zeros and bias from `up` on are its second projection
    int64_t up;
    float *sums;                   // workspace of a gated pair
};

struct AttnPromptArgs {
    const void *q, *k, *v;
    const int32_t *starts;
    void *y;
    int32_t n_seqs, total, q_heads, kv_heads, head_dim, dtype;
    float scale;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, y_token, y_head;
};

struct CacheArgs {
    void *k, *v;                   // the two tensors
    float *ks, *vs;                // scales of an 8-bit cache
    int32_t n_pages, page, dtype;
    FastDiv by_page;
    int64_t page_stride, token_stride, head_stride;
};

struct AttnTreeArgs {
    const void *q, *k, *v;
    const int32_t *starts, *table, *cached;
    const uint64_t *mask;          // nullptr: a chain
    void *y;
    float *partial;                // workspace
    CacheArgs cache;
    int32_t n_seqs, total, max_drafts, max_cached, q_heads, kv_heads, head_dim, dtype, table_stride;
    float scale;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, y_token, y_head;
};

struct CachePlanArgs {
    int32_t n_seqs, page, table_stride, n_free;
    int64_t n_slots;
    const int32_t *cached, *fresh, *free_pages;
    int32_t *table, *starts;
    int64_t *slots;
    int32_t *counts;
};

struct CacheStoreArgs {
    const void *k, *v;
    const int64_t *slots;
    CacheArgs cache;
    int32_t total, kv_heads, head_dim, dtype;
    int64_t k_token, k_head, v_token, v_head;
};

struct RotaryArgs {
    const void *x[2];              // queries, keys
    void *y[2];
    const int32_t *positions;
    const double *turns;
    int32_t total, q_heads, heads, head_dim, rotary_dim, layout, dtype;      // heads: of both
    float scale;
    int64_t x_token[2], x_head[2], y_token[2], y_head[2];
};

struct AdaptersArgs {
    const void *x, *a, *b, *base;
    const int32_t *ranks, *adapter;
    const float *scales;
    void *y;
    float *h;                      // workspace: the rows' inner sums
    int32_t M, N, K, n_adapters, max_rank, dtype;
    int64_t x_stride, base_stride, y_stride, a_adapter, a_row, b_adapter, b_row;
};

struct LogitsArgs {
    const void *x;
    const int32_t *past, *past_lens, *prompt_lens, *starts, *drafts;
    const uint64_t *mask;
    const float *penalties;
    const int32_t *bias_starts, *bias_ids;
    const float *bias_values;
    const uint32_t *allowed;
    const int32_t *allowed_row;
    void *y;
    int32_t n_seqs, total, vocab, dtype, past_stride, n_bias, n_allowed;
    int64_t allowed_stride, x_stride, y_stride;
};

hawq_status launch_linear_w4(const LinearW4Args &a, hipStream_t s);
size_t gated_w4_workspace(const LinearW4Args &a);
hawq_status launch_gated_w4(const LinearW4Args &a, hipStream_t s);
hawq_status launch_rotary(const RotaryArgs &a, hipStream_t s);
size_t adapters_workspace(const AdaptersArgs &a);
hawq_status launch_adapters(const AdaptersArgs &a, hipStream_t s);
hawq_status launch_logits(const LogitsArgs &a, hipStream_t s);
hawq_status launch_attn_prompt(const AttnPromptArgs &a, hipStream_t s);
size_t attn_tree_workspace(const AttnTreeArgs &a);
hawq_status launch_attn_tree(const AttnTreeArgs &a, hipStream_t s);
hawq_status launch_cache_plan(const CachePlanArgs &a, hipStream_t s);
hawq_status launch_cache_store(const CacheStoreArgs &a, hipStream_t s);

// Buffer of `bytes` bytes at p, both the same in every lane: made of scalars where the compiler does not see that they are.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t scalar_rsrc(const void *p, uint32_t bytes) {
    const uint64_t at = (uint64_t)p;
    const uint64_t s = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)) << 32;
    return __builtin_amdgcn_make_buffer_rsrc((void *)s, 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// Sum of v over the lanes up to this one; over all lanes; the largest of non-negative v.  Moves inside rows of 16 lanes, then of whole
// rows' ends: none waits for an exchange through LDS.  Every lane of the wave takes part.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int sum_up_to_lane(int v) {
    v += moved<0x111, 0xf>(v);      // from the lane 1, 2, 4, 8 below, 0 past the row's end
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);      // lane 15 of the row below to rows 1 and 3
    v += moved<0x143, 0xc>(v);      // lane 31 to rows 2 and 3
    return v;
}
__device__ __forceinline__ int sum_of_lanes(int v) { return __builtin_amdgcn_readlane(sum_up_to_lane(v), 63); }
__device__ __forceinline__ int max_of_lanes(int v) {
    v = max(v, moved<0x111, 0xf>(v));
    v = max(v, moved<0x112, 0xf>(v));
    v = max(v, moved<0x114, 0xf>(v));
    v = max(v, moved<0x118, 0xf>(v));
    v = max(v, moved<0x142, 0xa>(v));
    v = max(v, moved<0x143, 0xc>(v));
    return __builtin_amdgcn_readlane(v, 63);
}

// Pointers that the compiler knows to be global memory (a pointer put together from integers is not known to be), and to data that
// no kernel in flight writes, so that a load from the same place in every lane is a scalar one.
template <class X> using Global = const __attribute__((address_space(1))) X *;
template <class X> using Fixed = const __attribute__((address_space(4))) X *;

// Rows [from, to) of sequence b, whatever the starts hold: inside [0, total) and not negative in number.
__device__ __forceinline__ void sequence_rows(const int32_t *starts, int b, int total, int &from, int &to) {
    from = min(max(starts[b], 0), total);
    to = min(max(starts[b + 1], from), total);
}

}  // namespace hawq
