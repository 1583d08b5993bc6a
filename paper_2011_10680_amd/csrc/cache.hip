// The paged cache: room for new tokens (block tables, slots) and the store of their keys and values.
#include "lm.h"

namespace hawq {

namespace {

__device__ __forceinline__ int wave_scan(int v) {
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if ((int)(threadIdx.x & 63) >= d) v += o;
    }
    return v;
}

constexpr int kPlanThreads = 256;

// Every workgroup walks over all requests, kPlanThreads at a time with running totals, and writes of what it meets its own
// range of slots and (by the request's index) its own share of the table, the starts and the counts.
__global__ __launch_bounds__(kPlanThreads) void cache_plan(CachePlanArgs a, int slots_per_block) {
    __shared__ int tokens[kPlanThreads + 1], pages[kPlanThreads], held[kPlanThreads], have[kPlanThreads], wave_sum[2][kPlanThreads / 64];
    const int tid = threadIdx.x;
    const int64_t s0 = (int64_t)blockIdx.x * slots_per_block, s1 = min(s0 + slots_per_block, a.n_slots);
    int token_base = 0, page_base = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += kPlanThreads) {
        const int b = b0 + tid;
        const int c = b < a.n_seqs ? max(a.cached[b], 0) : 0, f = b < a.n_seqs ? max(a.fresh[b], 0) : 0;
        const int h = (int)(((int64_t)c + a.page - 1) / a.page), w = (int)min(((int64_t)c + f + a.page - 1) / a.page, (int64_t)a.table_stride);
        const int take = max(w - h, 0), ft = wave_scan(f), pt = wave_scan(take);
        if ((tid & 63) == 63) wave_sum[0][tid >> 6] = ft, wave_sum[1][tid >> 6] = pt;
        __syncthreads();
        int fb = token_base, pb = page_base;
        for (int i = 0; i < (tid >> 6); ++i) fb += wave_sum[0][i], pb += wave_sum[1][i];
        for (int i = 0; i < kPlanThreads / 64; ++i) token_base += wave_sum[0][i], page_base += wave_sum[1][i];
        tokens[tid] = fb + ft - f;
        pages[tid] = pb + pt - take;
        held[tid] = c;
        have[tid] = h;
        if (blockIdx.x == 0 && b < a.n_seqs) a.starts[b] = fb + ft - f;
        if (tid == 0) tokens[kPlanThreads] = token_base;
        if (b < a.n_seqs && b % gridDim.x == blockIdx.x)
            for (int p = h; p < w; ++p) {
                const int i = pb + pt - take + p - h;
                a.table[(int64_t)b * a.table_stride + p] = i < a.n_free ? a.free_pages[i] : -1;
            }
        __syncthreads();
        // slots of this chunk's tokens inside the block's range
        const int64_t lo = max(s0, (int64_t)tokens[0]), hi = min(s1, (int64_t)token_base);
        for (int64_t t = lo + tid; t < hi; t += kPlanThreads) {
            int l = 0, r = kPlanThreads - 1;
            while (l < r) {
                const int mid = (l + r + 1) >> 1;
                if (tokens[mid] <= t) l = mid; else r = mid - 1;
            }
            const int64_t at = (int64_t)held[l] + (t - tokens[l]), p = at / a.page;
            int page = -1;
            if (p < a.table_stride) {
                if (p < have[l]) page = a.table[(int64_t)(b0 + l) * a.table_stride + p];
                else {
                    const int64_t i = pages[l] + (p - have[l]);
                    if (i < a.n_free) page = a.free_pages[i];
                }
            }
            a.slots[t] = page >= 0 ? (int64_t)page * a.page + at % a.page : -1;
        }
        __syncthreads();
    }
    for (int64_t t = max(s0, (int64_t)token_base) + tid; t < s1; t += kPlanThreads) a.slots[t] = -1;
    if (blockIdx.x == 0 && tid == 0) {
        a.starts[a.n_seqs] = token_base;
        a.counts[0] = token_base;
        a.counts[1] = page_base;
    }
}

// one wave per row (token, head) of k (blockIdx.y = 0) or v
template <class T, bool CODES>
__global__ __launch_bounds__(256) void cache_store(CacheStoreArgs a) {
    typedef typename T::elem E;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (r >= (int64_t)a.total * a.kv_heads) return;
    const int t = (int)(r / a.kv_heads), h = (int)(r % a.kv_heads);
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= (int64_t)a.cache.n_pages * a.cache.page) return;
    const int64_t p = slot / a.cache.page, at = slot % a.cache.page;
    const E *x = blockIdx.y ? (const E *)a.v + t * a.v_token + h * a.v_head : (const E *)a.k + t * a.k_token + h * a.k_head;
    const int64_t e = p * a.cache.page_stride + at * a.cache.token_stride + h * a.cache.head_stride;
    if constexpr (!CODES) {
        E *y = (E *)(blockIdx.y ? a.cache.v : a.cache.k) + e;
        for (int i = lane; i < a.head_dim; i += 64) y[i] = x[i];
    } else {
        int8_t *y = (int8_t *)(blockIdx.y ? a.cache.v : a.cache.k) + e;
        float top = 0;
        bool finite = true;
        for (int i = lane; i < a.head_dim; i += 64) {
            const float v = fabsf((float)x[i]);
            finite &= v < INFINITY;
            top = fmaxf(top, v);
        }
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        finite = __all(finite);
        const float scale = finite ? top * (1.f / 127.f) : __builtin_nanf("");
        for (int i = lane; i < a.head_dim; i += 64) y[i] = scale > 0.f ? (int8_t)fminf(fmaxf(rintf((float)x[i] / scale), -127.f), 127.f) : 0;
        if (lane == 0) (blockIdx.y ? a.cache.vs : a.cache.ks)[slot * a.kv_heads + h] = scale;
    }
}

}  // namespace

hawq_status launch_cache_plan(const CachePlanArgs &a, hipStream_t s) {
    const int per = 1024;
    const int64_t blocks = a.n_slots > 0 ? (a.n_slots + per - 1) / per : 1;
    cache_plan<<<dim3((unsigned)blocks), kPlanThreads, 0, s>>>(a, per);
    return check_launch();
}

hawq_status launch_cache_store(const CacheStoreArgs &a, hipStream_t s) {
    const int64_t blocks = ((int64_t)a.total * a.kv_heads + 3) / 4;
    if (blocks > INT32_MAX) return HAWQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, 2);
    const bool codes = a.cache.dtype == HAWQ_S8;
    if (a.dtype == HAWQ_F16) {
        if (codes) cache_store<F16, true><<<grid, 256, 0, s>>>(a);
        else cache_store<F16, false><<<grid, 256, 0, s>>>(a);
    } else {
        if (codes) cache_store<BF16, true><<<grid, 256, 0, s>>>(a);
        else cache_store<BF16, false><<<grid, 256, 0, s>>>(a);
    }
    return check_launch();
}

}  // namespace hawq
