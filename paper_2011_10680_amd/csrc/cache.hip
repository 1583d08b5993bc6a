// The paged cache: room for new tokens (block tables, slots) and the store of their keys and values.
#include "lm.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr int kThreads = 1024, kEach = 2, kPass = kThreads * kEach;   // requests of a thread and of a pass
constexpr int kSlots = 4;                                             // slots of a thread under way (2000 requests: eight 13.9 us, four 12.0; few tokens alike)

// ceil(n / page) for n < 2^31
__device__ __forceinline__ int pages_of(int n, int page, FastDiv by_page) {
    const int q = (int)fdiv((uint32_t)n, by_page);
    return q + (q * page < n);
}

// A request in LDS: the tokens and the pages given before it, the tokens it holds
struct Request {
    int token, taken, held, unused;
};

// the last i < n with token (PAGES: taken) of i not above at: requests that get nothing share their neighbour's start and are passed over
template <bool PAGES>
__device__ __forceinline__ int holder(const Request *r, int n, int at) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((PAGES ? r[mid].taken : r[mid].token) <= at) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Every workgroup adds up the tokens and pages of all requests (2048 in a pass: two of a thread, then across the waves), so that one
// launch does without an order among workgroups, and writes its own share of the slots and of the pages taken.  A thread finds
// its first slot's request by bisection and walks on from there with the request in registers.  Bound by the chain of dependent steps
// -- lengths, sums, bisection, page numbers, stores: 5 requests 4.2 us (a pass with the host's call 5.7), 2000 with a million fresh tokens and two million
// slots 12.0, 16.3 MB written.
__global__ __launch_bounds__(kThreads) void cache_plan(CachePlanArgs a, FastDiv by_page, int slots_per_block, int pages_per_block) {
    __shared__ __align__(16) Request request[kPass + 1];
    __shared__ int wave_sum[2][kThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, last = gridDim.x - 1;
    const int64_t s0 = (int64_t)blockIdx.x * slots_per_block, s1 = min(s0 + slots_per_block, a.n_slots);
    const int64_t p0 = (int64_t)blockIdx.x * pages_per_block, p1 = (int)blockIdx.x == last ? INT32_MAX : p0 + pages_per_block;
    const bool vectors = (((uintptr_t)a.cached | (uintptr_t)a.fresh) & 7) == 0;
    int tokens_before = 0, pages_before = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += kPass) {
        const int n = min(kPass, a.n_seqs - b0);
        int c[kEach], f[kEach], take[kEach], sum_f = 0, sum_p = 0;
        if (vectors && tid * kEach + kEach <= n) {
            *(v2i *)c = *(const v2i *)(a.cached + b0 + tid * kEach);
            *(v2i *)f = *(const v2i *)(a.fresh + b0 + tid * kEach);
        } else {
            for (int i = 0; i < kEach; ++i) {
                const int at = b0 + min(tid * kEach + i, n - 1);
                c[i] = a.cached[at];
                f[i] = a.fresh[at];
            }
        }
        for (int i = 0; i < kEach; ++i) {
            const bool is = tid * kEach + i < n;
            c[i] = is ? max(c[i], 0) : 0;
            f[i] = is ? max(f[i], 0) : 0;
            const int end = (int)min((int64_t)c[i] + f[i], (int64_t)INT32_MAX);
            take[i] = max(min(pages_of(end, a.page, by_page), a.table_stride) - pages_of(c[i], a.page, by_page), 0);
            sum_f += f[i];
            sum_p += take[i];
        }
        const int upto_f = sum_up_to_lane(sum_f), upto_p = sum_up_to_lane(sum_p);
        if (lane == 63) wave_sum[0][wave] = upto_f, wave_sum[1][wave] = upto_p;
        __syncthreads();
        const int first_token = tokens_before, first_page = pages_before;
        int at_f = tokens_before + upto_f - sum_f, at_p = pages_before + upto_p - sum_p;
        for (int w = 0; w < kThreads / 64; ++w) {
            const int x = wave_sum[0][w], y = wave_sum[1][w];
            if (w < wave) at_f += x, at_p += y;
            tokens_before += x;
            pages_before += y;
        }
        for (int i = 0; i < kEach; ++i) {
            request[tid * kEach + i] = {at_f, at_p, c[i], 0};
            at_f += f[i];
            at_p += take[i];
        }
        if (tid == kThreads - 1) request[kPass] = {tokens_before, pages_before, 0, 0};
        __syncthreads();
        if (blockIdx.x == 0)
            for (int b = tid; b < n; b += kThreads) a.starts[b0 + b] = request[b].token;
        // pages of this pass in the block's share
        const int64_t pe = min(p1, (int64_t)pages_before);
        for (int64_t i = max(p0, (int64_t)first_page) + tid; i < pe; i += kThreads) {
            const int page = i < a.n_free ? a.free_pages[i] : -1, b = holder<true>(request, n, (int)i);
            const Request r = request[b];
            a.table[(int64_t)(b0 + b) * a.table_stride + pages_of(r.held, a.page, by_page) + (i - r.taken)] = page;
        }
        // slots of this pass in the block's share
        const int64_t se = min(s1, (int64_t)tokens_before);
        int64_t t = max(s0, (int64_t)first_token) + tid;
        if (t < se) {
            int b = holder<false>(request, n, (int)t);
            Request r = request[b];
            int next = request[b + 1].token, have = pages_of(r.held, a.page, by_page);
            for (; t < se; t += kSlots * kThreads) {
                // some slots at a time, so that their pages' numbers are under way together
                const int32_t *from[kSlots];
                uint32_t place[kSlots];
                int page[kSlots];
                for (int k = 0; k < kSlots; ++k) {
                    const int64_t tk = t + k * kThreads;
                    from[k] = nullptr;
                    if (tk >= se) continue;
                    if (next <= tk && b + 1 < n) {
                        do ++b; while (b + 1 < n && request[b + 1].token <= tk);
                        r = request[b];
                        next = request[b + 1].token;
                        have = pages_of(r.held, a.page, by_page);
                    }
                    const uint32_t at = (uint32_t)r.held + (uint32_t)(tk - r.token), p = fdiv(at, by_page);
                    place[k] = at - p * (uint32_t)a.page;
                    if (at >= INT32_MAX || p >= (uint32_t)a.table_stride) continue;      // (no request has more tokens than 32 bits count)
                    const int64_t i = (int64_t)r.taken + p - have;
                    if ((int)p < have) from[k] = a.table + (int64_t)(b0 + b) * a.table_stride + p;
                    else if (i < a.n_free) from[k] = a.free_pages + i;
                }
                for (int k = 0; k < kSlots; ++k) page[k] = from[k] ? *from[k] : -1;
                for (int k = 0; k < kSlots; ++k)
                    if (t + k * kThreads < se) a.slots[t + k * kThreads] = page[k] >= 0 ? (int64_t)page[k] * a.page + place[k] : -1;
            }
        }
        __syncthreads();
    }
    for (int64_t t = max(s0, (int64_t)tokens_before) + tid; t < s1; t += kThreads) a.slots[t] = -1;
    if (blockIdx.x == 0 && tid == 0) {
        a.starts[a.n_seqs] = tokens_before;
        a.counts[0] = tokens_before;
        a.counts[1] = pages_before;
    }
}

// Copies of whole vectors: 16 bytes of k (blockIdx.y = 0) or v a thread.  Bound by the bytes: 20001 tokens of 8 heads of 128 elements
// 34.9 us, 164 MB at 4.7 TB/s (a large copy on this device 5.2); two vectors a thread 35.5, four 38.7, eight 44.3.
__global__ __launch_bounds__(256) void cache_copy(CacheStoreArgs a, FastDiv by_piece, FastDiv by_head, uint32_t n) {
    const uint32_t at = blockIdx.x * 256 + threadIdx.x;
    if (at >= n) return;
    const uint32_t row = fdiv(at, by_piece), piece = at - row * (uint32_t)(a.head_dim >> 3), t = fdiv(row, by_head), h = row - t * a.kv_heads;
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= (int64_t)a.cache.n_pages * a.cache.page) return;
    int64_t p;
    if (slot < INT32_MAX) p = fdiv((uint32_t)slot, a.cache.by_page);
    else p = slot / a.cache.page;
    const uint16_t *x = blockIdx.y ? (const uint16_t *)a.v + t * a.v_token + h * a.v_head : (const uint16_t *)a.k + t * a.k_token + h * a.k_head;
    uint16_t *y = (uint16_t *)(blockIdx.y ? a.cache.v : a.cache.k) + p * a.cache.page_stride + (slot - p * a.cache.page) * a.cache.token_stride + h * a.cache.head_stride;
    *(v4u *)(y + piece * 8) = *(const v4u *)(x + piece * 8);
}

// Codes of whole vectors: a group of 8 to 32 lanes a row, eight elements a lane, the maximum by exchanges inside the group.  37 tokens of 8
// heads: 3.2 us, a launch and two dependent loads.
template <class T>
__global__ __launch_bounds__(256) void cache_codes(CacheStoreArgs a, FastDiv by_head, int group_bits) {
    typedef typename T::elem E;
    const int lane = threadIdx.x & 63, piece = lane & ((1 << group_bits) - 1);
    const int64_t r = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> group_bits;
    if (r >= (int64_t)a.total * a.kv_heads) return;
    const uint32_t t = fdiv((uint32_t)r, by_head), h = (uint32_t)r - t * a.kv_heads;
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= (int64_t)a.cache.n_pages * a.cache.page) return;
    const bool mine = piece * 8 < a.head_dim;
    const E *x = blockIdx.y ? (const E *)a.v + t * a.v_token + h * a.v_head : (const E *)a.k + t * a.k_token + h * a.k_head;
    typename T::v8 e = __builtin_bit_cast(typename T::v8, v4u{0, 0, 0, 0});
    if (mine) e = *(const typename T::v8 *)(x + piece * 8);
    float top = 0;
    bool finite = true;
    for (int i = 0; i < 8; ++i) {
        const float v = fabsf((float)e[i]);
        finite &= v < INFINITY;
        top = fmaxf(top, v);
    }
    if (!finite) top = INFINITY;                                // (stays the group's maximum)
    for (int d = 1 << group_bits >> 1; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float scale = top < INFINITY ? top * (1.f / 127.f) : __builtin_nanf("");
    int64_t p;
    if (slot < INT32_MAX) p = fdiv((uint32_t)slot, a.cache.by_page);
    else p = slot / a.cache.page;
    if (mine) {
        uint32_t q[2] = {0, 0};
        if (scale > 0.f)
            for (int i = 0; i < 8; ++i) q[i >> 2] |= ((uint32_t)(int)fminf(fmaxf(rintf((float)e[i] / scale), -127.f), 127.f) & 255u) << (8 * (i & 3));
        int8_t *y = (int8_t *)(blockIdx.y ? a.cache.v : a.cache.k) + p * a.cache.page_stride + (slot - p * a.cache.page) * a.cache.token_stride + h * a.cache.head_stride;
        *(v2u *)(y + piece * 8) = v2u{q[0], q[1]};
    }
    if (piece == 0) (blockIdx.y ? a.cache.vs : a.cache.ks)[slot * a.kv_heads + h] = scale;
}

// any head dimension, stride and alignment: one wave per row (token, head) of k (blockIdx.y = 0) or v
template <class T, bool CODES>
__global__ __launch_bounds__(256) void cache_store_any(CacheStoreArgs a) {
    typedef typename T::elem E;
    const int64_t r = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
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
    // one workgroup for a compute unit at most: each reads all lengths, and a thousand that read the same lines wait for one another
    const int64_t share = (a.n_slots + 255) / 256, per = share < kThreads ? kThreads : (share + kThreads - 1) / kThreads * kThreads;
    const int64_t blocks = a.n_slots > per ? (a.n_slots + per - 1) / per : 1;
    const int64_t pages = (a.n_slots / a.page + a.n_seqs + blocks - 1) / blocks;          // (a request's tokens may begin and end inside a page)
    cache_plan<<<dim3((unsigned)blocks), kThreads, 0, s>>>(a, fast_div((uint32_t)a.page), (int)per, (int)(pages < INT32_MAX ? pages : INT32_MAX));
    return check_launch();
}

hawq_status launch_cache_store(const CacheStoreArgs &all, hipStream_t s) {
    CacheStoreArgs a = all;
    const bool codes = a.cache.dtype == HAWQ_S8;
    const int64_t reads = a.k_token | a.k_head | a.v_token | a.v_head, writes = a.cache.page_stride | a.cache.token_stride | a.cache.head_stride;
    const uintptr_t from = (uintptr_t)a.k | (uintptr_t)a.v, to = (uintptr_t)a.cache.k | (uintptr_t)a.cache.v;
    // Whole vectors: as many tokens at a time as have fewer than 2^31 threads at 32 a row (the indices' divisions, and a launch)
    const int64_t at_once = INT32_MAX / 32 / a.kv_heads;
    if (a.head_dim % 8 == 0 && (reads | writes) % 8 == 0 && from % 16 == 0 && to % (codes ? 8 : 16) == 0 && at_once > 0) {
        const FastDiv by_head = fast_div((uint32_t)a.kv_heads);
        for (int64_t t = 0; t < all.total; t += at_once) {
            a.total = (int32_t)(all.total - t < at_once ? all.total - t : at_once);
            a.k = (const uint16_t *)all.k + t * a.k_token;
            a.v = (const uint16_t *)all.v + t * a.v_token;
            a.slots = all.slots + t;
            const int64_t rows = (int64_t)a.total * a.kv_heads;
            if (codes) {
                int bits = 3;
                while ((8 << bits) < a.head_dim) ++bits;
                const dim3 grid((unsigned)(((rows << bits) + 255) / 256), 2);
                if (a.dtype == HAWQ_F16) cache_codes<F16><<<grid, 256, 0, s>>>(a, by_head, bits);
                else cache_codes<BF16><<<grid, 256, 0, s>>>(a, by_head, bits);
            } else {
                const uint32_t n = (uint32_t)(rows * (a.head_dim / 8));
                cache_copy<<<dim3((n + 255) / 256, 2), 256, 0, s>>>(a, fast_div((uint32_t)a.head_dim / 8), by_head, n);
            }
            const hawq_status st = check_launch();
            if (st != HAWQ_OK) return st;
        }
        return HAWQ_OK;
    }
    const Grid g = spread(((int64_t)a.total * a.kv_heads + 3) / 4, 1, 256);
    if (g.x == 0) return HAWQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)g.x, 2, (unsigned)g.y);
    if (a.dtype == HAWQ_F16) {
        if (codes) cache_store_any<F16, true><<<grid, 256, 0, s>>>(a);
        else cache_store_any<F16, false><<<grid, 256, 0, s>>>(a);
    } else {
        if (codes) cache_store_any<BF16, true><<<grid, 256, 0, s>>>(a);
        else cache_store_any<BF16, false><<<grid, 256, 0, s>>>(a);
    }
    return check_launch();
}

}  // namespace hawq
