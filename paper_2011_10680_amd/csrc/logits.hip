// What a server does to the logits before it chooses: penalties for tokens that occurred, biases, grammar masks.
//
// A workgroup takes a part of the vocabulary for some rows.  It counts the past tokens of the row's request that fall into its part in LDS,
// one word a token (bit 31: occurred; below: how often the model wrote it), adds the drafted tokens that the row sees, and then
// passes over its logits once.  Integer counts: the order of the atomics does not matter.
#include "lm.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr int kThreads = 512, kPart = 8192;
constexpr uint32_t kOccurred = 0x80000000u;

// the request whose rows t belongs to, -1: none
__device__ __forceinline__ int request_of(const LogitsArgs &a, int t) {
    if (!a.starts) return t;
    int low = 0, high = a.n_seqs;                    // the first request that ends behind t
    while (low < high) {
        const int mid = low + (high - low) / 2;
        if (a.starts[mid + 1] > t) high = mid;
        else low = mid + 1;
    }
    return low < a.n_seqs && a.starts[low] <= t ? low : -1;
}

template <class T>
__global__ __launch_bounds__(kThreads) void logits_part(LogitsArgs a, int part) {
    typedef typename T::elem E;
    extern __shared__ uint32_t words[];
    const int t = (int)((int64_t)blockIdx.z * gridDim.y + blockIdx.y);
    if (t >= a.total) return;
    const int v0 = blockIdx.x * part, n = min(part, a.vocab - v0);
    const int b = request_of(a, t);
    if (b < 0) return;
    uint32_t *count = words, *listed = words + part;                // listed: the entry of the bias list, 0: none, i + 1 for entry i
    float r = 1, presence = 0, frequency = 0;
    const bool counts = a.penalties != nullptr;
    if (counts) r = a.penalties[3 * (int64_t)b], presence = a.penalties[3 * (int64_t)b + 1], frequency = a.penalties[3 * (int64_t)b + 2];
    const int first_bias = a.n_bias > 0 ? min(max(a.bias_starts[b], 0), a.n_bias) : 0, last_bias = a.n_bias > 0 ? min(max(a.bias_starts[b + 1], first_bias), a.n_bias) : 0;
    for (int i = threadIdx.x; i < n; i += kThreads) count[i] = 0, listed[i] = 0;
    __syncthreads();
    if (counts && a.past_stride > 0) {
        const int len = min(max(a.past_lens[b], 0), a.past_stride), prompt = a.prompt_lens ? a.prompt_lens[b] : 0;
        const int32_t *past = a.past + (int64_t)b * a.past_stride;
        for (int i = threadIdx.x; i < len; i += kThreads) {
            const uint32_t at = (uint32_t)past[i] - (uint32_t)v0;
            if (at < (uint32_t)n) {
                atomicOr(count + at, kOccurred);
                if (i >= prompt) atomicAdd(count + at, 1u);
            }
        }
    }
    if (counts && a.drafts) {
        int from = t, to = t + 1;
        if (a.starts) sequence_rows(a.starts, b, a.total, from, to);
        const int seen = a.mask ? min(to - from, 64) : t + 1 - from;
        for (int i = threadIdx.x; i < seen; i += kThreads) {
            const uint32_t at = (uint32_t)a.drafts[from + i] - (uint32_t)v0;
            if (at < (uint32_t)n && (!a.mask || (a.mask[t] >> i & 1))) {
                atomicOr(count + at, kOccurred);
                atomicAdd(count + at, 1u);
            }
        }
    }
    for (int i = first_bias + threadIdx.x; i < last_bias; i += kThreads) {
        const uint32_t at = (uint32_t)a.bias_ids[i] - (uint32_t)v0;
        if (at < (uint32_t)n) atomicMax(listed + at, (uint32_t)i + 1);
    }
    __syncthreads();
    const int mask_row = a.n_allowed == 0 ? -1 : a.allowed_row ? a.allowed_row[t] : t;
    const uint32_t *allowed = mask_row >= 0 && mask_row < a.n_allowed ? a.allowed + mask_row * a.allowed_stride : nullptr;
    const E *x = (const E *)a.x + t * a.x_stride + v0;
    E *y = (E *)a.y + t * a.y_stride + v0;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        float v = (float)x[i];
        const uint32_t c = count[i], bias = listed[i];
        if (c & kOccurred) v = v > 0 ? v / r : v * r;
        if (c & ~kOccurred) v = v - frequency * (float)(c & ~kOccurred) - presence;
        if (bias) v += a.bias_values[bias - 1];
        if (allowed && !(allowed[(v0 + i) >> 5] >> ((v0 + i) & 31) & 1)) v = -INFINITY;
        y[i] = (E)v;
    }
}

}  // namespace

hawq_status launch_logits(const LogitsArgs &a, hipStream_t s) {
    const int part = a.vocab < kPart ? (a.vocab + 31) / 32 * 32 : kPart;
    const int64_t along = a.total < kMostAlong ? a.total : kMostAlong;
    const dim3 grid((unsigned)(((int64_t)a.vocab + part - 1) / part), (unsigned)along, (unsigned)((a.total + along - 1) / along));
    if (a.dtype == HAWQ_F16) logits_part<F16><<<grid, kThreads, (size_t)part * 8, s>>>(a, part);
    else logits_part<BF16><<<grid, kThreads, (size_t)part * 8, s>>>(a, part);
    return check_launch();
}

}  // namespace hawq
