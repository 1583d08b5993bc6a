// Rotary positions of queries and keys.
//
//   (x, y) -> scale * (x cos a - y sin a, y cos a + x sin a),   a = 2 pi * position * turns[f]
//
// The angle's revolutions are a product of 64-bit floats, less the nearest whole number: a position of 2^20 keeps the angle to 2^-33 of a
// revolution, where a 32-bit product would keep 2^-5.  What is left is below half a revolution and goes on in 32 bits.
#include "lm.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr int kThreads = 256;

// One element pair, or one element past the turned ones, for each thread: tokens of a workgroup, heads, slots of a head.
template <class T>
__global__ __launch_bounds__(kThreads) void rotary_any(RotaryArgs a, int tokens, FastDiv by_slot, FastDiv by_head) {
    typedef typename T::elem E;
    extern __shared__ float2 turn[];                 // [token][rotary_dim / 2]
    const int half = a.rotary_dim >> 1, slots = half + a.head_dim - a.rotary_dim;
    const int64_t t0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * tokens;
    const int n = (int)min((int64_t)tokens, (int64_t)a.total - t0);
    for (int i = threadIdx.x; i < n * half; i += kThreads) {
        const int t = i / half, f = i - t * half;
        double r = (double)a.positions[t0 + t] * a.turns[f];
        r -= rint(r);
        float s, c;
        sincospif(2.f * (float)r, &s, &c);
        turn[i] = make_float2(c * a.scale, s * a.scale);
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < (uint32_t)n * a.heads * slots; i += kThreads) {
        const uint32_t row = fdiv(i, by_slot), t = fdiv(row, by_head);
        int slot = (int)(i - row * slots), h = (int)(row - t * a.heads);
        const int which = h >= a.q_heads;
        h -= which ? a.q_heads : 0;
        const E *x = (const E *)a.x[which] + (t0 + t) * a.x_token[which] + h * a.x_head[which];
        E *y = (E *)a.y[which] + (t0 + t) * a.y_token[which] + h * a.y_head[which];
        if (slot >= half) {
            slot += half;
            y[slot] = x[slot];
            continue;
        }
        const int e = a.layout == HAWQ_ROTARY_HALVES ? slot : 2 * slot, f = a.layout == HAWQ_ROTARY_HALVES ? slot + half : 2 * slot + 1;
        const float2 cs = turn[t * half + slot];
        const float u = (float)x[e], v = (float)x[f];
        y[e] = (E)(u * cs.x - v * cs.y);
        y[f] = (E)(v * cs.x + u * cs.y);
    }
}

}  // namespace

hawq_status launch_rotary(const RotaryArgs &a, hipStream_t s) {
    const int half = a.rotary_dim / 2, slots = half + a.head_dim - a.rotary_dim;
    int tokens = 1;
    while (tokens * 2 * half <= kThreads && a.total / tokens >= 2048 && (int64_t)tokens * 2 * a.heads * slots < INT32_MAX) tokens *= 2;
    const Grid g = spread(((int64_t)a.total + tokens - 1) / tokens, 1, kThreads);
    if (g.x == 0) return HAWQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)g.x, (unsigned)g.y);
    const size_t lds = (size_t)tokens * half * sizeof(float2);
    if (a.dtype == HAWQ_F16) rotary_any<F16><<<grid, kThreads, lds, s>>>(a, tokens, fast_div((uint32_t)slots), fast_div((uint32_t)a.heads));
    else rotary_any<BF16><<<grid, kThreads, lds, s>>>(a, tokens, fast_div((uint32_t)slots), fast_div((uint32_t)a.heads));
    return check_launch();
}

}  // namespace hawq
