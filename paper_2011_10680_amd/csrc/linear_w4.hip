// Linear layer with 4-bit weights and group scales.
#include "lm.h"

namespace hawq {

namespace {

template <class T>
__global__ __launch_bounds__(256) void linear_w4_any(LinearW4Args a) {
    typedef typename T::elem E;
    const int n = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, m = blockIdx.y;
    if (n >= a.N) return;
    const E *x = (const E *)a.x + m * a.x_stride, *s = (const E *)a.scales + (int64_t)n * a.groups;
    const uint8_t *w = a.w + (int64_t)n * (a.K / 2), *z = a.zeros ? a.zeros + (int64_t)n * a.groups : nullptr;
    float t = 0;
    for (int i = lane; i < a.K / 2; i += 64) {
        const int g = 2 * i / a.group, v = w[i];
        const int even = z ? (v & 15) - z[g] : ((v & 15) ^ 8) - 8, odd = z ? (v >> 4) - z[g] : ((v >> 4) ^ 8) - 8;
        t += ((float)x[2 * i] * (float)even + (float)x[2 * i + 1] * (float)odd) * (float)s[g];
    }
    for (int d = 32; d > 0; d >>= 1) t += __shfl_xor(t, d);
    if (lane == 0) ((E *)a.y)[m * a.y_stride + n] = (E)(t + (a.bias ? (float)((const E *)a.bias)[n] : 0.f));
}

}  // namespace

hawq_status launch_linear_w4(const LinearW4Args &a, hipStream_t s) {
    if (a.M > 65535) return HAWQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((a.N + 3) / 4), (unsigned)a.M);
    if (a.dtype == HAWQ_F16) linear_w4_any<F16><<<grid, 256, 0, s>>>(a);
    else linear_w4_any<BF16><<<grid, 256, 0, s>>>(a);
    return check_launch();
}

}  // namespace hawq
