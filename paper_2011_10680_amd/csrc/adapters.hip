// Low-rank adapters of the rows' own beside a projection that all rows share.
//
//   y[m,n] = base[m,n] + s_i * sum_j b[i,n,j] h[m,j],   h[m,j] = sum_k a[i,j,k] x[m,k],   i = adapter[m]
#include "lm.h"
#include "lm_launch.h"

namespace hawq {

namespace {

// the row's adapter, -1: none
__device__ __forceinline__ int adapter_of(const AdaptersArgs &a, int64_t m) {
    const int i = a.adapter[m];
    return i >= 0 && i < a.n_adapters ? i : -1;
}
__device__ __forceinline__ int rank_of(const AdaptersArgs &a, int i) { return i < 0 ? 0 : min(max(a.ranks[i], 0), a.max_rank); }

// one wave for an inner sum
template <class T>
__global__ __launch_bounds__(256) void inner_any(AdaptersArgs a) {
    typedef typename T::elem E;
    const int64_t e = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (e >= (int64_t)a.M * a.max_rank) return;
    const int64_t m = e / a.max_rank;
    const int j = (int)(e - m * a.max_rank), i = adapter_of(a, m);
    if (j >= rank_of(a, i)) return;
    const E *x = (const E *)a.x + m * a.x_stride, *row = (const E *)a.a + i * a.a_adapter + j * a.a_row;
    float v = 0;
    for (int k = lane; k < a.K; k += 64) v += (float)x[k] * (float)row[k];
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if (lane == 0) a.h[e] = v;
}

// one thread for an output
template <class T>
__global__ __launch_bounds__(256) void outer_any(AdaptersArgs a) {
    typedef typename T::elem E;
    const int64_t e = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
    if (e >= (int64_t)a.M * a.N) return;
    const int64_t m = e / a.N, n = e - m * a.N;
    const int i = adapter_of(a, m), rank = rank_of(a, i);
    const E *b = (const E *)a.b + i * a.b_adapter + n * a.b_row, *base = (const E *)a.base + m * a.base_stride + n;
    E *y = (E *)a.y + m * a.y_stride + n;
    if (rank == 0) {
        *y = *base;
        return;
    }
    float v = 0;
    for (int j = 0; j < rank; ++j) v += (float)b[j] * a.h[m * a.max_rank + j];
    *y = (E)((float)*base + a.scales[i] * v);
}

}  // namespace

size_t adapters_workspace(const AdaptersArgs &a) { return ((size_t)a.M * a.max_rank * 4 + 15) & ~(size_t)15; }

hawq_status launch_adapters(const AdaptersArgs &a, hipStream_t s) {
    const Grid g = spread(((int64_t)a.M * a.max_rank + 3) / 4, 1, 256), e = spread(((int64_t)a.M * a.N + 255) / 256, 1, 256);
    if (g.x == 0 || e.x == 0) return HAWQ_ERR_UNSUPPORTED;
    const dim3 inner((unsigned)g.x, (unsigned)g.y), outer((unsigned)e.x, (unsigned)e.y);
    if (a.dtype == HAWQ_F16) {
        if (a.n_adapters > 0) inner_any<F16><<<inner, 256, 0, s>>>(a);
        outer_any<F16><<<outer, 256, 0, s>>>(a);
    } else {
        if (a.n_adapters > 0) inner_any<BF16><<<inner, 256, 0, s>>>(a);
        outer_any<BF16><<<outer, 256, 0, s>>>(a);
    }
    return check_launch();
}

}  // namespace hawq
