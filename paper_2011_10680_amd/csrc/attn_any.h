// Attention of one row by one wave, for any head dimension up to 256, alignment and stride: what the matrix-core kernels leave.
#pragma once
#include "lm.h"

namespace hawq {

// keys(j): the j-th key the row may see, as {rows of k and v, their scales, 8-bit codes?}; visible(j): whether it does.
struct KeyRow {
    const void *k, *v;
    float ks, vs;
    bool codes;
};

template <class T>
__device__ __forceinline__ float row_elem(const void *row, bool codes, int i) {
    return codes ? (float)((const int8_t *)row)[i] : (float)((const typename T::elem *)row)[i];
}

// y = softmax over the visible keys of scale * q . k, times v: 64 keys at a time, a lane each, then a lane for each of the
// elements lane + 64 i of the result.  One running maximum and sum, everything in 32 bits; zeros where nothing is visible.
template <class T, class Keys, class Visible>
__device__ __forceinline__ void attend_row(const typename T::elem *q, typename T::elem *y, int head_dim, float scale, int n_keys, float *q_lds, Keys &&keys, Visible &&visible) {
    const int lane = threadIdx.x & 63;
    for (int i = lane; i < head_dim; i += 64) q_lds[i] = (float)q[i];
    __syncthreads();
    const float log2e = 1.4426950408889634f;
    float o[4] = {0, 0, 0, 0}, m = -INFINITY, total = 0;
    for (int j0 = 0; j0 < n_keys; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j < n_keys && visible(j);
        float s = -INFINITY;
        KeyRow r{};
        if (seen) {
            r = keys(j);
            float t = 0;
            for (int i = 0; i < head_dim; ++i) t += q_lds[i] * row_elem<T>(r.k, r.codes, i);
            s = t * (scale * r.ks);
        }
        // (a NaN score makes the row NaN: the maximum leaves it out, its own exponential does not)
        float top = s;
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        const float next = fmaxf(m, top), safe = next == -INFINITY ? 0.f : next;
        const float keep = __builtin_exp2f((m - safe) * log2e);
        const float p = seen ? __builtin_exp2f((s - safe) * log2e) : 0.f;
        float sum = p;
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        total = total * keep + sum;
        for (int i = 0; i < 4; ++i) o[i] *= keep;
        m = next;
        for (uint64_t left = __ballot(seen); left; left &= left - 1) {
            const int l = __builtin_ctzll(left);
            const KeyRow at = keys(j0 + l);
            const float pl = __shfl(p, l) * at.vs;
            for (int i = 0; i < 4; ++i)
                if (lane + 64 * i < head_dim) o[i] += pl * row_elem<T>(at.v, at.codes, lane + 64 * i);
        }
    }
    const float by = 1.f / total;
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < head_dim) y[lane + 64 * i] = (typename T::elem)(total == 0.f ? 0.f : o[i] * by);
}

}  // namespace hawq
