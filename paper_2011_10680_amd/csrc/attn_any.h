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

// One wave, one row: the visible keys of [from, to), 64 at a time with a lane each, then a lane for each of the elements
// lane + 64 i of the result.  One running maximum (of scale * q . k) and sum, everything in 32 bits; o is not yet divided by
// the sum.  q_lds: 256 floats of the wave's own.
struct RowSums {
    float m = -INFINITY, total = 0, o[4] = {0, 0, 0, 0};
};
template <class T, class Keys, class Visible>
__device__ __forceinline__ RowSums attend_row(const typename T::elem *q, int head_dim, float scale, int from, int to, float *q_lds, Keys &&keys, Visible &&visible) {
    const int lane = threadIdx.x & 63;
    __builtin_amdgcn_wave_barrier();
    for (int i = lane; i < head_dim; i += 64) q_lds[i] = (float)q[i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const float log2e = 1.4426950408889634f;
    RowSums a;
    for (int j0 = from; j0 < to; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j < to && visible(j);
        float s = -INFINITY;
        if (seen) {
            const KeyRow r = keys(j);
            float t = 0;
            for (int i = 0; i < head_dim; ++i) t += q_lds[i] * row_elem<T>(r.k, r.codes, i);
            s = t * (scale * r.ks);
        }
        // (a NaN score makes the row NaN: the maximum leaves it out, its own exponential does not)
        float top = s;
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        const float next = fmaxf(a.m, top), safe = next == -INFINITY ? 0.f : next;
        const float keep = __builtin_exp2f((a.m - safe) * log2e);
        const float p = seen ? __builtin_exp2f((s - safe) * log2e) : 0.f;
        float sum = p;
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        a.total = a.total * keep + sum;
        for (int i = 0; i < 4; ++i) a.o[i] *= keep;
        a.m = next;
        for (uint64_t left = __ballot(seen); left; left &= left - 1) {
            const int l = __builtin_ctzll(left);
            const KeyRow at = keys(j0 + l);
            const float pl = __shfl(p, l) * at.vs;
            for (int i = 0; i < 4; ++i)
                if (lane + 64 * i < head_dim) a.o[i] += pl * row_elem<T>(at.v, at.codes, lane + 64 * i);
        }
    }
    return a;
}

// y = o / total, zeros where nothing was visible
template <class T>
__device__ __forceinline__ void store_row(const RowSums &a, typename T::elem *y, int head_dim) {
    const int lane = threadIdx.x & 63;
    const float by = 1.f / a.total;
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < head_dim) y[lane + 64 * i] = (typename T::elem)(a.total == 0.f ? 0.f : a.o[i] * by);
}

}  // namespace hawq
