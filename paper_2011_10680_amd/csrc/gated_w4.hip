// The first half of a gated feed-forward block from 4-bit weights: which form of the kernel takes a call.
#include "linear_w4.h"

namespace hawq {

namespace {

template <class T, int PIECES, int ALIGN>
hawq_status pick_tiles(const LinearW4Args &a, hipStream_t s) {
    return a.M > 16 ? launch<T, 2, 2, PIECES, ALIGN, true>(a, s) : launch<T, 2, 1, PIECES, ALIGN, true>(a, s);
}

template <class T, int ALIGN>
hawq_status pick_pieces(const LinearW4Args &a, hipStream_t s) {
    return a.group % 128 == 0 ? pick_tiles<T, 1, ALIGN>(a, s) : a.group % 64 == 0 ? pick_tiles<T, 2, ALIGN>(a, s) : pick_tiles<T, 4, ALIGN>(a, s);
}

template <class T>
hawq_status pick_align(const LinearW4Args &a, hipStream_t s) {
    const bool x16 = ((uintptr_t)a.x & 15) == 0 && a.x_stride % 8 == 0 && a.x_stride < (1 << 25);      // (32-bit offsets inside 64 rows)
    if (x16 && a.K % 32 == 0 && ((uintptr_t)a.w & 15) == 0) return pick_pieces<T, 16>(a, s);
    if (x16 && a.K % 8 == 0 && ((uintptr_t)a.w & 3) == 0) return pick_pieces<T, 4>(a, s);
    return pick_pieces<T, 1>(a, s);
}

}  // namespace

size_t gated_w4_workspace(const LinearW4Args &) { return 0; }

hawq_status launch_gated_w4(const LinearW4Args &a, hipStream_t s) { return a.dtype == HAWQ_F16 ? pick_align<F16>(a, s) : pick_align<BF16>(a, s); }

}  // namespace hawq
