// Linear layer with 4-bit weights: which form of the kernel takes a call.
#include "linear_w4.h"

namespace hawq {

namespace {

// Tiles of a workgroup: a larger one reads x fewer times and has more to do for every 128 weights, and what does not come out even
// over the 256 compute units waits for its last round.  The times are those of a workgroup alone on its unit (K = 4096, groups of 128,
// us; the smaller forms leave room for a second one, which the rounds do not count); times the rounds they order the measured ones right, as for 30 rows of 4096 outputs 13.4 / 10.5 / 14.6 (16, 32, 64 outputs, 16
// rows) and 13.5 / 18.3 (32, 64 outputs, 32 rows), for 64 rows of 8192 (K = 8192) 81 / 53 / 42, 41 / 31 and 45 (64 outputs, 64 rows).
struct Tiles { int rt, mt; float us; };
constexpr Tiles kTiles[] = {{1, 1, 8.0f}, {2, 1, 10.0f}, {4, 1, 14.5f}, {2, 2, 13.5f}, {4, 2, 18.3f}, {4, 4, 27.5f}};

// the best of the forms whose bit is set in `forms`
int best_tiles(const LinearW4Args &a, unsigned forms) {
    int best = -1;
    double least = 0;
    for (int i = 0; i < 6; ++i) {
        if (!(forms >> i & 1)) continue;
        const Tiles &t = kTiles[i];
        const int64_t blocks = ((int64_t)a.N + 16 * t.rt - 1) / (16 * t.rt) * (((int64_t)a.M + 16 * t.mt - 1) / (16 * t.mt));
        const double us = t.us * (double)((blocks + 255) / 256);
        if (best < 0 || us < least) best = i, least = us;
    }
    return best;
}

template <class T, int PIECES, int ALIGN>
hawq_status pick_tiles(const LinearW4Args &a, hipStream_t s) {
    // Rows of w that are not read in whole vectors have the first and the fourth form only.  Read in 4 bytes they go by the best of all six,
    // its rows at least (8192 outputs of K = 4104: 13 rows 14.1 us in the first form, 15.7 in the fourth), element by element, where
    // x costs more, by the better of the two (K = 4096: 72 and 57).
    const int best = best_tiles(a, ALIGN == 1 ? 0x09 : 0x3f);
    if constexpr (ALIGN == 16) {
        if (best == 1) return launch<T, 2, 1, PIECES, ALIGN, false>(a, s);
        if (best == 2) return launch<T, 4, 1, PIECES, ALIGN, false>(a, s);
        if (best == 4) return launch<T, 4, 2, PIECES, ALIGN, false>(a, s);
        if (best == 5) return launch<T, 4, 4, PIECES, ALIGN, false>(a, s);
    }
    return best >= 3 ? launch<T, 2, 2, PIECES, ALIGN, false>(a, s) : launch<T, 1, 1, PIECES, ALIGN, false>(a, s);
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

hawq_status launch_linear_w4(const LinearW4Args &a, hipStream_t s) { return a.dtype == HAWQ_F16 ? pick_align<F16>(a, s) : pick_align<BF16>(a, s); }

}  // namespace hawq
