// Sizes of the language-model operators' launches: along x a launch holds less than 2^32 threads, along y and z 65535 workgroups.  Plain
// C++ without a device's headers, so that a host compiler's tests see the same functions.
#pragma once
#include <stdint.h>

namespace hawq {

constexpr int64_t kMostThreads = ((int64_t)1 << 32) - 1, kMostAlong = 65535;

// the workgroups of `threads` that one launch holds along x
inline int64_t most_blocks(int threads) { return kMostThreads / threads; }

// n times `unit` workgroups as x by y, x whole units and as many as there are or fit; the last of them may lie past n.  x = 0: too many
struct Grid {
    int64_t x, y;
};
inline Grid spread(int64_t n, int64_t unit, int threads) {
    const int64_t fit = most_blocks(threads) / unit, along = n < fit ? n : fit;
    if (along <= 0 || (n + along - 1) / along > kMostAlong) return {0, 0};
    return {along * unit, (n + along - 1) / along};
}

// Chunks of a part, a multiple of `waves`, to begin with where `all` chunks are to be shared out to `workgroups`: a part for each, were the
// requests alike.  No more than 2^27, which no request has: with numbers beyond that every request is one part.
constexpr int first_chunks(float all, unsigned workgroups, int waves) {
    const float each = all / (float)workgroups;
    return (int)(each < 0x1p27f ? each : 0x1p27f) / waves * waves + waves;
}

// Tokens of the vocabulary to a workgroup of the logits' copy: 16384, fewer where that gives the 256 compute units less than four workgroups each.
// And how many such parts there are.
inline int64_t logits_parts(int32_t vocab, int part) { return ((int64_t)vocab + part - 1) / part; }
inline int logits_part_of(int32_t total, int32_t vocab) {
    int part = 16384;
    while (part > 1024 && total * logits_parts(vocab, part) < 1024) part /= 2;
    return part;
}

}  // namespace hawq
