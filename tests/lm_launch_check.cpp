// Checks the launch sizes of the language-model operators on the host; prints the number of sizes looked at.
#include <cstdio>
#include <initializer_list>

#include "../paper_2011_10680_amd/csrc/lm_launch.h"

using namespace hawq;

int main() {
    long seen = 0;
    for (int threads : {64, 128, 256, 512, 1024})
        for (int64_t unit : {(int64_t)1, (int64_t)2, (int64_t)7, (int64_t)32, (int64_t)4096, (int64_t)65537, (int64_t)1 << 24, (int64_t)INT32_MAX})
            for (int64_t base = 1; base <= ((int64_t)1 << 42); base = base * 3 / 2 + 1)
                for (int64_t n : {base - 1, base, base + 1}) {
                    const Grid g = spread(n, unit, threads);
                    ++seen;
                    const int64_t fit = kMostThreads / threads / unit;
                    if (g.x == 0) {
                        if (n > 0 && fit > 0 && (n - 1) / fit + 1 <= kMostAlong) return std::printf("refused %lld x %lld x %d\n", (long long)n, (long long)unit, threads), 1;
                        continue;
                    }
                    const bool holds = g.x > 0 && g.x % unit == 0 && g.x * threads < ((int64_t)1 << 32) && g.y >= 1 && g.y <= 65535;
                    // all of them, and no whole row too many
                    if (!holds || g.x / unit * g.y < n || g.x / unit * (g.y - 1) >= n) return std::printf("wrong %lld x %lld x %d\n", (long long)n, (long long)unit, threads), 1;
                }
    for (int threads : {64, 256, 512})
        if (most_blocks(threads) * threads >= ((int64_t)1 << 32) || (most_blocks(threads) + 1) * threads < ((int64_t)1 << 32)) return 1;
    // Parts of listed work: requests of up to 2^26 chunks on up to 65535 heads of keys times row tiles.  From the first size on, the items
    // of 64 requests stay countable, whatever the requests are.
    for (int waves : {4, 8})
        for (int64_t tiles = 1; tiles <= 200000; tiles = tiles * 2 + 1)
            for (int64_t longest = 1; longest <= ((int64_t)1 << 26) + 2; longest = longest * 3 + 1)
                for (int like = 1; like <= 64; like += 9) {             // so many are as long as the longest, the rest have one chunk
                    float all = 0;
                    for (int b = 0; b < 64; ++b) all += (float)tiles * (float)(b < like ? longest : 1);
                    const int chunks = first_chunks(all, 512, waves);
                    ++seen;
                    if (chunks < waves || chunks % waves != 0) return std::printf("%d chunks of %lld\n", chunks, (long long)longest), 1;
                    const int64_t items = tiles * (like * ((longest + chunks - 1) / chunks) + 64 - like);
                    if (items > INT32_MAX / 2) return std::printf("%lld items\n", (long long)items), 1;
                }
    std::printf("%ld\n", seen);
    return 0;
}
