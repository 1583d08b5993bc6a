// Checks how the logits' copy shares its vocabulary out, on the host, with every overflow of a signed number an error; prints the number of sizes looked at.
#include <cstdio>
#include <initializer_list>

#include "../paper_2011_10680_amd/csrc/lm_launch.h"

using namespace hawq;

int main() {
    long seen = 0;
    const int64_t most = INT32_MAX - 4095;       // of the vocabulary
    for (int32_t total : {1, 2, 3, 7, 64, 171, 1000, 1023, 1024, 65535, (1 << 23) - 1})
        for (int64_t base = 1;; base = base * 5 / 4 + 1) {
            const bool last = base >= most;
            for (int64_t vocab : {base - 1, base, base + 1, last ? most - 16384 : base, last ? most - 8193 : base, last ? most : base}) {
                if (vocab < 1 || vocab > most) continue;
                const int part = logits_part_of(total, (int32_t)vocab);
                const int64_t parts = logits_parts((int32_t)vocab, part);
                ++seen;
                const bool shared = part == 1024 || total * parts >= 1024, wide = part == 16384 || total * ((vocab - 1) / (2 * part) + 1) < 1024;
                if (part < 1024 || part > 16384 || (part & (part - 1)) || parts * part < vocab || (parts - 1) * part >= vocab || !shared || !wide)
                    return std::printf("%d rows of %lld: %lld parts of %d\n", total, (long long)vocab, (long long)parts, part), 1;
                // a launch holds them, and each first token's number fits 32 bits (the last part ends with the vocabulary)
                if (parts * 512 >= ((int64_t)1 << 32) || (parts - 1) * part > INT32_MAX) return std::printf("%lld parts\n", (long long)parts), 1;
            }
            if (last) break;
        }
    std::printf("%ld\n", seen);
    return 0;
}
