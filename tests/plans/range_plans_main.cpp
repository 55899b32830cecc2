// Walks the lengths of the ranges into which the attention over pages cuts a step's sequences (csrc/ecco_plan.h) and prints the first step with
// more ranges than the launch and the workspace hold: B * Hkv + places.
#include <cstdio>
#include <vector>

#include "ecco_plan.h"

using namespace ecco;

int main() {
    long checked = 0;
    const int most = units_of(0x7FFFFFFF);
    unsigned state = 1;
    const auto draw = [&](int n) { return (int)((state = state * 1664525u + 1013904223u) >> 8) % n; };
    for (int places : {256, 512, 304, 608})
        for (int Hkv : {1, 2, 3, 7, 8, 16, 31, 32, 64, 100, 255})
            for (int B : {1, 2, 3, 8, 31, 32, 33, 63, 64, 65, 128, 255, 256}) {
                if ((long long)B * Hkv >= places || B > kRangeSequences) continue;
                for (int shape = 0; shape < 40; ++shape) {
                    // alike, from one unit to the longest, one long one beside short ones, or anything
                    static const int alike[] = {0, 1, 8, 9, 63, 64, 1000, 8191, 8400000, 9000000, 16777217, 33554432, most - 1, most};
                    std::vector<int> units(B);
                    for (int b = 0; b < B; ++b)
                        units[b] = shape < 14 ? alike[shape] : shape < 28 ? (b == 0 ? alike[shape - 14] : 1) : draw(shape % 2 ? 2000 : most) + 1;
                    float lanes[64] = {}, total = 0;
                    for (int l = 0; l < 64; ++l) {
                        int own = 0;  // four sequences of a lane fit an int
                        for (int b = l; b < B; b += 64) own += units[b];
                        lanes[l] = (float)own;
                    }
                    for (float t : lanes) total += t;
                    const int least = range_least(total, Hkv, places), step = std::max(1, least / 16);
                    for (int length : {least, least + least / 4, least + 63 * step}) {
                        long long ranges = 0;
                        for (int u : units) ranges += std::max(1, (u + length - 1) / length);
                        ++checked;
                        if (length < kRangeLeast || ranges * Hkv > (long long)B * Hkv + places) {
                            std::printf("%d sequences, %d heads, %d places, shape %d: %lld ranges of %d units\n", B, Hkv, places, shape, ranges, length);
                            return 1;
                        }
                    }
                }
            }
    std::printf("%ld conditions hold\n", checked);
    return 0;
}
