// Walks the launch plans of the attention over pages (csrc/ecco_plan.h) over their range of sizes and prints the first one that the kernel could not
// run: spans are positive multiples of 32 that make progress, everything fits the LDS that the plan asks for, and workgroups that are to share a
// compute unit take half of its LDS at most.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "ecco_plan.h"

using namespace ecco;

int main() {
    long checked = 0;
    const int most = units_of(0x7FFFFFFF);
    for (int S = 1; S <= kMaxS; S += S < 20 ? 1 : 11)
        for (int lk = 0; lk < 2; ++lk)
            for (int lv = 0; lv < 2; ++lv)
                for (int Sv : {S, 1, kMaxS})
                    for (int rows = 1; rows <= kFewRows; ++rows)
                        for (int units : {1, 2, 7, 8, 9, 12, 13, 24, 100, 256, 257, 100000, most})
                            for (size_t wgs : {(size_t)1, (size_t)256, (size_t)257, (size_t)600, (size_t)100000})
                                for (int cut = 0; cut < 2; ++cut) {
                                    const GqaPlan p = rows_plan(S, lk, Sv, lv, rows, wgs, units, 256, cut);
                                    const auto check = [&](bool ok, const char* what) {
                                        ++checked;
                                        if (ok) return;
                                        std::printf("%s at S %d/%d long %d/%d rows %d units %d workgroups %zu cut %d: waves %d span %d step %d lds %zu\n", what, S, Sv, lk, lv, rows,
                                                    units, wgs, cut, p.waves, p.span, p.step, p.lds);
                                        std::exit(1);
                                    };
                                    const bool share = rows_can_share(S, lk, Sv, lv, rows);
                                    const int wk = decode_table_words(S, lk), wv = decode_table_words(Sv, lv);
                                    check(p.waves == 8 || p.waves == 12, "wavefronts");
                                    check(!(lk || lv) || p.waves == (rows > 16 ? 8 : 12), "wavefronts of long codes");
                                    check(rows <= 16 || p.waves == (lk || lv ? 8 : 12), "wavefronts of more than 16 rows");
                                    check(p.span >= kUnitBlocks && p.span % kUnitBlocks == 0, "span");
                                    check(p.step >= kUnitBlocks && p.step % kUnitBlocks == 0 && p.step <= p.span, "step");
                                    check(p.table_words >= (p.both ? wk + wv : std::max(wk, wv)), "tables");
                                    check(p.lds <= (share && cut ? 80u : 160u) * 1024, "limit");
                                    check(p.lds >= 4 * ((size_t)p.table_words + (size_t)p.waves * (kUnitWords + kTileWords) + (size_t)rows * gqa_score_stride(p.span)), "room");
                                    check(p.lds >= 4 * ((size_t)gqa_state_words(p.waves) + (size_t)p.waves * 8 * kRedTile), "room of the sums");
                                    check(!share || p.waves == 8 || !cut, "sharing");
                                    // every wavefront can take a unit per span; with the largest models, long codes and 32 rows at least half of them
                                    check(p.span >= std::min(units, lk || lv ? p.waves / 2 : p.waves) * kUnitBlocks, "a round");
                                }
    for (int page = -5; page < 3000; ++page)
        for (int n : {-1, 0, 1, 7, 1 << 20, (1 << 27) - 1, 1 << 27, 0x7FFFFFFF}) {
            const bool want = (page == 16 || page == 32 || page == 64 || page == 128 || page == 256 || page == 512 || page == 1024) && n > 0 && (long long)page * n <= 0x7FFFFFFF;
            ++checked;
            if (pool_fits(page, n) != want) {
                std::printf("pool of %d pages of %d tokens\n", n, page);
                return 1;
            }
        }
    std::printf("%ld conditions hold\n", checked);
    return 0;
}
