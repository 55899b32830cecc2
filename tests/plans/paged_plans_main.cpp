// Draws sizes of the attention over pages (csrc/ecco_plan.h) and prints the first for which the workspace that is asked for does not hold the plan, or the
// one asked for by sizes that are nowhere larger; and follows lengths that a plan's bounds cover through its sums: tiles, units and ranges have to fit.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "ecco_plan.h"

using namespace ecco;

static unsigned long long state = 88172645463325252ull;
static long long draw(long long lo, long long hi) {  // spread over the logarithm, either end more often
    state ^= state << 13, state ^= state >> 7, state ^= state << 17;
    const unsigned long long r = state >> 11;
    if (r % 16 == 0) return lo;
    if (r % 16 == 1) return hi;
    int bits = 0;
    while ((hi - lo) >> bits) ++bits;
    const long long span = 1ll << ((r >> 4) % (bits + 1));
    return lo + (long long)((r >> 10) % (unsigned long long)std::min(span, hi - lo + 1));
}

struct Sizes {
    int n, B, max_new, max_kv;
    long long total;
};

int main() {
    const int most = 0x7FFFFFFF;
    long checked = 0;
    for (int i = 0; i < 3000000; ++i) {
        const int cus = i % 5 ? 256 : (int)draw(1, 400), grp = (int)draw(1, 16);
        Sizes a{};
        const int Hkv = (int)draw(1, i % 3 ? 64 : 4096);
        a.B = (int)draw(1, most / Hkv / (i % 3 ? 4096 : 1));
        a.n = (int)draw(1, most / (Hkv * grp));
        a.max_new = (int)draw(1, i % 4 ? a.n : most);
        a.max_kv = (int)draw(1, i % 2 ? 1 << 18 : most);
        a.total = draw(1, i % 2 ? (long long)a.B * a.max_kv : 1ll << 62);
        const Sizes b{(int)draw(1, a.n), (int)draw(1, a.B), (int)draw(1, a.max_new), (int)draw(1, a.max_kv), draw(1, a.total)};
        const PagedPlan p = paged_plan(a.n, a.B, Hkv * grp, Hkv, a.max_new, a.max_kv, a.total, cus);
        const size_t all = paged_workspace(a.n, a.B, Hkv * grp, Hkv, a.max_new, a.max_kv, a.total, cus);
        const size_t less = paged_workspace(b.n, b.B, Hkv * grp, Hkv, b.max_new, b.max_kv, b.total, cus);
        const auto check = [&](bool ok, const char* what) {
            ++checked;
            if (ok) return;
            std::printf("%s: %d units, %d/%d heads, rows %d of %d sequences, up to %d over %d, %lld together (%d, %d, %d, %d, %lld): plan %zu, asked %zu, less %zu; tiles %d of %d, splits %d, units %d\n",
                        what, cus, Hkv * grp, Hkv, a.n, a.B, a.max_new, a.max_kv, a.total, b.n, b.B, b.max_new, b.max_kv, b.total, p.bytes, all, less, p.wide_tiles, p.tile_rows,
                        p.wide_splits, p.wide_units);
            std::exit(1);
        };
        check(p.bytes <= all, "plan");
        check(less <= all, "less");
        check(p.few >= 0 && p.few <= kFewRows && p.few_rows >= p.few && (p.wide_tiles == 0 || (p.wide_splits >= 1 && p.wide_units >= 1)), "counts");
        check(p.wide_tiles == 0 || p.wide_splits == 1 || (long long)p.wide_tiles * Hkv * p.wide_splits <= cus, "splits");
        // lengths within the bounds, drawn until rows or tokens are used up
        if (p.wide_tiles == 0 || a.B > 4096 || i % 8) continue;
        long long rows = 0, tokens = 0, tiles = 0, units = 0;
        const bool equal = draw(0, 1);
        for (int s = 0; s < a.B; ++s) {
            const int n = (int)std::min<long long>(equal ? a.max_new : draw(0, std::min(a.max_new, a.n)), a.n - rows);
            const int kv = (int)std::min<long long>(draw(0, a.max_kv), a.total - tokens);
            rows += n, tokens += kv;
            if ((long long)n * grp <= p.few) continue;
            tiles += ((long long)n * grp - 1) / p.tile_rows + 1;
            units += kv > 0 ? units_of(kv) : 0;
        }
        check(tiles <= p.wide_tiles && (units <= p.wide_units || p.wide_units == most), "sums");
    }
    std::printf("%ld conditions hold\n", checked);
    return 0;
}
