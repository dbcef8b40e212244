// Host-only check of how paged attention shares out its work (csrc/paged_plan.h): what the host
// plans from the sizes against what the kernels find from the lengths, also where the lengths are
// wrong.  Built and run by tests/test_paged_plan.py, under sanitizers; with --planted items that
// stay whole are counted in units of four steps, and it has to catch that; with --resident it says
// how many workgroups of the row kernel the plan takes to be on a compute unit.
#include <stdio.h>
#include <string.h>

#include <random>
#include <vector>

#include "paged_plan.h"

using namespace attn;

namespace {

struct Call {
    int T, R, Hq, Hkv, d, max_q, page_log2, max_pages, window;
    std::vector<int> cu, kv;  // cu empty: one token of each
    bool right;               // the bounds are
};

// What a call would do with memory it has not asked for, or null.
const char* check(const Call& c, bool planted, bool memory = true) {
    const long long max_keys = (long long)c.max_pages << c.page_log2;
    const int window = c.window >= max_keys ? 0 : c.window;
    PagedLaunch l = paged_launch(c.T, c.R, c.Hq, c.Hkv, c.d, c.max_q, max_keys, window, 256);
    if (!memory) l.unsplit();
    if (!memory && (l.row_parts() || l.tile_parts())) return "parts without memory";
    PagedArgs a{};
    a.kv_lens = c.kv.data();
    a.cu = c.cu.empty() ? nullptr : c.cu.data();
    a.T = c.T;
    a.R = c.R;
    a.Hkv = c.Hkv;
    a.group = c.Hq / c.Hkv;
    a.page_log2 = c.page_log2;
    a.max_pages = c.max_pages;
    a.window = window;
    a.few = l.few;
    a.unit_log2 = planted ? 2 : l.unit_log2;
    long long units = 0, blocks = 0;
    for (int r = 0; r < c.R; ++r) {
        const PagedRequest x = paged_request(a, r);
        if (x.qn < 0 || (x.qn && (x.q0 < 0 || (long long)x.q0 + x.qn > c.T)))
            return "rows outside the queries";
        if (x.lo < 0 || x.kv < 0 || x.kv > max_keys) return "keys outside the table";
        const long long rows = (long long)x.qn * a.group;
        if (l.n_wg) {
            const Share s = share_of(a, x, 32 * l.waves);
            if (rows > l.few ? s.items != 0 : s.items < (rows > 0)) return "a request of nobody's";
            if (s.items && !l.shared && s.units != 1)
                return "an item of several units, and no memory for parts";
            units += (long long)s.items * s.units;
        }
        if (rows > l.few) blocks += (rows + kPagedTileRows - 1) / kPagedTileRows;
    }
    if (units > 2147483647) return "more units than a 32-bit number holds";
    if (c.right && l.items && blocks * c.Hkv > l.items) return "blocks without a workgroup";
    // items are requests' heads: no more than CUs, and short enough, they get eight waves
    if (l.n_wg && (long long)c.R * c.Hkv <= 256 && max_keys <= 8 * 128 && l.waves != 8)
        return "four waves to few items";
    if (l.n_wg && (l.few > l.block || l.n_wg < 1)) return "requests of more rows than a block";
    return nullptr;
}

}  // namespace

int main(int argc, char** argv) {
    const bool planted = argc > 1 && !strcmp(argv[1], "--planted");
    if (argc > 1 && !strcmp(argv[1], "--resident")) {
        for (int d : {64, 128})
            for (int block : {16, 32})
                printf("%d %d %d\n", d, block, paged_row_wgs_per_cu(d, block));
        return 0;
    }
    // single tokens in a window, the last bound far past the queries
    Call far = {16, 16, 32, 8, 128, 1, 4, 1250, 512, {}, {}, false};
    for (int r = 0; r <= 16; ++r) far.cu.push_back(r == 16 ? 20016 : r);
    far.kv.assign(16, 20000);
    const char* wrong = check(far, planted);
    std::mt19937 rng(11);
    auto below = [&](long long n) { return (long long)rng() % n; };
    auto spread = [&](long long lo, long long hi) {  // over the logarithm
        const double u = rng() / 4294967296.0;
        return (long long)(lo * pow((double)hi / lo, u));
    };
    int caught = wrong != nullptr, runs = 60000;
    if (wrong && !planted) return printf("one bound far past the queries: %s\n", wrong), 1;
    for (int i = 0; i < runs; ++i) {
        Call c;
        c.right = rng() % 3 != 0;
        c.Hkv = 1 + below(rng() % 2 ? 4 : 40);
        c.Hq = c.Hkv * (int)spread(1, rng() % 8 ? 12 : 200);
        c.d = rng() % 2 ? 64 : 128;
        c.R = (int)spread(1, 300);
        c.page_log2 = 3 + below(6);
        const long long keys = spread(1, rng() % 8 ? 60000 : 1 << 30);
        c.max_pages = (int)((keys >> c.page_log2) + 1);
        while ((long long)c.max_pages << c.page_log2 > 1 << 30) --c.max_pages;
        const long long most_keys = (long long)c.max_pages << c.page_log2;
        c.window = rng() % 2 ? 0 : (int)spread(1, 1 << 20);
        const int kind = rng() % 3;  // single tokens, drafts, all kinds
        int most = 0;
        std::vector<int> cu(1, 0);
        for (int r = 0; r < c.R; ++r) {
            const int n = kind == 0 ? 1 : kind == 1 ? below(9) : below(4) ? below(2) : spread(1, 700);
            most = std::max(most, n);
            cu.push_back(cu[r] + n);
            c.kv.push_back((int)(c.right ? std::max<long long>(std::min(most_keys, keys), 1)
                                         : below(4) ? below(most_keys + 1) : (int)rng()));
        }
        c.T = std::max(1, cu[c.R] + (int)below(3));
        c.max_q = rng() % 3 ? std::max(1, most) : 0;
        if (!c.right)
            for (int& x : cu)
                if (below(4) == 0) x = below(2) ? (int)rng() : x + (int)spread(1, 1 << 20);
        if (kind == 0 && c.right && rng() % 2 && cu[c.R] == c.R)
            c.T = c.R;
        else
            c.cu = cu;
        const char* what = check(c, planted);
        if (!what) what = check(c, planted, false);
        if (!what) continue;
        ++caught;
        if (planted) continue;
        return printf("case %d: T=%d R=%d heads %d/%d d=%d max_q=%d window=%d keys=%lld: %s\n", i, c.T,
                      c.R, c.Hq, c.Hkv, c.d, c.max_q, c.window, most_keys, what), 1;
    }
    if (planted) return printf(caught ? "caught %d times\n" : "not seen\n", caught), !caught;
    printf("paged_plan_check ok: %d calls\n", runs);
    return 0;
}
