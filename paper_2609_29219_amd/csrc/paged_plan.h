// How the work of a paged attention call is shared out: what the host plans from the sizes that it
// knows, and what the kernels find from the lengths that it does not.  Both compile for the host,
// where a test holds them against each other.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "paged.h"

namespace attn {

// ------------------------------------------------------------- the kernels --
__host__ __device__ __forceinline__ PagedRequest paged_request(const PagedArgs& a, int r) {
    const long long c0 = a.cu ? a.cu[r] : r, c1 = a.cu ? a.cu[r + 1] : r + 1;
    PagedRequest x;
    x.kv = std::max(a.kv_lens[r], 0);
    x.bad = x.kv > ((long long)a.max_pages << a.page_log2);
    x.q0 = (int)c0;
    x.qn = 0;
    if (c0 >= 0 && c1 > c0 && c0 < a.T) x.qn = (int)(std::min(c1, (long long)a.T) - c0);
    // Positions of the tokens that are there: bounds past the queries do not move the window, and
    // a request of few rows has as few steps as the host counted on.  (Positions less a window,
    // each of up to 2^30 tokens, are 32-bit.)
    x.pos0 = x.kv - x.qn;
    x.lo = a.window ? std::max(0, x.pos0 - a.window + 1) : 0;
    if (x.bad) x.kv = x.lo = 0;
    return x;
}

// The row kernel's items of a request: its key/value heads (all its rows are one block); their
// steps of step_keys keys, and their units of 2^unit_log2 steps.
struct Share {
    int items, steps, units;
};
__host__ __device__ __forceinline__ Share share_of(const PagedArgs& a, const PagedRequest& x,
                                                   int step_keys) {
    Share s = {0, 0, 0};
    const long long rows = (long long)x.qn * a.group;
    if (rows == 0 || rows > a.few) return s;
    s.items = a.Hkv;
    s.steps = x.kv > x.lo ? (int)((uint32_t)(x.kv + step_keys - 1) / (uint32_t)step_keys) -
                                (int)((uint32_t)x.lo / (uint32_t)step_keys)
                          : 1;
    s.units = (s.steps + (1 << a.unit_log2) - 1) >> a.unit_log2;
    return s;
}

// ---------------------------------------------------------------- the host --
constexpr int kPagedWholeLog2 = 24;  // more steps than 2^30 tokens have

// How a call is launched, from what the host knows of it.
struct PagedLaunch {
    int few = 0;                      // requests of up to so many rows: the row kernel's
    int block = 0, n_wg = 0;          // row kernel (n_wg 0: not launched): rows of an item, few of
                                      // them at most
    int waves = 4;                    // to its workgroups
    bool shared = false;              // its workgroups may share an item
    int unit_log2 = 0;
    long long items = 0;              // tile kernel: blocks of all heads at most (0: not launched)
    int splits = 1;
    long long row_parts() const { return shared ? 2LL * n_wg * block : 0; }
    long long tile_parts() const { return splits > 1 ? items * splits * kPagedTileRows : 0; }
    // as planned, but nobody has a part of anything, and no memory is used
    void unsplit() {
        shared = false;
        unit_log2 = kPagedWholeLog2;
        splits = 1;
    }
    size_t bytes(int d) const {
        return (size_t)(row_parts() + tile_parts()) * (d + 2) * sizeof(float) +
               (size_t)(n_wg + items) * kPagedMeta * sizeof(int);
    }
};

// The tile kernel's part, and whether it takes requests of few rows as well: by this estimate, in
// us on this card.  Rounds of workgroups, each with 6 us of start and end and 2 to a tile; where
// the keys are split, 4 us and the partial results' traffic; a row kernel beside it, 9 us and its
// keys' traffic.  (All rows are taken to be in requests of the most rows, so that a full batch is
// estimated as it is, or every fourth request has a block that is not full.  Keys as many as the
// table or the window allows, up to 16384.  What the device finds may need fewer splits, and the
// others end at once.)  Measured: 64 requests of 40 rows over 8192 keys in two splits 88 us, in
// four, as chosen, 67; 32 of 64 rows over 4096 keys of 8 heads in two 130 us, unsplit, as chosen,
// 110.  A prompt's 300 tokens twice and 10 single tokens, over 1000 to 3000 keys of 8 heads: by
// two kernels 67 us, by one, as chosen, 56; 512 twice and 30, over 3000 and 4000 keys: 154 and,
// as chosen, 159; 256 single tokens over 500 to 1500 keys where the most is not known: by two
// kernels, as chosen, 194, by one 248.
inline void plan_tiles(PagedLaunch* l, int R, long long rows, long long most, bool known, int Hkv, int d,
                int group, long long max_keys, int window, int num_cus) {
    const int block = kPagedTileRows;
    const bool exact = rows == R * most;
    double keys = std::min(16384.0, (double)max_keys);
    if (window) keys = std::min(keys, window + (double)block / group);
    auto estimate = [&](double items, int* splits) {
        double best = 0;
        for (int s = 1; s <= kPagedMaxSplits && (s == 1 || items * s <= 4.0 * num_cus); ++s) {
            const double rounds = items * s / num_cus;
            double t = (exact ? ceil(rounds) : std::max(1.0, rounds)) * (6 + 2 * keys / 64 / s);
            if (s > 1) t += 4 + items * s * block * d * 4 / 5e6;
            if (s == 1 || t < best) {
                best = t;
                *splits = s;
            }
        }
        return best;
    };
    const double full = (double)rows / most;     // requests, if all have the most rows
    const double few = std::max(0.0, R - full);  // at most so many have few
    double blocks = full * ((most + block - 1) / block);
    long long requests = std::min<long long>(R, rows / (l->few + 1));
    if (!exact) blocks = std::max(blocks, (double)rows / block + requests / 4.0);
    int all_splits = 1;
    const double apart = estimate(blocks * Hkv, &l->splits) + 9 + few * keys * Hkv * d * 4 / 6e6;
    // (a block of few rows takes about half the time of others)
    if (estimate((blocks + (known ? few / 2 : few)) * Hkv, &all_splits) < apart) {
        l->few = 0;
        l->splits = all_splits;
        requests = R;
    }
    // (all but one row of a block each may be missing from the requests' last blocks)
    l->items = (rows + requests * (block - 1)) / block * Hkv;
}

inline PagedLaunch paged_launch(int T, int R, int Hq, int Hkv, int d, int max_q, long long max_keys,
                         int window, int num_cus) {
    PagedLaunch l;
    const int group = Hq / Hkv;
    const long long rows = (long long)T * group;
    const long long most = (max_q ? std::min(max_q, T) : T) * (long long)group;  // of a request
    // Among several requests each kernel takes those of its kind, or the tile kernel all (see
    // below).  Without the tile kernel, what has more rows than the caller said is nobody's.
    const bool tiles = most > kPagedFewRows;
    l.few = tiles ? kPagedFewRows : (int)most;
    if (tiles) plan_tiles(&l, R, rows, most, max_q > 0, Hkv, d, group, max_keys, window, num_cus);
    if (l.few > 0) {
        l.block = most <= 16 ? 16 : 32;
        l.n_wg = paged_row_wgs_per_cu(d, l.block) * num_cus;
        // steps of a request at most (its tokens are no more than its rows)
        double steps = (double)max_keys / kPagedRowKeys + 1;
        if (window) steps = std::min(steps, ((double)window + l.few) / kPagedRowKeys + 2);
        const double items = (double)R * Hkv;
        // Few steps to every item: each is one workgroup's.  An item's steps one behind another
        // cost about 1 us each, adding up its parts a launch of 5 us.  Items no more than CUs:
        // workgroups of twice the waves have half the steps.  Measured: a token over 512 keys of
        // 8 heads, by four waves 11.0 us, by eight, as chosen, 9.7; over 1000 keys shared 13.0,
        // whole, as chosen, 13.5; sixteen tokens over 950 keys shared 22, whole, as chosen, 19;
        // 28 over 900 keys by four waves, shared, 26.5, by eight, as chosen, 22.5.
        if (items <= num_cus) l.waves = 8;
        l.shared = steps > (l.waves == 8 ? 9 : 6);
        if (l.shared)
            l.waves = 4;
        else
            l.n_wg = (int)std::min((double)l.n_wg, items);
        // one unit to an item, however long it turns out to be: no workgroup has a part of one
        if (!l.shared) l.unit_log2 = kPagedWholeLog2;
        // so few units that their number is 32-bit, whatever the lengths are
        while (items * (steps / (1 << l.unit_log2) + 1) >= 2147483647.0 &&
               l.unit_log2 < kPagedWholeLog2)
            ++l.unit_log2;
    }
    return l;
}

}  // namespace attn
