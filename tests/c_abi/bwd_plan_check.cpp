// Host-only sweep of the backward pass's plan (csrc/plan.cpp) and of the work that its
// workgroups find (bwd_work): every part of every block exactly once, each with at least
// one step, all of a block's steps dealt out, the workspace no smaller than what the parts
// take.  Built and run by tests/test_bwd_plan.py, under sanitizers.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <random>
#include <set>
#include <tuple>

#include "common.h"

using namespace attn;

static const char* check(int cus, int B, const BwdFold& q, int Hkv, int Skv, int d, bool planted) {
    BwdPlan p;
    const int Hq = q.Hq, Sq = q.Sq, causal = q.causal;
    if (!plan_bwd(cus, B, q, Hkv, Skv, d, &p)) return "no plan";
    const int group = Hq / Hkv, heads = B * Hkv, units = p.kv_units + p.q_units;
    if (p.grid != (long long)heads * units) return "grid";
    const int rows = bwd_block_rows(d);
    const BwdSize size = {rows, Sq, Skv, group, causal, q.diag};
    const int q_tiles = (Sq + 31) / 32 * group, per_block = rows / 32;
    if (p.kv_blocks != (Skv + rows - 1) / rows ||
        p.q_blocks != (q_tiles + per_block - 1) / per_block)
        return "blocks";
    if (!p.kv_chunk != !p.kv_parts || !p.q_chunk != !p.q_parts) return "parts without a chunk";
    if (p.ordered && (!causal || units > kBwdOrder)) return "an order";
    long long kv_most = 1, q_most = 1, kv_units = 0, q_units = 0;
    for (int b = 0; b < p.kv_blocks; ++b) {
        const int steps = size.kv_steps(b), n = bwd_parts(steps, p.kv_chunk);
        if (steps < 1 || n > steps) return "a part of keys without a step";
        kv_units += n;
        if (n > kv_most) kv_most = n;
        // the first query that any key of the block reaches lies in the first tile walked
        if (causal) {
            const long long first = (long long)b * rows - q.diag;  // (folded: of a position)
            const int qt0 = (Sq + 31) / 32 - steps / group;
            if (qt0 * 32 > (first > 0 ? first : 0)) return "tiles left out";
        }
    }
    for (int b = 0; b < p.q_blocks; ++b) {
        const int steps = size.q_steps(b), n = bwd_parts(steps, p.q_chunk);
        if (steps < 1 || n > steps || steps > (Skv + 31) / 32) return "steps of a query block";
        long long last = 0;  // query of any of the block's tiles
        for (int t = b * per_block; t < std::min((b + 1) * per_block, q_tiles); ++t)
            last = std::max(last, std::min(t / group * 32LL + 31, Sq - 1LL));
        const long long reach = causal && !q.period ? last + q.diag : Skv - 1;
        if (steps * 32LL <= reach) return "keys left out";
        if ((steps - 1) * 32LL > reach) return "a step past the keys";
        q_units += n;
        if (n > q_most) q_most = n;
    }
    if (kv_units != p.kv_units || q_units != p.q_units) return "units";
    if (p.kv_chunk && p.kv_parts != kv_most) return "parts of keys";
    if (p.q_chunk && p.q_parts != q_most) return "parts of queries";
    const long long row_values = (long long)B * Hq * ((Sq + 31) / 32) * 64;
    if (bwd_workspace_floats(p, B, q, Hkv, Skv, d) <
        row_values + (p.kv_chunk ? 2 * kv_most * heads * Skv * d : 0) +
            (p.q_chunk ? q_most * B * Hq * Sq * d : 0))
        return "workspace";
    if ((p.kv_chunk || p.q_chunk) &&
        bwd_workspace_floats(p, B, q, Hkv, Skv, d) * 4 > kBwdMaxWorkspaceBytes)
        return "a workspace over the limit";
    // no block outlasts the rest of the work many times over, if splitting can help it
    double total = 0.0, longest = 0.0;
    for (int b = 0; b < p.kv_blocks; ++b) {
        const double steps = size.kv_steps(b);
        total += 1.25 * steps * heads;
        longest = std::max(longest, 1.25 * steps / bwd_parts((int)steps, p.kv_chunk));
    }
    for (int b = 0; b < p.q_blocks; ++b) {
        const double steps = size.q_steps(b);
        total += steps * heads;
        longest = std::max(longest, steps / bwd_parts((int)steps, p.q_chunk));
    }
    if (cus == 256 && longest > 30.0 && longest > 4.0 * total / cus) return "a block that outlasts the rest";
    const BwdUnits u = {size,      p.kv_blocks, p.q_blocks, p.kv_units, p.q_units,
                        p.kv_chunk, p.q_chunk,   p.ordered};
    // all heads in one range, as on devices whose dies they do not divide evenly among, or
    // one die's
    for (const int hx : {heads, 1}) {
        if (p.grid / heads * hx > 200000) continue;
        std::set<std::tuple<int, int, int, int>> seen;
        for (int i = 0; i < units * hx; ++i) {
            BwdWork w = bwd_work(u, p.order.unit, hx, planted && i == 3 ? 2 : i);
            const int blocks = w.kv ? p.kv_blocks : p.q_blocks;
            if (w.head < 0 || w.head >= hx) return "head";
            if (w.block < 0 || w.block >= blocks) return "block";
            const int steps = w.kv ? size.kv_steps(w.block)
                                   : size.q_steps(w.block);
            if (w.splits != bwd_parts(steps, w.kv ? p.kv_chunk : p.q_chunk)) return "splits";
            if (w.split < 0 || w.split >= w.splits) return "split";
            if ((long long)steps * (w.split + 1) / w.splits <= (long long)steps * w.split / w.splits)
                return "an empty part";
            if (!seen.insert({w.kv, w.head, w.block, w.split}).second) return "twice";
        }
        if ((long long)seen.size() != (long long)units * hx) return "left out";
    }
    return nullptr;
}

// The problem as it is, or (folded) as the kernels get it.
static BwdFold problem(int Hq, int Hkv, int Sq, int Skv, int d, int causal, bool folded) {
    return folded ? bwd_fold(Hq, Hkv, Sq, Skv, d, causal) : BwdFold{Hq, Sq, causal, Skv - Sq, 0};
}

int main(int argc, char** argv) {
    const bool planted = argc > 1 && !strcmp(argv[1], "--planted");
    std::mt19937 rng(7);
    auto log_int = [&](double lo, double hi) {
        return (int)exp(std::uniform_real_distribution<double>(log(lo), log(hi))(rng));
    };
    const int groups[][2] = {{1, 1}, {1, 8}, {2, 4}, {8, 4}, {8, 8}, {16, 1}, {32, 1}, {3, 5},
                             {40, 1}, {1, 64}};
    int n = 0, split = 0, unordered = 0, periods = 0;
    for (; n < 1500; ++n) {
        const int* g = groups[rng() % 10];
        const int B = 1 + rng() % 5, causal = rng() % 2, d = rng() % 2 ? 64 : 128;
        int Sq = log_int(1, 70000), Skv = rng() % 2 ? Sq : log_int(1, 70000);
        if (causal && Skv < Sq) std::swap(Sq, Skv);
        const BwdFold q = problem(g[0] * g[1], g[0], Sq, Skv, d, causal, rng() % 2);
        const char* why = check(rng() % 8 ? 256 : 1 + rng() % 304, B, q, g[0], Skv, d, planted);
        periods += q.period > 0;
        if (why && planted) {
            printf("caught: %s\n", why);
            return 0;
        }
        if (why) {
            printf("B=%d Hq=%d Hkv=%d Sq=%d Skv=%d d=%d causal=%d: %s\n", B, g[0] * g[1], g[0], Sq,
                   Skv, d, causal, why);
            return 1;
        }
        BwdPlan p;
        plan_bwd(256, B, q, g[0], Skv, d, &p);
        split += p.kv_chunk || p.q_chunk;
        unordered += causal && !p.ordered;
    }
    // one key/value head of many query heads; few keys under many queries and the reverse
    const int corners[][7] = {{1, 64, 1, 8192, 8192, 128, 1}, {1, 128, 1, 30000, 30000, 64, 1},
                              {8, 16, 16, 16384, 77, 128, 0}, {1, 64, 1, 200000, 256, 128, 0},
                              {2, 8, 8, 5, 300000, 128, 1}, {1, 1, 1, 8000000, 1, 64, 0},
                              {1, 1, 1, 1, 8000000, 128, 1}, {4, 32, 8, 32768, 32768, 128, 1}};
    for (const auto& c : corners)
        if (const char* why = check(256, c[0], problem(c[1], c[2], c[3], c[4], c[5], c[6], false),
                                    c[2], c[4], c[5], false))
            return printf("Hq=%d Hkv=%d Sq=%d Skv=%d: %s\n", c[1], c[2], c[3], c[4], why), 1;
    // heads folded into one: without a mask, or of a single query, up to 2 GiB; with a mask,
    // of less than a tile
    const int folds[][9] = {{8, 2, 100, 128, 0, 2, 400, 0, 0}, {8, 2, 100, 128, 1, 8, 100, 1, 0},
                            {8, 2, 1, 64, 1, 2, 4, 0, 0},      {4, 4, 7, 64, 0, 4, 7, 0, 0},
                            {8, 2, 31, 64, 1, 2, 124, 1, 31},  {8, 2, 32, 64, 1, 8, 32, 1, 0},
                            {4, 4, 7, 64, 1, 4, 7, 1, 0},
                            {4, 1, 1 << 22, 64, 0, 4, 1 << 22, 0, 0},
                            {3, 1, 1 << 22, 64, 0, 1, 3 << 22, 0, 0}};
    for (const auto& f : folds) {
        const BwdFold q = bwd_fold(f[0], f[1], f[2], 1 << 23, f[3], f[4]);
        if (q.Hq != f[5] || q.Sq != f[6] || q.causal != f[7] || q.period != f[8] ||
            (q.causal && q.diag != (1 << 23) - f[2]))
            return printf("fold\n"), 1;
    }
    // the limits: too many workgroups for a grid is no plan, not an overflow
    BwdPlan p;
    if (plan_bwd(256, 1 << 20, BwdFold{1 << 12, 4096, 0, 0, 0}, 1 << 12, 4096, 64, &p) ||
        plan_bwd(256, 1, BwdFold{1 << 30, 1 << 20, 0, 0, 0}, 1, 1 << 20, 64, &p))
        return printf("limit\n"), 1;
    // a launch's threads are counted in 32 bits: 2^24 workgroups of 256 are too many, of the
    // products (two of each head here) and of the row values (d = 128: two of each tile)
    const int many[][4] = {{1 << 23, 1, 64, 0}, {(1 << 23) - 1, 1, 64, 1}, {1 << 16, 128, 128, 0},
                           {(1 << 18) - 1, 32, 128, 1}, {1 << 20, 32, 64, 0}};
    for (const auto& c : many) {
        const bool is = plan_bwd(256, c[0], BwdFold{c[1], 1, 0, 0, 0}, 1, 1, c[2], &p);
        if (is != !!c[3] || (is && p.grid >= 1LL << 24))
            return printf("B=%d Hq=%d: %d\n", c[0], c[1], is), 1;
    }
    if (!split || !unordered || !periods) return printf("the sweep missed a kind\n"), 1;
    printf("bwd_plan_check ok: %d shapes, %d split, %d without an order\n", n, split, unordered);
    return planted;
}
