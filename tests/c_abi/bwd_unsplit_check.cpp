// Host-only check of the backward pass's plan without splits (csrc/plan.cpp): every block in
// one part, no workspace but the row values, the launch of the blocks alone.  Built and run by
// tests/test_bwd_unsplit.py, under sanitizers.
#include <stdio.h>

#include <random>

#include "common.h"

using namespace attn;

int main() {
    std::mt19937 rng(7);
    int split = 0;
    const int n = 400;
    for (int i = 0; i < n; ++i) {
        const int d = rng() % 2 ? 64 : 128, causal = rng() % 2, B = 1 + rng() % 4;
        const int Hkv = 1 + rng() % 8, Hq = Hkv * (1 + rng() % 8);
        int Sq = 1 + rng() % (rng() % 2 ? 60 : 5000), Skv = 1 + rng() % 20000;
        if (causal && Skv < Sq) std::swap(Sq, Skv);
        const BwdFold q = bwd_fold(Hq, Hkv, Sq, Skv, d, causal);
        BwdPlan p, with;
        if (!plan_bwd(256, B, q, Hkv, Skv, d, &p, false) ||
            !plan_bwd(256, B, q, Hkv, Skv, d, &with, true))
            return printf("no plan\n"), 1;
        split += with.kv_chunk || with.q_chunk;
        const long long tiles = ((long long)q.Sq + 31) / 32;
        if (p.kv_chunk || p.q_chunk || p.kv_parts || p.q_parts || p.kv_units != p.kv_blocks ||
            p.q_units != p.q_blocks || p.grid != (long long)B * Hkv * (p.kv_blocks + p.q_blocks) ||
            bwd_workspace_floats(p, B, q, Hkv, Skv, d) != (long long)B * q.Hq * tiles * 64)
            return printf("B=%d Hq=%d Hkv=%d Sq=%d Skv=%d d=%d causal=%d\n", B, Hq, Hkv, Sq, Skv, d,
                          causal), 1;
    }
    if (!split) return printf("no shape would have been split\n"), 1;
    printf("bwd_unsplit_check ok: %d shapes, %d of them split otherwise\n", n, split);
    return 0;
}
