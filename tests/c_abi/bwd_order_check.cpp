// Host-only check that a plan holds no unset units (csrc/plan.cpp): its order, part of the
// causal kernels' arguments, is zero behind the units that it names, and all of it where it
// names none.  The stack is filled before each plan, so that unset ones are seen.  Built and run
// by tests/test_bwd_order.py.
#include <stdio.h>
#include <string.h>

#include <new>

#include "common.h"

using namespace attn;

__attribute__((noinline)) static int fill_stack() {
    volatile unsigned char place[65536];
    for (size_t i = 0; i < sizeof place; ++i) place[i] = 0xAB;
    return place[sizeof place / 2];
}

int main() {
    // named and unnamed, split and whole; without a mask
    const int shapes[][7] = {{1, 8, 8, 700, 900, 128, 1}, {1, 64, 1, 8192, 8192, 128, 1},
                             {2, 8, 2, 20, 5000, 64, 1},  {1, 1, 1, 1, 1, 64, 1},
                             {1, 2, 2, 300, 300, 128, 0}};
    int named = 0;
    for (const auto& s : shapes)
        for (int may_split = 0; may_split < 2; ++may_split) {
            alignas(BwdPlan) unsigned char place[sizeof(BwdPlan)];
            memset(place, fill_stack(), sizeof place);
            BwdPlan& p = *new (place) BwdPlan;
            if (!plan_bwd(256, s[0], bwd_fold(s[1], s[2], s[3], s[4], s[5], s[6]), s[2], s[4], s[5],
                          &p, may_split))
                return printf("no plan\n"), 1;
            const int units = p.ordered ? p.kv_units + p.q_units : 0;
            named += units > 0;
            for (int i = units; i < kBwdOrder; ++i)
                if (p.order.unit[i].kv || p.order.unit[i].block || p.order.unit[i].split)
                    return printf("Hq=%d Sq=%d Skv=%d: unit %d of %d is unset\n", s[1], s[3], s[4], i,
                                  units), 1;
        }
    if (!named) return printf("no plan with an order\n"), 1;
    printf("bwd_order_check ok\n");
    return 0;
}
