"""Sums of the weights as they are, in every form of paged attention: the bounds of the references
with nothing added to them (U |o| more would cover sums of weights rounded to bf16)."""
from __future__ import annotations

import math

import pytest
import torch

from tests import paged_refs as refs
from tests.gpu_common import announce
from tests.test_gpu_paged import BF16, DEV, ints, pa, scene  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [(4, 4), (32, 4)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("form", [dict(), dict(window=33, slopes=True), dict(softcap=20.0)],
                         ids=lambda f: "-".join(f) or "plain")
def test_without_a_log_sum_exp(pa, heads, form, d):  # noqa: F811
    announce(f"attn_paged sums without lse {heads} {form} d={d}")
    kw = dict(form)
    if kw.pop("slopes", None):
        kw["slopes"] = torch.linspace(0.02, 0.4, heads[0], device=DEV)
    s = scene([(1, 70), (300, 900), (9, 400), (0, 33), (33, 33)], *heads, d, 16)
    for dtype, step in ((BF16, refs.U), (torch.float32, 2.0 ** -24)):
        o = pa.attn_paged(s["q"], s["k"], s["v"], s["table"], ints(s["kv"]), ints(s["cu"]),
                          out_dtype=dtype, **kw)
        exact, _, bound, _ = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"],
                                               s["cu"], 1 / math.sqrt(d), out_step=step, **kw)
        refs.check(o, exact, bound, f"{dtype}")


@pytest.mark.parametrize("max_q", [1, 4, 8])
def test_beside_more_tokens_than_promised(pa, max_q):  # noqa: F811
    announce(f"attn_paged sums beside a broken max_q {max_q}")
    s = scene([(1, 500), (max_q, 900), (1, 33)], 8, 2, 64, 16)
    want, _, bound, _ = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"], s["cu"],
                                          0.125, out_step=2.0 ** -24)
    q = torch.cat([s["q"][:1], torch.randn(60, 8, 64, device=DEV).to(BF16), s["q"][1:]])
    table = torch.cat([s["table"][:1], s["table"]])
    o = pa.attn_paged(q, s["k"], s["v"], table, ints([500, 480, 900, 33]),
                      ints([0, 1, 61, 61 + max_q, 62 + max_q]), max_q=max_q)
    refs.check(torch.cat([o[:1], o[61:]]), want, bound, "the others")


def test_beside_bounds_that_make_no_sense(pa):  # noqa: F811
    announce("attn_paged sums beside wrong bounds")
    s = scene([(1, 300), (40, 500), (2, 70)], 8, 2, 64, 16)
    want, _, bound, _ = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"], s["cu"],
                                          0.125, out_step=2.0 ** -24)
    for cu, right in (([0, 1, 41, 2 ** 31 - 1], 41), ([0, 1, 0, -5], 1), ([0, 1, 1 << 30, 0], 1)):
        o = pa.attn_paged(s["q"], s["k"], s["v"], s["table"], ints(s["kv"]), ints(cu))
        refs.check(o[:right], want[:right], bound[:right], f"{cu}")
