"""Paged attention without memory for the parts of its sums."""
from __future__ import annotations

import math

import pytest
import torch

from tests import paged_refs as refs
from tests.gpu_common import announce
from tests.test_bwd_unsplit import new_stream, workspace_limit  # noqa: F401 (a fixture)
from tests.test_gpu_paged import call, pa, scene  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(1, 3000), (2, 1500), (1, 0), (0, 40)], [(200, 5000)],
                                  [(1, 9000), (200, 1500), (5, 77)], [(1, 100)]],
                         ids=lambda l: "-".join(f"{n}of{k}" for n, k in l))
@pytest.mark.parametrize("form", [dict(), dict(window=600), dict(softcap=30.0)],
                         ids=lambda f: "-".join(f) or "plain")
def test_attn_paged_without_memory_for_parts(pa, workspace_limit, lens, d, form):  # noqa: F811
    announce(f"attn_paged without memory for parts {lens} d={d} {form}")
    s = scene(lens, 8, 2, d, 16)
    with_parts = call(pa, s, **form)
    exact, lse, bound, lse_bound = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"],
                                                     s["cu"], 1 / math.sqrt(d),
                                                     out_step=2.0 ** -24, **form)
    torch.cuda.synchronize()
    workspace_limit(0)
    stream = new_stream()
    with torch.cuda.stream(stream):
        got, again = call(pa, s, **form), call(pa, s, **form)
    stream.synchronize()
    for name, pair in (("parts", with_parts), ("none", got)):
        refs.check(pair[0], exact, bound, f"{name}: o")
        refs.check(pair[1], lse, lse_bound, f"{name}: lse")
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    # with memory again, the same stream runs in parts
    workspace_limit(-1)
    with torch.cuda.stream(stream):
        later = call(pa, s, **form)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(with_parts, later))


def test_a_workspace_that_is_too_small_is_refused_all_the_same(pa):  # noqa: F811
    announce("attn_paged small workspace")
    s = scene([(1, 9000), (200, 1500)], 8, 2, 64, 16)
    ws = torch.empty(1024, dtype=torch.uint8, device="cuda")
    with pytest.raises(pa.AttnError) as e:
        call(pa, s, workspace=ws)
    assert e.value.code == pa.ATTN_EINVAL
