"""Paged attention with bounds of the requests past the queries' end: nothing but the results and
the workspace is written, and the requests that are right have their results.  (What the kernels
make of such bounds is held against the host's plan on the CPU, in test_paged_plan.py.)"""
from __future__ import annotations

import pytest
import torch

from tests.gpu_common import announce

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, I32 = torch.bfloat16, torch.int32


@pytest.mark.parametrize("window", [0, 60, 512])
@pytest.mark.parametrize("max_q", [1, 4, None])
@pytest.mark.parametrize("past", [1, 900, 20000, 2 ** 31 - 17])
def test_a_bound_far_past_the_queries(window, max_q, past):
    announce(f"attn_paged bound {past} past the queries, window={window} max_q={max_q}")
    import paper_2609_29219_amd as pa
    R, Hq, Hkv, d, page, kv = 16, 32, 8, 128, 16, 20000
    g = torch.Generator(device=DEV).manual_seed(past % 101)
    k, v = torch.randn(2, 40, Hkv, page, d, generator=g, device=DEV).to(BF16)
    q = torch.randn(R, Hq, d, generator=g, device=DEV).to(BF16)
    table = torch.randint(40, (R, kv // page), generator=g, device=DEV).int()
    kv_lens = torch.full((R,), kv, dtype=I32, device=DEV)
    cu = torch.arange(R + 1, dtype=I32, device=DEV)
    want = pa.attn_paged(q, k, v, table, kv_lens, cu, max_q=max_q, window=window)
    cu[R] = R + past
    n = pa.paged_workspace_bytes(R, R, Hq, Hkv, d, page, kv // page, max_q, window)
    ends = 1 << 20
    room = torch.full((n + 2 * ends,), 0x5a, dtype=torch.uint8, device=DEV)
    o = torch.full((R + 2, Hq, d), 7.0, device=DEV)
    pa.attn_paged(q, k, v, table, kv_lens, cu, max_q=max_q, window=window, o=o[1:-1],
                  workspace=room[ends:ends + n])
    assert torch.equal(o[1:R], want[:R - 1])
    assert (o[0] == 7.0).all() and (o[-1] == 7.0).all()
    assert (room[:ends] == 0x5a).all() and (room[ends + n:] == 0x5a).all()
