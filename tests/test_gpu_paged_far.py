"""Paged attention at positions that fp32 does not hold: distances are differences of integers."""
from __future__ import annotations

import math

import pytest
import torch

from tests import paged_refs as refs
from tests.gpu_common import announce

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, I32 = torch.bfloat16, torch.int32
PAGE = 1 << 16


@pytest.fixture(scope="module")
def pa():
    import paper_2609_29219_amd as pa
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    return pa


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("softcap", [0.0, 20.0])
@pytest.mark.parametrize("new,window", [(1, 300), (7, 1000), (300, 100), (513, 700)])
@pytest.mark.parametrize("kv", [(1 << 24) + 3, (1 << 24) + 801, (1 << 25) + 1027, (1 << 30) - 5])
def test_slopes_in_a_window_far_on(pa, kv, new, window, softcap, d):
    # a window behind position 2^24: the first tile of a block holds keys that are near
    announce(f"attn_paged kv={kv} new={new} window={window} softcap={softcap} d={d}")
    g = torch.Generator(device=DEV).manual_seed(kv % 1009 + new)
    Hq, Hkv = 4, 2
    # the keys that some token sees lie in two pages, the others nowhere
    lo = kv - new - window + 1
    first, last = lo // PAGE, (kv - 1) // PAGE
    table = torch.full((1, last + 1), 1 << 30, dtype=I32, device=DEV)
    table[0, first:] = torch.arange(last + 1 - first, dtype=I32, device=DEV).flip(0)
    k, v = (torch.full((2, Hkv, PAGE, d), math.nan, dtype=BF16, device=DEV) for _ in range(2))
    j = torch.arange(lo, kv, device=DEV)
    at = table[0].long()[j // PAGE], j % PAGE
    kd, vd = torch.randn(2, kv - lo, Hkv, d, generator=g, device=DEV).to(BF16)
    k[at[0], :, at[1]], v[at[0], :, at[1]] = kd, vd
    q = torch.randn(new, Hq, d, generator=g, device=DEV).to(BF16)
    slopes = torch.tensor([0.5, 0.03, 0.25, 1.0], device=DEV)
    o, lse = pa.attn_paged(q, k, v, table, torch.tensor([kv], dtype=I32, device=DEV),
                           torch.tensor([0, new], dtype=I32, device=DEV), window=window,
                           softcap=softcap, slopes=slopes, return_lse=True)
    pos = torch.arange(new, device=DEV) + (kv - new - lo)
    for h in range(Hq):
        n = h // (Hq // Hkv)
        eo, el, bo, bl = refs.attend(q[:, h], kd[:, n], vd[:, n], pos, d ** -0.5, True, window,
                                     softcap, float(slopes[h]), out_step=2.0 ** -24)
        refs.check(o[:, h], eo, bo, f"head {h}: o")
        refs.check(lse[:, h], el, bl, f"head {h}: lse")
