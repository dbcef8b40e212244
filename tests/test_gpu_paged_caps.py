"""Caps up to the largest number there is."""
from __future__ import annotations

import pytest
import torch

from tests.gpu_common import announce
from tests.test_gpu_paged import call, pa, scene  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("softcap", [1e30, 2.3e38, 2.4e38, 3.4028234e38])
def test_the_largest_caps(pa, softcap, d):  # noqa: F811
    # what a score may be off is past every score then: means of the values with weights that
    # are numbers
    announce(f"attn_paged softcap={softcap} d={d}")
    s = scene([(1, 100), (40, 200), (90, 90)], 8, 2, d, 16)
    o, lse = call(pa, s, softcap=softcap)
    most = s["v"][s["v"].isfinite()].abs().max().float()
    assert o.isfinite().all() and (o.abs() <= most * (1 + 2.0 ** -7)).all()
    assert lse.isfinite().all()
