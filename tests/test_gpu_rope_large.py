"""qk_norm_rope and qk_norm_rope_bwd over more than 256 MB, which run kernels of their own (past
the caches): every row against float64, and the same bits as smaller calls on parts."""
from __future__ import annotations

import pytest
import torch

import paper_2609_29219_amd as pa
from tests import test_gpu_training as small
from tests import training_refs as refs
from tests.gpu_common import announce

pytestmark = pytest.mark.gpu

# B, S, Hq, Hkv, d, rot: 4 bytes of each value pass 2^28 bytes by little
SHAPES = [(1, 8209, 48, 8, 128, 128), (1, 8209, 48, 8, 128, 96), (1, 16411, 48, 8, 64, 64)]


def slices(S):
    """Three parts of the tokens, each below 2^28 bytes in every direction and type."""
    cut = [0, S // 3, 2 * S // 3 + 5, S]
    return list(zip(cut, cut[1:]))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_qk_norm_rope_past_the_caches(shape, interleaved):
    announce(f"qk_norm_rope past the caches {shape} {interleaved}")
    B, S, Hq, Hkv, d, _ = shape
    assert B * S * (Hq + 2 * Hkv) * d * 4 > 1 << 28
    c = small.rope_case(*shape, interleaved=interleaved)
    got = pa.qk_norm_rope(**c)
    small.rope_check(c, got, f"{shape}")
    for s, e in slices(S):
        part = {**c, **{n: c[n][:, s:e] for n in "qkv"},
                "positions": torch.arange(s, e, device="cuda")}
        for a, b in zip(got, pa.qk_norm_rope(**part)):
            assert torch.equal(a[:, :, s:e], b)


@pytest.mark.parametrize("grads", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_qk_norm_rope_bwd_past_the_caches(shape, interleaved, grads):
    announce(f"qk_norm_rope_bwd past the caches {shape} {interleaved} {grads}")
    B, S, Hq, Hkv, d, _ = shape
    c = small.rope_case(*shape, interleaved=interleaved)
    c.pop("v")
    g = [small.randn(20 + i, B, H, S, d, dtype=grads) for i, H in enumerate((Hq, Hkv, Hkv))]
    got = pa.qk_norm_rope_bwd(*g, **c)
    small.rope_bwd_check(c, g, (*got[:3], None, None), f"{shape}")
    # The weights' sums: a lane adds up to 48 rows (a tile's 48 heads, or two tiles' 24), a
    # workgroup up to 32 lanes, the rest is in double precision: 80 roundings of 2^-24 of the
    # sum of absolute terms, whose own errors (cos and sin 2^-21, the norm, five products) are
    # less than 32 of them.
    a = small.case_angles(c)
    for n, grad, dw in (("q", g[0], got[3]), ("k", g[1], got[4])):
        _, exact, terms = refs.rope_backward(grad, c[n], c[n + "_weight"], a, c["eps"], interleaved)
        refs.check(dw, exact, terms * 2.0 ** -17, f"{shape}: d{n}_weight")
    assert all(torch.equal(x, y) for x, y in zip(got, pa.qk_norm_rope_bwd(*g, **c)))
    for s, e in slices(S):
        part = {**c, **{n: c[n][:, s:e] for n in "qk"},
                "positions": torch.arange(s, e, device="cuda")}
        for x, y in zip(got, pa.qk_norm_rope_bwd(*(t[:, :, s:e] for t in g), **part,
                                                 weight_grads=False)[:3]):
            assert torch.equal(x[:, s:e], y)
