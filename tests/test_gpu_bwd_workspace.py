"""A workspace that shares memory with a tensor of the call: the gradients' calls refuse it."""
from __future__ import annotations

import pytest
import torch

import paper_2609_29219_amd as pa
from tests.gpu_common import announce

pytestmark = pytest.mark.gpu


def randn(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def test_attn_bwd_refuses_a_shared_workspace():
    announce("attn_bwd workspace over tensors")
    B, Hq, Hkv, S, d = 1, 2, 1, 300, 64
    n = pa.bwd_workspace_bytes(B, Hq, Hkv, S, S, d, True)
    tensors = {"q": (Hq, S, d), "k": (Hkv, S, d), "v": (Hkv, S, d), "o": (Hq, S, d),
               "do": (Hq, S, d), "dq": (Hq, S, d), "dk": (Hkv, S, d), "dv": (Hkv, S, d)}
    # one buffer: the tensors (bf16), lse and dlse (fp32), then the workspace
    parts, at = {}, 0
    for name, (h, *rest) in tensors.items():
        parts[name] = (at, torch.bfloat16, (B, h, *rest), h * S * d * 2)
        at += h * S * d * 2
    for name in ("lse", "dlse"):
        parts[name] = (at, torch.float32, (B, Hq, S), Hq * S * 4)
        at += Hq * S * 4
    buf = torch.zeros(at + n + 64, dtype=torch.uint8, device="cuda")
    view = {name: buf[a:a + b].view(t).view(s) for name, (a, t, s, b) in parts.items()}
    for i, name in enumerate(("q", "k", "v", "do")):
        view[name].copy_(randn(i, *view[name].shape))
    o, lse = pa.attn_fwd(view["q"], view["k"], view["v"], causal=True, out_dtype=torch.bfloat16,
                         return_lse=True)
    view["o"].copy_(o)
    view["lse"].copy_(lse)
    kept = buf.clone()
    for name, (a, _, _, size) in parts.items():
        # over its first bytes, inside it, over its last ones
        for first in (a + 16 - n // 16 * 16, a, a + size - 16):
            if first < 0:
                continue
            with pytest.raises(pa.AttnError) as e:
                pa.attn_bwd(**view, causal=True, workspace=buf[first:first + n])
            assert e.value.code == pa.ATTN_EINVAL and "overlap" in str(e.value), name
    torch.cuda.synchronize()
    assert torch.equal(buf, kept)
    want = pa.attn_bwd(**{**view, "dq": None, "dk": None, "dv": None}, causal=True)
    got = pa.attn_bwd(**view, causal=True, workspace=buf[at:at + n])  # right behind them
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_qk_norm_rope_bwd_refuses_a_shared_workspace():
    announce("qk_norm_rope_bwd workspace over tensors")
    B, S, Hq, Hkv, d = 2, 40, 4, 2, 64
    c = dict(q=randn(1, B, S, Hq, d), k=randn(2, B, S, Hkv, d), q_weight=randn(3, d),
             k_weight=randn(4, d), inv_freq=torch.rand(d // 2, device="cuda"),
             positions=torch.arange(S, device="cuda"))
    g = [randn(5 + i, B, H, S, d) for i, H in enumerate((Hq, Hkv, Hkv))]
    n = pa.qk_norm_rope_bwd_workspace_bytes(B, S, Hq, Hkv, d)
    size = B * S * (Hq + 2 * Hkv) * d * 2
    buf = torch.full((size + n,), 0x3C, dtype=torch.uint8, device="cuda")
    out = buf[:size].view(torch.bfloat16).view(B, S, Hq + 2 * Hkv, d)
    outs = dict(dq_out=out[:, :, :Hq], dk_out=out[:, :, Hq:Hq + Hkv], dv_out=out[:, :, Hq + Hkv:])
    for first in (0, size - 16):
        with pytest.raises(pa.AttnError) as e:
            pa.qk_norm_rope_bwd(*g, **c, **outs, workspace=buf[first:first + n])
        assert e.value.code == pa.ATTN_EINVAL and "overlap" in str(e.value)
    torch.cuda.synchronize()
    assert (buf == 0x3C).all()
    want = pa.qk_norm_rope_bwd(*g, **c)
    got = pa.qk_norm_rope_bwd(*g, **c, **outs, workspace=buf[size:])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # without weight gradients the workspace is not used
    got = pa.qk_norm_rope_bwd(*g, **c, **outs, weight_grads=False, workspace=buf[:n])
    assert all(torch.equal(a, b) for a, b in zip(want[:3], got[:3]))
