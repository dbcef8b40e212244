"""CPU tests of the training operators: what they refuse on the host, and the float64
references that the GPU tests compare with, against autograd and against differences."""
import ctypes
import math

import pytest
import torch

import paper_2609_29219_amd as pa
from tests import training_refs as refs

HAS_GPU = torch.cuda.is_available()
A = 1 << 20  # a fake, 16-byte-aligned address: never dereferenced


MB = 1 << 20


def bwd(q=A, k=A, v=A, o=A, lse=A, do=A, dlse=None, dq=A + MB, dk=A + 2 * MB, dv=A + 3 * MB, B=1,
        Hq=2, Hkv=1, Sq=4, Skv=4, d=64, scale=0.125, causal=0, flags=0, ws=None, ws_bytes=0):
    return pa.lib.attn_bwd(q, k, v, o, lse, do, dlse, dq, dk, dv, B, Hq, Hkv, Sq, Skv, d, scale,
                           causal, flags, ws, ws_bytes)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), pa.ATTN_EINVAL), (dict(k=None), pa.ATTN_EINVAL),
    (dict(o=None), pa.ATTN_EINVAL), (dict(lse=None), pa.ATTN_EINVAL),
    (dict(do=None), pa.ATTN_EINVAL), (dict(dk=None), pa.ATTN_EINVAL),
    (dict(v=A + 8), pa.ATTN_EINVAL), (dict(dq=A + 4), pa.ATTN_EINVAL),
    (dict(lse=A + 2), pa.ATTN_EINVAL), (dict(dlse=A + 1), pa.ATTN_EINVAL),
    (dict(B=0), pa.ATTN_EINVAL), (dict(Hq=-2), pa.ATTN_EINVAL), (dict(Hkv=0), pa.ATTN_EINVAL),
    (dict(Hq=3, Hkv=2), pa.ATTN_EINVAL), (dict(Sq=0), pa.ATTN_EINVAL),
    (dict(Skv=-1), pa.ATTN_EINVAL), (dict(flags=2), pa.ATTN_EINVAL),
    (dict(flags=8), pa.ATTN_EINVAL), (dict(scale=float("nan")), pa.ATTN_EINVAL),
    (dict(d=96), pa.ATTN_EUNSUPPORTED), (dict(causal=1, Sq=5), pa.ATTN_EUNSUPPORTED),
    (dict(Skv=0x7FFFFFFF // 256 + 1, d=128), pa.ATTN_EUNSUPPORTED),
    (dict(Sq=0x7FFFFFFF // 256 + 1, d=128), pa.ATTN_EUNSUPPORTED),
    # results over operands or each other: dq is 2 * 4 * 64 fp32 values, 2048 bytes
    (dict(dq=A), pa.ATTN_EINVAL), (dict(dk=A + 1008), pa.ATTN_EINVAL),
    (dict(dv=A + 2 * MB), pa.ATTN_EINVAL), (dict(dk=A + MB + 2032), pa.ATTN_EINVAL),
    (dict(dlse=A + MB + 2044), pa.ATTN_EINVAL),
])
def test_bwd_rejects_on_host(kw, code):
    assert bwd(**kw) == code
    assert pa.last_error() != ""


def heads(B=2, S=4, H=2, d=64, **kw):
    h = dict(ptr=A, batch_stride=S * H * d, row_stride=H * d, head_stride=d)
    h.update(kw)
    return pa.Heads(h["ptr"], h["batch_stride"], h["row_stride"], h["head_stride"])


def ref(h):
    return None if h is None else ctypes.byref(h)


def rope(q=0, k=0, v=0, qo=0, ko=0, vo=0, wq=A, wk=A, freq=A, pos=None, pstride=0, B=2, S=4, Hq=2,
         Hkv=2, d=64, rot=64, eps=1e-6, flags=0):
    views = [ref(heads() if t == 0 else t) for t in (q, k, v, qo, ko, vo)]
    return pa.lib.attn_qk_norm_rope(*views, wq, wk, freq, pos, pstride, B, S, Hq, Hkv, d, rot, eps,
                                    flags)


ROPE_REFUSALS = [
    (dict(q=None), pa.ATTN_EINVAL), (dict(k=heads(ptr=None)), pa.ATTN_EINVAL),
    (dict(q=heads(ptr=A + 8)), pa.ATTN_EINVAL), (dict(wq=None), pa.ATTN_EINVAL),
    (dict(wk=A + 4), pa.ATTN_EINVAL), (dict(freq=None), pa.ATTN_EINVAL),
    (dict(freq=A + 2), pa.ATTN_EINVAL), (dict(pos=A + 2), pa.ATTN_EINVAL),
    (dict(pos=A + 4, flags=32), pa.ATTN_EINVAL), (dict(pos=A, pstride=-4), pa.ATTN_EINVAL),
    (dict(q=heads(row_stride=-128)), pa.ATTN_EINVAL),
    (dict(k=heads(head_stride=60)), pa.ATTN_EINVAL),
    (dict(B=0), pa.ATTN_EINVAL), (dict(S=0), pa.ATTN_EINVAL), (dict(Hq=0), pa.ATTN_EINVAL),
    (dict(Hkv=-1), pa.ATTN_EINVAL), (dict(eps=-1e-6), pa.ATTN_EINVAL),
    (dict(eps=float("nan")), pa.ATTN_EINVAL), (dict(eps=float("inf")), pa.ATTN_EINVAL),
    (dict(flags=1), pa.ATTN_EINVAL), (dict(d=96), pa.ATTN_EUNSUPPORTED),
    (dict(rot=0), pa.ATTN_EUNSUPPORTED), (dict(rot=24), pa.ATTN_EUNSUPPORTED),
    (dict(rot=80), pa.ATTN_EUNSUPPORTED),
]


@pytest.mark.parametrize("kw,code", ROPE_REFUSALS + [
    (dict(flags=64), pa.ATTN_EINVAL),
    (dict(vo=None), pa.ATTN_EINVAL), (dict(v=None), pa.ATTN_EINVAL),
    # output rows that share memory: no batch stride, heads half a row apart, interleaved
    (dict(qo=heads(batch_stride=0)), pa.ATTN_EINVAL),
    (dict(ko=heads(head_stride=32)), pa.ATTN_EINVAL),
    (dict(vo=heads(row_stride=64, head_stride=64)), pa.ATTN_EINVAL),
])
def test_qk_norm_rope_rejects_on_host(kw, code):
    assert rope(**kw) == code
    assert pa.last_error() != ""


def rope_bwd(q=0, k=0, gq=0, gk=0, gv=0, qo=0, ko=0, vo=0, wq=A, wk=A, freq=A, pos=None, pstride=0,
             dqw=A, dkw=A, B=2, S=4, Hq=2, Hkv=2, d=64, rot=64, eps=1e-6, flags=0, ws=None,
             ws_bytes=0):
    views = [ref(heads() if t == 0 else t) for t in (gq, gk, gv, q, k, qo, ko, vo)]
    return pa.lib.attn_qk_norm_rope_bwd(*views, wq, wk, freq, pos, pstride, dqw, dkw, B, S, Hq,
                                        Hkv, d, rot, eps, flags, ws, ws_bytes)


@pytest.mark.parametrize("kw,code", ROPE_REFUSALS + [
    (dict(gq=None), pa.ATTN_EINVAL), (dict(gk=heads(ptr=A + 2)), pa.ATTN_EINVAL),
    (dict(vo=None), pa.ATTN_EINVAL), (dict(gv=None), pa.ATTN_EINVAL),
    (dict(qo=heads(row_stride=0)), pa.ATTN_EINVAL),
    (dict(dqw=None), pa.ATTN_EINVAL), (dict(dkw=A + 2), pa.ATTN_EINVAL),
    (dict(flags=128), pa.ATTN_EINVAL),
])
def test_qk_norm_rope_bwd_rejects_on_host(kw, code):
    assert rope_bwd(**kw) == code
    assert pa.last_error() != ""


@pytest.mark.parametrize("call", [
    lambda: pa.lib.attn_bwd_workspace_bytes(1, 3, 2, 4, 4, 64, 0),
    lambda: pa.lib.attn_bwd_workspace_bytes(1, 2, 2, 0, 4, 64, 0),
    lambda: pa.lib.attn_qk_norm_rope_bwd_workspace_bytes(0, 1, 1, 1, 64),
])
def test_workspace_queries_reject_on_host(call):
    assert call() == pa.ATTN_EINVAL
    assert pa.last_error() != ""


@pytest.mark.skipif(HAS_GPU, reason="checks the no-device path")
def test_valid_calls_without_device_are_hip_errors():
    assert bwd() == pa.ATTN_EHIP
    assert bwd(flags=1 | 4, dlse=A, causal=1) == pa.ATTN_EHIP
    # results right behind one another and behind the operands
    assert bwd(dk=A + MB + 2048, dv=A + MB + 2048 + 1024) == pa.ATTN_EHIP
    assert bwd(dq=A + 2048, dlse=A + MB - 32) == pa.ATTN_EHIP
    assert rope() == pa.ATTN_EHIP
    assert rope(v=None, vo=None, flags=8 | 16 | 32, rot=16, pos=A) == pa.ATTN_EHIP
    # heads outside tokens, one element of any stride, a broadcast input
    assert rope(qo=heads(batch_stride=512, row_stride=64, head_stride=256)) == pa.ATTN_EHIP
    assert rope(B=1, qo=heads(batch_stride=0), q=heads(batch_stride=0)) == pa.ATTN_EHIP
    assert rope(q=heads(batch_stride=0, row_stride=0, head_stride=0)) == pa.ATTN_EHIP
    assert rope_bwd() == pa.ATTN_EHIP
    assert rope_bwd(gv=None, vo=None, dqw=None, dkw=None, flags=64) == pa.ATTN_EHIP
    assert pa.lib.attn_bwd_workspace_bytes(1, 2, 2, 4, 4, 64, 0) == pa.ATTN_EHIP


def test_more_than_a_launch_holds_is_refused_on_host():
    # 2^24 tiles of 16 tokens; products that pass 64 bits
    big = 1 << 28
    assert rope(B=1, S=big) == pa.ATTN_EUNSUPPORTED
    assert rope_bwd(B=big, S=1) == pa.ATTN_EUNSUPPORTED
    assert rope(B=0x7FFFFFFF, S=0x7FFFFFFF) == pa.ATTN_EUNSUPPORTED
    assert pa.lib.attn_qk_norm_rope_bwd_workspace_bytes(1, big, 1, 1, 64) == pa.ATTN_EUNSUPPORTED
    n = 0x7FFFFFFF
    assert bwd(B=n, Hq=n, Hkv=n, Sq=1 << 23) == pa.ATTN_EUNSUPPORTED
    assert pa.lib.attn_bwd_workspace_bytes(n, n, n, 4, 4, 64, 0) == pa.ATTN_EUNSUPPORTED


def test_packed_calls_reach_the_same_checks():
    # (the last number of each call, and one before it)
    def packed_bwd(d=64, scale=0.125):
        ptrs = [A] * 6 + [0, A + MB, A + 2 * MB, A + 3 * MB, 0, 0, 0]
        return pa.lib.attn__bwd_packed(pa._BWD_CALL.pack(*ptrs, 1, 2, 1, 4, 4, d, 0, 0, scale))

    h = (A, 512, 128, 64)

    def packed_rope(v=h, rot=64, eps=1e-6):
        return pa.lib.attn__qk_norm_rope_packed(pa._ROPE_CALL.pack(
            *h, *h, *v, *h, *h, *h, A, A, A, 0, 0, 0, 2, 4, 2, 2, 64, rot, 0, eps))

    def packed_rope_bwd(v=h, rot=64, eps=1e-6):
        return pa.lib.attn__qk_norm_rope_bwd_packed(pa._ROPE_BWD_CALL.pack(
            *h, *h, *v, *h, *h, *h, *h, *h, A, A, A, 0, 0, A, A, 0, 0, 0, 2, 4, 2, 2, 64, rot, 0,
            eps))

    assert packed_bwd(d=96) == pa.ATTN_EUNSUPPORTED and "head dim 96" in pa.last_error()
    assert packed_bwd(scale=math.inf) == pa.ATTN_EINVAL and "scale" in pa.last_error()
    for call in (packed_rope, packed_rope_bwd):
        assert call(rot=24) == pa.ATTN_EUNSUPPORTED and "rot (24)" in pa.last_error()
        assert call(eps=-1.0) == pa.ATTN_EINVAL and "eps" in pa.last_error()
        assert call(v=(0, 0, 0, 0)) == pa.ATTN_EINVAL and "go together" in pa.last_error()


# ------------------------------------------------------------ the references --
@pytest.mark.parametrize("causal", [False, True])
def test_attention_reference_is_the_gradient(causal):
    g = torch.Generator().manual_seed(3)
    q, do = (torch.randn(2, 4, 5, 64, generator=g, dtype=torch.float64) for _ in range(2))
    k, v = (torch.randn(2, 2, 9, 64, generator=g, dtype=torch.float64) for _ in range(2))
    dlse = torch.randn(2, 4, 5, generator=g, dtype=torch.float64)
    scale = 0.125
    (dq, dk, dv), _ = refs.attn_backward(q, k, v, do, scale, causal, dlse)

    def loss(q, k, v):
        o, lse = refs.attn_forward(q, k, v, scale, causal)
        return float((o * do).sum() + (lse * dlse).sum())

    # central differences: the error is h^2 times a third derivative (of order one) plus
    # 1e-16 times the loss (of order 100) over h
    h = 1e-5
    for name, x, dx in (("q", q, dq), ("k", k, dk), ("v", v, dv)):
        for seed in range(3):
            u = torch.randn(x.shape, generator=g, dtype=torch.float64)
            args = dict(q=q, k=k, v=v)
            up, down = (loss(**{**args, name: x + s * h * u}) for s in (1, -1))
            assert abs((up - down) / (2 * h) - float((dx * u).sum())) < 1e-6, name


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [64, 48, 16])
def test_rotation_reference_is_the_gradient(interleaved, rot):
    g = torch.Generator().manual_seed(4)
    x = torch.randn(2, 3, 2, 64, generator=g, dtype=torch.float64)
    w = 1 + 0.2 * torch.randn(64, generator=g, dtype=torch.float64)
    grad = torch.randn(2, 2, 3, 64, generator=g, dtype=torch.float64)
    freq = 0.5 ** torch.arange(rot // 2, dtype=torch.float64)
    a = refs.rope_angles(3, 2, freq, torch.tensor([[5, 6, 7], [100, 101, 102]]), "cpu")
    dx, dw, _ = refs.rope_backward(grad, x, w, a, 1e-6, interleaved)

    def loss(x, w):
        return float((refs.rope_forward(x, w, a, 1e-6, interleaved) * grad).sum())

    h = 1e-5
    for _ in range(3):
        u = torch.randn(x.shape, generator=g, dtype=torch.float64)
        want = (loss(x + h * u, w) - loss(x - h * u, w)) / (2 * h)
        assert abs(want - float((dx * u).sum())) < 1e-6
        u = torch.randn(w.shape, generator=g, dtype=torch.float64)
        want = (loss(x, w + h * u) - loss(x, w - h * u)) / (2 * h)
        assert abs(want - float((dw * u).sum())) < 1e-6


def test_rotation_reference_turns_pairs():
    # lengths of pairs are kept, and two equal heads at positions p and p + n have an inner
    # product that depends on n alone
    x = torch.randn(1, 4, 1, 64, dtype=torch.float64, generator=torch.Generator().manual_seed(5))
    x[:] = x[:, :1]
    w = torch.ones(64, dtype=torch.float64)
    freq = 0.7 ** torch.arange(32, dtype=torch.float64)
    for interleaved in (False, True):
        a = refs.rope_angles(4, 1, freq, torch.tensor([3, 8, 1000, 1005]), "cpu")
        y = refs.rope_forward(x, w, a, 0.0, interleaved)[0, 0]
        assert torch.allclose(y.square().sum(-1), torch.full((4,), 64.0, dtype=torch.float64))
        assert math.isclose(float(y[0] @ y[1]), float(y[2] @ y[3]), rel_tol=1e-9)


# ----------------------------------------------------- Python-side refusals --
def test_python_refuses_tensors_off_the_device():
    x = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)
    lse = torch.zeros(1, 1, 4)
    with pytest.raises(TypeError):
        pa.attn_bwd(x, x, x, x, x, lse)
    w, f = torch.ones(64, dtype=torch.bfloat16), torch.ones(32)
    with pytest.raises(TypeError):
        pa.qk_norm_rope(x, x, x, w, w, f)
    with pytest.raises(TypeError):
        pa.qk_norm_rope_bwd(x, x, x, x, x, w, w, f)
