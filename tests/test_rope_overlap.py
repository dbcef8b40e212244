"""Results of qk_norm_rope and qk_norm_rope_bwd that share memory with each other or with an
operand: the host's test for it against every byte (CPU), and the calls' refusals (GPU)."""
from __future__ import annotations

import ctypes
import random
import time

import pytest
import torch

import paper_2609_29219_amd as pa
from tests.gpu_common import announce

HP = ctypes.POINTER(pa.Heads)


def meet(a, b, B, S, Ha, Hb, d, size_a=2, size_b=2):
    f = pa.lib.attn__rows_meet
    f.argtypes = [HP, HP] + [ctypes.c_int] * 7
    return bool(f(pa.Heads(*a), pa.Heads(*b), B, S, Ha, Hb, d, size_a, size_b))


def touched(a, B, S, H, d, size):
    at, sb, ss, sh = a
    return {at + (b * sb + s * ss + h * sh) * size + i for b in range(B) for s in range(S)
            for h in range(H) for i in range(0, d * size, 8)}


def nested(rng, B, S, H, d):
    """Strides of an order of the dimensions, each with some room behind."""
    dims, span = [("b", B), ("s", S), ("h", H)], d
    rng.shuffle(dims)
    strides = {}
    for name, n in dims:
        strides[name] = span + rng.choice((0, 0, 8, d, 3 * d))
        span = strides[name] * n
    return strides["b"], strides["s"], strides["h"], span


def test_rows_meet_is_every_byte():
    # sizes in steps of 8 bytes, as the strides and addresses are
    rng = random.Random(5)
    seen = [0, 0]
    for _ in range(4000):
        B, S, Ha, Hb = (rng.randint(1, 4) for _ in range(4))
        d = rng.choice((16, 32))
        size_a, size_b = 2, rng.choice((2, 4))
        *sa, span = nested(rng, B, S, Ha, d)
        kind = rng.randrange(4)
        if kind == 0:  # the same strides: slices of one buffer
            sb = list(sa)
        elif kind == 1:
            *sb, _ = nested(rng, B, S, Hb, d)
        elif kind == 2:  # an input: any strides, broadcast ones among them
            sb = [8 * rng.randrange(0, 40) for _ in range(3)]
        else:  # the same buffer in another order
            sb = [sa[1], sa[0], sa[2]]
        a = (1 << 20, *sa)
        b = ((1 << 20) + 8 * rng.randrange(-span // 4 - 40, span // 4 + 40), *sb)
        want = not touched(a, B, S, Ha, d, size_a).isdisjoint(touched(b, B, S, Hb, d, size_b))
        assert meet(a, b, B, S, Ha, Hb, d, size_a, size_b) == want, (a, b, B, S, Ha, Hb, d, size_b)
        seen[want] += 1
    assert min(seen) > 500, seen


def test_rows_meet_at_full_size():
    # the heads of a fused projection, a cache's rows, both halves of a joint cache, far tensors
    B, S, Hq, Hkv, d = 4, 8192, 32, 8, 128
    W = Hq + 2 * Hkv
    fused = [(1 << 30) + 2 * d * h for h in (0, Hq, Hq + Hkv)]
    strides = (S * W * d, W * d, d)
    for i, (at, H) in enumerate(zip(fused, (Hq, Hkv, Hkv))):
        for j, (to, G) in enumerate(zip(fused, (Hq, Hkv, Hkv))):
            assert meet((at, *strides), (to, *strides), B, S, H, G, d) == (i == j)
    assert meet((fused[0], *strides), (fused[1] - 16, *strides), B, S, Hq, Hkv, d)
    # one batch's last row reaches the next one's first
    assert meet((fused[0], *strides), (fused[0] + 2 * strides[0] * (B - 1) + 2 * strides[0] - 16,
                                       *strides), B, S, W, W, d)
    L = 20000  # [B, Hkv, L, 2, d]: keys and values side by side
    cache = (Hkv * L * 2 * d, 2 * d, L * 2 * d)
    assert not meet((1 << 30, *cache), ((1 << 30) + 2 * d, *cache), B, S, Hkv, Hkv, d)
    assert meet((1 << 30, *cache), ((1 << 30) + 4 * d * (S - 1), *cache), B, S, Hkv, Hkv, d)
    assert not meet((1 << 30, *cache), ((1 << 30) + 4 * d * S, *cache), B, S, Hkv, Hkv, d)
    # token-major against head-major in one buffer, and beside it
    heads = (Hq * S * d, d, S * d)
    whole = (S * Hq * d, Hq * d, d)
    assert meet((1 << 30, *heads), (1 << 30, *whole), B, S, Hq, Hq, d)
    assert not meet((1 << 30, *heads), ((1 << 30) + 2 * B * S * Hq * d, *whole), B, S, Hq, Hq, d)
    # a strange pair is decided, or left open, in bounded time
    t = time.perf_counter()
    meet((1 << 30, 1 << 30, 72 * 999, 72), ((1 << 30) + 16, 8 * 100003, 8 * 10007, 8 * 1009), 4, 8192,
         100, 100, 8)
    assert time.perf_counter() - t < 0.1


def case(B=2, S=6, Hq=4, Hkv=2, d=64):
    g = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    return dict(q=mk(B, S, Hq, d), k=mk(B, S, Hkv, d), v=mk(B, S, Hkv, d), q_weight=mk(d),
                k_weight=mk(d), inv_freq=torch.rand(d // 2, device="cuda"),
                positions=torch.arange(B * S, device="cuda").view(B, S))


@pytest.mark.gpu
def test_qk_norm_rope_refuses_shared_results():
    announce("qk_norm_rope shared results")
    c = case()
    B, S, Hq, d = c["q"].shape
    Hkv = c["k"].shape[2]
    want = pa.qk_norm_rope(**c)
    kept = {n: t.clone() for n, t in c.items()}
    buf = torch.full((B, Hq + Hkv, S, d), 7.0, dtype=torch.bfloat16, device="cuda")
    small = torch.zeros(B * S * Hkv * d * 2, device="cuda")  # fp32 and bf16 views of it
    heads = small[:B * S * Hkv * d // 2].view(torch.bfloat16).view(B, Hkv, S, d)
    refused = [
        dict(q_out=buf[:, :Hq], k_out=buf[:, Hq - 1:-1]),        # a head in common
        dict(k_out=buf[:, :Hkv], v_out=buf[:, :Hkv]),
        dict(q_out=buf[:, :1].expand(B, Hq, S, d)),              # its own rows
        dict(k_out=c["v"].transpose(1, 2)),                      # another operand
        dict(v_out=c["k"].transpose(1, 2)),
        dict(k_out=c["k"].view(B, Hkv, S, d)),                   # the operand's, in another order
        dict(k_out=heads, inv_freq=small[16:16 + d // 2]),
        dict(k_out=heads, positions=small[64:64 + B * S * 2].view(torch.int64).view(B, S)),
        dict(v_out=heads, q_weight=heads[0, 1, 2]),
    ]
    for kw in refused:
        with pytest.raises(pa.AttnError) as e:
            pa.qk_norm_rope(**{**c, **kw})
        assert e.value.code == pa.ATTN_EINVAL and "overlap" in str(e.value)
    torch.cuda.synchronize()
    assert (buf == 7.0).all() and not small.any()
    assert all(torch.equal(c[n], t) for n, t in kept.items())
    # neighbours in one buffer, and in place
    got = pa.qk_norm_rope(**c, q_out=buf[:, :Hq], k_out=buf[:, Hq:])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    got = pa.qk_norm_rope(**c, k_out=c["k"].transpose(1, 2), v_out=c["v"].transpose(1, 2))
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.gpu
def test_qk_norm_rope_bwd_refuses_shared_results():
    announce("qk_norm_rope_bwd shared results")
    c = case()
    B, S, Hq, d = c["q"].shape
    Hkv = c["k"].shape[2]
    c.pop("v")
    g = [torch.randn(B, H, S, d, device="cuda").to(torch.bfloat16) for H in (Hq, Hkv, Hkv)]
    want = pa.qk_norm_rope_bwd(*g, **c)
    kept = [t.clone() for t in (*g, *c.values())]
    buf = torch.full((B, S, Hq + 2 * Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    refused = [
        dict(dq_out=buf[:, :, :Hq], dk_out=buf[:, :, Hq - 1:Hq + 1]),
        dict(dk_out=buf[:, :, :Hkv], dv_out=buf[:, :, 1:Hkv + 1]),
        dict(dq_out=c["q"]), dict(dk_out=c["k"]), dict(dv_out=c["k"]),
        dict(dq_out=g[0].transpose(1, 2)), dict(dk_out=g[2].transpose(1, 2)),
    ]
    for kw in refused:
        with pytest.raises(pa.AttnError) as e:
            pa.qk_norm_rope_bwd(*g, **c, **kw)
        assert e.value.code == pa.ATTN_EINVAL and "overlap" in str(e.value)
    torch.cuda.synchronize()
    assert (buf == 7.0).all()
    assert all(torch.equal(a, b) for a, b in zip(kept, (*g, *c.values())))
    got = pa.qk_norm_rope_bwd(*g, **c, dv_out=buf[:, :, :Hkv], dq_out=buf[:, :, Hkv:Hkv + Hq],
                              dk_out=buf[:, :, Hkv + Hq:])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
