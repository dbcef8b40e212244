"""GPU tests of attn_bwd, qk_norm_rope and qk_norm_rope_bwd against float64 references
(tests/training_refs.py), element by element within counted roundings."""
from __future__ import annotations

import math

import pytest
import torch

from tests import training_refs as refs
from tests.gpu_common import announce

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def pa():
    import paper_2609_29219_amd as pa
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    return pa


def randn(seed, *shape, mag=1.0, dtype=BF16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * mag).to(dtype)


def attn_case(B, Hq, Hkv, Sq, Skv, d, causal, scale=None, dlse=False, o=F32, mag=1.0, seed=1):
    """Inputs of attn_bwd, o and lse being the exact ones, rounded."""
    q, do = randn(seed, B, Hq, Sq, d, mag=mag), randn(seed + 1, B, Hq, Sq, d)
    k, v = randn(seed + 2, B, Hkv, Skv, d, mag=mag), randn(seed + 3, B, Hkv, Skv, d, mag=mag)
    sc = 1.0 / math.sqrt(d) if scale is None else scale
    out, lse = refs.attn_forward(q, k, v, sc, causal)
    return dict(q=q, k=k, v=v, do=do, o=out.to(o), lse=lse.float(), scale=scale, causal=causal,
                dlse=randn(seed + 4, B, Hq, Sq, dtype=F32) if dlse else None)


def attn_check(case, got, what, out_step=refs.U):
    sc = 1.0 / math.sqrt(case["q"].shape[-1]) if case["scale"] is None else case["scale"]
    exact, bound = refs.attn_backward(case["q"], case["k"], case["v"], case["do"], sc,
                                      case["causal"], case["dlse"],
                                      refs.U if case["o"].dtype is BF16 else 2.0 ** -24, out_step)
    for name, g, e, b in zip(("dq", "dk", "dv"), got, exact, bound):
        refs.check(g, e, b, f"{what}: {name}")


# query and key counts around tiles of 32, waves of 64 and blocks of 256; groups; splits
ATTN_SHAPES = [
    (1, 1, 1, 1, 1), (1, 1, 1, 1, 2), (2, 2, 1, 1, 300), (1, 1, 1, 5, 5), (1, 2, 2, 31, 33),
    (1, 1, 1, 32, 32), (2, 4, 2, 77, 131), (1, 8, 1, 64, 65), (1, 1, 1, 255, 257),
    (1, 3, 3, 256, 512), (1, 1, 1, 1000, 1000), (1, 2, 1, 129, 1500), (3, 6, 2, 300, 300),
    (1, 40, 40, 270, 290),
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", ATTN_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_attn_bwd(pa, shape, d, causal):
    announce(f"attn_bwd {shape} d={d} causal={causal}")
    case = attn_case(*shape, d, causal, dlse=shape[3] % 2 == 1)
    attn_check(case, pa.attn_bwd(**case), f"{shape} d={d}")


@pytest.mark.parametrize("shape", [(1, 64, 1, 700, 700, 64, True), (1, 96, 1, 400, 2000, 128, True),
                                   (2, 8, 8, 3000, 77, 128, False), (1, 16, 2, 1500, 1, 64, False),
                                   (1, 4, 1, 6000, 300, 128, False)],
                         ids=lambda s: "x".join(map(str, s)))
def test_attn_bwd_uneven(pa, shape):
    # many query heads on one key/value head (more units than the plan names in order), and
    # few keys under many queries: sums that are split into many parts
    announce(f"attn_bwd {shape}")
    case = attn_case(*shape)
    attn_check(case, pa.attn_bwd(**case), f"{shape}")


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", [(1, 5, 1, 100, 300), (2, 14, 2, 40, 40), (1, 24, 3, 8, 3000),
                                   (1, 7, 1, 33, 5000), (2, 32, 2, 130, 258), (1, 2, 2, 20, 128),
                                   (3, 3, 3, 600, 129), (1, 12, 4, 500, 385), (2, 7, 1, 31, 95),
                                   (1, 12, 4, 2, 40), (2, 9, 3, 17, 17), (1, 64, 1, 29, 700)],
                         ids=lambda s: "x".join(map(str, s)))
def test_attn_bwd_blocks_of_several_heads(pa, shape, d, causal):
    # tiles of several heads of a group in a block of queries, the last block not full, groups
    # that are no power of two; blocks of keys that are half empty; fewer queries than a tile,
    # whose heads share tiles, with a mask too
    B, Hq, Hkv, Sq, Skv = shape
    if causal and Sq > Skv:
        Sq, Skv = Skv, Sq
    announce(f"attn_bwd {shape} d={d} causal={causal}")
    case = attn_case(B, Hq, Hkv, Sq, Skv, d, causal, dlse=True)
    attn_check(case, pa.attn_bwd(**case), f"{shape} d={d}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [-0.1, 0.0, 0.3])
def test_attn_bwd_scales(pa, d, scale):
    announce(f"attn_bwd scale={scale} d={d}")
    case = attn_case(1, 4, 2, 100, 150, d, True, scale=scale)
    got = pa.attn_bwd(**case)
    attn_check(case, got, f"scale {scale}")
    if scale == 0.0:
        assert not got[0].any() and not got[1].any()


@pytest.mark.parametrize("o", [F32, BF16])
@pytest.mark.parametrize("out", [F32, BF16])
def test_attn_bwd_types(pa, o, out):
    announce(f"attn_bwd o={o} out={out}")
    for causal in (False, True):
        case = attn_case(1, 4, 2, 200, 230, 128, causal, o=o, dlse=True)
        got = pa.attn_bwd(**case, out_dtype=out)
        assert all(t.dtype is out for t in got)
        attn_check(case, got, f"{o} {out}", refs.U if out is BF16 else 2.0 ** -24)


def test_attn_bwd_large_scores(pa):
    # scores of up to some 60: most weights underflow, one key holds nearly all of a row
    announce("attn_bwd large scores")
    case = attn_case(1, 2, 2, 150, 150, 128, True, mag=2.5)
    attn_check(case, pa.attn_bwd(**case), "large scores")


def test_attn_bwd_against_differences(pa):
    # the derivative of <o, do> + <lse, dlse> in a direction, by central differences of the
    # exact forward pass in float64; the bound of the direction's sum is the elements'
    announce("attn_bwd differences")
    case = attn_case(1, 4, 2, 60, 90, 64, True, dlse=True)
    q, k, v, do, dlse = (case[n].double() for n in ("q", "k", "v", "do", "dlse"))
    got = pa.attn_bwd(**case, out_dtype=F32)
    _, bound = refs.attn_backward(case["q"], case["k"], case["v"], case["do"], 0.125, True,
                                  case["dlse"], out_step=2.0 ** -24)

    def loss(x):
        o, lse = refs.attn_forward(*x, 0.125, True)
        return float((o * do).sum() + (lse * dlse).sum())

    h = 1e-5
    for i in range(3):
        u = randn(90 + i, *(q, k, v)[i].shape, dtype=torch.float64)
        up, down = ([t + s * h * u if j == i else t for j, t in enumerate((q, k, v))]
                    for s in (1, -1))
        want = (loss(up) - loss(down)) / (2 * h)
        assert abs(want - float((got[i].double() * u).sum())) <= \
            float((bound[i] * u.abs()).sum()) + 1e-5


def test_attn_bwd_follows_attn_fwd(pa):
    # from the library's own output and log-sum-exp: attn_fwd's lse may be 2^-8 off, which
    # scales a row's weights by up to 1 + 2^-8 + 2^-17, and its o 2 u of its absolute terms
    announce("attn_bwd after attn_fwd")
    for d, out in ((64, F32), (128, BF16)):
        case = attn_case(2, 8, 2, 333, 333, d, True)
        o, lse = pa.attn_fwd(case["q"], case["k"], case["v"], causal=True, out_dtype=out,
                             return_lse=True)
        case.update(o=o, lse=lse)
        got = pa.attn_bwd(**case)
        exact, bound = refs.attn_backward(case["q"], case["k"], case["v"], case["do"],
                                          1 / math.sqrt(d), True)
        loose = refs.attn_backward(case["q"], case["k"], case["v"].abs(), case["do"].abs(),
                                   1 / math.sqrt(d), True, o_step=3 * refs.U)[1]
        for name, g, e, b, b2 in zip(("dq", "dk", "dv"), got, exact, bound, loose):
            refs.check(g, e, 2 * b + 2 * b2, f"after attn_fwd d={d}: {name}")


def test_attn_bwd_outputs_and_determinism(pa):
    # given outputs, prefilled with NaN inside guard values; the same bits each time
    announce("attn_bwd given outputs")
    for shape in ((1, 2, 1, 129, 1500), (2, 4, 2, 77, 131)):
        for out in (F32, BF16):
            case = attn_case(*shape, 128, True)
            first = pa.attn_bwd(**case, out_dtype=out)
            outs, bufs = [], []
            for t in first:
                buf = torch.full((t.numel() + 512,), 7.0, dtype=out, device=DEV)
                buf[256:-256] = float("nan")
                bufs.append(buf)
                outs.append(buf[256:-256].view(t.shape))
            got = pa.attn_bwd(**case, dq=outs[0], dk=outs[1], dv=outs[2])
            for a, b, g, buf in zip(first, got, outs, bufs):
                assert b.data_ptr() == g.data_ptr()
                assert torch.equal(a, b)
                assert (buf[:256] == 7.0).all() and (buf[-256:] == 7.0).all()


def test_attn_bwd_workspace(pa):
    announce("attn_bwd workspace")
    shape = (1, 2, 1, 129, 1500)
    case = attn_case(*shape, 64, True)
    want = pa.attn_bwd(**case)
    B, Hq, Hkv, Sq, Skv = shape
    n = pa.bwd_workspace_bytes(B, Hq, Hkv, Sq, Skv, 64, True)
    buf = torch.full((n + 256,), 0x5A, dtype=torch.uint8, device=DEV)
    got = pa.attn_bwd(**case, workspace=buf[:n])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert (buf[n:] == 0x5A).all()
    with pytest.raises(pa.AttnError):
        pa.attn_bwd(**case, workspace=buf[:n - 16])
    with pytest.raises(pa.AttnError):
        pa.attn_bwd(**case, workspace=buf[8:])
    with pytest.raises(TypeError):
        pa.attn_bwd(**case, workspace=torch.empty(n, dtype=torch.uint8))


def test_attn_bwd_refusals(pa):
    announce("attn_bwd refusals")
    case = attn_case(1, 2, 1, 40, 50, 64, False)
    for name, bad, error in (
            ("q", case["q"].float(), TypeError), ("do", case["do"].float(), TypeError),
            ("lse", case["lse"].double(), TypeError), ("o", case["o"].half(), TypeError),
            ("o", case["o"][:, :, :39], ValueError), ("lse", case["lse"][:, :1], ValueError),
            ("dlse", case["lse"][:, :, :39], ValueError),
            ("k", case["k"].transpose(2, 3).contiguous().transpose(2, 3), ValueError),
            ("do", case["do"].cpu(), TypeError)):
        with pytest.raises(error):
            pa.attn_bwd(**{**case, name: bad})
    with pytest.raises(ValueError):
        pa.attn_bwd(**case, out_dtype=torch.float16)
    with pytest.raises(TypeError):
        pa.attn_bwd(**case, dq=torch.empty_like(case["q"]), dk=case["k"].float())
    for n in ("dq", "dk"):  # a result in an operand's place, or in another result's
        with pytest.raises(pa.AttnError):
            pa.attn_bwd(**case, **{n: case["q" if n == "dq" else "k"]})
    both = torch.empty_like(case["k"])
    with pytest.raises(pa.AttnError):
        pa.attn_bwd(**case, dk=both, dv=both)
    wide = attn_case(1, 1, 1, 50, 50, 64, True)
    with pytest.raises(pa.AttnError):  # causal with fewer keys than queries
        pa.attn_bwd(**{**wide, "k": wide["k"][:, :, :40].contiguous(),
                       "v": wide["v"][:, :, :40].contiguous()})


def test_attn_bwd_streams(pa):
    # two streams at once, each with its own workspace, against one call at a time
    announce("attn_bwd streams")
    cases = [attn_case(1, 4, 2, 400, 900, 128, True, seed=s) for s in (10, 20)]
    want = [pa.attn_bwd(**c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(5):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                got[i].append(pa.attn_bwd(**c))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(want[i], g))


def replayed(fn, outs, refill, times=4):
    """Captures fn, then replays it with eager work in between; yields after each."""
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        fn()
    for i in range(times):
        refill(i)
        for o in outs:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        yield i


def test_attn_bwd_captured(pa):
    announce("attn_bwd captured")
    shape = (1, 4, 2, 300, 1100)
    cases = [attn_case(*shape, 128, True, dlse=True, seed=s) for s in (30, 40, 50, 60)]
    want = [pa.attn_bwd(**c) for c in cases]
    held = {n: t.clone() if isinstance(t, torch.Tensor) else t for n, t in cases[0].items()}
    outs = [torch.empty_like(t) for t in want[0]]
    torch.cuda.synchronize()

    def refill(i):
        for n, t in held.items():
            if isinstance(t, torch.Tensor):
                t.copy_(cases[i][n])

    for i in replayed(lambda: pa.attn_bwd(**held, dq=outs[0], dk=outs[1], dv=outs[2]), outs,
                      refill):
        assert all(torch.equal(a, b) for a, b in zip(want[i], outs)), f"replay {i}"
        other = pa.attn_bwd(**cases[(i + 1) % 4])  # eager, in between
        assert all(torch.equal(a, b) for a, b in zip(want[(i + 1) % 4], other))


# ------------------------------------------------------- norm and rotation --
def rope_case(B, S, Hq, Hkv, d, rot, start=0, fused=True, weight=BF16, seed=1, eps=1e-6,
              interleaved=False, pos=torch.int64):
    if fused:
        q, k, v = randn(seed, B, S, Hq + 2 * Hkv, d).split((Hq, Hkv, Hkv), dim=2)
    else:
        q, k, v = (randn(seed + i, B, S, H, d) for i, H in enumerate((Hq, Hkv, Hkv)))
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    positions = None
    if start:
        first = torch.arange(B, device=DEV)[:, None] * 1001 + start
        positions = (first + torch.arange(S, device=DEV)).to(pos)
    return dict(q=q, k=k, v=v, q_weight=(1 + 0.2 * randn(seed + 5, d, dtype=F32)).to(weight),
                k_weight=(1 + 0.2 * randn(seed + 6, d, dtype=F32)).to(weight),
                inv_freq=torch.pow(10000.0, -2 * i / rot).float(), positions=positions, eps=eps,
                interleaved=interleaved)


def case_angles(c):
    B, S = c["q"].shape[:2]
    return refs.rope_angles(S, B, c["inv_freq"], c["positions"], DEV)


def rope_check(c, got, what):
    """Products of a value of up to 12 x weight with cos and sin: each fp32 operation and the
    angle's 2^-22 turn the sum of absolute terms (a value and its pair) by less than 2^-18."""
    a = case_angles(c)
    for n, y in zip(("q", "k"), got):
        e = refs.rope_forward(c[n], c[n + "_weight"], a, c["eps"], c["interleaved"])
        size = refs.rope_forward(c[n], c[n + "_weight"], 0 * a, c["eps"], c["interleaved"]).abs()
        pair = size.amax(-1, keepdim=True)
        refs.check(y, e, e.abs() * refs.U + pair * 2.0 ** -18 + 1e-30, f"{what}: {n}")
    if c["v"] is None:
        assert got[2] is None
    else:
        assert torch.equal(got[2], c["v"].transpose(1, 2))


def rope_bwd_check(c, g, got, what):
    """fp32 operations: 2^-18 of the absolute terms, and 2^-20 of those of the weights' sums."""
    a = case_angles(c)
    dq, dk, dv, dqw, dkw = got
    for n, grad, dx, dw in (("q", g[0], dq, dqw), ("k", g[1], dk, dkw)):
        ex, ew, absw = refs.rope_backward(grad, c[n], c[n + "_weight"], a, c["eps"],
                                             c["interleaved"])
        x = c[n].double()
        r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + c["eps"])
        # |gw| and |n| mean(|gw n|) are at most the row's largest |g w| times 1 + |n|
        top = r * (grad.double().abs().amax(-1).transpose(1, 2)[..., None] * 2 *
                   c[n + "_weight"].double().abs().max()) * (1 + (x * r).abs().amax(-1, keepdim=True))
        refs.check(dx, ex, ex.abs() * refs.U + top * 2.0 ** -18 + 1e-30, f"{what}: d{n}")
        if dw is not None:
            refs.check(dw, ew, absw * 2.0 ** -20 + 1e-30, f"{what}: d{n}_weight")
    if g[2] is not None:
        assert torch.equal(dv, g[2].transpose(1, 2).to(BF16))


ROPE_SHAPES = [  # B, S, Hq, Hkv, d, rot
    (1, 1, 1, 1, 64, 64), (1, 1, 32, 8, 128, 128), (64, 1, 8, 1, 128, 64), (2, 3, 5, 5, 64, 16),
    (3, 50, 1, 1, 128, 96), (1, 333, 7, 1, 64, 48), (2, 177, 16, 16, 128, 128),
    (1, 4099, 4, 2, 64, 32), (5, 1000, 2, 1, 128, 16), (1, 20000, 1, 1, 64, 64),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", ROPE_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_qk_norm_rope(pa, shape, interleaved):
    announce(f"qk_norm_rope {shape} {interleaved}")
    i = ROPE_SHAPES.index(shape)
    c = rope_case(*shape, start=(0, 77)[i % 2], fused=i % 3 != 0, weight=(BF16, F32)[i % 2],
                  interleaved=interleaved, pos=(torch.int64, torch.int32)[i // 2 % 2])
    rope_check(c, pa.qk_norm_rope(**c), f"{shape}")


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", ROPE_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_qk_norm_rope_bwd(pa, shape, interleaved):
    announce(f"qk_norm_rope_bwd {shape} {interleaved}")
    i = ROPE_SHAPES.index(shape)
    B, S, Hq, Hkv, d, _ = shape
    c = rope_case(*shape, start=(77, 0)[i % 2], fused=i % 3 == 0, weight=(F32, BF16)[i % 2],
                  interleaved=interleaved, pos=(torch.int64, torch.int32)[i // 2 % 2])
    g = [randn(20 + j, B, H, S, d, dtype=(BF16, F32)[i // 2 % 2])
         for j, H in enumerate((Hq, Hkv, Hkv))]
    del c["v"]
    rope_bwd_check(c, g, pa.qk_norm_rope_bwd(*g, **c), f"{shape}")


def test_qk_norm_rope_far_positions(pa):
    # positions to 2^31 and below zero: the angles stay those of the exact product
    announce("qk_norm_rope far positions")
    c = rope_case(1, 8, 4, 2, 128, 128)
    for dtype, pos in ((torch.int64, [0, 1, 131071, 1 << 20, (1 << 24) + 1, -1, -4097, 10 ** 7]),
                       (torch.int32, [5, 4, 3, 2, 1, 0, -2, 9999999])):
        c["positions"] = torch.tensor(pos, dtype=dtype, device=DEV)
        rope_check(c, pa.qk_norm_rope(**c), f"positions {pos}")
    # at 2^31 the fp64 product is off by up to 2^-22 turns times 2^31 / 2^31: still 2^-18
    c["positions"] = torch.tensor([2 ** 31 - 1 - i for i in range(8)], device=DEV)
    rope_check(c, pa.qk_norm_rope(**c), "positions near 2^31")


def test_qk_norm_rope_strides_and_cache(pa):
    # batch and token dimensions exchanged, a broadcast batch, rows of a cache: the rest
    # of the cache is left as it was
    announce("qk_norm_rope strides")
    c = rope_case(3, 5, 4, 2, 64, 64, fused=False)
    c["q"] = c["q"].transpose(0, 1).contiguous().transpose(0, 1)
    c["k"] = c["k"][:1].expand(3, -1, -1, -1)
    caches = [torch.full((3, 2, 40, 64), 9.0, dtype=BF16, device=DEV) for _ in range(2)]
    views = [t[:, :, 17:22] for t in caches]
    q_out = torch.empty((5, 3, 4, 64), dtype=BF16, device=DEV).permute(1, 2, 0, 3)
    got = pa.qk_norm_rope(**c, q_out=q_out, k_out=views[0], v_out=views[1])
    assert got[0] is q_out and got[1] is views[0]
    rope_check(c, got, "strides")
    for t in caches:
        assert (t[:, :, :17] == 9.0).all() and (t[:, :, 22:] == 9.0).all()
    # one token into every row of the cache in turn, as decoding does
    c = rope_case(3, 1, 4, 2, 64, 64)
    for row in (0, 39):
        c["positions"] = torch.full((3, 1), row, device=DEV)
        got = pa.qk_norm_rope(**c, k_out=caches[0][:, :, row:row + 1],
                              v_out=caches[1][:, :, row:row + 1])
        rope_check(c, got, f"cache row {row}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_qk_norm_rope_in_place(pa, d, interleaved):
    announce(f"qk_norm_rope in place d={d} {interleaved}")
    for S, rot in ((1, d), (700, d), (333, d // 2)):
        c = rope_case(2, S, 5, 2, d, rot, start=9, interleaved=interleaved)
        want = pa.qk_norm_rope(**c)
        outs = {n + "_out": c[n].transpose(1, 2) for n in ("q", "k", "v")}
        got = pa.qk_norm_rope(**c, **outs)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        assert got[0].data_ptr() == c["q"].data_ptr()


def test_operators_on_streams(pa):
    # each stream's work behind its own copies, two streams at once
    announce("norm and rotation on streams")
    cs = [rope_case(2, 900, 8, 2, 128, 128, seed=s) for s in (1, 2)]
    gs = [[randn(90 + 3 * s + i, 2, H, 900, 128) for i, H in enumerate((8, 2, 2))]
          for s in range(2)]
    back = [{n: t for n, t in c.items() if n != "v"} for c in cs]
    want = [(*pa.qk_norm_rope(**c), *pa.qk_norm_rope_bwd(*g, **b))
            for c, g, b in zip(cs, gs, back)]
    torch.cuda.synchronize()
    got = [[], []]
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((*pa.qk_norm_rope(**cs[i]),
                               *pa.qk_norm_rope_bwd(*gs[i], **back[i])))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(want[i], g))


def test_qk_norm_rope_without_values(pa):
    announce("qk_norm_rope without values")
    c = rope_case(2, 9, 4, 2, 64, 32)
    c["v"] = None
    got = pa.qk_norm_rope(**c)
    rope_check(c, got, "no v")
    del c["v"]
    g = [randn(30 + i, 2, H, 9, 64) for i, H in enumerate((4, 2))] + [None]
    back = pa.qk_norm_rope_bwd(*g, **c, weight_grads=False)
    assert back[2] is None and back[3] is None and back[4] is None
    rope_bwd_check(c, g, back, "no v")


def test_qk_norm_rope_edge_values(pa):
    # a row of zeros stays zero, and its gradient is that of 1/sqrt(eps); huge and tiny rows
    announce("qk_norm_rope edge values")
    c = rope_case(1, 6, 2, 1, 128, 128, fused=False, eps=1e-5)
    c["q"][0, 0] = 0
    c["q"][0, 1] *= 1e15
    c["q"][0, 2] *= 1e-12
    rope_check(c, pa.qk_norm_rope(**c), "edges")
    assert not pa.qk_norm_rope(**c)[0][0, :, 0].any()
    v = c.pop("v")
    g = [randn(40 + i, 1, H, 6, 128) for i, H in enumerate((2, 1, 1))]
    rope_bwd_check(c, g, pa.qk_norm_rope_bwd(*g, **c), "edges")
    # a NaN row stays its own
    c["v"] = v
    c["q"][0, 3, 0, 5] = float("nan")
    y = pa.qk_norm_rope(**c)[0]
    assert torch.isnan(y[0, 0, 3]).all()
    y[0, 0, 3] = 0
    assert torch.isfinite(y).all()


def test_qk_norm_rope_bwd_against_differences(pa):
    announce("qk_norm_rope_bwd differences")
    c = rope_case(2, 7, 3, 1, 64, 48, start=1000, weight=F32)
    v = c.pop("v")
    g = [randn(50 + i, 2, H, 7, 64, dtype=F32) for i, H in enumerate((3, 1, 1))]
    dq, dk, dv, dqw, dkw = pa.qk_norm_rope_bwd(*g, **c)
    a = case_angles(c)
    h = 1e-5
    for n, grad, dx, dw in (("q", g[0], dq, dqw), ("k", g[1], dk, dkw)):
        x, w = c[n].double(), c[n + "_weight"].double()

        def loss(x, w):
            return float((refs.rope_forward(x, w, a, c["eps"], False) * grad.double()).sum())

        u = randn(60, *x.shape, dtype=torch.float64)
        want = (loss(x + h * u, w) - loss(x - h * u, w)) / (2 * h)
        # each element of dx is rounded by up to u of its value
        assert abs(want - float((dx.double() * u).sum())) <= \
            float((dx.double().abs() * u.abs()).sum()) * (refs.U + 2.0 ** -14) + 1e-5
        u = randn(61, 64, dtype=torch.float64)
        want = (loss(x, w + h * u) - loss(x, w - h * u)) / (2 * h)
        absw = refs.rope_backward(grad, x, w, a, c["eps"], False)[2]
        assert abs(want - float((dw.double() * u).sum())) <= \
            float((absw * u.abs()).sum()) * 2.0 ** -20 + 1e-5
    assert torch.equal(dv, g[2].transpose(1, 2).to(BF16))


def test_qk_norm_rope_bwd_outputs(pa):
    # by default the heads of one fused tensor; given ones, strided; the same bits
    announce("qk_norm_rope_bwd outputs")
    B, S, Hq, Hkv, d = 2, 700, 4, 2, 64
    c = rope_case(B, S, Hq, Hkv, d, 64)
    del c["v"]
    g = [randn(70 + i, B, H, S, d) for i, H in enumerate((Hq, Hkv, Hkv))]
    first = pa.qk_norm_rope_bwd(*g, **c)
    base = first[0]._base
    assert base.shape == (B, S, Hq + 2 * Hkv, d) and first[2]._base is base
    out = torch.full((B, S, Hq + 2 * Hkv + 1, d), 5.0, dtype=BF16, device=DEV)
    n = pa.qk_norm_rope_bwd_workspace_bytes(B, S, Hq, Hkv, d)
    ws = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device=DEV)
    again = pa.qk_norm_rope_bwd(*g, **c, dv_out=out[:, :, 1:3], dk_out=out[:, :, 3:5],
                                dq_out=out[:, :, 5:], workspace=ws[:n])
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    assert (out[:, :, 0] == 5.0).all() and (ws[n:] == 0x5A).all()
    with pytest.raises(pa.AttnError):
        pa.qk_norm_rope_bwd(*g, **c, workspace=ws[:n - 16])


def test_qk_norm_rope_refusals(pa):
    announce("qk_norm_rope refusals")
    c = rope_case(2, 6, 4, 2, 64, 32, start=5, fused=False)
    for name, bad, error in (
            ("q", c["q"].float(), TypeError), ("k", c["k"][:, :5], ValueError),
            ("v", c["v"][..., :32], ValueError), ("q", c["q"][0], ValueError),
            ("k", c["k"].transpose(2, 3).contiguous().transpose(2, 3), ValueError),
            ("q_weight", c["q_weight"][:32], ValueError),
            ("k_weight", c["k_weight"].float(), TypeError),
            ("inv_freq", c["inv_freq"].double(), TypeError),
            ("inv_freq", c["inv_freq"][:3].contiguous(), pa.AttnError),  # rot 6
            ("positions", c["positions"].float(), TypeError),
            ("positions", c["positions"][:, :5], ValueError),
            ("positions", c["positions"].t().contiguous().t(), ValueError),
            ("positions", c["positions"].cpu(), TypeError)):
        with pytest.raises(error):
            pa.qk_norm_rope(**{**c, name: bad})
    k_out = torch.empty(2, 1, 6, 64, dtype=BF16, device=DEV).expand(2, 2, 6, 64)
    with pytest.raises(pa.AttnError):  # two heads to one place
        pa.qk_norm_rope(**c, k_out=k_out)
    odd = torch.empty(2, 6, 4, 68, dtype=BF16, device=DEV)[..., :64]
    with pytest.raises(pa.AttnError):  # rows that are not 16-byte aligned
        pa.qk_norm_rope(**{**c, "q": odd})
    with pytest.raises(ValueError):
        pa.qk_norm_rope(**{**c, "v": None}, v_out=k_out)


def test_qk_norm_rope_captured(pa):
    announce("qk_norm_rope captured")
    cs = [rope_case(2, 100, 4, 2, 64, 64, start=100 * s, fused=False, seed=s) for s in (1, 2, 3, 4)]
    gs = [[randn(80 + 3 * s + i, 2, H, 100, 64) for i, H in enumerate((4, 2, 2))]
          for s in range(4)]
    want = []
    for c, g in zip(cs, gs):
        want.append((*pa.qk_norm_rope(**c),
                     *pa.qk_norm_rope_bwd(*g, **{n: t for n, t in c.items() if n != "v"})))
    held = {n: t.clone() if isinstance(t, torch.Tensor) else t for n, t in cs[0].items()}
    grads = [t.clone() for t in gs[0]]
    got = []
    torch.cuda.synchronize()

    def refill(i):
        for n, t in held.items():
            if isinstance(t, torch.Tensor):
                t.copy_(cs[i][n])
        for t, x in zip(grads, gs[i]):
            t.copy_(x)

    def both():
        got.extend((*pa.qk_norm_rope(**held), *pa.qk_norm_rope_bwd(
            *grads, **{n: t for n, t in held.items() if n != "v"})))

    for i in replayed(both, got, refill):
        assert all(torch.equal(a, b) for a, b in zip(want[i], got)), f"replay {i}"
        again = pa.qk_norm_rope(**cs[i])
        assert all(torch.equal(a, b) for a, b in zip(want[i], again))


# ----------------------------------------------------------- the whole layer --
@pytest.mark.parametrize("interleaved", [False, True])
def test_layer_gradients(pa, interleaved):
    """Projections -> qk_norm_rope -> attn_fwd -> attn_bwd -> qk_norm_rope_bwd, against
    autograd of the float64 formulas.  In the 2-norm, each of the eight roundings on the way
    (q, k, P, o, P and dS again, the gradients of q and k, those of the projections) turns a
    result by at most u, but for those of q and k, which the scores (up to some 6) amplify:
    8 + 2 * 6 roundings, 20 u."""
    announce("layer gradients")
    B, S, Hq, Hkv, d = 2, 150, 4, 2, 64
    c = rope_case(B, S, Hq, Hkv, d, 64, start=300, weight=F32, interleaved=interleaved)
    do = randn(9, B, Hq, S, d)
    q, k, v = pa.qk_norm_rope(**c)
    o, lse = pa.attn_fwd(q, k, v, causal=True, return_lse=True)
    dq, dk, dv = pa.attn_bwd(do, q, k, v, o, lse, causal=True)
    got = pa.qk_norm_rope_bwd(dq, dk, dv, **{n: t for n, t in c.items() if n != "v"})
    a = case_angles(c)
    leaves = [c[n].double().detach().requires_grad_() for n in ("q", "k", "v", "q_weight",
                                                                "k_weight")]
    qx = refs.rope_forward(leaves[0], leaves[3], a, c["eps"], interleaved)
    kx = refs.rope_forward(leaves[1], leaves[4], a, c["eps"], interleaved)
    vx = leaves[2].transpose(1, 2)
    loss = 0
    for b in range(B):
        for h in range(Hq):
            n = h // (Hq // Hkv)
            p = torch.softmax(refs.scores(qx[b, h], kx[b, n], 1 / math.sqrt(d), True), -1)
            loss = loss + ((p @ vx[b, n]) * do[b, h].double()).sum()
    want = torch.autograd.grad(loss, leaves)
    for n, g, w in zip(("q", "k", "v", "q_weight", "k_weight"), got, want):
        off = float((g.double() - w).norm() / w.norm())
        print(f"[layer] d{n}: {off:.2e}", flush=True)
        assert off <= 20 * refs.U, f"d{n}: {off}"


# ------------------------------------------------------------- large tensors --
def test_attn_bwd_past_32_bit_offsets(pa):
    # 2.3e9 values of q: the last batch, against float64 (gradients from the library's own o
    # and lse, so the bounds are those of test_attn_bwd_follows_attn_fwd)
    announce("attn_bwd past 32-bit offsets")
    B, Hq, S, d = 140, 128, 1024, 128
    q = torch.empty(B, Hq, S, d, dtype=BF16, device=DEV)
    do = torch.empty_like(q)
    for b in range(B):
        q[b], do[b] = randn(b, Hq, S, d), randn(1000 + b, Hq, S, d)
    k, v = randn(1, B, 1, S, d), randn(2, B, 1, S, d)
    o, lse = pa.attn_fwd(q, k, v, causal=True, out_dtype=BF16, return_lse=True)
    dq, dk, dv = pa.attn_bwd(do, q, k, v, o, lse, causal=True)
    last = slice(B - 1, B)
    args = (q[last], k[last], v[last], do[last], 1 / math.sqrt(d), True)
    exact, bound = refs.attn_backward(*args)
    loose = refs.attn_backward(args[0], args[1], args[2].abs(), args[3].abs(), *args[4:],
                               o_step=3 * refs.U)[1]
    for n, g, e, b1, b2 in zip(("dq", "dk", "dv"), (dq, dk, dv), exact, bound, loose):
        refs.check(g[last], e, 2 * b1 + 2 * b2, n)


def test_qk_norm_rope_past_32_bit_offsets(pa):
    announce("qk_norm_rope past 32-bit offsets")
    B, S, Hq, Hkv, d = 5, 1 << 16, 48, 8, 128  # 2.7e9 values, and the gradients in float32
    x = torch.empty(B, S, Hq + 2 * Hkv, d, dtype=BF16, device=DEV)
    x[-1] = randn(1, S, Hq + 2 * Hkv, d)
    x[:-1] = 1.0
    q, k, v = x.split((Hq, Hkv, Hkv), dim=2)
    c = rope_case(1, 1, 1, 1, d, d)
    c.update(q=q, k=k, v=v)
    tail = {n: t[-1:, -64:] if n in "qkv" else t for n, t in c.items()}
    tail["positions"] = torch.arange(S - 64, S, device=DEV)
    got = pa.qk_norm_rope(**c)
    rope_check(tail, [t[-1:, :, -64:] for t in got], "tail")
    del got, c["v"]
    g = [torch.zeros(B, H, S, d, device=DEV) for H in (Hq, Hkv, Hkv)]
    for t in g:
        t[-1, :, -64:] = torch.randn(t.shape[1], 64, d, device=DEV)
    back = pa.qk_norm_rope_bwd(*g, **c)
    rope_bwd_check(tail, [t[-1:, :, -64:] for t in g],
                   (*[t[-1:, -64:] for t in back[:3]], *back[3:]), "tail")
