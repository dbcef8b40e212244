"""GPU tests of the paged cache's operators against their definitions (tests/paged_refs.py),
element by element within counted roundings.  Whatever a call must not read holds NaN (rows of
the cache) or numbers far outside (tables)."""
from __future__ import annotations

import math
import random

import pytest
import torch

from tests import paged_refs as refs
from tests.gpu_common import announce

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def pa():
    import paper_2609_29219_amd as pa
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    return pa


def ints(values):
    return torch.tensor(values, dtype=I32, device=DEV)


def scene(lens, Hq, Hkv, d, page, token_major=False, seed=1, mag=1.0, padded=0, hidden=None):
    """Requests of (new tokens, tokens in all): q, a cache, tables.  hidden: of each request, how
    many of its first keys no token sees."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)

    def randn(*shape):
        return (torch.randn(shape, generator=g, device=DEV) * mag).to(BF16)

    held = [-(-kv // page) for _, kv in lens]
    pages, most = sum(held) + 3, max(held + [1]) + 2
    order = list(range(pages))
    rng.shuffle(order)
    table = torch.full((len(lens), most), 1 << 30, dtype=I32)
    shape = (pages, page, Hkv, d) if token_major else (pages, Hkv, page, d)
    k, v = torch.full(shape, math.nan, dtype=BF16, device=DEV), \
        torch.full(shape, math.nan, dtype=BF16, device=DEV)
    if token_major:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    for r, (_, kv) in enumerate(lens):
        mine = [order.pop() for _ in range(held[r])]
        table[r, :held[r]] = ints(mine).cpu()
        for i, p in enumerate(mine):
            n = min(page, kv - i * page)
            k[p, :, :n], v[p, :, :n] = randn(Hkv, n, d), randn(Hkv, n, d)
    new = [n for n, _ in lens]
    cu = [sum(new[:r]) for r in range(len(new) + 1)]
    table = table.to(DEV)
    poisoned = table, k, v
    if hidden:  # keys out of every token's sight
        table2, k2, v2 = table.clone(), k.clone(), v.clone()
        for r, n in enumerate(hidden):
            for j in range(n):
                p = int(table[r, j // page])
                k2[p, :, j % page] = math.nan
                v2[p, :, j % page] = math.nan
            table2[r, :n // page] = -7
        poisoned = table2, k2, v2
    return dict(q=randn(sum(new) + padded, Hq, d), k=k, v=v, table=table, kv=[n for _, n in lens],
                cu=cu, poisoned=poisoned)


def call(pa, s, **kw):
    table, k, v = s["poisoned"]
    return pa.attn_paged(s["q"], k, v, table, ints(s["kv"]), ints(s["cu"]), return_lse=True, **kw)


def verify(pa, s, what, scale=None, out_dtype=F32, max_q=None, **kw):
    sc = 1.0 / math.sqrt(s["q"].shape[-1]) if scale is None else scale
    o, lse = call(pa, s, scale=scale, out_dtype=out_dtype, max_q=max_q, **kw)
    assert o.dtype is out_dtype
    step = refs.U if out_dtype is BF16 else 2.0 ** -24
    eo, else_, bo, bl = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"], s["cu"], sc,
                                          out_step=step, **kw)
    n = s["cu"][-1]
    refs.check(o[:n], eo[:n], bo[:n], f"{what}: o")
    refs.check(lse[:n], else_[:n], bl[:n], f"{what}: lse")


HEADS = [(1, 1), (8, 8), (8, 2), (32, 4), (14, 2), (40, 1)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_single_tokens(pa, heads, d):
    announce(f"attn_paged tokens {heads} d={d}")
    lens = [(1, n) for n in (1, 2, 31, 32, 33, 127, 128, 129, 500, 1000, 7)]
    verify(pa, scene(lens, *heads, d, 16), f"{heads}", max_q=1)


@pytest.mark.parametrize("page", [8, 16, 64, 256])
@pytest.mark.parametrize("token_major", [False, True])
def test_pages(pa, page, token_major):
    announce(f"attn_paged page={page} token_major={token_major}")
    lens = [(1, 300), (5, 5), (3, 257), (1, 1), (70, 513), (2, 8)]
    verify(pa, scene(lens, 8, 2, 128, page, token_major), f"page {page}")
    verify(pa, scene(lens, 8, 2, 64, page, token_major), f"page {page}")


# new tokens around blocks of rows; no context, some, much
CHUNKS = [(1, 1), (2, 2), (7, 100), (8, 8), (9, 40), (16, 16), (31, 31), (32, 700), (33, 33),
          (63, 64), (64, 65), (65, 1000), (127, 127), (128, 128), (129, 300), (255, 256),
          (256, 1500), (300, 300), (0, 50), (513, 513)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [(1, 1), (4, 1), (14, 2), (6, 6)],
                         ids=lambda h: "x".join(map(str, h)))
def test_chunks(pa, heads, d, causal):
    announce(f"attn_paged chunks {heads} d={d} causal={causal}")
    verify(pa, scene(CHUNKS, *heads, d, 16), f"{heads}", causal=causal)


@pytest.mark.parametrize("lens", [[c] for c in CHUNKS if c[0]] + [[(2000, 2000)], [(100, 9000)],
                                                                 [(1, 20000)], [(3, 6000)]],
                         ids=lambda c: "x".join(map(str, c[0])))
@pytest.mark.parametrize("heads", [(4, 1), (16, 8)], ids=lambda h: "x".join(map(str, h)))
def test_one_request(pa, lens, heads):
    announce(f"attn_paged {lens} {heads}")
    s = scene(lens, *heads, 128, 32)
    verify(pa, s, f"{lens}")
    verify(pa, s, f"{lens}, max_q", max_q=lens[0][0], out_dtype=BF16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [1, 2, 16, 100, 129, 1000])
def test_window(pa, window, d):
    announce(f"attn_paged window={window} d={d}")
    lens = [(1, 1), (1, 700), (4, 300), (40, 130), (300, 1200), (129, 129), (600, 600), (2, 2000)]
    hidden = [max(0, kv - new - window + 1) for new, kv in lens]
    verify(pa, scene(lens, 8, 2, d, 16, hidden=hidden), f"window {window}", window=window)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", [dict(softcap=5.0), dict(softcap=50.0), dict(slopes=True),
                                  dict(softcap=20.0, slopes=True),
                                  dict(softcap=20.0, slopes=True, window=65),
                                  dict(slopes=True, causal=False),
                                  dict(softcap=3.0, causal=False)],
                         ids=lambda f: "-".join(f"{k}{v}" for k, v in f.items()))
def test_scores(pa, form, d):
    announce(f"attn_paged {form} d={d}")
    lens = [(1, 1), (1, 700), (4, 300), (40, 130), (300, 1200), (129, 129), (7, 2000)]
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = torch.exp2(-torch.arange(1, 9, device=DEV).float())
    verify(pa, scene(lens, 8, 2, d, 16, mag=1.5), f"{form}", **form)


@pytest.mark.parametrize("scale", [-0.1, 0.0, 0.4])
def test_scales(pa, scale):
    announce(f"attn_paged scale={scale}")
    lens = [(1, 300), (200, 260), (6, 40)]
    verify(pa, scene(lens, 8, 2, 128, 16), f"scale {scale}", scale=scale)
    verify(pa, scene(lens, 8, 2, 64, 16), f"scale {scale}", scale=scale, softcap=10.0)


def test_rows_without_keys(pa):
    # an empty request, one with fewer tokens than new ones, and one without new ones
    announce("attn_paged rows without keys")
    lens = [(2, 0), (10, 4), (0, 0), (1, 0), (300, 100), (1, 60), (0, 9)]
    verify(pa, scene(lens, 8, 2, 128, 16), "no keys")
    verify(pa, scene(lens, 8, 2, 64, 16), "no keys, window", window=3)
    verify(pa, scene(lens, 8, 2, 64, 16), "no keys, all", causal=False)


@pytest.mark.parametrize("R", [255, 256, 257, 1000])
def test_many_requests(pa, R):
    announce(f"attn_paged R={R}")
    rng = random.Random(R)
    lens = [(rng.choice([0, 1, 1, 1, 2, 5]), rng.randint(5, 90)) for _ in range(R)]
    lens[R // 2] = (130, 150)
    verify(pa, scene(lens, 4, 2, 64, 8), f"R {R}")


def test_rows_behind_the_last(pa):
    announce("attn_paged padding")
    s = scene([(1, 40), (0, 7), (30, 90)], 8, 2, 128, 16, padded=9)
    o, lse = (torch.full((40, 8, 128), 7.0, device=DEV), None)
    got, lse = call(pa, s, o=o)
    assert got is o and (o[31:] == 7.0).all()
    exact, _, bound, _ = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"], s["cu"],
                                           1 / math.sqrt(128), out_step=2.0 ** -24)
    refs.check(o[:31], exact[:31], bound[:31], "padding")


def test_without_sums(pa):
    # one token of each request, strided queries, no list of where they begin
    announce("attn_paged without cu_seqlens")
    s = scene([(1, n) for n in (5, 100, 33)], 8, 4, 128, 16)
    wide = torch.randn(3, 24, 128, device=DEV).to(BF16)
    s["q"] = wide[:, 3:11]
    o = pa.attn_paged(s["q"], s["k"], s["v"], s["table"], ints(s["kv"]))
    exact, _, bound, _ = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"], s["cu"],
                                           1 / math.sqrt(128), out_step=2.0 ** -24)
    refs.check(o, exact, bound, "strided")
    head_major = s["q"].transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(o, pa.attn_paged(head_major, s["k"], s["v"], s["table"], ints(s["kv"])))


@pytest.mark.parametrize("new", [1, 3, 40, 300])
def test_bad_pages(pa, new):
    # a page number outside the cache, or more tokens than the table holds: that request's results
    # are NaN, the others' are as they were
    announce(f"attn_paged bad pages new={new}")
    lens = [(new, 400), (new, 350), (new, 310), (2, 90)]
    s = scene(lens, 8, 2, 128, 16)
    want, _ = call(pa, s)
    table = s["table"].clone()
    table[0, 3], table[1, 0] = -1, s["k"].shape[0]
    kv = list(s["kv"])
    kv[2] = table.shape[1] * 16 + 1
    o, lse = pa.attn_paged(s["q"], s["k"], s["v"], table, ints(kv), ints(s["cu"]),
                           return_lse=True)
    at = s["cu"][3]
    assert torch.equal(o[at:], want[at:])
    assert o[:at].isnan().all() and lse[:at].isnan().all()


def test_same_bits(pa):
    announce("attn_paged same bits")
    s = scene([(1, 3000), (200, 1500), (5, 77), (1, 1)], 16, 4, 128, 16)
    first = call(pa, s)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, call(pa, s)))


def test_large_scores(pa):
    # one key holds nearly all of a row; most weights underflow
    announce("attn_paged large scores")
    verify(pa, scene([(1, 300), (150, 400)], 4, 2, 128, 16, mag=3.0), "large")


def test_caller_workspace(pa):
    announce("attn_paged workspace")
    s = scene([(1, 3000), (200, 1500), (5, 77)], 16, 4, 128, 16)
    n = pa.paged_workspace_bytes(206, 3, 16, 4, 128, 16, s["table"].shape[1])
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    want = call(pa, s)
    got = call(pa, s, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    with pytest.raises(pa.AttnError) as e:
        call(pa, s, workspace=ws[:n - 16])
    assert e.value.code == pa.ATTN_EINVAL


def test_a_cache_past_32_bits(pa):
    # pages 2^31 values and more from the first
    announce("attn_paged large cache")
    pages = (1 << 32) // (8 * 16 * 128) + 40
    k = torch.zeros(pages, 8, 16, 128, dtype=BF16, device=DEV)
    v = torch.zeros(pages, 8, 16, 128, dtype=BF16, device=DEV)
    s = scene([(1, 200), (70, 300)], 16, 8, 128, 16)
    small = s["k"].shape[0]
    move = torch.tensor([pages - 1 - 2 * i if i % 2 else i for i in range(small)], device=DEV)
    k[move], v[move] = s["k"], s["v"]
    used = s["table"] < small
    table = torch.where(used, move[s["table"].clamp(0, small - 1).long()].int(), s["table"])
    want = pa.attn_paged(s["q"], s["k"], s["v"], s["table"], ints(s["kv"]), ints(s["cu"]))
    got = pa.attn_paged(s["q"], k, v, table, ints(s["kv"]), ints(s["cu"]))
    assert torch.equal(want, got)
    # and written there
    slots = ints([int(move[-1]) * 16 + 3, 5, -1, pages * 16, 2 ** 31 - 1])
    kn, vn = torch.randn(2, 5, 8, 128, device=DEV).to(BF16).unbind()
    k0 = k.clone()
    pa.paged_store(kn, vn, slots, k, v)
    k0[int(move[-1]), :, 3], k0[0, :, 5] = kn[0], kn[1]
    same = torch.equal(k.view(torch.int16), k0.view(torch.int16))  # (rows hold NaN)
    assert same
    assert torch.equal(v[int(move[-1]), :, 3], vn[0]) and torch.equal(v[0, :, 5], vn[1])


# ------------------------------------------------------------------ tables --
def extend_case(seed, R, page, most, spare, T_more=0, max_pages=None):
    rng = random.Random(seed)
    seq = [rng.choice([0, page, rng.randint(0, 5 * page)]) for _ in range(R)]
    new = [rng.choice([0, 1, rng.randint(0, most)]) for _ in range(R)]
    held = [-(-s // page) for s in seq]
    need = [-(-(s + n) // page) for s, n in zip(seq, new)]
    max_pages = max_pages or max(need) + 1
    order = list(range(1000, 1000 + sum(need) + 50))
    rng.shuffle(order)
    table = [[order.pop() if i < min(h, max_pages) else -9 for i in range(max_pages)] for h in held]
    n_free = sum(need) - sum(held) + spare
    return table, seq, new, order, max(n_free, 0), page, sum(new) + T_more


@pytest.mark.parametrize("case", [(1, 1, 16, 1, 3), (2, 1, 16, 5000, 0), (3, 7, 8, 30, 2, 5),
                                  (4, 256, 16, 40, 9), (5, 1024, 16, 9, 1, 3000),
                                  (6, 1025, 64, 20, 4), (7, 3000, 16, 6, 0, 1), (8, 5, 256, 900, 7),
                                  (9, 40, 16, 60, -5), (10, 40, 16, 300, 4, 0, 6),
                                  (11, 3, 8, 100, -40)],
                         ids=lambda c: "-".join(map(str, c)))
def test_extend(pa, case):
    announce(f"paged_extend {case}")
    table, seq, new, free, n_free, page, T = extend_case(*case)
    T = max(T, 1)
    *want, want_table = refs.extend(table, seq, new, free, n_free, page, T)
    got_table = ints(table)
    got = pa.paged_extend(got_table, ints(seq), ints(new), ints(free), ints([n_free]), page, T)
    for name, g, w in zip(("slots", "positions", "cu", "kv", "n_left"), got, want):
        assert g.tolist() == (w if isinstance(w, list) else [w]), name
    assert got_table.tolist() == want_table


def test_extend_again_after_a_release(pa):
    # too few pages; the same call after some came back
    announce("paged_extend again")
    page, table = 8, ints([[5, 6, -1, -1], [7, -1, -1, -1], [8, 9, 10, -1]])
    seq, new = ints([16, 3, 24]), ints([9, 4, 0])
    free, n_free = ints([3, 0, 0, 0, 0]), ints([1])
    *_, left = pa.paged_extend(table, seq, new, free, n_free, page, 13)
    assert left.tolist() == [-1]
    n_free = pa.paged_release(table, ints([0, 0, 24]), ints([0, 0, 1]), free, n_free, page)
    assert n_free.tolist() == [3] and free.tolist() == [3, 9, 10, 0, 0]
    slots, _, _, kv, left = pa.paged_extend(table, seq, new, free, n_free, page, 13)
    assert left.tolist() == [1] and kv.tolist() == [25, 7, 24]
    assert table.tolist()[0] == [5, 6, 10, 9] and (slots >= 0).all()


@pytest.mark.parametrize("case", [(1, 1, 16), (2, 9, 8), (3, 600, 16), (4, 2000, 32)],
                         ids=lambda c: "-".join(map(str, c)))
def test_release(pa, case):
    announce(f"paged_release {case}")
    seed, R, page = case
    rng = random.Random(seed)
    seq = [rng.choice([0, page, rng.randint(0, 700)]) for _ in range(R)]
    keep = [rng.choice([0, s, rng.randint(0, s), s + 100]) for s in seq]
    held = [-(-s // page) for s in seq]
    table = [[rng.randrange(1 << 20) if i < h else -9 for i in range(max(held) + 1)] for h in held]
    for room in (sum(held) + 20, max(3, sum(held) // 2)):
        free = [rng.randrange(1 << 20) for _ in range(room)]
        n_free = min(4, room)
        n_left, want = refs.release(table, seq, keep, free, n_free, page)
        got = ints(free)
        left = pa.paged_release(ints(table), ints(seq), ints(keep), got, ints([n_free]), page)
        assert left.tolist() == [n_left] and got.tolist() == want


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,Hkv", [(1, 1), (3, 8), (77, 5), (1000, 2)])
@pytest.mark.parametrize("token_major", [False, True])
def test_store(pa, T, Hkv, d, token_major):
    announce(f"paged_store T={T} Hkv={Hkv} d={d} token_major={token_major}")
    g = torch.Generator(device=DEV).manual_seed(T)
    page, pages = 16, T // 16 + 4
    shape = (pages, page, Hkv, d) if token_major else (pages, Hkv, page, d)
    k, v = (torch.randn(shape, generator=g, device=DEV).to(BF16) for _ in range(2))
    if token_major:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    x = torch.randn(T, 2 * Hkv, d, generator=g, device=DEV).to(BF16)
    kn, vn = x.split(Hkv, 1)
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:T].int()
    slots[::5] = -1
    if T > 3:
        slots[1] = pages * page
    want = [k.clone(), v.clone()]
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            want[0][s // page, :, s % page], want[1][s // page, :, s % page] = kn[t], vn[t]
    pa.paged_store(kn, vn, slots, k, v)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


# ---------------------------------------------------------- as they are used --
@pytest.mark.parametrize("heads", [(4, 4), (32, 4)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("form", [dict(), dict(window=33, slopes=True)],
                         ids=lambda f: "-".join(f) or "plain")
def test_without_lse(pa, heads, form):
    # sums of the weights as rounded to bf16: off by as much again as the weights themselves
    announce(f"attn_paged without lse {heads} {form}")
    kw = dict(form)
    if kw.pop("slopes", None):
        kw["slopes"] = torch.linspace(0.02, 0.4, heads[0], device=DEV)
    for d in (64, 128):
        s = scene([(1, 70), (300, 900), (9, 400), (0, 33), (33, 33)], *heads, d, 16)
        o = pa.attn_paged(s["q"], s["k"], s["v"], s["table"], ints(s["kv"]), ints(s["cu"]),
                          out_dtype=BF16, **kw)
        exact, _, bound, _ = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"],
                                               s["cu"], 1 / math.sqrt(d), **kw)
        refs.check(o, exact, bound + 1.01 * refs.U * exact.abs(), f"d={d}")


@pytest.mark.parametrize("d", [64, 128])
def test_a_run_of_steps(pa, d):
    # prompts, single tokens, drafts of which some are taken back, a request that ends and another
    # in its place; each step normalised and rotated, stored, and attended to
    announce(f"paged steps d={d}")
    Hq, Hkv, page, P, most = 8, 2, 16, 64, 30
    g = torch.Generator(device=DEV).manual_seed(d)
    freq = 10000.0 ** (-torch.arange(0, d, 2, device=DEV).float() / d)
    wq, wk = (torch.rand(d, generator=g, device=DEV) + 0.5 for _ in range(2))
    cache = torch.full((P, page, 2, Hkv, d), math.nan, dtype=BF16, device=DEV)
    k_pages, v_pages = (cache[:, :, i].transpose(1, 2) for i in range(2))
    table = torch.full((4, most), -1, dtype=I32, device=DEV)
    free = torch.randperm(P, generator=g, device=DEV).int()
    n_free, seq = ints([P]), ints([0, 0, 0, 0])
    mine = [[torch.zeros(Hkv, 0, d, dtype=BF16, device=DEV)] * 2 for _ in range(4)]
    steps = [([37, 5, 300, 1], None), ([1, 20, 1, 1], None), ([4, 4, 4, 4], [1, 3, 4, 2]),
             ([1, 1, 50, 0], [1, 1, 50, -2]), ([1, 1, 1, 60], None), ([2, 2, 2, 2], [2, 0, 1, 2])]
    for at, (new, keep) in enumerate(steps):
        T = sum(new) + at % 3
        qkv = torch.randn(1, T, Hq + 2 * Hkv, d, generator=g, device=DEV).to(BF16)
        slots, pos, cu, kv, left = pa.paged_extend(table, seq, ints(new), free, n_free, page, T)
        q, k, _ = pa.qk_norm_rope(qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], None, wq, wk, freq, pos)
        q, k, v = q[0].transpose(0, 1), k[0].transpose(0, 1), qkv[0, :, Hq + Hkv:]
        pa.paged_store(k, v, slots, k_pages, v_pages)
        o, lse = pa.attn_paged(q, k_pages, v_pages, table, kv, cu, max_q=max(new),
                               return_lse=True)
        starts = cu.tolist()
        for r, n in enumerate(new):
            a, b = starts[r], starts[r + 1]
            mine[r] = [torch.cat([old, x[a:b].transpose(0, 1)], 1)
                       for old, x in zip(mine[r], (k, v))]
            S = mine[r][0].shape[1]
            assert kv.tolist()[r] == S
            for h in range(Hq if n else 0):
                eo, el, bo, bl = refs.attend(q[a:b, h], *(x[h // (Hq // Hkv)] for x in mine[r]),
                                             torch.arange(S - n, S, device=DEV), 1 / math.sqrt(d),
                                             True, out_step=2.0 ** -24)
                refs.check(o[a:b, h], eo, bo, f"step {at} request {r}: o")
                refs.check(lse[a:b, h], el, bl, f"step {at} request {r}: lse")
        n_free, seq = left, kv
        if keep:  # (-2: the request ends)
            held = [0 if n == -2 else s - m + n for s, m, n in zip(kv.tolist(), new, keep)]
            n_free = pa.paged_release(table, kv, ints(held), free, left, page)
            seq = ints(held)
            mine = [[x[:, :n] for x in old] for old, n in zip(mine, held)]
        live = sum(-(-n // page) for n in seq.tolist())
        assert n_free.tolist() == [P - live]
        used = [table[r, i].item() for r in range(4) for i in range(-(-seq.tolist()[r] // page))]
        assert sorted(used + free[:P - live].tolist()) == list(range(P))


def test_replayed_steps(pa):
    # a step of decoding as one graph, its lengths and tables going on from replay to replay;
    # another graph on the same workspace, and eager calls between
    announce("paged steps in a graph")
    R, Hq, Hkv, d, page, P = 5, 16, 4, 128, 16, 400
    g = torch.Generator(device=DEV).manual_seed(9)

    def start():
        s = dict(table=torch.full((R, 100), -1, dtype=I32, device=DEV), seq=ints([0] * R),
                 free=torch.arange(P, dtype=I32, device=DEV), n_free=ints([P]))
        s["k"], s["v"] = (torch.zeros(P, Hkv, page, d, dtype=BF16, device=DEV) for _ in range(2))
        s["q_in"] = torch.zeros(R, Hq + 2 * Hkv, d, dtype=BF16, device=DEV)
        s["outs"] = [ints([0] * n) for n in (R, R, R + 1, R, 1)]
        s["o"] = torch.zeros(R, Hq, d, dtype=BF16, device=DEV)
        return s

    ones = ints([1] * R)

    def step(s):
        x = s["q_in"]
        names = ("slots", "positions", "cu_seqlens", "kv_lens", "n_left")
        slots, _, cu, kv, left = pa.paged_extend(s["table"], s["seq"], ones, s["free"], s["n_free"],
                                                 page, R, **dict(zip(names, s["outs"])))
        pa.paged_store(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], slots, s["k"], s["v"])
        pa.attn_paged(x[:, :Hq], s["k"], s["v"], s["table"], kv, cu, max_q=1, o=s["o"])
        torch.add(kv, 0, out=s["seq"])
        torch.add(left, 0, out=s["n_free"])

    prompt = [40, 700, 1, 333, 90]
    kv = torch.randn(2, sum(prompt), Hkv, d, generator=g, device=DEV).to(BF16)
    states = [start() for _ in range(3)]  # eager, and of two graphs
    for s in states:
        slots, _, _, lens, left = pa.paged_extend(s["table"], s["seq"], ints(prompt), s["free"],
                                                  s["n_free"], page, sum(prompt))
        pa.paged_store(kv[0], kv[1], slots, s["k"], s["v"])
        s["seq"], s["n_free"] = lens, left
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = []
    for s in states[1:]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            step(s)
    for i in range(5):
        x = torch.randn(R, Hq + 2 * Hkv, d, generator=g, device=DEV).to(BF16)
        for s in states:
            s["q_in"].copy_(x)
            s["o"].fill_(math.nan)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            step(states[0])
        torch.cuda.synchronize()
        assert states[0]["o"].isfinite().all()
        for s in states[1:]:
            for name in ("o", "table", "seq", "n_free"):
                assert torch.equal(s[name], states[0][name]), f"replay {i}: {name}"
    assert states[1]["seq"].tolist() == [n + 5 for n in prompt]


def test_two_streams_at_once(pa):
    announce("attn_paged on two streams")
    scenes = [scene([(1, 3000), (200, 1500), (5, 77)], 16, 4, 128, 16, seed=n) for n in (1, 2)]
    want = [call(pa, s) for s in scenes]
    streams = [torch.cuda.Stream() for _ in scenes]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for s, on in zip(scenes, streams):
            with torch.cuda.stream(on):
                got.append(call(pa, s))
    torch.cuda.synchronize()
    for i, pair in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(pair, want[i % 2]))


def test_workspace_of_any_content(pa):
    announce("attn_paged workspace content")
    s = scene([(1, 3000), (200, 1500), (5, 77), (0, 50), (1, 0)], 16, 4, 128, 16)
    n = pa.paged_workspace_bytes(207, 5, 16, 4, 128, 16, s["table"].shape[1])
    want = call(pa, s)
    for fill in (0, 0x7f, 0xff):
        ws = torch.full((n,), fill, dtype=torch.uint8, device=DEV)
        assert all(torch.equal(a, b) for a, b in zip(want, call(pa, s, workspace=ws)))


def test_workspace_over_an_operand(pa):
    announce("attn_paged workspace overlaps")
    s = scene([(1, 3000), (2, 1500)], 16, 4, 128, 16)
    n = pa.paged_workspace_bytes(3, 2, 16, 4, 128, 16, s["table"].shape[1])
    room = torch.empty(n + 3 * 16 * 128 * 2, dtype=torch.uint8, device=DEV)
    q = room[n - n % 16 - 16:][:3 * 16 * 128 * 2].view(BF16).view(3, 16, 128)
    with pytest.raises(pa.AttnError) as e:
        pa.attn_paged(q, s["k"], s["v"], s["table"], ints(s["kv"]), ints(s["cu"]),
                      workspace=room[:n])
    assert e.value.code == pa.ATTN_EINVAL


@pytest.mark.parametrize("page,max_pages", [(1024, 3), (8, 4000), (65536, 1)])
def test_extreme_pages(pa, page, max_pages):
    # a wide table, a cache of one page, pages longer than their request
    announce(f"attn_paged pages of {page}")
    lens = [(1, 2000)] if max_pages == 1 else [(1, 2000), (70, 300), (3, 1100), (1, 9)]
    s = scene(lens, 8, 2, 64, page)
    if max_pages == 1:
        p = int(s["table"][0, 0])
        s["k"], s["v"], s["table"] = s["k"][p:p + 1], s["v"][p:p + 1], ints([[0]])
    elif max_pages > s["table"].shape[1]:
        wide = torch.full((len(lens), max_pages + 100), 1 << 30, dtype=I32, device=DEV)
        wide[:, :s["table"].shape[1]] = s["table"]
        s["table"] = wide[:, :max_pages]
    s["poisoned"] = s["table"], s["k"], s["v"]
    verify(pa, s, f"page {page}")
    verify(pa, s, f"page {page}", window=100)


@pytest.mark.parametrize("R", [65, 300])
def test_many_long_requests(pa, R):
    # more requests than a wave, or a workgroup, finds its own among in one go
    announce(f"attn_paged {R} requests of many rows")
    lens = [(17 + r % 9 if r % 3 else 1, 40 + 13 * (r % 17)) for r in range(R)]
    verify(pa, scene(lens, 8, 2, 64, 16), f"{R}")


def test_a_window_without_end(pa):
    # (with more new tokens than tokens: positions below zero less the largest window)
    announce("attn_paged largest windows")
    s = scene([(1, 100), (40, 200), (1, 3)], 8, 2, 64, 16)
    s["kv"] = [100, 30, 3]
    want = call(pa, s)
    for window in (2 ** 31 - 1, 2 ** 31 - 2, s["table"].shape[1] * 16):
        got = call(pa, s, window=window)
        assert all(torch.equal(a, b) for a, b in zip(want, got)), window
    verify(pa, s, "no window")
    verify(pa, s, "window", window=201)


@pytest.mark.parametrize("max_q", [1, 4, 8])
def test_more_tokens_than_promised(pa, max_q):
    # the others' results are as they were
    announce(f"attn_paged broken max_q {max_q}")
    lens = [(1, 500), (max_q, 900), (1, 33)]
    s = scene(lens, 8, 2, 64, 16)
    want, _, bound, _ = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"], s["cu"],
                                          0.125, out_step=2.0 ** -24)
    q = torch.cat([s["q"][:1], torch.randn(60, 8, 64, device=DEV).to(BF16), s["q"][1:]])
    table = torch.cat([s["table"][:1], s["table"]])
    o = pa.attn_paged(q, s["k"], s["v"], table, ints([500, 480, 900, 33]),
                      ints([0, 1, 61, 61 + max_q, 62 + max_q]), max_q=max_q)
    refs.check(torch.cat([o[:1], o[61:]]), want, bound + refs.U * want.abs(), "the others")


def test_softcap_of_nothing(pa):
    # scores past the cap: all keys weigh the same
    announce("attn_paged tiny softcap")
    s = scene([(1, 100), (40, 200)], 8, 2, 64, 16)
    verify(pa, s, "tiny cap", softcap=1e-30)


def test_lengths_that_make_no_sense(pa):
    # bounds past the queries' end, or falling: only the rows of the requests that are right are
    # defined, and nothing outside the tensors is touched
    announce("attn_paged wrong bounds")
    s = scene([(1, 300), (40, 500), (2, 70)], 8, 2, 64, 16)
    want, _, bound, _ = refs.attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"], s["cu"],
                                          0.125, out_step=2.0 ** -24)
    bound = bound + refs.U * want.abs()  # (sums of rounded weights)
    room = torch.full((45, 8, 64), 7.0, device=DEV)
    for cu, right in (([0, 1, 41, 2 ** 31 - 1], 41), ([0, 1, 0, -5], 1), ([0, 1, 1 << 30, 0], 1)):
        for window in (0, 50):
            room.fill_(7.0)
            pa.attn_paged(s["q"], s["k"], s["v"], s["table"], ints(s["kv"]), ints(cu),
                          o=room[1:44], window=window)
            if not window:
                refs.check(room[1:1 + right], want[:right], bound[:right], f"{cu}")
            assert (room[0] == 7.0).all() and (room[44] == 7.0).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(1, 150000)], [(40, 70001)], [(1, 90000), (1, 3), (20, 40000)]],
                         ids=lambda l: "-".join(f"{n}of{k}" for n, k in l))
def test_long_requests(pa, lens, d):
    announce(f"attn_paged long {lens} d={d}")
    verify(pa, scene(lens, 4, 1, d, 32), "long")


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("scale", [0.0, 1e-7, -0.2, 3.0])
def test_slopes_of_any_scale(pa, scale, causal):
    # rising and falling with distance, by both kernels
    announce(f"attn_paged slopes scale={scale} causal={causal}")
    for d in (64, 128):
        slopes = torch.tensor([0.5, -0.01, 0.0, 3.0], device=DEV)
        verify(pa, scene([(1, 300), (90, 400), (200, 200)], 4, 2, d, 16), f"d={d}", scale=scale,
               causal=causal, slopes=slopes)
