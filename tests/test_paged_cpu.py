"""CPU tests of the paged cache's operators: what they refuse on the host, and the references
that the GPU tests compare with."""
import ctypes
import math
import random

import pytest
import torch

import paper_2609_29219_amd as pa
from tests import paged_refs as refs

A = 1 << 20  # fake, aligned addresses: never dereferenced
MB = 1 << 20
EINVAL, EUNSUPPORTED = pa.ATTN_EINVAL, pa.ATTN_EUNSUPPORTED


def heads(ptr, batch, row, head):
    return pa.Heads(ptr, batch, row, head)


def ref(h):
    return None if h is None else ctypes.byref(h)


def cache(at, Hkv=2, page=16, d=64, **kw):
    h = dict(ptr=at, batch=Hkv * page * d, row=d, head=page * d)
    h.update(kw)
    return heads(**h)


def extend(table=A, stride=8, seq=A + MB, new=A + 2 * MB, free=A + 3 * MB, n_list=20,
           n_free=A + 4 * MB, slots=A + 5 * MB, pos=A + 6 * MB, cu=A + 7 * MB, kv=A + 8 * MB,
           left=A + 9 * MB, R=4, max_pages=8, page=16, T=10):
    return pa.lib.attn_paged_extend(table, stride, seq, new, free, n_list, n_free, slots, pos, cu,
                                    kv, left, R, max_pages, page, T)


@pytest.mark.parametrize("kw,code", [
    *[({n: None}, EINVAL) for n in ("table", "seq", "new", "free", "n_free", "slots", "pos", "cu",
                                    "kv", "left")],
    *[({n: A + 30 * MB + 2}, EINVAL) for n in ("table", "seq", "free", "slots", "cu", "left")],
    (dict(R=0), EINVAL), (dict(T=0), EINVAL), (dict(max_pages=0), EINVAL),
    (dict(n_list=0), EINVAL), (dict(stride=7), EINVAL), (dict(stride=-8), EINVAL),
    (dict(page=0), EUNSUPPORTED), (dict(page=4), EUNSUPPORTED), (dict(page=24), EUNSUPPORTED),
    (dict(page=-16), EUNSUPPORTED), (dict(page=1 << 17), EUNSUPPORTED),
    (dict(max_pages=1 << 27, stride=1 << 27), EUNSUPPORTED),
    (dict(T=(1 << 30) + 1), EUNSUPPORTED), (dict(R=(1 << 30) + 1), EUNSUPPORTED),
    # results over operands and over each other
    (dict(kv=A + MB), EINVAL), (dict(left=A + 4 * MB), EINVAL), (dict(cu=A + MB + 12), EINVAL),
    (dict(pos=A + 5 * MB + 36), EINVAL), (dict(slots=A + 124), EINVAL),
    (dict(free=A + 5 * MB), EINVAL),
])
def test_extend_rejects_on_host(kw, code):
    assert extend(**kw) == code
    assert pa.last_error() != ""


def release(table=A, stride=8, seq=A + MB, keep=A + 2 * MB, free=A + 3 * MB, n_list=20,
            n_free=A + 4 * MB, left=A + 5 * MB, R=4, max_pages=8, page=16):
    return pa.lib.attn_paged_release(table, stride, seq, keep, free, n_list, n_free, left, R,
                                     max_pages, page)


@pytest.mark.parametrize("kw,code", [
    *[({n: None}, EINVAL) for n in ("table", "seq", "keep", "free", "n_free", "left")],
    (dict(keep=A + 30 * MB + 1), EINVAL), (dict(R=-1), EINVAL), (dict(n_list=0), EINVAL),
    (dict(stride=4), EINVAL), (dict(page=12), EUNSUPPORTED), (dict(left=A + 4 * MB), EINVAL),
    (dict(free=A + 64), EINVAL), (dict(left=A + 3 * MB + 76), EINVAL), (dict(n_free=A + 3 * MB), EINVAL),
])
def test_release_rejects_on_host(kw, code):
    assert release(**kw) == code
    assert pa.last_error() != ""


def store(k=0, v=0, slots=A + 2 * MB, kp=0, vp=0, T=3, Hkv=2, d=64, pages=5, page=16):
    k = heads(A, 0, 128, 64) if k == 0 else k
    v = heads(A + MB, 0, 128, 64) if v == 0 else v
    kp = cache(A + 8 * MB) if kp == 0 else kp
    vp = cache(A + 16 * MB) if vp == 0 else vp
    return pa.lib.attn_paged_store(ref(k), ref(v), slots, ref(kp), ref(vp), T, Hkv, d, pages, page)


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), EINVAL), (dict(v=heads(None, 0, 128, 64)), EINVAL), (dict(kp=None), EINVAL),
    (dict(slots=None), EINVAL), (dict(slots=A + 2 * MB + 1), EINVAL),
    (dict(k=heads(A + 8, 0, 128, 64)), EINVAL), (dict(v=heads(A, 0, 100, 64)), EINVAL),
    (dict(T=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(pages=0), EINVAL),
    (dict(d=96), EUNSUPPORTED), (dict(page=4), EUNSUPPORTED),
    (dict(pages=1 << 27), EUNSUPPORTED),
    (dict(kp=cache(A + 8 * MB, row=1 << 27)), EUNSUPPORTED),
    (dict(vp=heads(A + 16 * MB, 1 << 36, 64, 1024)), EUNSUPPORTED),
    # a cache whose rows overlap, or lie over the other side's, or over k
    (dict(kp=cache(A + 8 * MB, batch=0)), EINVAL), (dict(vp=cache(A + 16 * MB, row=32)), EINVAL),
    (dict(vp=cache(A + 8 * MB)), EINVAL), (dict(vp=cache(A + 8 * MB + 64)), EINVAL),
    (dict(k=heads(A + 8 * MB, 0, 128, 64)), EINVAL), (dict(slots=A + 8 * MB), EINVAL),
])
def test_store_rejects_on_host(kw, code):
    assert store(**kw) == code
    assert pa.last_error() != ""


def attend(q=0, kp=0, vp=0, o=A + MB, lse=None, table=A + 2 * MB, stride=8, kv=A + 3 * MB,
           cu=A + 4 * MB, slopes=None, T=6, R=4, max_q=0, Hq=4, Hkv=2, d=64, pages=5, page=16,
           max_pages=8, scale=0.125, softcap=0.0, window=0, causal=1, flags=0, ws=None,
           ws_bytes=0):
    q = heads(A, 0, 256, 64) if q == 0 else q
    kp = cache(A + 8 * MB) if kp == 0 else kp
    vp = cache(A + 16 * MB) if vp == 0 else vp
    return pa.lib.attn_paged(ref(q), ref(kp), ref(vp), o, lse, table, stride, kv, cu, slopes, T, R,
                             max_q, Hq, Hkv, d, pages, page, max_pages, scale, softcap, window,
                             causal, flags, ws, ws_bytes)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), EINVAL), (dict(kp=None), EINVAL), (dict(vp=heads(None, 0, 0, 0)), EINVAL),
    (dict(o=None), EINVAL), (dict(table=None), EINVAL), (dict(kv=None), EINVAL),
    (dict(q=heads(A + 2, 0, 256, 64)), EINVAL), (dict(q=heads(A, 0, 250, 64)), EINVAL),
    (dict(o=A + MB + 8), EINVAL), (dict(lse=A + 5 * MB + 2), EINVAL),
    (dict(cu=A + 4 * MB + 1), EINVAL), (dict(slopes=A + 4 * MB + 3), EINVAL),
    (dict(kv=A + 3 * MB + 2), EINVAL), (dict(T=0), EINVAL), (dict(R=0), EINVAL),
    (dict(Hq=3), EINVAL), (dict(Hkv=0), EINVAL), (dict(pages=0), EINVAL),
    (dict(max_pages=0), EINVAL), (dict(stride=7), EINVAL), (dict(max_q=-1), EINVAL),
    (dict(cu=None), EINVAL),  # six tokens of four requests
    (dict(flags=2), EINVAL), (dict(scale=math.nan), EINVAL), (dict(scale=math.inf), EINVAL),
    (dict(softcap=-1.0), EINVAL), (dict(softcap=math.nan), EINVAL),
    (dict(softcap=math.inf), EINVAL), (dict(window=-1), EINVAL),
    (dict(window=4, causal=0), EUNSUPPORTED), (dict(d=80), EUNSUPPORTED),
    (dict(page=1), EUNSUPPORTED), (dict(max_pages=1 << 27, stride=1 << 27), EUNSUPPORTED),
    (dict(T=1 << 29, q=heads(A, 0, 256, 64)), EUNSUPPORTED),
    (dict(kp=cache(A + 8 * MB, row=1 << 27)), EUNSUPPORTED),
    (dict(vp=heads(A + 16 * MB, 1 << 36, 64, 1024)), EUNSUPPORTED),
    (dict(Hq=(1 << 15) + 1, Hkv=1, q=heads(A, 0, 1 << 22, 64), T=1, R=1, o=A + 64 * MB),
     EUNSUPPORTED),
    (dict(T=(1 << 30) + 1, Hq=1, Hkv=1), EUNSUPPORTED),
    (dict(R=(1 << 30) + 1), EUNSUPPORTED),
    (dict(max_pages=1 << 26, page=32, stride=1 << 26), EUNSUPPORTED),
    # results over operands and each other: o is 6 * 4 * 64 floats, 6144 bytes
    (dict(o=A), EINVAL), (dict(lse=A + MB + 6140), EINVAL), (dict(o=A + 2 * MB - 6128), EINVAL),
    (dict(o=A + 8 * MB + 16), EINVAL), (dict(lse=A + 3 * MB + 12), EINVAL),
    (dict(lse=A + 4 * MB + 16), EINVAL), (dict(slopes=A + MB), EINVAL),
])
def test_attn_paged_rejects_on_host(kw, code):
    assert attend(**kw) == code
    assert pa.last_error() != ""


@pytest.mark.parametrize("args", [(0, 1, 0, 2, 1, 64, 16, 4, 0), (1, 0, 0, 2, 1, 64, 16, 4, 0),
                                  (1, 1, 0, 3, 2, 64, 16, 4, 0), (1, 1, 0, 2, 1, 96, 16, 4, 0),
                                  (1, 1, -1, 2, 1, 64, 16, 4, 0), (1, 1, 0, 2, 1, 64, 12, 4, 0),
                                  (1, 1, 0, 2, 1, 64, 16, 0, 0), (1, 1, 0, 2, 1, 64, 16, 4, -1),
                                  (1 << 30, 1, 0, 2, 1, 64, 16, 4, 0)])
def test_workspace_query_rejects_on_host(args):
    assert pa.lib.attn_paged_workspace_bytes(*args) < 0
    assert pa.last_error() != ""


def test_python_rejects_tensors_of_the_wrong_kind():
    t = torch.zeros(4, 8, dtype=torch.int32)
    n = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    p = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    for call in (lambda: pa.paged_extend(t, n, n, n, n[:1], 16, 4),
                 lambda: pa.paged_release(t, n, n, n, n[:1], 16),
                 lambda: pa.paged_store(x, x, n, p, p), lambda: pa.attn_paged(x, p, p, t, n),
                 lambda: pa.attn_paged(x.float(), p, p, t, n)):
        with pytest.raises(TypeError):
            call()


# ------------------------------------------------------------ the references --
def test_reference_attention_against_torch():
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(n, 64, generator=g, dtype=torch.float64) for n in (7, 40, 40))
    pos = torch.arange(7) + 33
    o, lse, bound, _ = refs.attend(q, k, v, pos, 0.125, True, window=20, slope=0.3)
    away = pos[:, None] - torch.arange(40)
    bias = torch.where((away < 0) | (away >= 20), -math.inf, -0.3 * away.abs().double())
    want = torch.nn.functional.scaled_dot_product_attention(q[None], k[None], v[None],
                                                            attn_mask=bias, scale=0.125)[0]
    assert torch.allclose(o, want, atol=1e-12)
    assert (bound > 0).all() and torch.isfinite(lse).all()
    o, lse, _, _ = refs.attend(q, k, v, pos, 0.125, True, softcap=2.0)
    x = 2.0 * torch.tanh(q @ k.t() * 0.125 / 2.0)
    x = x.masked_fill(away < 0, -math.inf)
    assert torch.allclose(o, torch.softmax(x, -1) @ v, atol=1e-12)
    assert torch.allclose(lse, torch.logsumexp(x, -1), atol=1e-12)


def test_reference_tables_give_every_row_once():
    rng = random.Random(5)
    page, table = 8, [[-1] * 12 for _ in range(6)]
    free, n_free, seq = list(range(40)), 40, [0] * 6
    rows = {}
    for _ in range(30):
        new = [rng.randint(0, 9) if s < 70 else 0 for s in seq]
        slots, pos, cu, kv, left, table2 = refs.extend(table, seq, new, free, n_free, page,
                                                       sum(new) + 3)
        assert slots[cu[-1]:] == [-1] * 3 and pos[cu[-1]:] == [0] * 3
        if left >= 0:
            table, seq, n_free = table2, kv, left
            for r in range(6):
                for t in range(cu[r], cu[r + 1]):
                    assert slots[t] not in rows.values()
                    rows[r, pos[t]] = slots[t]
        keep = [rng.choice([s, s, max(0, s - 4), 0]) for s in seq]
        n_free, free = refs.release(table, seq, keep, free, n_free, page)
        rows = {k: s for k, s in rows.items() if k[1] < keep[k[0]]}
        seq = keep
        assert n_free + sum(-(-s // page) for s in seq) == 40
        assert len(set(free[:n_free])) == n_free
