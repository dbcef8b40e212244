"""A serving step over a paged key/value cache, and how fast its operators run.

Four operators: ``paged_extend`` (pages, slots and positions of a step's new tokens from the
requests' lengths), ``paged_release`` (pages given back), ``paged_store`` (keys and values into
the cache) and ``attn_paged`` (new tokens of requests of any lengths against the cache).  A case
is one call.  ``run`` computes it in plain torch in float32, or with ``own`` by this library's
kernels; ``exact`` gives the definitions in float64.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
# no drawn case does more than the largest listed ones
MAX_PAIRS = 32 * 8192 * 8192       # (new token, key) pairs over all heads, requests as long as the longest
MAX_CACHE = 16 * 8192 * 8 * 128    # keys' values in the cache, requests as long as the longest
MAX_VALUES = 16384 * 8 * 128       # keys' values of a store
MAX_TABLE = 1024 * 2048            # page numbers of a table


# ------------------------------------------------------------------ cases --
def _attn(name, R, new, ctx, Hq, Hkv, d, page, causal=True, window=0, softcap=0.0, slopes=False,
          lse=False, token_major=False, pick=1):
    """R requests with new[0]..new[1] new tokens each, behind ctx[0]..ctx[1] that are in the cache
    (the first request has the most of both)."""
    return {"name": name, "op": "attn", "R": R, "new_min": new[0], "new_max": new[1],
            "ctx_min": ctx[0], "ctx_max": ctx[1], "Hq": Hq, "Hkv": Hkv, "d": d, "page": page,
            "causal": causal, "window": window, "softcap": softcap, "slopes": slopes, "lse": lse,
            "token_major": token_major, "pick": pick}


def _tables(name, op, R, new, ctx, page, max_pages, pick=1):
    return {"name": name, "op": op, "R": R, "new_min": new[0], "new_max": new[1],
            "ctx_min": ctx[0], "ctx_max": ctx[1], "page": page, "max_pages": max_pages,
            "pick": pick}


def _store(name, T, Hkv, d, page, token_major, fused, padded, pick=1):
    return {"name": name, "op": "store", "T": T, "Hkv": Hkv, "d": d, "page": page,
            "token_major": token_major, "fused": fused, "padded": padded, "pick": pick}


def listed():
    return [
        # the next token of a single conversation: the smallest attention call
        _attn("attn_token", 1, (1, 1), (511, 511), 32, 8, 128, 16),
        # the next token of a full batch of requests of all lengths up to 8192
        _attn("attn_decode", 16, (1, 1), (1000, 8191), 32, 8, 128, 16),
        # a few drafted tokens of each request to be verified, capped scores, pages that hold
        # whole tokens, a log-sum-exp
        _attn("attn_drafts", 32, (2, 8), (100, 4000), 16, 8, 64, 32, softcap=30.0, lse=True,
              token_major=True),
        # a chunk of a long prompt behind what is in the cache already
        _attn("attn_chunk", 1, (512, 512), (15872, 15872), 32, 8, 128, 16),
        # a whole prompt, one key/value head to a query head: the largest
        _attn("attn_prompt", 1, (8192, 8192), (0, 0), 32, 32, 128, 64),
        # chunks of prompts among requests in the middle of their answers, a sliding window,
        # scores that fall with distance, large pages
        _attn("attn_mixed", 16, (1, 500), (1, 3500), 16, 4, 128, 128, window=1024, slopes=True),
        # one request takes one token, for which it needs a page: the smallest
        _tables("extend_token", "extend", 1, (1, 1), (512, 512), 16, 512),
        # a large server's step: prompts' chunks and single tokens of a thousand requests
        _tables("extend_batch", "extend", 1024, (0, 256), (0, 30000), 16, 2048),
        # drafted tokens that were not accepted, a few of each request
        _tables("release_drafts", "release", 64, (1, 8), (100, 4000), 16, 512),
        # a thousand requests end
        _tables("release_batch", "release", 1024, (0, 30000), (0, 2000), 16, 2048),
        # a token of each of a few requests
        _store("store_tokens", 16, 8, 128, 16, False, True, 0),
        # a long prompt's keys and values, out of one projection, some rows empty
        _store("store_prompt", 16384, 8, 128, 16, True, True, 100),
    ]


def _log(rng, lo, hi):
    """Spread over the logarithm; 0 stands below 1."""
    return int(round(math.exp(rng.uniform(math.log(max(lo, 0.5)), math.log(hi)))))


def _draw_attn(rng):
    Hkv, group = rng.choice([(1, 1), (1, 8), (2, 4), (2, 7), (4, 4), (4, 8), (8, 1), (8, 4), (8, 8),
                             (16, 1), (16, 2), (32, 1), (1, 40)])
    R = _log(rng, 1, 128)
    kind = rng.choice(["token", "drafts", "chunk", "mixed"])
    if kind == "token":
        new = (1, 1)
    elif kind == "drafts":
        new = (1, rng.randint(2, 12))
    else:
        most = max(1, _log(rng, 8, 8192))
        new = (0 if kind == "mixed" else max(1, most // 2), most)
    most = 0 if rng.random() < 0.15 else _log(rng, 16, 65536)
    ctx = (rng.choice([0, most // 8, most]), most)
    causal = rng.random() < 0.9
    return _attn("", R, new, ctx, Hkv * group, Hkv, rng.choice([64, 128, 128]),
                 rng.choice([8, 16, 16, 32, 64, 256]), causal,
                 _log(rng, 16, 8192) if causal and rng.random() < 0.25 else 0,
                 rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]), rng.random() < 0.25,
                 rng.random() < 0.4, rng.random() < 0.4, rng.randrange(1 << 20))


def _draw_any(rng):
    op = rng.choice(["attn", "attn", "attn", "attn", "extend", "release", "store"])
    if op == "attn":
        return _draw_attn(rng)
    page = rng.choice([8, 16, 16, 32, 64, 256])
    if op == "store":
        T = _log(rng, 1, 65536)
        return _store("", T, rng.choice([1, 2, 4, 7, 8, 16, 32]), rng.choice([64, 128]), page,
                      rng.random() < 0.5, rng.random() < 0.5, rng.choice([0, T // 7]),
                      rng.randrange(1 << 20))
    R = _log(rng, 1, 4096)
    new = _log(rng, 1, 4096)
    ctx = _log(rng, 0, 32768)
    pages = (new + ctx) // page + 1
    return _tables("", op, R, (rng.choice([0, 1, new]), new), (0, ctx), page,
                   pages + rng.randrange(pages), rng.randrange(1 << 20))


def draw(rng):
    while True:
        case = _draw_any(rng)
        if case["op"] == "attn":
            keys = case["R"] * (case["new_max"] + case["ctx_max"])
            if keys * case["new_max"] * case["Hq"] > MAX_PAIRS or \
                    keys * case["Hkv"] * case["d"] > MAX_CACHE:
                continue
        elif case["op"] == "store":
            if case["T"] * case["Hkv"] * case["d"] > MAX_VALUES:
                continue
        elif case["R"] * case["max_pages"] > MAX_TABLE or case["R"] * case["new_max"] > 1 << 22:
            continue
        del case["name"]
        return case


def _lens(case):
    """New tokens of each request, and its tokens in the cache before them."""
    rng = random.Random(case["pick"])
    new, ctx = [case["new_max"]], [case["ctx_max"]]
    for _ in range(case["R"] - 1):
        new.append(rng.randint(case["new_min"], case["new_max"]))
        ctx.append(rng.randint(case["ctx_min"], case["ctx_max"]))
    if case["op"] == "attn" and case["new_min"] < 2 and case["new_max"] > 64:
        # most requests of a mixed batch are in the middle of their answers
        new = [n if i % 4 == 0 else min(n, 1) for i, n in enumerate(new)]
    return new, ctx


# ----------------------------------------------------------------- inputs --
def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pages_of(n, page):
    return -(-n // page)


def _table(g, held, max_pages, pages):
    """Each request's pages, from all over the cache; -1 behind them; and the pages left."""
    order = torch.randperm(pages, generator=g, device=DEV).int()
    held = torch.tensor(held, device=DEV)
    first = held.cumsum(0) - held
    cols = torch.arange(max_pages, device=DEV)
    at = (first[:, None] + cols).clamp(max=pages - 1)
    table = torch.where(cols < held[:, None], order[at], -1)
    return table, order[int(held.sum()):]


def _cache(g, pages, Hkv, page, d, token_major):
    """[pages, Hkv, page, d]; in memory a page's heads one by one, or its tokens."""
    if token_major:
        return _randn(g, pages, page, Hkv, d).transpose(1, 2)
    return _randn(g, pages, Hkv, page, d)


def prepare(case, seed):
    """Unit-normal bf16 queries, keys and values; pages of a request lie anywhere in the cache,
    whose other rows hold what earlier requests left there."""
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    page = case["page"]
    state = {"case": case}
    if case["op"] == "store":
        T, Hkv, d = case["T"], case["Hkv"], case["d"]
        pages = _pages_of(T, page) + 3
        slots = torch.randperm(pages, generator=g, device=DEV)[:, None] * page + \
            torch.arange(page, device=DEV)
        slots = slots.reshape(-1)[:T].int()
        state["tokens"] = T - case["padded"]
        slots[state["tokens"]:] = -1
        if case["fused"]:  # one projection of keys and values
            k, v = _randn(g, T, 2 * Hkv, d).split(Hkv, 1)
        else:
            k, v = _randn(g, T, Hkv, d), _randn(g, T, Hkv, d)
        state.update(k=k, v=v, slots=slots)
        for n in ("k_pages", "v_pages"):
            state[n] = _cache(g, pages, Hkv, page, d, case["token_major"])
        return state
    new, ctx = _lens(case)
    if case["op"] == "attn":
        T, kv = sum(new), [n + c for n, c in zip(new, ctx)]
        held = [_pages_of(n, page) for n in kv]
        max_pages = max(held) + 2
        pages = sum(held) + 5
        state["table"], _ = _table(g, held, max_pages, pages)
        state["kv_lens"] = _ints(kv)
        state["cu"] = _ints([0] + new).cumsum(0).int()
        state["max_q"], state["max_kv"] = max(new), max(kv)
        state["q"] = _randn(g, T, case["Hq"], case["d"])
        for n in ("k_pages", "v_pages"):
            state[n] = _cache(g, pages, case["Hkv"], page, case["d"], case["token_major"])
        state["slopes"] = None
        if case["slopes"]:  # a power of two to each head, as usual
            h = torch.arange(1, case["Hq"] + 1, device=DEV)
            state["slopes"] = torch.exp2(-8.0 * h / case["Hq"]).float()
        return state
    if case["op"] == "extend":
        state["table"], free = _table(g, [_pages_of(c, page) for c in ctx], case["max_pages"],
                                      sum(_pages_of(n + c, page) for n, c in zip(new, ctx)) + 7)
        state["tokens"] = sum(new) + 5  # of the buffers that the step fills
    else:
        state["table"], free = _table(g, [_pages_of(n + c, page) for n, c in zip(new, ctx)],
                                      case["max_pages"],
                                      sum(_pages_of(n + c, page) for n, c in zip(new, ctx)) + 7)
        # the list has room for every page of the cache
        gone = sum(_pages_of(n + c, page) for n, c in zip(new, ctx))
        free = torch.cat((free, torch.full((gone,), -1, dtype=torch.int32, device=DEV)))
        state["n_free"] = _ints([len(free) - gone])
        state["seq_lens"], state["keep_lens"] = _ints([n + c for n, c in zip(new, ctx)]), _ints(ctx)
        state["free"] = free
        return state
    state.update(free=free, n_free=_ints([len(free)]), seq_lens=_ints(ctx), new_lens=_ints(new))
    return state


# ---------------------------------------------------------- the plain forms --
def _plain_extend(state):
    page, T = state["case"]["page"], state["tokens"]
    seq, new, table = state["seq_lens"].long(), state["new_lens"].long(), state["table"]
    kv = seq + new
    cu = torch.cat((new.new_zeros(1), new.cumsum(0)))
    held = (seq + page - 1) // page
    need = (kv + page - 1) // page - held
    first = need.cumsum(0) - need
    cols = torch.arange(table.shape[1], device=DEV)
    fresh = (cols >= held[:, None]) & (cols < (held + need)[:, None])
    at = state["n_free"].long() - 1 - (first[:, None] + cols - held[:, None])
    table = torch.where(fresh, state["free"][at.clamp(0, len(state["free"]) - 1)], table)
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(cu[1:], t, right=True)
    there = r < len(seq)
    r = r.clamp(max=len(seq) - 1)
    pos = torch.where(there, seq[r] + t - cu[r], 0)
    slots = torch.where(there, table[r, pos // page].long() * page + pos % page, -1)
    return (slots.int(), pos.int(), cu.int(), kv.int(),
            (state["n_free"] - need.sum()).int(), table)


def _plain_release(state):
    page = state["case"]["page"]
    kept = (state["keep_lens"].long() + page - 1) // page
    held = (state["seq_lens"].long() + page - 1) // page
    gone = held - kept
    first = gone.cumsum(0) - gone
    cols = torch.arange(state["table"].shape[1], device=DEV)
    back = (cols >= kept[:, None]) & (cols < held[:, None])
    # where in the list (one place more than it has: nowhere)
    at = state["n_free"].long() + first[:, None] + cols - kept[:, None]
    free = torch.cat((state["free"], state["free"][:1]))
    free = free.scatter(0, torch.where(back, at, len(free) - 1).reshape(-1),
                        state["table"].reshape(-1))
    return (state["n_free"] + gone.sum()).int(), free[:-1]


def _plain_store(state):
    page = state["case"]["page"]
    slots = state["slots"][:state["tokens"]].long()
    for x, pages in ((state["k"], state["k_pages"]), (state["v"], state["v_pages"])):
        pages[slots // page, :, slots % page] = x[:state["tokens"]]
    return state["k_pages"], state["v_pages"]


def _plain_attn(state):
    """All requests padded to the longest."""
    case = state["case"]
    page, Hq, Hkv, d = (case[n] for n in ("page", "Hq", "Hkv", "d"))
    R, G, Sq = case["R"], Hq // Hkv, state["max_q"]
    kv, cu = state["kv_lens"].long(), state["cu"].long()
    new = cu[1:] - cu[:-1]
    tok = torch.arange(Sq, device=DEV)
    row = (cu[:-1, None] + tok).clamp(max=len(state["q"]) - 1)
    q = state["q"][row].float().view(R, Sq, Hkv, G, d).permute(0, 2, 1, 3, 4)
    n = _pages_of(state["max_kv"], page)
    Skv = n * page
    table = state["table"][:, :n].long().clamp(min=0)
    keys = torch.arange(Skv, device=DEV)
    there = (keys < kv[:, None])[:, None, :, None]
    k, v = (state[x][table].permute(0, 2, 1, 3, 4).reshape(R, Hkv, Skv, d).float()
            .masked_fill_(~there, 0.0) for x in ("k_pages", "v_pages"))
    s = q.reshape(R, Hkv, Sq * G, d) @ (k.transpose(-1, -2) / math.sqrt(d))
    del k
    if case["softcap"]:
        s = s.div_(case["softcap"]).tanh_().mul_(case["softcap"])
    s = s.view(R, Hkv, Sq, G, Skv)
    pos = (kv - new)[:, None] + tok  # of every new token
    away = pos[:, :, None] - keys
    if case["slopes"]:
        s -= state["slopes"].view(1, Hkv, 1, G, 1) * away.abs()[:, None, :, None].float()
    seen = (keys < kv[:, None])[:, None].expand(R, Sq, Skv)
    if case["causal"]:
        seen = seen & (away >= 0)
    if case["window"]:
        seen = seen & (away < case["window"])
    s.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = s.sum(-1, keepdim=True)
    o = (s.view(R, Hkv, Sq * G, Skv) @ v).view(R, Hkv, Sq, G, d)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (top + total.log())[..., 0]
    # each request's own tokens, one request behind another
    t = torch.arange(len(state["q"]), device=DEV)
    r = torch.searchsorted(cu[1:], t, right=True)
    o = o.permute(0, 2, 1, 3, 4).reshape(R, Sq, Hq, d)[r, t - cu[r]].bfloat16()
    if not case["lse"]:
        return o
    return o, lse.permute(0, 2, 1, 3).reshape(R, Sq, Hq)[r, t - cu[r]]


def run(state):
    case = state["case"]
    if own:
        import paper_2609_29219_amd as pa
    if case["op"] == "attn":
        if own:
            return pa.attn_paged(state["q"], state["k_pages"], state["v_pages"], state["table"],
                                 state["kv_lens"], state["cu"], max_q=state["max_q"],
                                 causal=case["causal"], window=case["window"],
                                 softcap=case["softcap"], slopes=state["slopes"],
                                 out_dtype=torch.bfloat16, return_lse=case["lse"])
        return _plain_attn(state)
    if case["op"] == "extend":
        if own:
            return (*pa.paged_extend(state["table"], state["seq_lens"], state["new_lens"],
                                     state["free"], state["n_free"], case["page"],
                                     state["tokens"]), state["table"])
        return _plain_extend(state)
    if case["op"] == "release":
        if own:
            return pa.paged_release(state["table"], state["seq_lens"], state["keep_lens"],
                                    state["free"], state["n_free"], case["page"]), state["free"]
        return _plain_release(state)
    if own:
        pa.paged_store(state["k"], state["v"], state["slots"], state["k_pages"],
                       state["v_pages"])
        return state["k_pages"], state["v_pages"]
    return _plain_store(state)


# -------------------------------------------------------------------- work --
def work(case):
    """Operands read once, results written once.  attn: two products of 2 d operations for each
    (query, key) pair that is seen; of the cache, the keys that any new token sees."""
    if case["op"] == "store":
        n = case["T"] - case["padded"]
        return {"bytes": 8 * n * case["Hkv"] * case["d"] + 4 * case["T"], "flops": 0}
    new, ctx = _lens(case)
    page, R = case["page"], case["R"]
    if case["op"] == "extend":
        fresh = sum(_pages_of(n + c, page) - _pages_of(c, page) for n, c in zip(new, ctx))
        # lengths in; positions and slots, sums and lengths out; a number of every page met
        met = sum(_pages_of(n + c, page) - c // page for n, c in zip(new, ctx) if n)
        return {"bytes": 8 * R + 8 * (sum(new) + 5) + 8 * R + 8 * fresh + 4 * (met - fresh),
                "flops": 0}
    if case["op"] == "release":
        gone = sum(_pages_of(n + c, page) - _pages_of(c, page) for n, c in zip(new, ctx))
        return {"bytes": 8 * R + 8 * gone + 8, "flops": 0}
    Hq, Hkv, d, w = (case[n] for n in ("Hq", "Hkv", "d", "window"))
    pairs = keys = 0
    for n, c in zip(new, ctx):
        kv = n + c
        if not case["causal"]:
            pairs, keys = pairs + n * kv, keys + (kv if n else 0)
            continue
        # token i sees the keys up to c + i, at most w of them
        full = n * c + n * (n + 1) // 2
        if w:
            far = max(0, kv - w)  # by how many the last token's are cut
            cut = min(far, n)
            full -= cut * far - cut * (cut - 1) // 2
        pairs += full
        keys += min(kv, w + n - 1) if w and n else kv if n else 0
    T = sum(new)
    return {"bytes": 4 * keys * Hkv * d + 4 * T * Hq * d + (4 * T * Hq if case["lse"] else 0),
            "flops": 4 * d * pairs * Hq}


# ------------------------------------------------------------------- exact --
def exact(case, seed):
    """Attention request by request and head by head; the others give whole numbers, or rows as
    they were."""
    if case["op"] != "attn":
        return None
    state = prepare(case, seed)
    Hq, Hkv, d, page = (case[n] for n in ("Hq", "Hkv", "d", "page"))
    q, cu, kv = state["q"], state["cu"].tolist(), state["kv_lens"].tolist()
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for r in range(case["R"]):
        first, end, S = cu[r], cu[r + 1], kv[r]
        if first == end or S == 0:
            continue
        slots = torch.arange(S, device=DEV)
        where = state["table"][r].long()[slots // page], slots % page
        step = max(1, (1 << 27) // S)
        for n in range(Hkv):
            K, V = (state[x][where[0], n, where[1]].double() for x in ("k_pages", "v_pages"))
            Kt = K.t().contiguous()
            for h in range(n * (Hq // Hkv), (n + 1) * (Hq // Hkv)):
                for a in range(first, end, step):
                    b = min(a + step, end)
                    x = q[a:b, h].double() @ Kt / math.sqrt(d)
                    if case["softcap"]:
                        x = case["softcap"] * torch.tanh(x / case["softcap"])
                    i = torch.arange(a - first, b - first, device=DEV)[:, None] + S - (end - first)
                    if case["slopes"]:
                        x = x - float(state["slopes"][h]) * (i - slots).abs()
                    hidden = torch.zeros_like(x, dtype=torch.bool)
                    if case["causal"]:
                        hidden |= slots > i
                    if case["window"]:
                        hidden |= slots <= i - case["window"]
                    x = x.masked_fill(hidden, -math.inf)
                    lse[a:b, h] = torch.logsumexp(x, -1)
                    o[a:b, h] = torch.exp(x - lse[a:b, h, None]) @ V
    return (o, lse) if case["lse"] else o
