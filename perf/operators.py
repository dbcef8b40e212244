"""The training step of an attention layer around ``attn_fwd``, and how fast its operators run.

Three operators: ``attn_bwd`` (the gradients of ``attn_fwd``), ``qk_norm_rope`` (RMS norm of
every query and key head, then the position rotation, token-major projections in, the
head-major tensors that ``attn_fwd`` reads out) and ``qk_norm_rope_bwd`` (its gradients).  A
case is one call.  ``run`` computes it in plain torch in float32, or with ``own`` by this
library's kernels; ``exact`` gives the definitions in float64.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
# no drawn case does more than the largest listed ones
MAX_PAIRS = 32 * 8192 * 8192    # (query, key) pairs over all heads
MAX_VALUES = 4 * 8192 * 48 * 128  # projected values of queries, keys and values


# ------------------------------------------------------------------ cases --
def _attn(name, B, Hq, Hkv, Sq, Skv, d, causal, o="fp32", dlse=False, mag=1.0):
    return {"name": name, "op": "attn_bwd", "B": B, "Hq": Hq, "Hkv": Hkv, "Sq": Sq, "Skv": Skv,
            "d": d, "causal": causal, "o": o, "dlse": dlse, "mag": mag}


def _rope(name, op, B, S, Hq, Hkv, d, rot, interleaved=False, start=0, weight="bf16", fused=True,
          grad="bf16"):
    return {"name": name, "op": op, "B": B, "S": S, "Hq": Hq, "Hkv": Hkv, "d": d, "rot": rot,
            "interleaved": interleaved, "start": start, "weight": weight, "fused": fused,
            "grad": grad}


def listed():
    return [
        # one short head of an encoder-sized model: the smallest backward pass, bound by
        # its launches
        _attn("bwd_single_head", 1, 1, 1, 256, 256, 64, False),
        # a training batch, causal, as many key/value heads as query heads
        _attn("bwd_causal", 4, 16, 16, 2048, 2048, 128, True),
        # one long sequence without a mask: the largest backward pass
        _attn("bwd_long", 1, 32, 32, 8192, 8192, 128, False, mag=0.5),
        # a grouped-query model on sequences that fill no tile, from a bf16 output
        _attn("bwd_gqa_ragged", 2, 32, 8, 1777, 1777, 128, True, o="bf16"),
        # a chunk of new tokens behind a long context, merged with other parts by its
        # log-sum-exp, which therefore has a gradient too
        _attn("bwd_chunk", 1, 32, 8, 512, 16384, 128, True, dlse=True),
        # 64-dimensional heads, no mask (an encoder batch)
        _attn("bwd_d64", 4, 16, 16, 2048, 2048, 64, False),
        # one new token of one sequence at a far position: the smallest call of serving
        _rope("rope_token", "rope", 1, 1, 32, 8, 128, 128, start=131071),
        # prompts that fill no tile, interleaved pairs, part of the dimensions rotated,
        # separate projections, float32 weights
        _rope("rope_ragged", "rope", 2, 1777, 16, 16, 64, 32, interleaved=True, weight="fp32",
              fused=False),
        # a training batch of long sequences from one fused projection: the largest
        _rope("rope_long", "rope", 4, 8192, 32, 8, 128, 128),
        # one short head, its gradients in float32
        _rope("rope_bwd_single_head", "rope_bwd", 1, 256, 1, 1, 64, 64, grad="fp32"),
        # sequences that fill no tile, interleaved pairs, part of the dimensions rotated
        _rope("rope_bwd_ragged", "rope_bwd", 2, 1777, 16, 16, 64, 32, interleaved=True,
              weight="fp32", fused=False),
        # a training batch of long sequences: the largest
        _rope("rope_bwd_long", "rope_bwd", 4, 8192, 32, 8, 128, 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_any(rng):
    op = rng.choice(["attn_bwd", "attn_bwd", "rope", "rope_bwd"])
    d = rng.choice([64, 128, 128])
    Hkv, group = rng.choice([(1, 1), (1, 8), (2, 4), (4, 8), (8, 4), (8, 8), (16, 1), (16, 2),
                             (32, 1)])
    if op == "attn_bwd":
        causal = rng.random() < 0.6
        if rng.random() < 0.25:  # new tokens behind a context
            Sq = _log(rng, 1, 1024)
            Skv = Sq + _log(rng, 256, 32768)
        else:
            # (with a single key the softmax is constant and dq, dk are sums of roundings)
            Sq = Skv = _log(rng, 4, 8192)
        return _attn("", rng.choice([1, 1, 2, 3, 4, 8]), Hkv * group, Hkv, Sq, Skv, d, causal,
                     rng.choice(["fp32", "bf16"]), rng.random() < 0.25, rng.choice([1.0, 0.5]))
    rot = rng.choice([d, d, d // 2, 3 * d // 4, 16])
    return _rope("", op, rng.choice([1, 1, 2, 3, 4, 8, 16, 64]), _log(rng, 1, 16384),
                 Hkv * group, Hkv, d, rot, rng.random() < 0.5,
                 rng.choice([0, 0, _log(rng, 1, 1 << 20)]), rng.choice(["fp32", "bf16"]),
                 rng.random() < 0.6, rng.choice(["fp32", "bf16"]))


def draw(rng):
    while True:
        case = _draw_any(rng)
        if case["op"] == "attn_bwd":
            if case["B"] * case["Hq"] * case["Sq"] * case["Skv"] > MAX_PAIRS:
                continue
        elif case["B"] * case["S"] * (case["Hq"] + 2 * case["Hkv"]) * case["d"] > MAX_VALUES:
            continue
        del case["name"]
        return case


# ----------------------------------------------------------------- inputs --
def _randn(g, *shape, dtype=torch.bfloat16, mag=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * mag).to(dtype)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _forward(q, k, v, causal):
    """Output and log-sum-exp in float32: what the forward pass left behind."""
    B, Hq, Sq, d = q.shape
    Hkv, Skv = k.shape[1], k.shape[2]
    s = q.float().view(B, Hkv, -1, d) @ (k.float().transpose(-1, -2) / math.sqrt(d))
    if causal:
        hidden = torch.ones(Sq, Skv, dtype=torch.bool, device=DEV).triu(Skv - Sq + 1)
        s.view(B, Hkv, -1, Sq, Skv).masked_fill_(hidden, -math.inf)
    lse = torch.logsumexp(s, dim=-1)
    o = s.sub_(lse.unsqueeze(-1)).exp_() @ v.float()
    return o.view(B, Hq, Sq, d), lse.view(B, Hq, Sq)


def prepare(case, seed):
    """Unit-normal bf16 operands (queries, keys and values of normalised layers, the
    gradients that come back); ``mag`` scales them.  Norm weights lie around one; the
    rotation's frequencies fall from 1 to 1e-4 as usual."""
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    B, Hq, Hkv, d = (case[n] for n in ("B", "Hq", "Hkv", "d"))
    state = {"case": case}
    if case["op"] == "attn_bwd":
        Sq, Skv, mag = case["Sq"], case["Skv"], case["mag"]
        q, k, v = (_randn(g, B, Hq, Sq, d, mag=mag), _randn(g, B, Hkv, Skv, d, mag=mag),
                   _randn(g, B, Hkv, Skv, d, mag=mag))
        o, lse = _forward(q, k, v, case["causal"])
        state.update(q=q, k=k, v=v, o=o.to(_dtype(case["o"])), lse=lse,
                     do=_randn(g, B, Hq, Sq, d),
                     dlse=_randn(g, B, Hq, Sq, dtype=torch.float32) if case["dlse"] else None)
        return state
    S, R = case["S"], case["rot"]
    if case["fused"]:  # one projection, query heads first
        x = _randn(g, B, S, Hq + 2 * Hkv, d)
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    else:
        q, k, v = _randn(g, B, S, Hq, d), _randn(g, B, S, Hkv, d), _randn(g, B, S, Hkv, d)
    state.update(q=q, k=k, v=v)
    for n in ("q_weight", "k_weight"):
        state[n] = (1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(_dtype(case["weight"]))
    i = torch.arange(R // 2, dtype=torch.float64, device=DEV)
    state["inv_freq"] = torch.pow(10000.0, -2.0 * i / R).float()
    state["positions"] = None
    if case["start"]:  # each sequence begins somewhere up to there
        first = torch.randint(case["start"] // 2, case["start"] + 1, (B, 1), generator=g, device=DEV)
        state["positions"] = first + torch.arange(S, device=DEV)
    if case["op"] == "rope_bwd":
        for n, H in (("dq", Hq), ("dk", Hkv), ("dv", Hkv)):
            state[n] = _randn(g, B, H, S, d, dtype=_dtype(case["grad"]))
    return state


# ---------------------------------------------------------- the plain forms --
def _plain_attn_bwd(q, k, v, o, lse, do, dlse, causal):
    B, Hq, Sq, d = q.shape
    Hkv, Skv = k.shape[1], k.shape[2]
    scale = 1.0 / math.sqrt(d)
    delta = (do.float() * o.float()).sum(-1)  # sum_j P_ij dP_ij
    if dlse is not None:
        delta = delta - dlse
    # the query heads of one key/value head are rows of one matrix
    qf, dof = q.float().view(B, Hkv, -1, d), do.float().view(B, Hkv, -1, d)
    kf, vf = k.float(), v.float()
    p = (qf @ kf.transpose(-1, -2)).mul_(scale).sub_(lse.view(B, Hkv, -1, 1)).exp_()
    if causal:
        hidden = torch.ones(Sq, Skv, dtype=torch.bool, device=DEV).triu(Skv - Sq + 1)
        p.view(B, Hkv, -1, Sq, Skv).masked_fill_(hidden, 0.0)
    dv = p.transpose(-1, -2) @ dof
    ds = (dof @ vf.transpose(-1, -2)).sub_(delta.view(B, Hkv, -1, 1)).mul_(p).mul_(scale)
    dq = (ds @ kf).view(B, Hq, Sq, d)
    dk = ds.transpose(-1, -2) @ qf
    return dq.bfloat16(), dk.bfloat16(), dv.bfloat16()


def _cos_sin(state):
    """Of every token and pair, [B or 1, S, 1, R/2]; the angles in float64."""
    pos = state["positions"]
    if pos is None:
        pos = torch.arange(state["q"].shape[1], device=DEV)[None]
    angle = pos.double()[..., None, None] * state["inv_freq"].double()
    return angle.cos().float(), angle.sin().float()


def _rotate(x, cos, sin, interleaved):
    R = 2 * cos.shape[-1]
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((turned, x[..., R:]), dim=-1)


def _plain_rope(state, eps):
    case = state["case"]
    cos, sin = _cos_sin(state)
    outs = []
    for n in ("q", "k"):
        x = state[n].float()
        y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * state[n + "_weight"].float()
        outs.append(_rotate(y, cos, sin, case["interleaved"]))
    outs.append(state["v"])
    return tuple(t.bfloat16().transpose(1, 2).contiguous() for t in outs)


def _plain_rope_bwd(state, eps):
    case = state["case"]
    cos, sin = _cos_sin(state)
    dx, dw = [], []
    for n in ("q", "k"):
        x, grad = state[n].float(), state["d" + n].float().transpose(1, 2)
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)
        n_hat = x * r
        grad = _rotate(grad, cos, -sin, case["interleaved"])  # the rotation's transpose
        dw.append((grad * n_hat).sum((0, 1, 2)))
        grad = grad * state[n + "_weight"].float()
        dx.append((r * (grad - n_hat * (grad * n_hat).mean(-1, keepdim=True))).bfloat16())
    dx.append(state["dv"].transpose(1, 2).bfloat16())
    return (*dx, *dw)


def run(state):
    case = state["case"]
    if own:
        import paper_2609_29219_amd as pa
    if case["op"] == "attn_bwd":
        args = (state["q"], state["k"], state["v"], state["o"], state["lse"])
        if own:
            return pa.attn_bwd(state["do"], *args, causal=case["causal"], dlse=state["dlse"])
        return _plain_attn_bwd(*args, state["do"], state["dlse"], case["causal"])
    if case["op"] == "rope":
        if own:
            return pa.qk_norm_rope(state["q"], state["k"], state["v"], state["q_weight"],
                                   state["k_weight"], state["inv_freq"],
                                   positions=state["positions"], interleaved=case["interleaved"])
        return _plain_rope(state, 1e-6)
    if own:
        return pa.qk_norm_rope_bwd(state["dq"], state["dk"], state["dv"], state["q"], state["k"],
                                   state["q_weight"], state["k_weight"], state["inv_freq"],
                                   positions=state["positions"], interleaved=case["interleaved"])
    return _plain_rope_bwd(state, 1e-6)


# -------------------------------------------------------------------- work --
def work(case):
    """Operands read once, results written once.  attn_bwd: five products of 2 d operations
    for each (query, key) pair that the mask allows.  The others: some 7 operations for each
    query and key value forward, 16 backward."""
    B, Hq, Hkv, d = (case[n] for n in ("B", "Hq", "Hkv", "d"))
    if case["op"] == "attn_bwd":
        Sq, Skv = case["Sq"], case["Skv"]
        rows = B * Hq * Sq
        pairs = Sq * Skv - (Sq * (Sq - 1) // 2 if case["causal"] else 0)
        o = 2 if case["o"] == "bf16" else 4
        # q, do, dq; o; lse and its gradient; k, v, dk, dv
        return {"bytes": rows * d * (6 + o) + rows * (8 if case["dlse"] else 4)
                + 8 * B * Hkv * Skv * d, "flops": 10 * d * pairs * B * Hq}
    tokens, heads = B * case["S"], Hq + 2 * Hkv
    w = 2 * d * (2 if case["weight"] == "bf16" else 4)
    small = w + 2 * case["rot"] + (8 * tokens if case["start"] else 0)
    if case["op"] == "rope":
        return {"bytes": 4 * tokens * heads * d + small, "flops": 7 * tokens * (Hq + Hkv) * d}
    g = 2 if case["grad"] == "bf16" else 4
    # gradients in, q and k in, their gradients and the values' out, the weights' out
    return {"bytes": tokens * d * (heads * (g + 2) + 2 * (Hq + Hkv)) + small + 8 * d,
            "flops": 16 * tokens * (Hq + Hkv) * d}


# ------------------------------------------------------------------- exact --
def _exact_attn_bwd(state):
    """Head by head from the definition: softmax, then its differential."""
    case = state["case"]
    q, k, v, do = (state[n] for n in ("q", "k", "v", "do"))
    B, Hq, Sq, d = q.shape
    Hkv, Skv = k.shape[1], k.shape[2]
    dq = torch.empty(B, Hq, Sq, d, dtype=torch.float64, device=DEV)
    dk = torch.zeros(B, Hkv, Skv, d, dtype=torch.float64, device=DEV)
    dv = torch.zeros_like(dk)
    keys = torch.arange(Skv, device=DEV)
    step = max(1, (1 << 26) // Skv)  # query rows whose scores are held at once
    for b in range(B):
        for h in range(Hq):
            n = h // (Hq // Hkv)
            kk, vv = k[b, n].double(), v[b, n].double()
            kt, vt = kk.t().contiguous(), vv.t().contiguous()
            for r in range(0, Sq, step):
                qq, gg = q[b, h, r:r + step].double(), do[b, h, r:r + step].double()
                s = (qq @ kt) / math.sqrt(d)
                if case["causal"]:
                    last = torch.arange(r, r + qq.shape[0], device=DEV) + (Skv - Sq)
                    s.masked_fill_(keys[None, :] > last[:, None], -math.inf)
                p = torch.softmax(s, dim=-1)
                gp = gg @ vt
                gs = gp - (p * gp).sum(-1, keepdim=True)
                if state["dlse"] is not None:
                    gs += state["dlse"][b, h, r:r + step, None].double()
                gs = gs * p / math.sqrt(d)
                dq[b, h, r:r + step] = gs @ kk
                dk[b, n] += gs.t().contiguous() @ qq
                dv[b, n] += p.t().contiguous() @ gg
    return dq, dk, dv


def _exact_rope(state, q, k, qw, kw):
    """Rotation by complex multiplication, on float64 leaves."""
    case = state["case"]
    R, S = case["rot"], q.shape[1]
    pos = state["positions"]
    pos = torch.arange(S, device=DEV).expand(q.shape[0], S) if pos is None else pos
    angle = pos.double()[:, :, None] * state["inv_freq"].double()
    turn = torch.polar(torch.ones_like(angle), angle)[:, :, None, :]
    outs = []
    for x, w in ((q, qw), (k, kw)):
        y = w * x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + 1e-6)
        head, tail = y[..., :R], y[..., R:]
        if case["interleaved"]:
            pairs = head.reshape(*head.shape[:-1], R // 2, 2)
        else:
            pairs = torch.stack(head.chunk(2, dim=-1), dim=-1)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z.flatten(-2) if case["interleaved"] else torch.cat((z[..., 0], z[..., 1]), dim=-1)
        outs.append(torch.cat((z, tail), dim=-1).permute(0, 2, 1, 3))
    return outs


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "attn_bwd":
        return _exact_attn_bwd(state)
    leaves = [state[n].double().requires_grad_(case["op"] == "rope_bwd")
              for n in ("q", "k", "q_weight", "k_weight")]
    q, k = _exact_rope(state, *leaves)
    if case["op"] == "rope":
        return q, k, state["v"].double().permute(0, 2, 1, 3)
    dq, dk, dqw, dkw = torch.autograd.grad([q, k], leaves, [state["dq"].double(),
                                                            state["dk"].double()])
    return dq, dk, state["dv"].double().permute(0, 2, 1, 3), dqw, dkw
