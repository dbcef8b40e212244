"""The training operators in float64, with bounds on what their kernels may be off.

Everything is computed head by head from the definitions.  A bound counts roundings:
u = 2^-8 is half a step of bf16 relative to the value, and the fp32 sums in between are
allowed 2^-14 (scores of absolute sum up to 100, summed in up to ten roundings of 2^-24
each, give the exponent an error of 100 * 10 * 2^-24 < 2^-14; the other sums less).
"""
from __future__ import annotations

import math

import torch

U = 2.0 ** -8
SUMS = 2.0 ** -14


def scores(q, k, scale, causal):
    """fp64 scores of one head, hidden ones -inf."""
    s = q @ k.t().contiguous() * scale
    if causal:
        n, m = s.shape
        s = s.masked_fill(torch.ones(n, m, dtype=torch.bool, device=s.device).triu(m - n + 1),
                          -math.inf)
    return s


def attn_forward(q, k, v, scale, causal):
    """o and lse of [B,H,S,d] inputs in fp64."""
    B, Hq, Sq, d = q.shape
    group = Hq // k.shape[1]
    o = torch.empty(B, Hq, Sq, d, dtype=torch.float64, device=q.device)
    lse = torch.empty(B, Hq, Sq, dtype=torch.float64, device=q.device)
    for b in range(B):
        for h in range(Hq):
            s = scores(q[b, h].double(), k[b, h // group].double(), scale, causal)
            lse[b, h] = torch.logsumexp(s, -1)
            o[b, h] = torch.exp(s - lse[b, h][:, None]) @ v[b, h // group].double()
    return o, lse


def attn_backward(q, k, v, do, scale, causal, dlse=None, o_step=2.0 ** -24, out_step=U):
    """Exact (dq, dk, dv) and a bound on the error of each: P and dS rounded to bf16, the
    given o off by o_step of its values, the result rounded by out_step."""
    B, Hq, Sq, d = q.shape
    Hkv = k.shape[1]
    group = Hq // Hkv
    f64 = dict(dtype=torch.float64, device=q.device)
    exact = [torch.zeros(t.shape, **f64) for t in (q, k, v)]
    bound = [torch.zeros(t.shape, **f64) for t in (q, k, v)]
    for b in range(B):
        for h in range(Hq):
            n = h // group
            Q, K, V, G = (t.double() for t in (q[b, h], k[b, n], v[b, n], do[b, h]))
            p = torch.softmax(scores(Q, K, scale, causal), -1)
            dp = G @ V.t().contiguous()
            o = p @ V
            ds = dp - (p * dp).sum(-1, keepdim=True)
            if dlse is not None:
                ds = ds + dlse[b, h, :, None].double()
            ds = p * ds
            # dS: its own rounding, P's fp32 error, and dP - delta off by its sums and o's step
            absdp = G.abs() @ V.abs().t().contiguous()
            absdelta = (G.abs() * o.abs()).sum(-1, keepdim=True)
            if dlse is not None:
                absdelta = absdelta + dlse[b, h, :, None].double().abs()
            eds = ds.abs() * (U + SUMS) + p * ((absdp + absdelta) * 2.0 ** -20 + absdelta * o_step)
            sc = abs(scale)
            exact[0][b, h] = ds @ K * scale
            bound[0][b, h] = (eds + ds.abs() * SUMS) @ K.abs() * sc
            exact[1][b, n] += ds.t().contiguous() @ Q * scale
            bound[1][b, n] += (eds + ds.abs() * SUMS).t().contiguous() @ Q.abs() * sc
            exact[2][b, n] += p.t().contiguous() @ G
            bound[2][b, n] += p.t().contiguous() @ G.abs() * (U + 2 * SUMS)
    bound = [e * (1 + out_step) + x.abs() * out_step + 1e-30 for e, x in zip(bound, exact)]
    return exact, bound


def check(got, exact, bound, what):
    """Every element within its bound."""
    g = got.double()
    assert g.shape == exact.shape, f"{what}: shape {tuple(g.shape)} vs {tuple(exact.shape)}"
    assert torch.isfinite(g).all(), f"{what}: non-finite values"
    over = (g - exact).abs() / bound
    worst = float(over.max())
    assert worst <= 1.0, f"{what}: {worst:.3f} times the bound, {int((over > 1).sum())} elements"
    return worst


# ------------------------------------------------------ norm and rotation --
def rope_angles(S, B, inv_freq, positions, device):
    pos = torch.arange(S, device=device) if positions is None else positions.to(device)
    return pos.double().expand(B, S)[..., None] * inv_freq.double()


def rope_forward(x, w, angles, eps, interleaved):
    """fp64 [B,H,S,d] of x [B,S,H,d]."""
    x, w = x.double(), w.double()
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w
    R = 2 * angles.shape[-1]
    c, s = angles.cos()[:, :, None], angles.sin()[:, :, None]
    out = y.clone()
    if interleaved:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        out[..., 0:R:2], out[..., 1:R:2] = a * c - b * s, b * c + a * s
    else:
        a, b = y[..., :R // 2], y[..., R // 2:R]
        out[..., :R // 2], out[..., R // 2:R] = a * c - b * s, b * c + a * s
    return out.transpose(1, 2)


def rope_backward(g, x, w, angles, eps, interleaved):
    """fp64 gradients of x [B,S,H,d] and of w [d] from g [B,H,S,d], and the sum of the
    absolute terms of w's.  A term is g' n with g' = a cos + b sin; cos and sin are off by up
    to 2^-22 (the angle's rounding) + 2^-23 (their own), absolutely, so g' by 2^-21 (|a| + |b|)
    however small it is: the absolute term is (|a| + |b|) |n|."""
    g, x, w = g.double().transpose(1, 2), x.double(), w.double()
    R = 2 * angles.shape[-1]
    c, s = angles.cos()[:, :, None], angles.sin()[:, :, None]
    t, tabs = g.clone(), g.abs()
    first, second = (slice(0, R, 2), slice(1, R, 2)) if interleaved else \
        (slice(0, R // 2), slice(R // 2, R))
    a, b = g[..., first], g[..., second]
    t[..., first], t[..., second] = a * c + b * s, b * c - a * s
    tabs[..., first] = tabs[..., second] = a.abs() + b.abs()
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    n = x * r
    dw = (t * n).sum((0, 1, 2))
    gw = t * w
    dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
    return dx, dw, (tabs * n.abs()).sum((0, 1, 2))
