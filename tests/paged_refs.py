"""The paged cache's operators from their definitions: attention in float64 with a bound on what
its kernels may be off, the tables in Python integers.

A bound counts roundings: u = 2^-8 is half a step of bf16 relative to the value, 2^-14 what the
fp32 sums are allowed (up to 2^9 additions of 2^-24 each, one behind another, and as many scores'
steps).
"""
from __future__ import annotations

import math

import torch

U = 2.0 ** -8
SUMS = 2.0 ** -14


def attend(q, k, v, pos, scale, causal, window=0, softcap=0.0, slope=0.0, out_step=U):
    """o, lse, and bounds on the error of each, of one head's queries q [n,d] at positions pos over
    the keys and values k, v [m,d] of one request."""
    q, k, v = q.double(), k.double(), v.double()
    raw = q @ k.t().contiguous() * scale
    # the exponent: the products' sums, the cap (2^-22 of it, and what the score's error
    # becomes), the distance's product, all in fp32
    err = (q.abs() @ k.abs().t().contiguous() * abs(scale) + raw.abs()) * 2.0 ** -20
    x = raw
    if softcap:
        x = softcap * torch.tanh(raw / softcap)
        err = err + softcap * 2.0 ** -21
    keys = torch.arange(k.shape[0], device=q.device)
    away = (pos[:, None] - keys).double()
    if slope:
        x = x - slope * away.abs()
        err = err + slope * away.abs() * 2.0 ** -21
    seen = torch.ones_like(x, dtype=torch.bool)
    if causal:
        seen &= away >= 0
    if window:
        seen &= away < window
    x = x.masked_fill(~seen, -math.inf)
    none = ~seen.any(-1)
    lse = torch.logsumexp(x, -1)
    # the difference to the maximum is taken in fp32 as well
    top = x.amax(-1, keepdim=True).masked_fill(none[:, None], 0.0)
    err = err + (x - top).abs().masked_fill(~seen, 0.0) * 2.0 ** -22 + top.abs() * 2.0 ** -22
    w = torch.exp(x - lse[:, None]).masked_fill(none[:, None], 0.0)
    o = w @ v
    off = (w * err).sum(-1, keepdim=True)
    bound = (w * (U + SUMS + err)) @ v.abs() + o.abs() * (off + SUMS)
    bound = bound * (1 + out_step) + o.abs() * out_step + 1e-30
    return o, lse, bound, off[:, 0] + SUMS + lse.abs().masked_fill(none, 0.0) * 2.0 ** -22


def attend_paged(q, k_pages, v_pages, table, kv_lens, cu, scale, causal=True, window=0,
                 softcap=0.0, slopes=None, out_step=U):
    """The same of a whole call; lengths as lists.  Rows behind the last request's are NaN."""
    T, Hq, d = q.shape
    Hkv, page = k_pages.shape[1:3]
    f64 = dict(dtype=torch.float64, device=q.device)
    o, bound = torch.full((T, Hq, d), math.nan, **f64), torch.ones((T, Hq, d), **f64)
    lse, lse_bound = torch.full((T, Hq), math.nan, **f64), torch.ones((T, Hq), **f64)
    for r, S in enumerate(kv_lens):
        a, b = cu[r], cu[r + 1]
        if a == b:
            continue
        j = torch.arange(S, device=q.device)
        at = table[r].long()[j // page], j % page
        pos = torch.arange(b - a, device=q.device) + S - (b - a)
        for h in range(Hq):
            n = h // (Hq // Hkv)
            if S == 0:
                o[a:b, h], lse[a:b, h], bound[a:b, h] = 0.0, -math.inf, 1e-30
                continue
            o[a:b, h], lse[a:b, h], bound[a:b, h], lse_bound[a:b, h] = attend(
                q[a:b, h], k_pages[at[0], n, at[1]], v_pages[at[0], n, at[1]], pos, scale, causal,
                window, softcap, 0.0 if slopes is None else float(slopes[h]), out_step)
    return o, lse, bound, lse_bound


def check(got, exact, bound, what):
    """Every element within its bound; infinities where they belong."""
    g = got.double()
    assert g.shape == exact.shape, f"{what}: shape {tuple(g.shape)} vs {tuple(exact.shape)}"
    finite = torch.isfinite(exact)
    assert torch.equal(g[~finite], exact[~finite]), f"{what}: infinities"
    assert torch.isfinite(g[finite]).all(), f"{what}: non-finite values"
    over = ((g - exact).abs() / bound)[finite]
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3f} times the bound, {int((over > 1).sum())} elements"
    return worst


def extend(table, seq, new, free, n_free, page, T):
    """(slots, positions, cu, kv, n_left) and the table, as lists."""
    table = [list(row) for row in table]
    slots, positions, cu, kv, taken = [], [], [0], [], 0
    for r, (s, n) in enumerate(zip(seq, new)):
        for p in range(s, s + n):
            i = p // page
            if i < len(table[r]) and i >= -(-s // page) and p % page == 0:
                table[r][i] = free[n_free - 1 - taken] if taken < n_free else -1
                taken += 1
            entry = table[r][i] if i < len(table[r]) else -1
            slots.append(entry * page + p % page if entry >= 0 else -1)
            positions.append(p)
        cu.append(cu[-1] + n)
        kv.append(s + n)
    pad = T - len(slots)
    return slots + [-1] * pad, positions + [0] * pad, cu, kv, n_free - taken, table


def release(table, seq, keep, free, n_free, page):
    """n_left and the list."""
    free = list(free)
    for row, s, k in zip(table, seq, keep):
        for i in range(-(-k // page), min(-(-s // page), len(row))):
            if n_free < len(free):
                free[n_free] = row[i]
                n_free += 1
    return n_free, free
