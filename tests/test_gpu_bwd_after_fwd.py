"""attn_bwd from attn_fwd's own o and log-sum-exp: what the forward pass's rounding of the
weights adds to the gradients, bounded element by element."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_29219_amd as pa
from tests import training_refs as refs
from tests.gpu_common import announce

pytestmark = pytest.mark.gpu

U, SUMS = refs.U, refs.SUMS


def exact_and_bound(q, k, v, do, scale, causal, o_bf16):
    """With p the exact weights of a row: the forward pass sums and applies p_j (1 + e_j),
    |e_j| <= U, so its normaliser is off by a factor 1 + e, |e| <= U, which the log-sum-exp
    passes on.  The backward pass's weights are p / (1 + e), rounded once more: off by at most
    2 U + 2 U^2 of p.  o is off by (e_j - e) / (1 + e), at most 2 U + 3 U^2, of its absolute terms,
    and by its own rounding; delta by as much of |do|.  The rest as in refs.attn_backward."""
    B, Hq, Sq, d = q.shape
    group = Hq // k.shape[1]
    twice = 2 * U + 4 * U * U
    exact = [torch.zeros(t.shape, dtype=torch.float64, device=q.device) for t in (q, k, v)]
    bound = [torch.zeros_like(t) for t in exact]
    lse = torch.zeros(B, Hq, Sq, dtype=torch.float64, device=q.device)
    for b in range(B):
        for h in range(Hq):
            n = h // group
            Q, K, V, G = (t.double() for t in (q[b, h], k[b, n], v[b, n], do[b, h]))
            s = refs.scores(Q, K, scale, causal)
            lse[b, h] = torch.logsumexp(s, -1)
            p = torch.softmax(s, -1)
            dp, o = G @ V.t().contiguous(), p @ V
            delta = (G * o).sum(-1, keepdim=True)
            ds = p * (dp - delta)
            off = (p @ V.abs()) * (twice + SUMS)
            if o_bf16:
                off = off + (o.abs() + off) * U
            absdp = G.abs() @ V.abs().t().contiguous()
            absdelta = (G.abs() * o.abs()).sum(-1, keepdim=True)
            inner = (absdp + absdelta) * 2.0 ** -20 + (G.abs() * off).sum(-1, keepdim=True)
            eds = ds.abs() * (twice + 2 * SUMS) + p * (1 + 2 * twice) * inner
            exact[0][b, h] = ds @ K * scale
            bound[0][b, h] = eds @ K.abs() * scale
            exact[1][b, n] += ds.t().contiguous() @ Q * scale
            bound[1][b, n] += eds.t().contiguous() @ Q.abs() * scale
            exact[2][b, n] += p.t().contiguous() @ G
            bound[2][b, n] += p.t().contiguous() @ G.abs() * (twice + 2 * SUMS)
    return exact, [e * (1 + U) + x.abs() * U + 1e-30 for e, x in zip(bound, exact)], lse


@pytest.mark.parametrize("o_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 2, 2, 2, 2, 64, True), (1, 4, 2, 40, 40, 128, True),
                                   (2, 8, 2, 333, 333, 64, True), (1, 8, 1, 100, 1500, 128, False),
                                   (1, 2, 1, 7, 9000, 64, True)],
                         ids=lambda s: "x".join(map(str, s)))
def test_attn_bwd_from_the_forward_pass(shape, o_type):
    announce(f"attn_bwd after attn_fwd {shape} {o_type}")
    B, Hq, Hkv, Sq, Skv, d, causal = shape
    g = torch.Generator(device="cuda").manual_seed(11)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    q, do, k, v = mk(B, Hq, Sq, d), mk(B, Hq, Sq, d), mk(B, Hkv, Skv, d), mk(B, Hkv, Skv, d)
    o, lse = pa.attn_fwd(q, k, v, causal=causal, out_dtype=o_type, return_lse=True)
    got = pa.attn_bwd(do, q, k, v, o, lse, causal=causal)
    exact, bound, want = exact_and_bound(q, k, v, do, 1 / math.sqrt(d), causal,
                                         o_type is torch.bfloat16)
    # the log-sum-exp as the contract has it: the normaliser's factor, and fp32
    assert float((lse.double() - want).abs().max()) <= -math.log(1 - U) + SUMS
    for name, x, e, b in zip(("dq", "dk", "dv"), got, exact, bound):
        print(f"[after attn_fwd] {shape} {name}: {refs.check(x, e, b, f'{shape}: {name}'):.3f} of "
              "its bound", flush=True)
