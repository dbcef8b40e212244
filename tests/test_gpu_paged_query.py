"""The workspace that paged_workspace_bytes names is what attn_paged takes, with every argument
that both have left as it is by default."""
from __future__ import annotations

import pytest
import torch

from tests.gpu_common import announce

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, I32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def pa():
    import paper_2609_29219_amd as pa
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    return pa


@pytest.mark.parametrize("heads", [(32, 8), (32, 1), (8, 8), (40, 1), (2, 2)],
                         ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens_with_default_arguments(pa, heads, d):
    Hq, Hkv = heads
    page = 16
    k, v = torch.randn(2, 8, Hkv, page, d, device=DEV).to(BF16)
    for R in (1, 2, 3, 8, 32, 64, 65, 256):
        q = torch.randn(R, Hq, d, device=DEV).to(BF16)
        kv = torch.arange(R, dtype=I32, device=DEV) % 100 + 1
        cu = torch.arange(R + 1, dtype=I32, device=DEV)
        for keys in (128, 512, 1024, 4096, 32768):
            announce(f"attn_paged queried workspace {heads} d={d} R={R} keys={keys}")
            table = torch.randint(8, (R, keys // page), device=DEV).int()
            n = pa.paged_workspace_bytes(R, R, Hq, Hkv, d, page, keys // page)
            ws = torch.empty(n, dtype=torch.uint8, device=DEV)
            args = (q, k, v, table, kv)
            assert torch.equal(pa.attn_paged(*args, workspace=ws), pa.attn_paged(*args))
            assert torch.equal(pa.attn_paged(*args, cu, workspace=ws), pa.attn_paged(*args, cu))
            n = pa.paged_workspace_bytes(R, R, Hq, Hkv, d, page, keys // page, max_q=1)
            assert torch.equal(pa.attn_paged(*args, max_q=1, workspace=ws[:n]),
                               pa.attn_paged(*args, max_q=1))
