"""Sizes that qk_norm_rope and qk_norm_rope_bwd refuse on the host (CPU)."""
from __future__ import annotations

import pytest

import paper_2609_29219_amd as pa
from tests import test_training_cpu as host


@pytest.mark.parametrize("n", [(1 << 30) + 1, 0x7FFFFFFF])
def test_more_heads_than_the_kernels_count_are_refused(n):
    # their head numbers are 32-bit integers that run up to a step past the last head
    for kw in (dict(Hq=n), dict(Hkv=n)):
        assert host.rope(B=1, S=1, **kw) == pa.ATTN_EUNSUPPORTED
        assert "heads" in pa.last_error()
        assert host.rope_bwd(B=1, S=1, **kw) == pa.ATTN_EUNSUPPORTED
        assert pa.lib.attn_qk_norm_rope_bwd_workspace_bytes(
            1, 1, kw.get("Hq", 1), kw.get("Hkv", 1), 64) == pa.ATTN_EUNSUPPORTED
