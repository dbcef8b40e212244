"""Largest calls of the paged cache's operators (CPU: refused on the host, or by the missing
device)."""
from __future__ import annotations

import pytest

import paper_2609_29219_amd as pa
from tests.test_paged_cpu import A, attend, heads

M = 1 << 30


@pytest.mark.parametrize("T,Hq,Hkv", [(M - 1, 2, 1), (M - 128, 2, 1), (M - 128, 2, 2)])
def test_rows_of_the_last_block_are_numbered_too(T, Hq, Hkv):
    # up to 255 rows more than there are: 2^31 - 256 rows and more would not be 32-bit numbers
    assert pa.lib.attn_paged_workspace_bytes(T, 1, 0, Hq, Hkv, 64, 16, 4, 0) == \
        pa.ATTN_EUNSUPPORTED
    assert "query rows" in pa.last_error()
    assert attend(T=T, Hq=Hq, Hkv=Hkv, q=heads(A, 0, Hq * 64, 64), o=A + (1 << 50)) == \
        pa.ATTN_EUNSUPPORTED
    assert "query rows" in pa.last_error()


def test_as_many_rows_as_there_are_numbers():
    got = pa.lib.attn_paged_workspace_bytes(M - 129, 1, 0, 2, 1, 64, 16, 4, 0)
    assert got != pa.ATTN_EUNSUPPORTED or "query rows" not in pa.last_error()
