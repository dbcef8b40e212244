"""The counters that the benchmark line quotes are of the sources as they stand (CPU): after a
change to the files in bench.KERNEL_SOURCES the profiles are taken again, by the commands that
they name, or the line has no traffic and no MFMA share."""
from __future__ import annotations

import pytest

import bench
from attn_inputs import BY_NAME

PREFILL = ("prefill_b1_h32_s8192_d128", "prefill_b4_h16_s2048_d128_causal")
DECODE = ("decode_b16_h32_s8192_d128", "decode_b1_h32_s131072_d128")


@pytest.mark.parametrize("kind,workload", [("prefill", w) for w in PREFILL] +
                         [("decode", w) for w in DECODE] + [("gemm", bench.GEMM_WORKLOAD)])
def test_traffic_is_of_these_sources(kind, workload):
    traffic = bench.profiled_traffic(kind, workload)
    assert traffic is not None, f"profiles/traffic_{workload}.txt is of other sources"
    # no less than the operands and results once (within 1%: the counters' accuracy); the GEMM
    # reads its operands several times
    if kind == "gemm":
        needed = bench.gemm_bytes()
    else:
        w = BY_NAME[workload]
        needed = w.B * w.H * w.d * (2 * (w.Sq + 2 * w.Skv) + 4 * w.Sq)
    assert 0.99 * needed <= traffic <= 5 * needed


@pytest.mark.parametrize("workload", PREFILL)
def test_mfma_share_is_of_these_sources(workload):
    share = bench.profiled_mfma_busy(workload)
    assert share is not None, f"profiles/mfma_{workload}.txt is of other sources"
    assert 0.0 < share < 1.0
