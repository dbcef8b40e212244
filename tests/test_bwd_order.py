"""A plan of the backward pass holds no unset units (CPU): tests/c_abi/bwd_order_check.cpp."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

from tests.test_bwd_plan import CSRC, ROOT, run


def test_no_unit_is_unset(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    out = str(tmp_path / "bwd_order_check")
    cmd = [gxx, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(CSRC, "plan.cpp"),
           os.path.join(ROOT, "tests", "c_abi", "bwd_order_check.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    r = run(out)
    assert r.returncode == 0 and "bwd_order_check ok" in r.stdout, (r.stdout + r.stderr)[-2000:]
