"""How paged attention shares out its work, under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU): tests/c_abi/paged_plan_check.cpp, and with a planted mistake."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

from tests.test_bwd_plan import CSRC, ROOT, run


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    out = str(tmp_path_factory.mktemp("plan") / "paged_plan_check")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
           os.path.join(ROOT, "tests", "c_abi", "paged_plan_check.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    return out


def test_no_part_without_memory(check):
    r = run(check)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "paged_plan_check ok" in r.stdout


def test_a_planted_mistake_is_caught(check):
    r = run(check, "--planted")
    assert r.returncode == 0 and "caught" in r.stdout, (r.stdout + r.stderr)[-2000:]
