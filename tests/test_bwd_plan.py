"""The backward pass's plan under AddressSanitizer and UndefinedBehaviorSanitizer (CPU):
tests/c_abi/bwd_plan_check.cpp over a seeded sweep of shapes, and with a planted mistake."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_29219_amd", "csrc")


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    out = str(tmp_path_factory.mktemp("plan") / "bwd_plan_check")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
           os.path.join(CSRC, "plan.cpp"),
           os.path.join(ROOT, "tests", "c_abi", "bwd_plan_check.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    return out


def run(exe, *args):
    env = dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    env.pop("LD_PRELOAD", None)
    return subprocess.run([exe, *args], capture_output=True, text=True, timeout=300, env=env)


def test_every_part_of_every_block_once(check):
    r = run(check)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "bwd_plan_check ok" in r.stdout


def test_a_planted_mistake_is_caught(check):
    r = run(check, "--planted")
    assert r.returncode == 0 and "caught" in r.stdout, (r.stdout + r.stderr)[-2000:]
