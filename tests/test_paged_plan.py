"""How paged attention shares out its work, under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU): tests/c_abi/paged_plan_check.cpp, and with a planted mistake."""
from __future__ import annotations

import os
import re
import shutil
import subprocess

import pytest

from paper_2609_29219_amd import build
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


def test_as_many_workgroups_as_are_resident(check):
    # the row kernel as compiled: registers and LDS of its workgroups of four waves
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    r = subprocess.run([build.HIPCC, *build.CFLAGS, "--cuda-device-only", "-S", "-o", os.devnull,
                        "-Rpass-analysis=kernel-resource-usage",
                        os.path.join(CSRC, "paged_rows.hip")],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    found = {}
    for text in r.stderr.split("Function Name: ")[1:]:
        m = re.match(r"\S*paged_rows_kernelILi(\d+)ELi(\d)ELi4E", text)
        if m:
            waves = int(re.search(r"Occupancy \[waves/SIMD\]: (\d+)", text)[1])
            lds = int(re.search(r"LDS Size \[bytes/block\]: (\d+)", text)[1])
            assert re.search(r"VGPRs Spill: 0\b", text) and "ScratchSize [bytes/lane]: 0 " in text
            # a wave of each workgroup to a SIMD
            found[int(m[1]), 16 * int(m[2])] = min(waves, 160 * 1024 // lds)
    said = {}
    for line in run(check, "--resident").stdout.splitlines():
        d, block, n = map(int, line.split())
        said[d, block] = n
    assert len(found) == 4 and found == said
