"""The backward pass without memory for the parts of its sums: the plan (CPU, under
AddressSanitizer and UndefinedBehaviorSanitizer) and the call."""
from __future__ import annotations

import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2609_29219_amd as pa
from tests import training_refs as refs
from tests.gpu_common import announce
from tests.test_bwd_plan import CSRC, ROOT, run


def test_the_plan_without_splits(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    out = str(tmp_path / "bwd_unsplit_check")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           os.path.join(CSRC, "plan.cpp"),
           os.path.join(ROOT, "tests", "c_abi", "bwd_unsplit_check.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    r = run(out)
    assert r.returncode == 0 and "bwd_unsplit_check ok" in r.stdout, (r.stdout + r.stderr)[-2000:]


@pytest.fixture
def workspace_limit():
    """Sets the largest buffer that the library's workspaces get."""
    f = pa.lib.attn__workspace_limit
    f.argtypes = [ctypes.c_longlong]
    yield f
    f(-1)


def new_stream():
    """A stream that no call has used (torch hands out pooled ones); never destroyed."""
    handle = ctypes.c_void_p()
    create = pa.lib.hipStreamCreate  # of the runtime that the library is linked with
    create.argtypes = [ctypes.POINTER(ctypes.c_void_p)]
    assert create(ctypes.byref(handle)) == 0
    return torch.cuda.ExternalStream(handle.value)


def randn(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 2, 1, 129, 1500, 128, True), (1, 8, 2, 20, 5000, 64, True),
                                   (1, 4, 4, 700, 900, 64, False)],
                         ids=lambda s: "x".join(map(str, s)))
def test_attn_bwd_without_memory_for_parts(workspace_limit, shape):
    announce(f"attn_bwd without memory for parts {shape}")
    B, Hq, Hkv, Sq, Skv, d, causal = shape
    q, do = randn(1, B, Hq, Sq, d), randn(2, B, Hq, Sq, d)
    k, v = randn(3, B, Hkv, Skv, d), randn(4, B, Hkv, Skv, d)
    sc = d ** -0.5
    o, lse = refs.attn_forward(q, k, v, sc, causal)
    args = (do, q, k, v, o.float(), lse.float())
    exact, bound = refs.attn_backward(q, k, v, do, sc, causal)
    with_parts = pa.attn_bwd(*args, causal=causal)
    # what the row values take: 256 bytes for every 32 rows of a head, a power of two; the
    # call with parts needs more
    limit = 1 << 16
    assert B * Hq * ((Sq + 31) // 32) * 256 <= limit < pa.bwd_workspace_bytes(
        B, Hq, Hkv, Sq, Skv, d, causal)
    torch.cuda.synchronize()
    workspace_limit(limit)
    stream = new_stream()
    with torch.cuda.stream(stream):
        got = pa.attn_bwd(*args, causal=causal)
        again = pa.attn_bwd(*args, causal=causal)
    stream.synchronize()
    for name, g, a, w, e, b in zip(("dq", "dk", "dv"), got, again, with_parts, exact, bound):
        refs.check(g, e, b, f"{shape}: {name}")
        refs.check(w, e, b, f"{shape}: {name} in parts")
        assert torch.equal(g, a), name
    # no memory at all is an error, and nothing is written
    workspace_limit(0)
    outs = [torch.full_like(t, 7.0) for t in (q, k, v)]
    torch.cuda.synchronize()
    stream = new_stream()
    with torch.cuda.stream(stream), pytest.raises(pa.AttnError) as e:
        pa.attn_bwd(*args, causal=causal, dq=outs[0], dk=outs[1], dv=outs[2])
    assert e.value.code == pa.ATTN_ENOMEM
    torch.cuda.synchronize()
    assert all((t == 7.0).all() for t in outs)
    # with memory again, the same stream runs in parts
    workspace_limit(-1)
    with torch.cuda.stream(stream):
        later = pa.attn_bwd(*args, causal=causal)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(with_parts, later))
