"""Tiled exact attention on MI355X (gfx950): Python binding of libattn.so.

This module only marshals arguments into the C ABI declared in
``include/attn.h``; every step of the computation runs in the HIP kernels of
``libattn.so``.  PyTorch is used for device memory and the current stream.
There is no fallback: if the library is missing, importing this package
raises ImportError, and the compute calls raise AttnError without a gfx950
device.

    o = attn_fwd(q, k, v, scale=None, causal=False)  # q [B,H,Sq,d], k/v [B,H,Skv,d] bf16
    o = attn_decode(q, k, v, n_splits=0)             # q [B,H,d], k/v [B,H,Skv,d] bf16
    dq, dk, dv = attn_bwd(do, q, k, v, o, lse)       # the gradients of attn_fwd
    q, k, v = qk_norm_rope(q, k, v, wq, wk, freq)    # [B,S,H,d] projections to [B,H,S,d]

Requests of different lengths, over a cache in pages:

    slots, positions, cu, kv_lens, n_left = paged_extend(table, seq_lens, new_lens, free_pages,
                                                         n_free, page_size, n_tokens)
    paged_store(k, v, slots, k_pages, v_pages)       # k, v [T,Hkv,d] into [P,Hkv,page,d]
    o = attn_paged(q, k_pages, v_pages, table, kv_lens, cu)         # q [T,Hq,d]
    n_free = paged_release(table, kv_lens, keep_lens, free_pages, n_left, page_size)
"""
from __future__ import annotations

import ctypes
import math
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libattn.so")

ATTN_OK = 0
ATTN_EINVAL = -1
ATTN_EUNSUPPORTED = -2
ATTN_EHIP = -3
ATTN_ENOMEM = -4
KIND_FWD = 0
KIND_DECODE = 1
ATTN_OUT_BF16 = 1
ATTN_GEMM_B_NK = 2
ATTN_O_BF16 = 4
ATTN_ROPE_INTERLEAVED = 8
ATTN_WEIGHT_F32 = 16
ATTN_POSITIONS_I64 = 32
ATTN_GRAD_F32 = 64

# Entry points declared in include/attn.h.
EXPORTED = ("attn_fwd", "attn_decode", "attn_fwd_ex", "attn_decode_ex",
            "attn_decode_workspace_bytes", "attn_set_stream", "attn_get_stream",
            "attn_last_error", "attn_query_device", "attn_measure_device", "attn_get_plan",
            "attn_get_plan_for", "attn_get_plan_ex", "attn_gemm", "attn_gemm_plan", "attn_decode_noalloc",
            "attn_bwd", "attn_bwd_workspace_bytes", "attn_qk_norm_rope",
            "attn_qk_norm_rope_bwd", "attn_qk_norm_rope_bwd_workspace_bytes",
            "attn_paged_extend", "attn_paged_release", "attn_paged_store", "attn_paged",
            "attn_paged_workspace_bytes")
NOALLOC_SCRATCH_BYTES = 16 << 20  # ATTN_NOALLOC_SCRATCH_BYTES


class AttnError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"attn error {code}: {msg}")
        self.code = code


class Heads(ctypes.Structure):
    """attn_heads: rows of d values by batch, token and head, strides in elements."""
    _fields_ = [("ptr", ctypes.c_void_p), ("batch_stride", ctypes.c_longlong),
                ("row_stride", ctypes.c_longlong), ("head_stride", ctypes.c_longlong)]


class DeviceDesc(ctypes.Structure):
    _fields_ = [
        ("arch", ctypes.c_char * 32),
        ("num_cus", ctypes.c_int),
        ("num_xcds", ctypes.c_int),
        ("simds_per_cu", ctypes.c_int),
        ("wave_size", ctypes.c_int),
        ("lds_bytes_per_cu", ctypes.c_int),
        ("vgprs_per_simd_lane", ctypes.c_int),
        ("max_waves_per_simd", ctypes.c_int),
        ("clock_ghz", ctypes.c_double),
        ("mfma_bf16_flops_per_clk_cu", ctypes.c_double),
        ("valu_lanes_per_clk_simd", ctypes.c_double),
        ("trans_cycles_per_op", ctypes.c_double),
        ("lds_bytes_per_clk_cu", ctypes.c_double),
        ("l2_bytes_per_clk_xcd", ctypes.c_double),
        ("hbm_bytes_per_s", ctypes.c_double),
        ("hbm_latency_us", ctypes.c_double),
        ("launch_us", ctypes.c_double),
        ("issue_cycles_per_score", ctypes.c_double),
        ("valu_mfma_overlap", ctypes.c_double),
        ("tile_sync_cycles", ctypes.c_double),
        ("tile_latency_cycles", ctypes.c_double),
    ]

    def as_dict(self) -> dict:
        d = {name: getattr(self, name) for name, _ in self._fields_}
        d["arch"] = self.arch.decode()
        return d


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python paper_2609_29219_amd/build.py` "
            "(or __graft_entry__.build())")
    # One HIP runtime per process: torch ships its own libamdhip64, and the
    # library must bind to that one (loaded first, it satisfies the library's
    # dependency), not load the system copy beside it.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.attn_fwd.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, ci]
    lib.attn_decode.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci]
    lib.attn_fwd_ex.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, ci, ci]
    lib.attn_decode_ex.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, vp,
                                   ctypes.c_size_t]
    lib.attn_decode_noalloc.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci]
    lib.attn_decode_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci]
    lib.attn_decode_workspace_bytes.restype = ctypes.c_longlong
    lib.attn_set_stream.argtypes = [vp]
    lib.attn_get_stream.argtypes = []
    lib.attn_get_stream.restype = vp
    lib.attn_last_error.argtypes = []
    lib.attn_last_error.restype = ctypes.c_char_p
    lib.attn_query_device.argtypes = [ctypes.POINTER(DeviceDesc)]
    lib.attn_measure_device.argtypes = [ctypes.POINTER(DeviceDesc)]
    lib.attn_get_plan.argtypes = [ci, ci, ci, ci, ci, ci, ci, ci, ctypes.c_char_p, ci]
    lib.attn_get_plan_for.argtypes = [ctypes.POINTER(DeviceDesc), ci, ci, ci, ci, ci, ci, ci,
                                      ci, ctypes.c_char_p, ci]
    lib.attn_get_plan_ex.argtypes = [ctypes.POINTER(DeviceDesc), ci, ci, ci, ci, ci, ci, ci, ci,
                                     ci, ctypes.c_char_p, ci]
    lib.attn__fwd_candidates.argtypes = [ctypes.POINTER(DeviceDesc), ci, ci, ci, ci, ci, ci, ci,
                                         ci, ctypes.c_char_p, ci]
    lib.attn_gemm.argtypes = [vp, vp, vp, ci, ci, ci, ci]
    lib.attn_gemm_plan.argtypes = [ctypes.POINTER(DeviceDesc), ci, ci, ci, ci, ctypes.c_char_p,
                                   ci]
    lib.attn__gemm_candidates.argtypes = [ctypes.POINTER(DeviceDesc), ci, ci, ci, ci, ci,
                                          ctypes.c_char_p, ci]
    lib.attn_bwd.argtypes = [vp] * 10 + [ci] * 6 + [cf, ci, ci, vp, ctypes.c_size_t]
    lib.attn_bwd_workspace_bytes.argtypes = [ci] * 7
    lib.attn_bwd_workspace_bytes.restype = ctypes.c_longlong
    ll = ctypes.c_longlong
    lib.attn_qk_norm_rope.argtypes = [vp] * 6 + [vp] * 4 + [ll] + [ci] * 6 + [cf, ci]
    lib.attn_qk_norm_rope_bwd.argtypes = [vp] * 8 + [vp] * 4 + [ll, vp, vp] + [ci] * 6 + \
        [cf, ci, vp, ctypes.c_size_t]
    lib.attn_qk_norm_rope_bwd_workspace_bytes.argtypes = [ci] * 5
    lib.attn_qk_norm_rope_bwd_workspace_bytes.restype = ctypes.c_longlong
    lib.attn_paged_extend.argtypes = [vp, ll, vp, vp, vp, ci] + [vp] * 6 + [ci] * 4
    lib.attn_paged_release.argtypes = [vp, ll, vp, vp, vp, ci, vp, vp] + [ci] * 3
    lib.attn_paged_store.argtypes = [vp] * 5 + [ci] * 5
    lib.attn_paged.argtypes = [vp] * 6 + [ll, vp, vp, vp] + [ci] * 9 + [cf, cf, ci, ci, ci, vp,
                                                                       ctypes.c_size_t]
    lib.attn_paged_workspace_bytes.argtypes = [ci] * 9
    lib.attn_paged_workspace_bytes.restype = ctypes.c_longlong
    for fn in (lib.attn__bwd_packed, lib.attn__qk_norm_rope_packed,
               lib.attn__qk_norm_rope_bwd_packed, lib.attn__paged_extend_packed,
               lib.attn__paged_release_packed, lib.attn__paged_store_packed,
               lib.attn__paged_packed):
        fn.argtypes = [ctypes.c_char_p]
        fn.restype = ci
    for fn in (lib.attn_paged_extend, lib.attn_paged_release, lib.attn_paged_store,
               lib.attn_paged, lib.attn_bwd, lib.attn_qk_norm_rope, lib.attn_qk_norm_rope_bwd,
               lib.attn_fwd, lib.attn_decode, lib.attn_fwd_ex, lib.attn_decode_ex,
               lib.attn_decode_noalloc,
               lib.attn_set_stream, lib.attn_query_device,
               lib.attn_measure_device, lib.attn_get_plan, lib.attn_get_plan_for,
               lib.attn_get_plan_ex,
               lib.attn__fwd_candidates, lib.attn_gemm, lib.attn_gemm_plan,
               lib.attn__gemm_candidates):
        fn.restype = ci
    return lib


lib = _load()


def last_error() -> str:
    return lib.attn_last_error().decode()


def _check(rc: int):
    if rc != ATTN_OK:
        raise AttnError(rc, last_error())


# The host path is most of the time of the smallest calls (kernels of a few
# microseconds): the stream is read as a raw handle, without a Python stream
# object around it, and _require passes a good tensor in one expression.
try:
    from torch._C import _cuda_getCurrentRawStream as _raw_stream
except ImportError:
    def _raw_stream(index: int) -> int:
        import torch
        return torch.cuda.current_stream(index).cuda_stream


def _set_stream(t) -> None:
    lib.attn_set_stream(_raw_stream(t.get_device()))


def _require(t, dtype, shape, name):
    import torch
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.shape == shape and \
            t.is_contiguous():
        return
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_cuda:
        raise TypeError(f"{name} must be a {dtype} tensor on a HIP device")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def attn_fwd(q, k, v, o=None, scale: float | None = None, causal: bool = False,
             out_dtype=None, return_lse: bool = False):
    """Prefill attention; returns o [B,Hq,Sq,d] (fp32, or out_dtype bf16),
    and with return_lse also the fp32 row log-sum-exp [B,Hq,Sq].  k and v
    may have fewer heads than q (grouped-query heads: Hkv divides Hq)."""
    import torch
    B, Hq, Sq, d = q.shape
    Hkv, Skv = k.shape[1], k.shape[2]
    _require(q, torch.bfloat16, (B, Hq, Sq, d), "q")
    _require(k, torch.bfloat16, (B, Hkv, Skv, d), "k")
    _require(v, torch.bfloat16, (B, Hkv, Skv, d), "v")
    if out_dtype is None:
        out_dtype = o.dtype if o is not None else torch.float32
    if out_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
    if o is None:
        o = torch.empty((B, Hq, Sq, d), dtype=out_dtype, device=q.device)
    else:
        _require(o, out_dtype, (B, Hq, Sq, d), "o")
    lse = None
    if return_lse:
        lse = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    _set_stream(q)
    flags = ATTN_OUT_BF16 if out_dtype == torch.bfloat16 else 0
    _check(lib.attn_fwd_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                           lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Sq, Skv, d,
                           float(scale), int(bool(causal)), flags))
    return (o, lse) if return_lse else o


def attn_decode(q, k, v, o=None, n_splits: int = 0, workspace=None, return_lse: bool = False):
    """Split-KV single-query attention; returns o fp32 [B,Hq,d], and with
    return_lse also the row log-sum-exp [B,Hq].  k and v may have fewer heads
    than q (grouped-query heads).  workspace: None (the library's), or a
    device tensor of at least decode_workspace_bytes(...) bytes."""
    import torch
    B, Hq, d = q.shape
    Hkv, Skv = k.shape[1], k.shape[2]
    _require(q, torch.bfloat16, (B, Hq, d), "q")
    _require(k, torch.bfloat16, (B, Hkv, Skv, d), "k")
    _require(v, torch.bfloat16, (B, Hkv, Skv, d), "v")
    if o is None:
        o = torch.empty((B, Hq, d), dtype=torch.float32, device=q.device)
    else:
        _require(o, torch.float32, (B, Hq, d), "o")
    lse = None
    if return_lse:
        lse = torch.empty((B, Hq), dtype=torch.float32, device=q.device)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or \
                not workspace.is_contiguous():
            raise TypeError("workspace must be a contiguous tensor on a HIP device")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _set_stream(q)
    _check(lib.attn_decode_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                              lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Skv, d,
                              int(n_splits), ws_ptr, ws_bytes))
    return (o, lse) if return_lse else o


def attn_decode_noalloc(q, k, v, o, n_splits: int = 0, lse=None):
    """attn_decode with its split partials in the library's static device
    scratch: allocates nothing, so o (fp32 [B,Hq,d]) and the optional lse
    (fp32 [B,Hq]) must be given.  Calls that can overlap on one device race
    on the scratch."""
    import torch
    B, Hq, d = q.shape
    Hkv, Skv = k.shape[1], k.shape[2]
    _require(q, torch.bfloat16, (B, Hq, d), "q")
    _require(k, torch.bfloat16, (B, Hkv, Skv, d), "k")
    _require(v, torch.bfloat16, (B, Hkv, Skv, d), "v")
    _require(o, torch.float32, (B, Hq, d), "o")
    if lse is not None:
        _require(lse, torch.float32, (B, Hq), "lse")
    _set_stream(q)
    _check(lib.attn_decode_noalloc(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                   lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Skv,
                                   d, int(n_splits)))
    return o


def decode_workspace_bytes(B: int, Hq: int, Hkv: int, Skv: int, d: int, n_splits: int = 0) -> int:
    """Bytes of workspace attn_decode needs with a caller-provided buffer."""
    n = lib.attn_decode_workspace_bytes(B, Hq, Hkv, Skv, d, int(n_splits))
    if n < 0:
        raise AttnError(int(n), last_error())
    return int(n)


def gemm(a, b, c=None, b_nk: bool = False, out_dtype=None):
    """C = A B on bf16 MFMA with fp32 accumulation.  a: bf16 [M,K]; b: bf16
    [K,N], or [N,K] with b_nk; returns c [M,N] fp32 (or out_dtype bf16)."""
    import torch
    M, K = a.shape
    N = b.shape[0] if b_nk else b.shape[1]
    _require(a, torch.bfloat16, (M, K), "a")
    _require(b, torch.bfloat16, (N, K) if b_nk else (K, N), "b")
    if out_dtype is None:
        out_dtype = c.dtype if c is not None else torch.float32
    if out_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
    if c is None:
        c = torch.empty((M, N), dtype=out_dtype, device=a.device)
    else:
        _require(c, out_dtype, (M, N), "c")
    flags = (ATTN_OUT_BF16 if out_dtype == torch.bfloat16 else 0) | \
        (ATTN_GEMM_B_NK if b_nk else 0)
    _set_stream(a)
    _check(lib.attn_gemm(a.data_ptr(), b.data_ptr(), c.data_ptr(), M, N, K, flags))
    return c


# The operands of the calls below, packed as csrc/api.hip's PackedBwd, PackedRope and
# PackedRopeBwd: ctypes converts an argument in 0.08 us, and these calls have up to 30 numbers
# (qk_norm_rope of one token 15.6 us with them as arguments, 12.9 packed).
_BWD_CALL = struct.Struct("13Q8if")
_ROPE_CALL = struct.Struct("24q4QqQ7if")
_ROPE_BWD_CALL = struct.Struct("32q4Qq5Q7if")


def _require_on(t, dtype, shape, name, dev) -> None:
    """_require, on device dev (one expression for a good tensor)."""
    if getattr(t, "dtype", None) is dtype and t.get_device() == dev and t.shape == shape and \
            t.is_contiguous():
        return
    _require(t, dtype, shape, name)
    raise ValueError(f"{name} is on another device than the first operand")


def _call_on(dev, fn, packed) -> None:
    """A C call on device dev."""
    import torch
    if torch._C._cuda_getDevice() != dev:
        with torch.cuda.device(dev):
            return _call_on(dev, fn, packed)
    _check(fn(packed))


def _workspace(workspace, dev):
    """Address and bytes of a caller's workspace (None: the library's)."""
    import torch
    if workspace is None:
        return 0, 0
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or \
            not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous tensor on a HIP device")
    if workspace.get_device() != dev:
        raise ValueError("workspace is on another device than the first operand")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def attn_bwd(do, q, k, v, o, lse, scale: float | None = None, causal: bool = False, dlse=None,
             dq=None, dk=None, dv=None, out_dtype=None, workspace=None):
    """Gradients of attn_fwd; returns (dq, dk, dv), bf16 (or out_dtype fp32).

    q, k, v, scale, causal: as attn_fwd got them; o (fp32 or bf16) and lse: what it
    returned (return_lse=True).  do: the gradient of o, bf16 [B,Hq,Sq,d]; dlse: that of
    lse, fp32 [B,Hq,Sq], or None.  workspace: None (the library's), or a device tensor of
    at least bwd_workspace_bytes(...) bytes."""
    import torch
    B, Hq, Sq, d = qs = q.shape
    Hkv, Skv = k.shape[1], k.shape[2]
    ks = (B, Hkv, Skv, d)
    bf16, f32 = torch.bfloat16, torch.float32
    dev = q.get_device()
    if dev < 0:
        raise TypeError("q must be on a HIP device")
    _require_on(q, bf16, qs, "q", dev)
    _require_on(k, bf16, ks, "k", dev)
    _require_on(v, bf16, ks, "v", dev)
    _require_on(do, bf16, qs, "do", dev)
    o_bf16 = getattr(o, "dtype", None) is bf16
    _require_on(o, bf16 if o_bf16 else f32, qs, "o", dev)
    _require_on(lse, f32, (B, Hq, Sq), "lse", dev)
    if dlse is not None:
        _require_on(dlse, f32, (B, Hq, Sq), "dlse", dev)
    if out_dtype is None:
        given = dq if dq is not None else dk if dk is not None else dv
        out_dtype = bf16 if given is None else given.dtype
    if out_dtype not in (f32, bf16):
        raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
    if dq is None:
        dq = torch.empty_like(q, dtype=out_dtype)
    else:
        _require_on(dq, out_dtype, qs, "dq", dev)
    if dk is None:
        dk = torch.empty_like(k, dtype=out_dtype)
    else:
        _require_on(dk, out_dtype, ks, "dk", dev)
    if dv is None:
        dv = torch.empty_like(v, dtype=out_dtype)
    else:
        _require_on(dv, out_dtype, ks, "dv", dev)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    flags = (ATTN_OUT_BF16 if out_dtype is bf16 else 0) | (ATTN_O_BF16 if o_bf16 else 0)
    _call_on(dev, lib.attn__bwd_packed, _BWD_CALL.pack(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), do.data_ptr(),
        0 if dlse is None else dlse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
        *_workspace(workspace, dev), _raw_stream(dev), B, Hq, Hkv, Sq, Skv, d,
        1 if causal else 0, flags, scale))
    return dq, dk, dv


def bwd_workspace_bytes(B: int, Hq: int, Hkv: int, Sq: int, Skv: int, d: int,
                        causal: bool = False) -> int:
    """Bytes of workspace attn_bwd needs with a caller-provided buffer."""
    n = lib.attn_bwd_workspace_bytes(B, Hq, Hkv, Sq, Skv, d, int(bool(causal)))
    if n < 0:
        raise AttnError(int(n), last_error())
    return int(n)


def _rows(t, dtype, shape, name, dev):
    """A 4-dimensional tensor whose rows (last dimension) are contiguous, checked; its
    strides."""
    if getattr(t, "dtype", None) is dtype and t.get_device() == dev and t.shape == shape:
        strides = t.stride()
        if strides[3] == 1:
            return strides
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() < 0:
        raise TypeError(f"{name} must be a {dtype} tensor on a HIP device")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on another device than the first operand")
    raise ValueError(f"{name} must be contiguous in its last dimension")


def _head_major_out(out, B, S, H, d, name, like):
    """An output [B,H,S,d] (the given one, checked, or a new bf16 one as like is) and its
    fields."""
    import torch
    if out is None:
        out = like.new_empty((B, H, S, d))
        return out, (out.data_ptr(), H * S * d, d, S * d)
    return out, _head_major(out, torch.bfloat16, (B, H, S, d), name, like.get_device())


def _token_major(t, dtype, shape, name, dev):
    """The fields of attn_heads for [B,S,H,d]."""
    b, s, h, _ = _rows(t, dtype, shape, name, dev)
    return t.data_ptr(), b, s, h


def _head_major(t, dtype, shape, name, dev):
    """The fields of attn_heads for [B,H,S,d]."""
    b, h, s, _ = _rows(t, dtype, shape, name, dev)
    return t.data_ptr(), b, s, h


_NO_HEADS = (0, 0, 0, 0)  # no tensor


def _rope_common(q, k, q_weight, k_weight, inv_freq, positions, interleaved):
    """Dimensions, checked small operands and flags of the two rotation calls."""
    import torch
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must be [B,S,H,d]")
    B, S, Hq, d = q.shape
    dev = q.get_device()
    if dev < 0:
        raise TypeError("q must be on a HIP device")
    w_f32 = getattr(q_weight, "dtype", None) is torch.float32
    wdtype = torch.float32 if w_f32 else torch.bfloat16
    _require_on(q_weight, wdtype, (d,), "q_weight", dev)
    _require_on(k_weight, wdtype, (d,), "k_weight", dev)
    if not isinstance(inv_freq, torch.Tensor) or inv_freq.dim() != 1:
        raise TypeError("inv_freq must be a one-dimensional tensor")
    half = inv_freq.shape[0]
    _require_on(inv_freq, torch.float32, (half,), "inv_freq", dev)
    flags = (ATTN_ROPE_INTERLEAVED if interleaved else 0) | (ATTN_WEIGHT_F32 if w_f32 else 0)
    pos_ptr = pos_stride = 0
    if positions is not None:
        if not isinstance(positions, torch.Tensor) or not positions.is_cuda or \
                positions.dtype not in (torch.int32, torch.int64):
            raise TypeError("positions must be an int32 or int64 tensor on a HIP device")
        if positions.shape not in ((S,), (B, S)):
            raise ValueError(f"positions has shape {tuple(positions.shape)}, expected "
                             f"{(S,)} or {(B, S)}")
        if positions.get_device() != dev:
            raise ValueError("positions is on another device than the first operand")
        if S > 1 and positions.stride(-1) != 1:
            raise ValueError("positions must be contiguous in its last dimension")
        if B > 1 and positions.dim() == 2:
            pos_stride = positions.stride(0)
        pos_ptr = positions.data_ptr()
        if positions.dtype is torch.int64:
            flags |= ATTN_POSITIONS_I64
    small = (q_weight.data_ptr(), k_weight.data_ptr(), inv_freq.data_ptr(), pos_ptr, pos_stride)
    return B, S, Hq, k.shape[2], d, 2 * half, dev, flags, small


def qk_norm_rope(q, k, v, q_weight, k_weight, inv_freq, positions=None, eps: float = 1e-6,
                 interleaved: bool = False, q_out=None, k_out=None, v_out=None):
    """RMS norm of every query and key head and rotation by position, from token-major
    projections to what attn_fwd and attn_decode read; returns (q, k, v), bf16 [B,H,S,d].

    q: bf16 [B,S,Hq,d], k, v: bf16 [B,S,Hkv,d], any strides with contiguous rows (views
    of one fused projection); v may be None (None is returned for it).  q_weight, k_weight:
    [d], bf16 or fp32.  inv_freq: fp32 [rot/2]; pair i is (i, i + rot/2), or interleaved
    (2i, 2i+1), and turns by position * inv_freq[i].  positions: int32 or int64 [S] or
    [B,S]; None: 0..S-1.  q_out, k_out, v_out: [B,H,S,d], any strides with contiguous rows
    (for a step of decoding, the cache's rows: k_out=cache[:, :, pos:pos + S]; in place:
    q_out=q.transpose(1, 2)), that share no memory with each other or, unless in place, with
    the projections."""
    import torch
    B, S, Hq, Hkv, d, rot, dev, flags, small = _rope_common(q, k, q_weight, k_weight, inv_freq,
                                                            positions, interleaved)
    bf16 = torch.bfloat16
    q_in = _token_major(q, bf16, (B, S, Hq, d), "q", dev)
    k_in = _token_major(k, bf16, (B, S, Hkv, d), "k", dev)
    q_out, q_to = _head_major_out(q_out, B, S, Hq, d, "q_out", q)
    k_out, k_to = _head_major_out(k_out, B, S, Hkv, d, "k_out", q)
    v_in = v_to = _NO_HEADS
    if v is not None:
        v_in = _token_major(v, bf16, (B, S, Hkv, d), "v", dev)
        v_out, v_to = _head_major_out(v_out, B, S, Hkv, d, "v_out", q)
    elif v_out is not None:
        raise ValueError("v_out without v")
    _call_on(dev, lib.attn__qk_norm_rope_packed, _ROPE_CALL.pack(
        *q_in, *k_in, *v_in, *q_to, *k_to, *v_to, *small, _raw_stream(dev), B, S, Hq, Hkv, d,
        rot, flags, eps))
    return q_out, k_out, v_out


def qk_norm_rope_bwd(dq, dk, dv, q, k, q_weight, k_weight, inv_freq, positions=None,
                     eps: float = 1e-6, interleaved: bool = False, dq_out=None, dk_out=None,
                     dv_out=None, weight_grads: bool = True, workspace=None):
    """Gradients of qk_norm_rope; returns those of q, k and v (bf16 [B,S,H,d]) and of
    q_weight and k_weight (fp32 [d]; None without weight_grads).

    dq, dk, dv: gradients of its results, bf16 or fp32 [B,H,S,d], any strides with
    contiguous rows (dv may be None); the rest as qk_norm_rope got it.  dq_out, dk_out,
    dv_out: any strides with contiguous rows, sharing no memory with each other or the
    inputs; without them, they are the heads of one fused [B,S,Hq+2*Hkv,d] tensor in this
    order.  workspace: None (the library's), or a device
    tensor of at least qk_norm_rope_bwd_workspace_bytes(...) bytes."""
    import torch
    B, S, Hq, Hkv, d, rot, dev, flags, small = _rope_common(q, k, q_weight, k_weight, inv_freq,
                                                            positions, interleaved)
    bf16, f32 = torch.bfloat16, torch.float32
    g_type = bf16
    if getattr(dq, "dtype", None) is f32:
        g_type = f32
        flags |= ATTN_GRAD_F32
    q_shape, k_shape = (B, S, Hq, d), (B, S, Hkv, d)
    dq_in = _head_major(dq, g_type, (B, Hq, S, d), "dq", dev)
    dk_in = _head_major(dk, g_type, (B, Hkv, S, d), "dk", dev)
    q_in = _token_major(q, bf16, q_shape, "q", dev)
    k_in = _token_major(k, bf16, k_shape, "k", dev)
    if dq_out is None or dk_out is None or (dv_out is None and dv is not None):
        parts = q.new_empty((B, S, Hq + 2 * Hkv, d)).split_with_sizes((Hq, Hkv, Hkv), 2)
        dq_out = parts[0] if dq_out is None else dq_out
        dk_out = parts[1] if dk_out is None else dk_out
        if dv is not None and dv_out is None:
            dv_out = parts[2]
    dq_to = _token_major(dq_out, bf16, q_shape, "dq_out", dev)
    dk_to = _token_major(dk_out, bf16, k_shape, "dk_out", dev)
    dv_in = dv_to = _NO_HEADS
    if dv is not None:
        dv_in = _head_major(dv, g_type, (B, Hkv, S, d), "dv", dev)
        dv_to = _token_major(dv_out, bf16, k_shape, "dv_out", dev)
    elif dv_out is not None:
        raise ValueError("dv_out without dv")
    dqw = dkw = None
    dqw_ptr = dkw_ptr = 0
    if weight_grads:
        dqw, dkw = torch.empty((2, d), dtype=f32, device=q.device).unbind()
        dqw_ptr, dkw_ptr = dqw.data_ptr(), dkw.data_ptr()
    _call_on(dev, lib.attn__qk_norm_rope_bwd_packed, _ROPE_BWD_CALL.pack(
        *dq_in, *dk_in, *dv_in, *q_in, *k_in, *dq_to, *dk_to, *dv_to, *small, dqw_ptr, dkw_ptr,
        *_workspace(workspace, dev), _raw_stream(dev), B, S, Hq, Hkv, d, rot, flags, eps))
    return dq_out, dk_out, dv_out, dqw, dkw


def qk_norm_rope_bwd_workspace_bytes(B: int, S: int, Hq: int, Hkv: int, d: int) -> int:
    """Bytes of workspace qk_norm_rope_bwd needs with a caller-provided buffer."""
    n = lib.attn_qk_norm_rope_bwd_workspace_bytes(B, S, Hq, Hkv, d)
    if n < 0:
        raise AttnError(int(n), last_error())
    return int(n)


# csrc/paged_api.hip's PackedExtend, PackedRelease, PackedStore and PackedPaged
_EXTEND_CALL = struct.Struct("Qq10Q5i")
_RELEASE_CALL = struct.Struct("Qq6Q4i")
_STORE_CALL = struct.Struct("16qQQ5i")
_PAGED_CALL = struct.Struct("12q3Qq6Q12i2f")


try:
    from torch import bfloat16 as _BF16, float32 as _F32, int32 as _I32
except ImportError:
    _BF16 = _F32 = _I32 = None


def _ints(t, shape, name, dev) -> int:
    """Address of an int32 tensor, checked."""
    if getattr(t, "dtype", None) is _I32 and t.get_device() == dev and t.shape == shape and \
            t.is_contiguous():
        return t.data_ptr()
    _require_on(t, _I32, shape, name, dev)
    return t.data_ptr()


def _new_ints(given, sizes, names, like, dev):
    """Int32 results of the given sizes: those given, checked, and the others from one new
    tensor."""
    if all(t is None for t in given):
        return like.new_empty(sum(sizes)).split_with_sizes(sizes)
    out = []
    for t, n, name in zip(given, sizes, names):
        if t is None:
            t = like.new_empty(n)
        else:
            _require_on(t, _I32, (n,), name, dev)
        out.append(t)
    return out


def _block_table(table, R):
    """Device, address, row stride and pages to a row of a block table of R rows."""
    if getattr(table, "dtype", None) is not _I32 or not table.is_cuda:
        raise TypeError("block_table must be an int32 tensor on a HIP device")
    if table.dim() != 2 or (R is not None and table.shape[0] != R):
        raise ValueError(f"block_table has shape {tuple(table.shape)}, expected "
                         f"({'R' if R is None else R}, max_pages)")
    stride, one = table.stride()
    if one != 1 and table.shape[1] > 1:
        raise ValueError("block_table must be contiguous in its last dimension")
    return table.get_device(), table.data_ptr(), stride, table.shape[1]


def _list(free_pages, dev):
    """Address and length of a list of free pages."""
    if getattr(free_pages, "dtype", None) is not _I32 or free_pages.dim() != 1:
        raise TypeError("free_pages must be a one-dimensional int32 tensor")
    return _ints(free_pages, free_pages.shape, "free_pages", dev), free_pages.shape[0]


def paged_extend(block_table, seq_lens, new_lens, free_pages, n_free, page_size: int,
                 n_tokens: int, slots=None, positions=None, cu_seqlens=None, kv_lens=None,
                 n_left=None):
    """Pages, slots and positions of a step's new tokens, on the GPU; returns (slots, positions,
    cu_seqlens, kv_lens, n_left).  All tensors are int32.

    block_table: [R,max_pages], holds the pages of each request's tokens and gets those of the
    new ones, in place.  seq_lens, new_lens: [R], each request's tokens in the cache and its new
    ones.  free_pages: the list of free pages, n_free: [1], how many of it are; they are taken
    from its end.  n_tokens: at least the sum of new_lens.  slots (page * page_size + row) and
    positions: [n_tokens], one request's tokens behind another's, -1 and 0 behind the last;
    cu_seqlens: [R+1]; kv_lens: [R], seq_lens + new_lens; n_left: [1], the next call's n_free, or
    negative: so many pages were missing (-1 in the table and in slots), and the call can be made
    again, with the n_free from before it, when some were released behind those.  A step that goes
    on instead takes n_left as it is (none are free).  The results may be given; they must not be
    the operands."""
    if seq_lens.dim() != 1:
        raise ValueError("seq_lens must be [R]")
    R = seq_lens.shape[0]
    dev, table_ptr, stride, max_pages = _block_table(block_table, R)
    seq_ptr, new_ptr = _ints(seq_lens, (R,), "seq_lens", dev), _ints(new_lens, (R,), "new_lens", dev)
    list_ptr, list_len = _list(free_pages, dev)
    free_ptr = _ints(n_free, (1,), "n_free", dev)
    slots, positions, cu_seqlens, kv_lens, n_left = _new_ints(
        (slots, positions, cu_seqlens, kv_lens, n_left), (n_tokens, n_tokens, R + 1, R, 1),
        ("slots", "positions", "cu_seqlens", "kv_lens", "n_left"), block_table, dev)
    _call_on(dev, lib.attn__paged_extend_packed, _EXTEND_CALL.pack(
        table_ptr, stride, seq_ptr, new_ptr, list_ptr, free_ptr, slots.data_ptr(),
        positions.data_ptr(), cu_seqlens.data_ptr(), kv_lens.data_ptr(), n_left.data_ptr(),
        _raw_stream(dev), list_len, R, max_pages, page_size, n_tokens))
    return slots, positions, cu_seqlens, kv_lens, n_left


def paged_release(block_table, seq_lens, keep_lens, free_pages, n_free, page_size: int,
                  n_left=None):
    """Pages given back: of each request those behind its first keep_lens tokens, into free_pages
    behind the n_free in it, in place; returns n_left, [1], how many are free then.  Pages that
    were missing (below zero in the table) are left out.  Tensors as for paged_extend (keep_lens:
    [R], 0 where a request ends); the table is not changed."""
    if seq_lens.dim() != 1:
        raise ValueError("seq_lens must be [R]")
    R = seq_lens.shape[0]
    dev, table_ptr, stride, max_pages = _block_table(block_table, R)
    seq_ptr, keep_ptr = _ints(seq_lens, (R,), "seq_lens", dev), _ints(keep_lens, (R,), "keep_lens",
                                                                      dev)
    list_ptr, list_len = _list(free_pages, dev)
    free_ptr = _ints(n_free, (1,), "n_free", dev)
    n_left, = _new_ints((n_left,), (1,), ("n_left",), block_table, dev)
    _call_on(dev, lib.attn__paged_release_packed, _RELEASE_CALL.pack(
        table_ptr, stride, seq_ptr, keep_ptr, list_ptr, free_ptr, n_left.data_ptr(),
        _raw_stream(dev), list_len, R, max_pages, page_size))
    return n_left


def _packed_rows(t, name, dev=None):
    """Shape, device and fields of attn_heads for [T,H,d], any strides with contiguous rows."""
    if getattr(t, "dtype", None) is not _BF16 or not t.is_cuda:
        raise TypeError(f"{name} must be a torch.bfloat16 tensor on a HIP device")
    if t.dim() != 3:
        raise ValueError(f"{name} must be [T,H,d]")
    row, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    return t.shape, t.get_device(), (t.data_ptr(), 0, row, head)


def _cache_pages(k_pages, v_pages, Hkv, d, dev):
    """Pages, page size and fields of attn_heads of both sides of a cache."""
    if len(getattr(k_pages, "shape", ())) != 4:
        raise ValueError("k_pages must be [P,Hkv,page_size,d]")
    n_pages, heads, page_size, _ = k_pages.shape
    if Hkv is None:
        Hkv = heads
    shape = (n_pages, Hkv, page_size, d)
    k = _head_major(k_pages, _BF16, shape, "k_pages", dev)
    return Hkv, n_pages, page_size, k, _head_major(v_pages, _BF16, shape, "v_pages", dev)


def paged_store(k, v, slots, k_pages, v_pages) -> None:
    """Keys and values of new tokens into the cache.  k, v: bf16 [T,Hkv,d]; slots: int32 [T] (as
    from paged_extend; negative: left out; none twice); k_pages, v_pages: bf16
    [P,Hkv,page_size,d].  Any strides with contiguous rows: heads of one projection, a cache whose
    pages are token by token ([P,page_size,Hkv,d].transpose(1, 2)); qk_norm_rope's k as
    k[0].transpose(0, 1)."""
    (T, Hkv, d), dev, k_in = _packed_rows(k, "k")
    v_shape, v_dev, v_in = _packed_rows(v, "v")
    if v_shape != (T, Hkv, d) or v_dev != dev:
        raise ValueError(f"v has shape {tuple(v_shape)}, expected {(T, Hkv, d)} on k's device")
    _, n_pages, page_size, k_to, v_to = _cache_pages(k_pages, v_pages, Hkv, d, dev)
    _call_on(dev, lib.attn__paged_store_packed, _STORE_CALL.pack(
        *k_in, *v_in, *k_to, *v_to, _ints(slots, (T,), "slots", dev), _raw_stream(dev), T, Hkv, d,
        n_pages, page_size))


def attn_paged(q, k_pages, v_pages, block_table, kv_lens, cu_seqlens=None, max_q: int | None = None,
               scale: float | None = None, causal: bool = True, window: int = 0,
               softcap: float = 0.0, slopes=None, o=None, out_dtype=None,
               return_lse: bool = False, workspace=None):
    """Attention of the new tokens of R requests over a paged cache that holds them already;
    returns o [T,Hq,d] (fp32, or out_dtype bf16), and with return_lse also the fp32 row
    log-sum-exp [T,Hq].

    q: bf16 [T,Hq,d], any strides with contiguous rows: each request's new tokens, one request
    behind another, from cu_seqlens[r] (int32 [R+1]; None: one token of each).  k_pages, v_pages:
    bf16 [P,Hkv,page_size,d], as for paged_store; Hkv divides Hq.  block_table: int32
    [R,max_pages]; kv_lens: int32 [R], each request's tokens, the new ones among them.  max_q: no
    request has more new tokens (None: not known; a small number spares kernels that only longer
    requests need).  causal: a token sees the keys up to its own; window: and only so many of
    them; softcap: scores become softcap * tanh(score / softcap); slopes: fp32 [Hq], scores fall
    by slopes[h] for every position of distance.  A token that sees no key has o = 0, lse = -inf;
    rows of q behind the last request's are left as they were.  workspace: None (the library's),
    or a device tensor of at least paged_workspace_bytes(...) bytes."""
    (T, Hq, d), dev, q_in = _packed_rows(q, "q")
    Hkv, n_pages, page_size, k_in, v_in = _cache_pages(k_pages, v_pages, None, d, dev)
    if kv_lens.dim() != 1:
        raise ValueError("kv_lens must be [R]")
    R = kv_lens.shape[0]
    table_dev, table_ptr, stride, max_pages = _block_table(block_table, R)
    if table_dev != dev:
        raise ValueError("block_table is on another device than the first operand")
    kv_ptr = _ints(kv_lens, (R,), "kv_lens", dev)
    cu_ptr = 0
    if cu_seqlens is not None:
        cu_ptr = _ints(cu_seqlens, (R + 1,), "cu_seqlens", dev)
    elif T != R:
        raise ValueError(f"{T} tokens of {R} requests without cu_seqlens")
    slopes_ptr = 0
    if slopes is not None:
        _require_on(slopes, _F32, (Hq,), "slopes", dev)
        slopes_ptr = slopes.data_ptr()
    if out_dtype is None:
        out_dtype = o.dtype if o is not None else _F32
    if out_dtype not in (_F32, _BF16):
        raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
    if o is None:
        o = q.new_empty((T, Hq, d), dtype=out_dtype)
    else:
        _require_on(o, out_dtype, (T, Hq, d), "o", dev)
    lse = q.new_empty((T, Hq), dtype=_F32) if return_lse else None
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if max_q is None:
        max_q = 0 if cu_seqlens is not None else 1
    elif max_q < 1:
        raise ValueError("max_q must be positive")
    _call_on(dev, lib.attn__paged_packed, _PAGED_CALL.pack(
        *q_in, *k_in, *v_in, o.data_ptr(), 0 if lse is None else lse.data_ptr(), table_ptr, stride,
        kv_ptr, cu_ptr, slopes_ptr, *_workspace(workspace, dev), _raw_stream(dev), T, R, max_q, Hq,
        Hkv, d, n_pages, page_size, max_pages, window, 1 if causal else 0,
        ATTN_OUT_BF16 if out_dtype is _BF16 else 0, scale, softcap))
    return (o, lse) if return_lse else o


def paged_workspace_bytes(T: int, R: int, Hq: int, Hkv: int, d: int, page_size: int,
                          max_pages: int, max_q: int | None = None, window: int = 0) -> int:
    """Bytes of workspace attn_paged needs with a caller-provided buffer, for a call of these
    sizes, max_q and window.  (Without max_q and with T = R, which a call without cu_seqlens takes
    for one token of each request and a call with it does not: of both the larger number.)"""
    most = [max_q or 0]
    if max_q is None and T == R:
        most.append(1)
    sizes = [int(lib.attn_paged_workspace_bytes(T, R, n, Hq, Hkv, d, page_size, max_pages, window))
             for n in most]
    if min(sizes) < 0:
        raise AttnError(min(sizes), last_error())
    return max(sizes)


def gemm_plan(M: int, N: int, K: int, b_nk: bool = False, desc: DeviceDesc | None = None) -> str:
    buf = ctypes.create_string_buffer(512)
    ptr = ctypes.byref(desc) if desc is not None else None
    rc = lib.attn_gemm_plan(ptr, M, N, K, ATTN_GEMM_B_NK if b_nk else 0, buf, 512)
    if rc < 0:
        raise AttnError(rc, last_error())
    return buf.value.decode()


def gemm_candidates(M: int, N: int, K: int, b_nk: bool = False, desc: DeviceDesc | None = None,
                    device_footprint: bool = False, analytic_only: bool = False,
                    deep: bool = False) -> list[dict]:
    """Every feasible GEMM candidate with its modelled time (not ABI; for the
    block-size ablation) of the generic and the hand-scheduled kernel, and with
    deep of the deep-pipeline kernel.  analytic_only: without the measured
    per-variant costs."""
    buf = ctypes.create_string_buffer(1 << 17)
    ptr = ctypes.byref(desc) if desc is not None else None
    flags = int(bool(device_footprint)) | (2 if analytic_only else 0) | (4 if deep else 0)
    rc = lib.attn__gemm_candidates(ptr, M, N, K, ATTN_GEMM_B_NK if b_nk else 0, flags, buf,
                                   1 << 17)
    if rc < 0:
        raise AttnError(rc, last_error())
    return [parse_plan(l) for l in buf.value.decode().splitlines() if l.strip()]


def query_device() -> dict:
    desc = DeviceDesc()
    lib.attn_query_device(ctypes.byref(desc))
    return desc.as_dict()


def measure_device() -> dict:
    """Run the device microbenchmarks (needs a gfx950 device)."""
    desc = DeviceDesc()
    _check(lib.attn_measure_device(ctypes.byref(desc)))
    return desc.as_dict()


def get_plan(kind: int, B: int, H: int, Sq: int, Skv: int, d: int, causal: bool = False,
             n_splits: int = 0, desc: DeviceDesc | None = None, Hkv: int | None = None) -> str:
    """The plan line of a call with H query heads and Hkv (default H) key/value
    heads."""
    buf = ctypes.create_string_buffer(512)
    ptr = ctypes.byref(desc) if desc is not None else None
    rc = lib.attn_get_plan_ex(ptr, kind, B, H, H if Hkv is None else Hkv, Sq, Skv, d,
                              int(bool(causal)), n_splits, buf, 512)
    if rc < 0:
        raise AttnError(rc, last_error())
    return buf.value.decode()


def fwd_candidates(B: int, H: int, Sq: int, Skv: int, d: int, causal: bool = False,
                   desc: DeviceDesc | None = None, device_footprint: bool = False,
                   analytic_only: bool = False, group: int = 0) -> list[dict]:
    """Every feasible prefill candidate with its modelled time (not ABI; for
    the block-size ablation).  desc None: this device's description and the
    compiled kernels' real register/occupancy footprint; with a desc, the
    footprint is estimated unless device_footprint is set.  analytic_only:
    without the measured per-variant tile costs.  group 0: the plain form only;
    else every form of a call with that many query heads to a key/value head."""
    buf = ctypes.create_string_buffer(1 << 20)
    ptr = ctypes.byref(desc) if desc is not None else None
    flags = int(bool(device_footprint)) | (2 if analytic_only else 0)
    rc = lib.attn__fwd_candidates(ptr, B, H, Sq, Skv, d, int(bool(causal)), group, flags, buf,
                                  1 << 20)
    if rc < 0:
        raise AttnError(rc, last_error())
    return [parse_plan(l) for l in buf.value.decode().splitlines() if l.strip()]


def parse_plan(line: str) -> dict:
    out = {}
    for tok in line.split():
        key, _, val = tok.partition("=")
        try:
            out[key] = int(val)
        except ValueError:
            try:
                out[key] = float(val)
            except ValueError:
                out[key] = val
    return out
