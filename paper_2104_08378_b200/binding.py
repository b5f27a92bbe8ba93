"""Binding of the sp24 C ABI (include/sp24.h): argument marshalling only, by ctypes and, for the short calls, natively.

Every function takes torch CUDA tensors (PyTorch is used for device memory and streams only),
passes their device pointers and the current stream to ``libsp24.so`` and raises
``Sp24Error`` on a non-zero status.  There is no CPU fallback: if the library is missing the
import fails, and every call needs a CUDA device.

16-bit matrices may be torch.float16 / torch.bfloat16 or raw torch.int16 / uint16 bit patterns
(then pass ``dtype=`` explicitly); int8 matrices are torch.int8.
"""
from __future__ import annotations

import ctypes
import functools
import os
from ctypes import byref
from typing import NamedTuple

import torch

from .build import LIB_PATH

OK = 0
F16, BF16, I8, F32, I32, E4M3, E5M2 = 0, 1, 2, 3, 4, 5, 6
META_CANONICAL, META_TCGEN05 = 0, 1
ROW_MAJOR, COL_MAJOR = 0, 1
DTYPE_CODE = {"f16": F16, "bf16": BF16, "i8": I8, "f32": F32, "i32": I32, "e4m3": E4M3, "e5m2": E5M2}
TORCH_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8, "f32": torch.float32,
               "i32": torch.int32, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_FROM_TORCH = {torch.float16: "f16", torch.bfloat16: "bf16", torch.int8: "i8", torch.float32: "f32",
               torch.int32: "i32", torch.float8_e4m3fn: "e4m3", torch.float8_e5m2: "e5m2"}

EXPORTS = [
    "sp24_status_string", "sp24_values_bytes", "sp24_meta_bytes", "sp24_prune", "sp24_compress",
    "sp24_decompress", "sp24_prune_compress", "sp24_gemm_workspace_bytes", "sp24_gemm", "sp24_gemm_status",
    "sp24_im2col_nhwc_3x3", "sp24_pipeline_host", "sp24_gemm_static_ws", "sp24_gemm_i8_dequant",
    "sp24_conv3x3_nhwc", "sp24_kept_magnitude", "sp24_apply_mask", "sp24_prune_2d",
    "sp24_gemm_static_ws_status", "sp24_set_tile_override", "sp24_test_set_fault_hooks", "sp24_gemm_f16acc",
    "sp24_gemm_plan", "sp24_rms_norm", "sp24_rms_norm_backward_workspace_bytes", "sp24_rms_norm_backward",
    "sp24_gated_act", "sp24_gated_act_backward", "sp24_act_backward_workspace_bytes", "sp24_act_backward",
    "sp24_linear", "sp24_route", "sp24_route_backward", "sp24_expert_rows", "sp24_expert_order_workspace_bytes", "sp24_expert_order", "sp24_expert_gather",
    "sp24_expert_combine", "sp24_expert_combine_backward", "sp24_expert_linear", "sp24_expert_linear_dx", "sp24_expert_linear_dw",
    "sp24_expert_act_backward_workspace_bytes", "sp24_expert_act_backward",
]


class Sp24Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: sp24 status {status} ({status_string(status)})")


class GemmDesc(ctypes.Structure):
    _fields_ = [("ab_type", ctypes.c_int), ("cd_type", ctypes.c_int),
                ("M", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("lda", ctypes.c_int64), ("ldb", ctypes.c_int64), ("ldc", ctypes.c_int64),
                ("ldd", ctypes.c_int64),
                ("order_b", ctypes.c_int), ("order_c", ctypes.c_int), ("order_d", ctypes.c_int),
                ("a_is_dense", ctypes.c_int)]


class LinearEpilogue(ctypes.Structure):
    _fields_ = [("row_scale", ctypes.c_void_p), ("col_scale", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("act", ctypes.c_int),
                ("residual", ctypes.c_void_p), ("pre", ctypes.c_void_p), ("ld_pre", ctypes.c_int64)]


class ExpertDesc(ctypes.Structure):
    _fields_ = [("ab_type", ctypes.c_int), ("cd_type", ctypes.c_int)] + [
        (name, ctypes.c_int64) for name in ("E", "M", "K", "rows", "lda", "ldx", "ldd", "ld_residual", "ld_pre")] + [("a_is_dense", ctypes.c_int)]


class ExpertEpilogue(ctypes.Structure):
    _fields_ = [("row_scale", ctypes.c_void_p), ("col_scale", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("act", ctypes.c_int),
                ("residual", ctypes.c_void_p), ("pre", ctypes.c_void_p)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2104_08378_b200.build` "
                          "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    i64, vp, ci, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.sp24_status_string.argtypes = [ci]
    lib.sp24_status_string.restype = ctypes.c_char_p
    lib.sp24_values_bytes.argtypes = [ci, i64, i64]
    lib.sp24_values_bytes.restype = sz
    lib.sp24_meta_bytes.argtypes = [ci, i64, i64, ci]
    lib.sp24_meta_bytes.restype = sz
    lib.sp24_prune.argtypes = [ci, i64, i64, vp, i64, vp, i64, vp]
    lib.sp24_compress.argtypes = [ci, i64, i64, vp, i64, vp, i64, vp, ci, vp, vp]
    lib.sp24_decompress.argtypes = [ci, i64, i64, vp, i64, vp, ci, vp, i64, vp]
    lib.sp24_prune_compress.argtypes = [ci, i64, i64, vp, i64, vp, i64, vp, i64, vp, ci, vp, vp]
    lib.sp24_gemm_workspace_bytes.argtypes = [ctypes.POINTER(GemmDesc)]
    lib.sp24_gemm_workspace_bytes.restype = sz
    lib.sp24_gemm.argtypes = [ctypes.POINTER(GemmDesc), vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sp24_gemm_plan.argtypes = [ctypes.POINTER(GemmDesc), ctypes.POINTER(ci), ctypes.POINTER(ci), ctypes.POINTER(ci)]
    lib.sp24_gemm_plan.restype = ci
    lib.sp24_gemm_f16acc.argtypes = lib.sp24_gemm.argtypes
    lib.sp24_gemm_f16acc.restype = ci
    lib.sp24_gemm_static_ws.argtypes = [ctypes.POINTER(GemmDesc), vp, vp, vp, vp, vp, vp, vp, vp]
    lib.sp24_gemm_static_ws.restype = ci
    lib.sp24_gemm_i8_dequant.argtypes = [ctypes.POINTER(GemmDesc), vp, vp, vp, vp, vp, ci, ctypes.c_float, vp, vp,
                                         sz, vp]
    lib.sp24_gemm_i8_dequant.restype = ci
    lib.sp24_conv3x3_nhwc.argtypes = [ctypes.POINTER(GemmDesc), i64, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sp24_conv3x3_nhwc.restype = ci
    lib.sp24_kept_magnitude.argtypes = [ci, i64, i64, vp, i64, vp, vp, vp]
    lib.sp24_apply_mask.argtypes = [ci, i64, i64, vp, i64, vp, ci, vp, i64, vp]
    lib.sp24_prune_2d.argtypes = [ci, i64, i64, vp, i64, vp, i64, vp]
    for name in ("sp24_kept_magnitude", "sp24_apply_mask", "sp24_prune_2d"):
        getattr(lib, name).restype = ci
    lib.sp24_gemm_status.argtypes = [vp, vp]
    lib.sp24_gemm_static_ws_status.argtypes = [vp]
    lib.sp24_gemm_static_ws_status.restype = ci
    lib.sp24_set_tile_override.argtypes = [ci, ci, ci, ci]
    lib.sp24_set_tile_override.restype = ci
    lib.sp24_test_set_fault_hooks.argtypes = [ctypes.c_longlong, ci]
    lib.sp24_test_set_fault_hooks.restype = ci
    lib.sp24_im2col_nhwc_3x3.argtypes = [ci, i64, i64, i64, i64, vp, vp, i64, vp]
    lib.sp24_pipeline_host.argtypes = [ctypes.POINTER(GemmDesc)] + [vp] * 13 + [sz, vp]
    lib.sp24_rms_norm.argtypes = [ci, i64, i64, vp, i64, vp, i64, vp, ci, ctypes.c_float, vp, i64, ci, vp, i64, vp, vp, vp]
    lib.sp24_rms_norm_backward_workspace_bytes.argtypes = [i64, i64]
    lib.sp24_rms_norm_backward_workspace_bytes.restype = sz
    lib.sp24_rms_norm_backward.argtypes = [ci, i64, i64, vp, i64, vp, i64, vp, ci, vp, vp, i64, vp, i64, vp, vp, sz, vp]
    lib.sp24_gated_act.argtypes = [ci, ci, i64, i64, vp, i64, vp, i64, ci, vp, i64, vp, vp]
    lib.sp24_gated_act_backward.argtypes = [ci, ci, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    lib.sp24_act_backward_workspace_bytes.argtypes = [i64, i64, ci]
    lib.sp24_act_backward_workspace_bytes.restype = sz
    lib.sp24_act_backward.argtypes = [ci, ci, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, ci, vp, sz, vp]
    lib.sp24_linear.argtypes = [ctypes.POINTER(GemmDesc), ctypes.POINTER(LinearEpilogue), vp, vp, vp, vp, vp, sz, vp]
    cf = ctypes.c_float
    lib.sp24_route.argtypes = [ci, i64, i64, vp, i64, ci, vp, ci, ci, ci, ci, ci, cf, vp, vp, vp]
    lib.sp24_route_backward.argtypes = [ci, i64, i64, vp, vp, i64, vp, ci, ci, ci, cf, vp, i64, vp]
    lib.sp24_expert_rows.argtypes = [i64, i64, i64]
    lib.sp24_expert_rows.restype = i64
    lib.sp24_expert_order_workspace_bytes.argtypes = [i64, i64]
    lib.sp24_expert_order_workspace_bytes.restype = sz
    lib.sp24_expert_order.argtypes = [i64, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    lib.sp24_expert_gather.argtypes = [ci, i64, i64, vp, i64, vp, ci, vp, i64, vp, vp, i64, vp, vp]
    lib.sp24_expert_combine.argtypes = [ci, i64, i64, i64, vp, i64, ci, vp, vp, vp, i64, vp, i64, vp]
    lib.sp24_expert_combine_backward.argtypes = [ci, i64, i64, i64, vp, i64, vp, i64, ci, vp, vp, vp, vp, i64, vp, vp]
    lib.sp24_expert_linear.argtypes = [ctypes.POINTER(ExpertDesc), ctypes.POINTER(ExpertEpilogue), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sp24_expert_linear_dx.argtypes = [ctypes.POINTER(ExpertDesc), vp, vp, vp, vp, vp, sz, vp]
    lib.sp24_expert_linear_dw.argtypes = [ctypes.POINTER(ExpertDesc), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sp24_expert_act_backward_workspace_bytes.argtypes = [i64, i64, i64]
    lib.sp24_expert_act_backward_workspace_bytes.restype = sz
    lib.sp24_expert_act_backward.argtypes = [ci, ci, i64, i64, i64, vp, i64, vp, i64, vp, vp, i64, vp, vp, sz, vp]
    for name in ("sp24_route", "sp24_route_backward", "sp24_expert_order", "sp24_expert_gather", "sp24_expert_combine", "sp24_expert_combine_backward",
                 "sp24_expert_linear", "sp24_expert_linear_dx", "sp24_expert_linear_dw", "sp24_expert_act_backward"):
        getattr(lib, name).restype = ci
    for name in ("sp24_linear", "sp24_rms_norm", "sp24_rms_norm_backward", "sp24_gated_act", "sp24_gated_act_backward", "sp24_act_backward"):
        getattr(lib, name).restype = ci
    for name in ("sp24_prune", "sp24_compress", "sp24_decompress", "sp24_gemm", "sp24_gemm_status",
                 "sp24_im2col_nhwc_3x3", "sp24_pipeline_host"):
        getattr(lib, name).restype = ci
    return lib


lib = _load()

if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    from . import _native      # compiled beside libsp24.so (csrc/sp24_native.cpp); missing: the import fails
else:                          # a CPU-only build of torch has no CUDA tensors: every call is for the functions below
    class _native:
        gemm = gemm_i8_dequant = conv3x3_nhwc = compress = apply_mask = staticmethod(lambda *args: None)
        rms_norm = rms_norm_backward = gated_act = gated_act_backward = act_backward = linear = linear_backward = staticmethod(
            lambda *args: None)
        route = route_backward = expert_order = expert_gather = expert_combine = expert_combine_backward = staticmethod(lambda *args: None)
        expert_linear = expert_linear_backward = staticmethod(lambda *args: None)

# Addresses for the native form of the short calls, which does what the functions below do if all arguments are of the
# ordinary kind, and returns None if not (then they do it themselves) or the status of a call that was refused.
_GEMM, _DEQUANT, _CONV, _COMPRESS, _META_BYTES, _APPLY_MASK = (
    ctypes.cast(getattr(lib, name), ctypes.c_void_p).value
    for name in ("sp24_gemm", "sp24_gemm_i8_dequant", "sp24_conv3x3_nhwc", "sp24_compress", "sp24_meta_bytes", "sp24_apply_mask"))
_RMS_NORM, _RMS_NORM_BACKWARD, _RMS_NORM_BYTES, _GATED, _GATED_BACKWARD, _ACT_BACKWARD, _ACT_BYTES, _LINEAR = (
    ctypes.cast(getattr(lib, name), ctypes.c_void_p).value
    for name in ("sp24_rms_norm", "sp24_rms_norm_backward", "sp24_rms_norm_backward_workspace_bytes", "sp24_gated_act",
                 "sp24_gated_act_backward", "sp24_act_backward", "sp24_act_backward_workspace_bytes", "sp24_linear"))
(_ROUTE, _ROUTE_BACKWARD, _ORDER, _ROWS, _ORDER_BYTES, _GATHER, _COMBINE, _COMBINE_BACKWARD, _EXPERT_LINEAR, _EXPERT_DX, _EXPERT_DW, _EXPERT_ACT,
 _EXPERT_ACT_BYTES) = (
    ctypes.cast(getattr(lib, name), ctypes.c_void_p).value
    for name in ("sp24_route", "sp24_route_backward", "sp24_expert_order", "sp24_expert_rows", "sp24_expert_order_workspace_bytes", "sp24_expert_gather",
                 "sp24_expert_combine", "sp24_expert_combine_backward", "sp24_expert_linear", "sp24_expert_linear_dx", "sp24_expert_linear_dw",
                 "sp24_expert_act_backward", "sp24_expert_act_backward_workspace_bytes"))


def status_string(status: int) -> str:
    return lib.sp24_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise Sp24Error(status, where)


# (None on a CPU-only build of torch; the call below then fails in current_device(), which says so)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    """The current device's current stream as a handle (no Stream object is made for it)."""
    return _raw_stream(torch.cuda.current_device())


def _dtype_of(t: torch.Tensor, dtype: str | None) -> str:
    if dtype is not None:
        return dtype
    return _FROM_TORCH[t.dtype]


def _ptr(t):
    return None if t is None else t.data_ptr()


def values_bytes(dtype: str, M: int, K: int) -> int:
    return lib.sp24_values_bytes(DTYPE_CODE[dtype], M, K)


@functools.lru_cache(maxsize=256)
def meta_bytes(dtype: str, M: int, K: int, layout: int = META_TCGEN05) -> int:
    return lib.sp24_meta_bytes(DTYPE_CODE[dtype], M, K, layout)


def prune(x: torch.Tensor, out: torch.Tensor | None = None, dtype: str | None = None) -> torch.Tensor:
    """sp24_prune on a 2-D row-major tensor (row stride = leading dimension)."""
    dt = _dtype_of(x, dtype)
    M, K = x.shape
    if out is None:
        out = torch.empty((M, K), dtype=x.dtype, device=x.device)
    assert x.stride(1) == 1 or K <= 1
    _check(lib.sp24_prune(DTYPE_CODE[dt], M, K, _ptr(x), x.stride(0) if M > 1 else K, _ptr(out),
                          out.stride(0) if M > 1 else K, _stream()), "sp24_prune")
    return out


def compress(x: torch.Tensor, layout: int = META_TCGEN05, dtype: str | None = None,
             count_dropped: bool = False):
    """sp24_compress: returns (vals [M, K/2], meta uint8 [meta_bytes], dropped tensor or None)."""
    if dtype is None and count_dropped is False:
        done = _native.compress(_COMPRESS, _META_BYTES, x, layout)
        if done is not None:
            return done if type(done) is not int else _check(done, "sp24_compress")
    dt = _dtype_of(x, dtype)
    M, K = x.shape
    vals = x.new_empty((M, K // 2))
    meta = x.new_empty(meta_bytes(dt, M, K, layout), dtype=torch.uint8)
    dropped = torch.zeros(1, dtype=torch.int64, device=x.device) if count_dropped else None
    _check(lib.sp24_compress(DTYPE_CODE[dt], M, K, _ptr(x), x.stride(0) if M > 1 else K, _ptr(vals),
                             K // 2, _ptr(meta), layout, _ptr(dropped), _stream()), "sp24_compress")
    return vals, meta, dropped


def compress_into(x, vals, meta, layout: int = META_TCGEN05, dtype: str | None = None, dropped=None):
    dt = _dtype_of(x, dtype)
    M, K = x.shape
    _check(lib.sp24_compress(DTYPE_CODE[dt], M, K, _ptr(x), x.stride(0) if M > 1 else K, _ptr(vals),
                             vals.stride(0) if M > 1 else K // 2, _ptr(meta), layout, _ptr(dropped),
                             _stream()), "sp24_compress")


def prune_compress(x: torch.Tensor, layout: int = META_TCGEN05, dtype: str | None = None, count_dropped: bool = False,
                   pruned: torch.Tensor | None = None, vals: torch.Tensor | None = None,
                   meta: torch.Tensor | None = None):
    """sp24_prune_compress: one pass; returns (pruned [M, K], vals [M, K/2], meta, dropped tensor or None)."""
    dt = _dtype_of(x, dtype)
    M, K = x.shape
    pruned = torch.empty_like(x) if pruned is None else pruned
    vals = x.new_empty((M, K // 2)) if vals is None else vals
    meta = x.new_empty(meta_bytes(dt, M, K, layout), dtype=torch.uint8) if meta is None else meta
    dropped = torch.zeros(1, dtype=torch.int64, device=x.device) if count_dropped else None
    _check(lib.sp24_prune_compress(DTYPE_CODE[dt], M, K, _ptr(x), x.stride(0) if M > 1 else K, _ptr(pruned),
                                   pruned.stride(0) if M > 1 else K, _ptr(vals), vals.stride(0) if M > 1 else K // 2,
                                   _ptr(meta), layout, _ptr(dropped), _stream()), "sp24_prune_compress")
    return pruned, vals, meta, dropped


def decompress(vals: torch.Tensor, meta: torch.Tensor, layout: int = META_TCGEN05,
               dtype: str | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    dt = _dtype_of(vals, dtype)
    M, K2 = vals.shape
    y = torch.empty((M, 2 * K2), dtype=vals.dtype, device=vals.device) if out is None else out
    _check(lib.sp24_decompress(DTYPE_CODE[dt], M, 2 * K2, _ptr(vals), vals.stride(0) if M > 1 else K2,
                               _ptr(meta), layout, _ptr(y), y.stride(0) if M > 1 else 2 * K2, _stream()),
           "sp24_decompress")
    return y


def make_desc(ab: str, cd: str, M: int, N: int, K: int, lda: int, ldb: int, ldc: int, ldd: int,
              a_is_dense: bool = False, b_row_major: bool = False, cd_col_major: bool = False) -> GemmDesc:
    cd_order = COL_MAJOR if cd_col_major else ROW_MAJOR
    return GemmDesc(DTYPE_CODE[ab], DTYPE_CODE[cd], M, N, K, lda, ldb, ldc, ldd,
                    ROW_MAJOR if b_row_major else COL_MAJOR, cd_order, cd_order, 1 if a_is_dense else 0)


@functools.lru_cache(maxsize=512)
def _desc_ref(*args):
    """A reference to make_desc(*args) for the calls below, which only read it: a problem is described once."""
    return byref(make_desc(*args))


def _scalar(ab: str, v):
    return ctypes.c_float(float(v)) if ab != "i8" else ctypes.c_int32(int(v))


# The scalars of most calls, made once (the library only reads them).
_FLOAT_ONE, _FLOAT_ZERO = byref(ctypes.c_float(1.0)), byref(ctypes.c_float(0.0))


def _scalar_refs(ab: str, alpha, beta):
    if ab == "i8":
        return byref(ctypes.c_int32(int(alpha))), byref(ctypes.c_int32(int(beta)))
    return (_FLOAT_ONE if type(alpha) is float and alpha == 1.0 else byref(ctypes.c_float(float(alpha))),
            _FLOAT_ZERO if type(beta) is float and beta == 0.0 else byref(ctypes.c_float(float(beta))))


_workspaces: dict = {}


def workspace(device, stream: int | None = None) -> torch.Tensor:
    if type(device) is not torch.device:
        device = torch.device(device)
    key = (device.index, _stream() if stream is None else stream)
    ws = _workspaces.get(key)
    if ws is None:
        ws = _workspaces.setdefault(key, torch.zeros(256, dtype=torch.uint8, device=device))
    return ws


def gemm(A: torch.Tensor, meta: torch.Tensor | None, Bt: torch.Tensor, *, alpha=1.0, beta=0.0,
         C: torch.Tensor | None = None, out: torch.Tensor | None = None, cd: str | None = None,
         ab: str | None = None, a_is_dense: bool = False, ws: torch.Tensor | None = None,
         b_row_major: bool = False, cd_col_major: bool = False, acc_f16: bool = False) -> torch.Tensor:
    """sp24_gemm (sp24_gemm_f16acc with acc_f16=True).  A: vals [M, K/2] (or dense [M, K]); Bt: [N, K]
    (K contiguous), or with b_row_major=True the K x N matrix itself, [K, N] (N contiguous); C/D: [M, N],
    or with cd_col_major=True their transposes [N, M] (M contiguous)."""
    if ab is None and acc_f16 is False:
        done = _native.gemm(_GEMM, _workspaces, A, meta, Bt, alpha, beta, C, out, cd, a_is_dense, ws, b_row_major, cd_col_major)
        if done is not None:
            return done if type(done) is not int else _check(done, "sp24_gemm")
    ab = _dtype_of(A, ab)
    a_shape, b_shape = A.shape, Bt.shape
    M = a_shape[0]
    K = a_shape[1] if a_is_dense else 2 * a_shape[1]
    N = b_shape[1 if b_row_major else 0]
    assert b_shape[0 if b_row_major else 1] == K
    cd = cd or ("i32" if ab == "i8" else ("bf16" if ab in ("e4m3", "e5m2") else ab))
    if out is None:
        out = A.new_empty((N, M) if cd_col_major else (M, N), dtype=TORCH_DTYPE[cd])
    stream = _stream()
    ws = ws if ws is not None else workspace(A.device, stream)
    desc = _desc_ref(ab, cd, M, N, K, A.stride(0), Bt.stride(0),
                     C.stride(0) if C is not None else (M if cd_col_major else N), out.stride(0), a_is_dense,
                     b_row_major, cd_col_major)
    a, b = _scalar_refs(ab, alpha, beta)
    fn = lib.sp24_gemm_f16acc if acc_f16 else lib.sp24_gemm
    _check(fn(desc, a, _ptr(A), _ptr(meta), _ptr(Bt), b, _ptr(C), _ptr(out), _ptr(ws), ws.numel(), stream),
           "sp24_gemm_f16acc" if acc_f16 else "sp24_gemm")
    return out


def gemm_plan(desc: GemmDesc) -> str:
    """sp24_gemm_plan: the tile shape the library picks for this problem, as "<ctas>x<block_n>x<mblk>"."""
    c, n, m = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(lib.sp24_gemm_plan(byref(desc), byref(c), byref(n), byref(m)), "sp24_gemm_plan")
    return f"{c.value}x{n.value}x{m.value}"


def gemm_status(ws: torch.Tensor | None = None, device=None) -> int:
    """sp24_gemm_status: 0, or SP24_ERR_TIMEOUT (9) if a wait expired in any launch on this workspace
    since the last read (the record is then cleared)."""
    ws = ws if ws is not None else workspace(device or "cuda")
    return lib.sp24_gemm_status(_ptr(ws), _stream())


def gemm_static_ws_status() -> int:
    """sp24_gemm_static_ws_status: the same for the library's own workspace array on the current device."""
    return lib.sp24_gemm_static_ws_status(_stream())


def set_tile_override(tile: str | None = None, band: int = 0):
    """sp24_set_tile_override: tile = "<ctas>x<block_n>x<mblk>" forces that tile shape, None restores
    the automatic choice (benchmarks and tests)."""
    c, n, m = (0, 0, 0) if not tile else (list(map(int, tile.split("x"))) + [1])[:3]
    _check(lib.sp24_set_tile_override(c, n, m, band), "sp24_set_tile_override")


def set_fault_hooks(wait_cycles: int = 0, skip_stage: bool | int = False):
    """sp24_test_set_fault_hooks (failure-path tests only)."""
    _check(lib.sp24_test_set_fault_hooks(int(wait_cycles), int(skip_stage)), "sp24_test_set_fault_hooks")


def im2col_nhwc_3x3(x: torch.Tensor, dtype: str | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    dt = _dtype_of(x, dtype)
    Nb, H, W, C = x.shape
    if out is None:
        out = torch.empty((Nb * H * W, 9 * C), dtype=x.dtype, device=x.device)
    _check(lib.sp24_im2col_nhwc_3x3(DTYPE_CODE[dt], Nb, H, W, C, _ptr(x), _ptr(out), out.stride(0), _stream()),
           "sp24_im2col_nhwc_3x3")
    return out


def gemm_static_ws(A: torch.Tensor, meta: torch.Tensor | None, Bt: torch.Tensor, *, alpha=1.0, beta=0.0,
                   C: torch.Tensor | None = None, out: torch.Tensor, cd: str | None = None,
                   ab: str | None = None, a_is_dense: bool = False) -> torch.Tensor:
    """sp24_gemm_static_ws: the GEMM for callers that cannot allocate device memory (the workspace is
    a fixed array inside the library).  `out` must be provided: nothing is allocated here either."""
    ab = _dtype_of(A, ab)
    M = A.shape[0]
    K = A.shape[1] if a_is_dense else 2 * A.shape[1]
    N = Bt.shape[0]
    cd = cd or ("i32" if ab == "i8" else ("bf16" if ab in ("e4m3", "e5m2") else ab))
    desc = _desc_ref(ab, cd, M, N, K, A.stride(0), Bt.stride(0), C.stride(0) if C is not None else N,
                     out.stride(0), a_is_dense)
    a, b = _scalar_refs(ab, alpha, beta)
    _check(lib.sp24_gemm_static_ws(desc, a, _ptr(A), _ptr(meta), _ptr(Bt), b, _ptr(C), _ptr(out), _stream()),
           "sp24_gemm_static_ws")
    return out


def gemm_i8_dequant(A: torch.Tensor, meta: torch.Tensor | None, Bt: torch.Tensor, row_scale: torch.Tensor, *,
                    bias: torch.Tensor | None = None, relu: bool = False, out_scale: float = 1.0, cd: str = "bf16",
                    out: torch.Tensor | None = None, a_is_dense: bool = False, ws: torch.Tensor | None = None,
                    b_row_major: bool = False, cd_col_major: bool = False) -> torch.Tensor:
    """sp24_gemm_i8_dequant: int8 sparse GEMM, D = act(row_scale[i] * acc + bias[i]) as cd (bf16/f16/f32/i8)."""
    done = _native.gemm_i8_dequant(_DEQUANT, _workspaces, A, meta, Bt, row_scale, bias, relu, out_scale, cd, out, a_is_dense,
                                   ws, b_row_major, cd_col_major)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_gemm_i8_dequant")
    a_shape = A.shape
    M = a_shape[0]
    K = a_shape[1] if a_is_dense else 2 * a_shape[1]
    N = Bt.shape[1 if b_row_major else 0]
    if out is None:
        out = A.new_empty((N, M) if cd_col_major else (M, N), dtype=TORCH_DTYPE[cd])
    stream = _stream()
    ws = ws if ws is not None else workspace(A.device, stream)
    desc = _desc_ref("i8", cd, M, N, K, A.stride(0), Bt.stride(0), M if cd_col_major else N, out.stride(0),
                     a_is_dense, b_row_major, cd_col_major)
    _check(lib.sp24_gemm_i8_dequant(desc, _ptr(A), _ptr(meta), _ptr(Bt), _ptr(row_scale), _ptr(bias),
                                    1 if relu else 0, out_scale, _ptr(out), _ptr(ws), ws.numel(), stream),
           "sp24_gemm_i8_dequant")
    return out


def conv3x3_nhwc(A: torch.Tensor, meta: torch.Tensor | None, x: torch.Tensor, *, alpha=1.0, beta=0.0,
                 C: torch.Tensor | None = None, out: torch.Tensor | None = None, cd: str | None = None,
                 ab: str | None = None, a_is_dense: bool = False, ws: torch.Tensor | None = None,
                 nhwc_out: bool = False) -> torch.Tensor:
    """sp24_conv3x3_nhwc: x [Nb, H, W, Cin] -> D [Kout, Nb*H*W] (or NHWC [Nb*H*W, Kout] with nhwc_out)."""
    if ab is None:
        done = _native.conv3x3_nhwc(_CONV, _workspaces, A, meta, x, alpha, beta, C, out, cd, a_is_dense, ws, nhwc_out)
        if done is not None:
            return done if type(done) is not int else _check(done, "sp24_conv3x3_nhwc")
    ab = _dtype_of(A, ab)
    Nb, H, W, Cin = x.shape
    M = A.shape[0]
    K, N = 9 * Cin, Nb * H * W
    cd = cd or ("i32" if ab == "i8" else ("bf16" if ab in ("e4m3", "e5m2") else ab))
    if out is None:
        out = A.new_empty((N, M) if nhwc_out else (M, N), dtype=TORCH_DTYPE[cd])
    stream = _stream()
    ws = ws if ws is not None else workspace(A.device, stream)
    desc = _desc_ref(ab, cd, M, N, K, A.stride(0), K, C.stride(0) if C is not None else (M if nhwc_out else N),
                     out.stride(0), a_is_dense, False, nhwc_out)
    a, b = _scalar_refs(ab, alpha, beta)
    _check(lib.sp24_conv3x3_nhwc(desc, Nb, H, W, Cin, a, _ptr(A), _ptr(meta), _ptr(x), b, _ptr(C), _ptr(out), _ptr(ws),
                                 ws.numel(), stream),
           "sp24_conv3x3_nhwc")
    return out


def kept_magnitude(x: torch.Tensor, perm: torch.Tensor | None = None, dtype: str | None = None) -> torch.Tensor:
    """sp24_kept_magnitude: total magnitude 2:4 pruning keeps under a column permutation (device double[1])."""
    dt = _dtype_of(x, dtype)
    M, K = x.shape
    res = torch.zeros(1, dtype=torch.float64, device=x.device)
    _check(lib.sp24_kept_magnitude(DTYPE_CODE[dt], M, K, _ptr(x), x.stride(0) if M > 1 else K, _ptr(perm), _ptr(res),
                                   _stream()), "sp24_kept_magnitude")
    return res


def apply_mask(w: torch.Tensor, meta: torch.Tensor, layout: int = META_TCGEN05, out: torch.Tensor | None = None,
               dtype: str | None = None) -> torch.Tensor:
    """sp24_apply_mask: zero every position of w the metadata does not name as kept."""
    if out is not None and dtype is None:
        done = _native.apply_mask(_APPLY_MASK, w, meta, layout, out)
        if done is not None:
            return done if type(done) is not int else _check(done, "sp24_apply_mask")
    dt = _dtype_of(w, dtype)
    M, K = w.shape
    if out is None:
        out = torch.empty_like(w)
    _check(lib.sp24_apply_mask(DTYPE_CODE[dt], M, K, _ptr(w), w.stride(0) if M > 1 else K, _ptr(meta), layout, _ptr(out),
                               out.stride(0) if M > 1 else K, _stream()), "sp24_apply_mask")
    return out


def prune_2d(x: torch.Tensor, out: torch.Tensor | None = None, dtype: str | None = None) -> torch.Tensor:
    """sp24_prune_2d: 2:4 along rows and columns of every 4 x 4 block (exhaustive search)."""
    dt = _dtype_of(x, dtype)
    M, K = x.shape
    if out is None:
        out = torch.empty_like(x)
    _check(lib.sp24_prune_2d(DTYPE_CODE[dt], M, K, _ptr(x), x.stride(0) if M > 1 else K, _ptr(out),
                             out.stride(0) if M > 1 else K, _stream()), "sp24_prune_2d")
    return out


# ---- the operators around the products -----------------------------------------------------------------------------------
# Their tensors may be on another device than the current one (all on the same): the call is then made with that one current,
# on its current stream.  What torch knows about the tensors is checked here, the rest by the library.  Their results carry no
# gradient for autograd (nor do those of the products above): the gradients are calls of their own.
ERR_DTYPE, ERR_SHAPE, ERR_STRIDE, ERR_UNSUPPORTED = 2, 3, 4, 6
_QUANT = ("i8", "e4m3", "e5m2")
ACT = {None: 0, "relu": 1, "gelu": 2, "silu": 3, "gelu_tanh": 4}


def _refuse(condition, status: int, where: str):
    if condition:
        raise Sp24Error(status, where)


def _matrix(t: torch.Tensor, where: str, like: torch.Tensor | None = None, shape=None, dtype=None) -> int:
    """The leading dimension of a CUDA matrix whose rows are contiguous; refused if it is not one, on another device than
    `like`, or not of the shape or type given."""
    _refuse(t.dim() != 2 or (shape is not None and tuple(t.shape) != tuple(shape)), ERR_SHAPE, where)
    _refuse(not t.is_cuda or (like is not None and t.device != like.device), ERR_UNSUPPORTED, where)
    _refuse(dtype is not None and t.dtype != dtype, ERR_DTYPE, where)
    _refuse(t.shape[1] > 1 and t.stride(1) != 1, ERR_STRIDE, where)
    return t.stride(0) if t.shape[0] > 1 else max(1, t.shape[1])


def _vector(t: torch.Tensor | None, n: int, where: str, like: torch.Tensor, dtypes=(torch.float32,)):
    """The same for a contiguous vector of n values, or None."""
    if t is None:
        return
    _refuse(t.dim() != 1 or t.shape[0] != n, ERR_SHAPE, where)
    _refuse(not t.is_cuda or t.device != like.device, ERR_UNSUPPORTED, where)
    _refuse(t.dtype not in dtypes, ERR_DTYPE, where)
    _refuse(n > 1 and t.stride(0) != 1, ERR_STRIDE, where)


def _on_device_of(name: str):
    """Makes the device of the first argument, `name`, current for the call where it is not."""
    def wrap(fn):
        @functools.wraps(fn)
        def call(*args, **kwargs):
            t = args[0] if args else kwargs[name]
            if not t.is_cuda or t.get_device() == torch.cuda.current_device():
                return fn(*args, **kwargs)
            with torch.cuda.device(t.device):
                return fn(*args, **kwargs)
        return call
    return wrap


def _float_code(t: torch.Tensor, where: str) -> int:
    code = _FROM_TORCH.get(t.dtype)
    _refuse(code not in ("f16", "bf16", "f32"), ERR_DTYPE, where)
    return DTYPE_CODE[code]


def _act_code(act: str | None, where: str) -> int:
    _refuse(act not in ACT, ERR_UNSUPPORTED, where)
    return ACT[act]


def rms_norm(x: torch.Tensor, weight: torch.Tensor | None = None, *, eps: float = 1e-6, residual: torch.Tensor | None = None,
             quant: str | None = None, with_rstd: bool = False, h_out: torch.Tensor | None = None,
             out: torch.Tensor | None = None):
    """sp24_rms_norm on the rows of x [rows, K]: returns (y, h, scale, rstd).  h = x + residual (None without residual), y its
    norm times weight [K] (x's type or float32; None: ones).  quant = "i8", "e4m3" or "e5m2": y in 8 bits and scale [rows],
    else scale is None.  rstd [rows] with with_rstd, else None.  h_out and out may be x or residual themselves."""
    done = _native.rms_norm(_RMS_NORM, x, weight, eps, residual, quant, with_rstd, h_out, out)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_rms_norm")
    return _rms_norm(x, weight, eps=eps, residual=residual, quant=quant, with_rstd=with_rstd, h_out=h_out, out=out)


@_on_device_of("x")
def _rms_norm(x, weight, *, eps, residual, quant, with_rstd, h_out, out):
    where = "sp24_rms_norm"
    t = _float_code(x, where)
    ldx = _matrix(x, where)
    rows, K = x.shape
    _refuse(quant is not None and quant not in _QUANT, ERR_DTYPE, where)
    _refuse(residual is None and h_out is not None, ERR_UNSUPPORTED, where)
    ldr = ldh = ldx
    h = None
    if residual is not None:
        ldr = _matrix(residual, where, x, x.shape, x.dtype)
        h = x.new_empty((rows, K)) if h_out is None else h_out
        ldh = _matrix(h, where, x, x.shape, x.dtype)
    _vector(weight, K, where, x, (x.dtype, torch.float32))
    out_dtype = x.dtype if quant is None else TORCH_DTYPE[quant]
    y = x.new_empty((rows, K), dtype=out_dtype) if out is None else out
    ldy = _matrix(y, where, x, x.shape, out_dtype)
    scale = x.new_empty(rows, dtype=torch.float32) if quant is not None else None
    rstd = x.new_empty(rows, dtype=torch.float32) if with_rstd else None
    _check(lib.sp24_rms_norm(t, rows, K, _ptr(x), ldx, _ptr(residual), ldr, _ptr(weight),
                             F32 if weight is None else DTYPE_CODE[_FROM_TORCH[weight.dtype]], eps, _ptr(h), ldh,
                             t if quant is None else DTYPE_CODE[quant], _ptr(y), ldy, _ptr(scale), _ptr(rstd), _stream()), where)
    return y, h, scale, rstd


def rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor | None, rstd: torch.Tensor, *,
                      dh: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """sp24_rms_norm_backward: (dx, dweight) from the gradient of y, the h that rms_norm normalised (x without residual), its
    weight and its rstd; dh is the gradient that arrives at h along the residual.  dweight is float32, None without weight.
    out may be dy, h or dh."""
    done = _native.rms_norm_backward(_RMS_NORM_BACKWARD, _RMS_NORM_BYTES, dy, h, weight, rstd, dh, out)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_rms_norm_backward")
    return _rms_norm_backward(dy, h, weight, rstd, dh=dh, out=out)


@_on_device_of("dy")
def _rms_norm_backward(dy, h, weight, rstd, *, dh, out):
    where = "sp24_rms_norm_backward"
    t = _float_code(dy, where)
    lddy = _matrix(dy, where)
    rows, K = dy.shape
    ldh = _matrix(h, where, dy, dy.shape, dy.dtype)
    lddh = lddy if dh is None else _matrix(dh, where, dy, dy.shape, dy.dtype)
    _vector(weight, K, where, dy, (dy.dtype, torch.float32))
    _refuse(rstd is None, 1, where)
    _vector(rstd, rows, where, dy)
    dx = dy.new_empty((rows, K)) if out is None else out
    lddx = _matrix(dx, where, dy, dy.shape, dy.dtype)
    dweight = ws = None
    ws_bytes = 0
    if weight is not None:
        dweight = dy.new_empty(K, dtype=torch.float32)
        ws_bytes = lib.sp24_rms_norm_backward_workspace_bytes(rows, K)
        ws = dy.new_empty(ws_bytes, dtype=torch.uint8)
    _check(lib.sp24_rms_norm_backward(t, rows, K, _ptr(dy), lddy, _ptr(h), ldh, _ptr(weight),
                                      F32 if weight is None else DTYPE_CODE[_FROM_TORCH[weight.dtype]], _ptr(rstd), _ptr(dh),
                                      lddh, _ptr(dx), lddx, _ptr(dweight), _ptr(ws), ws_bytes, _stream()), where)
    return dx, dweight


def gated_act(g: torch.Tensor, u: torch.Tensor | None = None, *, act: str | None = "silu", quant: str | None = None,
              out: torch.Tensor | None = None):
    """sp24_gated_act: (y, scale) with y = act(g) * u on rows [rows, F] (act(g) without u; act: "relu", "gelu", "silu",
    "gelu_tanh" or None).  quant = "i8", "e4m3" or "e5m2": y in 8 bits and scale [rows], else scale is None.  g and u may be
    slices of one matrix; out may be g or u."""
    done = _native.gated_act(_GATED, g, u, act, quant, out)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_gated_act")
    return _gated_act(g, u, act=act, quant=quant, out=out)


@_on_device_of("g")
def _gated_act(g, u, *, act, quant, out):
    where = "sp24_gated_act"
    t, code = _float_code(g, where), _act_code(act, where)
    ldg = _matrix(g, where)
    rows, F = g.shape
    ldu = ldg if u is None else _matrix(u, where, g, g.shape, g.dtype)
    _refuse(quant is not None and quant not in _QUANT, ERR_DTYPE, where)
    out_dtype = g.dtype if quant is None else TORCH_DTYPE[quant]
    y = g.new_empty((rows, F), dtype=out_dtype) if out is None else out
    ldy = _matrix(y, where, g, g.shape, out_dtype)
    scale = g.new_empty(rows, dtype=torch.float32) if quant is not None else None
    _check(lib.sp24_gated_act(t, code, rows, F, _ptr(g), ldg, _ptr(u), ldu, t if quant is None else DTYPE_CODE[quant], _ptr(y),
                              ldy, _ptr(scale), _stream()), where)
    return y, scale


def gated_act_backward(dy: torch.Tensor, g: torch.Tensor, u: torch.Tensor | None = None, *, act: str | None = "silu",
                       dg: torch.Tensor | None = None, du: torch.Tensor | None = None):
    """sp24_gated_act_backward: (dg, du) from the gradient of y = act(g) * u; du is None without u.  dg and du may be given,
    as slices of one matrix for instance."""
    done = _native.gated_act_backward(_GATED_BACKWARD, dy, g, u, act, dg, du)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_gated_act_backward")
    return _gated_act_backward(dy, g, u, act=act, dg=dg, du=du)


@_on_device_of("dy")
def _gated_act_backward(dy, g, u, *, act, dg, du):
    where = "sp24_gated_act_backward"
    t, code = _float_code(dy, where), _act_code(act, where)
    lddy = _matrix(dy, where)
    rows, F = dy.shape
    ldg = _matrix(g, where, dy, dy.shape, dy.dtype)
    dg = dy.new_empty((rows, F)) if dg is None else dg
    lddg = _matrix(dg, where, dy, dy.shape, dy.dtype)
    ldu = lddu = lddy
    if u is not None:
        ldu = _matrix(u, where, dy, dy.shape, dy.dtype)
        du = dy.new_empty((rows, F)) if du is None else du
        lddu = _matrix(du, where, dy, dy.shape, dy.dtype)
    _check(lib.sp24_gated_act_backward(t, code, rows, F, _ptr(dy), lddy, _ptr(g), ldg, _ptr(u), ldu, _ptr(dg), lddg, _ptr(du),
                                       lddu, _stream()), where)
    return dg, du


def act_backward(dy: torch.Tensor, pre: torch.Tensor | None, *, act: str | None, cd_col_major: bool = False,
                 transposed: bool = True, bias: bool = True, out: torch.Tensor | None = None):
    """sp24_act_backward: (dz, dz transposed or None, dbias or None) from the gradient of act(pre).  cd_col_major as in the
    product that made pre: True: dy and pre are [N, M], else [M, N]; dbias [M] sums over the N tokens.  Without an activation
    dz is dy itself (with `out`: a copy of it there) and pre is not read.  out may be dy or pre."""
    done = _native.act_backward(_ACT_BACKWARD, _ACT_BYTES, dy, pre, act, cd_col_major, transposed, bias, out)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_act_backward")
    return _act_backward(dy, pre, act=act, cd_col_major=cd_col_major, transposed=transposed, bias=bias, out=out)


@_on_device_of("dy")
def _act_backward(dy, pre, *, act, cd_col_major, transposed, bias, out):
    where = "sp24_act_backward"
    t, code = _float_code(dy, where), _act_code(act, where)
    lddy = ldz = _matrix(dy, where)
    rows, cols = dy.shape
    dz = out
    if code:
        _refuse(pre is None, 1, where)
        ldz = _matrix(pre, where, dy, dy.shape, dy.dtype)
        dz = dy.new_empty((rows, cols)) if out is None else out
    lddz = lddy if dz is None else _matrix(dz, where, dy, dy.shape, dy.dtype)
    dzt = dy.new_empty((cols, rows)) if transposed else None
    dbias = ws = None
    ws_bytes = 0
    if bias:
        dbias = dy.new_empty(cols if cd_col_major else rows, dtype=torch.float32)
        ws_bytes = lib.sp24_act_backward_workspace_bytes(rows, cols, 1 if cd_col_major else 0)
        ws = dy.new_empty(ws_bytes, dtype=torch.uint8)
    _check(lib.sp24_act_backward(t, code, rows, cols, _ptr(dy), lddy, _ptr(pre) if code else None, ldz, _ptr(dz), lddz, _ptr(dzt),
                                 max(1, rows), _ptr(dbias), 1 if cd_col_major else 0, _ptr(ws), ws_bytes, _stream()), where)
    return dy if dz is None else dz, dzt, dbias


def linear(A: torch.Tensor, meta: torch.Tensor | None, Bt: torch.Tensor, *, bias: torch.Tensor | None = None,
           act: str | None = None, residual: torch.Tensor | None = None, row_scale: torch.Tensor | None = None,
           col_scale: torch.Tensor | None = None, pre: bool | torch.Tensor = False, out: torch.Tensor | None = None,
           cd: str | None = None, a_is_dense: bool = False, b_row_major: bool = False, cd_col_major: bool = False,
           ws: torch.Tensor | None = None):
    """sp24_linear: D = act(row_scale[i] * col_scale[j] * (A B)[i, j] + bias[i]) + residual[i, j].  A, meta, Bt, cd,
    a_is_dense, b_row_major, cd_col_major as for gemm (cd defaults to A's type, bf16 for 8-bit operands); bias and row_scale
    [M], col_scale [N] float32 (col_scale: 8-bit operands); residual in D's type and shape, and may be `out`.  Returns D, or
    with pre=True (or a tensor for it) (D, what act was applied to).  M, N and K are multiples of 16, with 8-bit operands of
    32, as for gemm: other numbers of tokens are padded by the caller."""
    done = _native.linear(_LINEAR, _workspaces, _META_BYTES, A, meta, Bt, bias, act, residual, row_scale, col_scale, pre,
                          out, cd, a_is_dense, b_row_major, cd_col_major, ws)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_linear")
    return _linear(A, meta, Bt, bias=bias, act=act, residual=residual, row_scale=row_scale, col_scale=col_scale, pre=pre,
                   out=out, cd=cd, a_is_dense=a_is_dense, b_row_major=b_row_major, cd_col_major=cd_col_major, ws=ws)


@_on_device_of("A")
def _linear(A, meta, Bt, *, bias, act, residual, row_scale, col_scale, pre, out, cd, a_is_dense, b_row_major,
            cd_col_major, ws):
    where = "sp24_linear"
    ab = _FROM_TORCH.get(A.dtype)
    _refuse(ab is None or ab == "i32", ERR_DTYPE, where)
    lda, ldb = _matrix(A, where), _matrix(Bt, where, A, None, A.dtype)
    M, K = A.shape[0], A.shape[1] * (1 if a_is_dense else 2)
    N = Bt.shape[1 if b_row_major else 0]
    _refuse(Bt.shape[0 if b_row_major else 1] != K, ERR_SHAPE, where)
    if not a_is_dense:
        _refuse(meta is None, 1, where)
        _vector(meta, meta_bytes(ab, M, K), where, A, (torch.uint8,))
    cd = cd or ("bf16" if ab in _QUANT else ab)
    _refuse(cd not in TORCH_DTYPE, ERR_DTYPE, where)
    shape, dtype = ((N, M) if cd_col_major else (M, N)), TORCH_DTYPE[cd]
    if out is None:
        out = A.new_empty(shape, dtype=dtype)
    ldd = ldc = _matrix(out, where, A, shape, dtype)
    if residual is not None:
        ldc = _matrix(residual, where, A, shape, dtype)
    for v, n in ((bias, M), (row_scale, M), (col_scale, N)):
        _vector(v, n, where, A)
    z, ld_pre = None, 0
    if pre is not False and pre is not None:
        z = torch.empty_like(out) if pre is True else pre
        ld_pre = _matrix(z, where, A, shape, dtype)
    stream = _stream()
    ws = ws if ws is not None else workspace(A.device, stream)
    order = COL_MAJOR if cd_col_major else ROW_MAJOR
    desc = GemmDesc(DTYPE_CODE[ab], DTYPE_CODE[cd], M, N, K, lda, ldb, ldc, ldd, ROW_MAJOR if b_row_major else COL_MAJOR, order,
                    order, 1 if a_is_dense else 0)
    epilogue = LinearEpilogue(_ptr(row_scale), _ptr(col_scale), _ptr(bias), _act_code(act, where), _ptr(residual), _ptr(z), ld_pre)
    _check(lib.sp24_linear(byref(desc), byref(epilogue), _ptr(A), _ptr(meta), _ptr(Bt), _ptr(out), _ptr(ws), ws.numel(), stream),
           where)
    return out if z is None else (out, z)


def linear_backward(dy: torch.Tensor, pre: torch.Tensor | None, Bt: torch.Tensor, W: torch.Tensor, *, act: str | None = None,
                    meta: torch.Tensor | None = None, b_row_major: bool = False, cd_col_major: bool = False,
                    ws: torch.Tensor | None = None):
    """Gradients of linear (16-bit operands, or float32 in the TF32 mode without meta) from dy, its `pre` (None without an activation) and Bt, and the pruned
    weights W [M, K] themselves: (dBt, dW, dbias).  dy and pre are [N, M] with cd_col_major, else [M, N]; Bt [N, K], or [K, N]
    with b_row_major; dBt has Bt's form.  dy and pre may have any leading dimension and alignment, Bt and W those of gemm's operands.  With meta the entries of dW that the 2:4 pattern leaves out are zeros.  The
    residual's gradient is dy.  sp24_act_backward, then two dense products (and sp24_apply_mask).  dz = dy act'(pre) is an operand of
    both products, so it is rounded to dy's type before them (float32: the tensor cores read it as TF32); dbias is not."""
    done = _native.linear_backward(_ACT_BACKWARD, _ACT_BYTES, _GEMM, _META_BYTES, _APPLY_MASK, _workspaces, dy, pre, Bt, W, act,
                                   meta, b_row_major, cd_col_major, ws)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_linear_backward")
    return _linear_backward(dy, pre, Bt, W, act=act, meta=meta, b_row_major=b_row_major, cd_col_major=cd_col_major, ws=ws)


@_on_device_of("dy")
def _linear_backward(dy, pre, Bt, W, *, act, meta, b_row_major, cd_col_major, ws):
    where = "sp24_linear_backward"
    _float_code(dy, where)
    _matrix(dy, where)
    _matrix(W, where, dy, None, dy.dtype)
    _matrix(Bt, where, dy, None, dy.dtype)
    M, K = W.shape
    N = Bt.shape[1 if b_row_major else 0]
    _refuse(tuple(Bt.shape) != ((K, N) if b_row_major else (N, K)) or tuple(dy.shape) != ((N, M) if cd_col_major else (M, N)),
            ERR_SHAPE, where)
    _refuse(M % 16 or N % 16 or K % 16, ERR_SHAPE, where)
    _refuse(meta is not None and dy.dtype == torch.float32, ERR_DTYPE, where)   # (apply_mask knows the 2:4 pattern only)
    if meta is not None:
        _vector(meta, meta_bytes(_FROM_TORCH[W.dtype], M, K), where, dy, (torch.uint8,))
    if N == 0:
        return Bt.new_empty(Bt.shape), torch.zeros_like(W), dy.new_zeros(M, dtype=torch.float32)
    # (without an activation dz is dy itself, where a product can take it)
    out = dy.new_empty(dy.shape) if act is None and (dy.data_ptr() % 16 or dy.stride(0) * dy.element_size() % 16) else None
    dz, dzt, dbias = act_backward(dy, pre, act=act, cd_col_major=cd_col_major, out=out)
    tokens, features = (dz, dzt) if cd_col_major else (dzt, dz)          # [N, M], [M, N]
    dBt = gemm(tokens, None, W, a_is_dense=True, b_row_major=True, cd_col_major=b_row_major, ws=ws)
    dW = gemm(features, None, Bt, a_is_dense=True, b_row_major=not b_row_major, ws=ws)
    if meta is not None:
        apply_mask(dW, meta, out=dW)
    return dBt, dW, dbias


# ---- experts -------------------------------------------------------------------------------------------------------------------
SCORE = {"softmax": 0, "sigmoid": 1}
GROUP_SCORE = {"max": 0, "top2": 1}


class ExpertOrder(NamedTuple):
    """Where the slots (token, number) of a routing lie in the experts' order: the first row of each expert and the end [E + 1], the row of
    each slot [T, k] and the slot, T * k of them, of each row [rows]; -1 where there is none.  All int32."""
    offsets: torch.Tensor
    position: torch.Tensor
    source: torch.Tensor


def route(logits: torch.Tensor, k: int, *, score: str = "softmax", bias: torch.Tensor | None = None, groups: int = 1, top_groups: int | None = None,
          group_score: str = "max", renorm: bool = True, scale: float = 1.0):
    """sp24_route: (weights [T, k] float32, experts [T, k] int32) from the logits [T, E] (f16, bf16 or f32), the best expert first.  score: "softmax" or
    "sigmoid"; bias [E] float32 is added to the scores for the choice only; groups of E / groups experts, of which the top_groups (default: all) best by
    group_score ("max", or "top2": the sum of the two largest) stay; renorm: the weights of a token add up to scale.  Logits of -inf are never chosen;
    a slot that is left over has expert -1 and weight 0."""
    done = _native.route(_ROUTE, logits, k, score, bias, groups, top_groups, group_score, renorm, scale)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_route")
    return _route(logits, k, score, bias, groups, groups if top_groups is None else top_groups, group_score, renorm, scale)


@_on_device_of("logits")
def _route(logits, k, score, bias, groups, top_groups, group_score, renorm, scale):
    where = "sp24_route"
    t = _float_code(logits, where)
    ld = _matrix(logits, where)
    T, E = logits.shape
    _refuse(score not in SCORE or group_score not in GROUP_SCORE, ERR_UNSUPPORTED, where)
    _vector(bias, E, where, logits)
    _refuse(not 1 <= k <= max(1, E) or not 1 <= groups <= max(1, E) or not 1 <= top_groups <= groups, ERR_SHAPE, where)
    weights = logits.new_empty((T, k), dtype=torch.float32)
    experts = logits.new_empty((T, k), dtype=torch.int32)
    _check(lib.sp24_route(t, T, E, _ptr(logits), ld, SCORE[score], _ptr(bias), groups, top_groups, GROUP_SCORE[group_score], k, 1 if renorm else 0, scale,
                          _ptr(weights), _ptr(experts), _stream()), where)
    return weights, experts


def _slots(t: torch.Tensor, where: str, like: torch.Tensor, dtype, shape=None):
    """A contiguous [T, k] of the type, on the device of `like`."""
    _refuse(t.dim() != 2 or (shape is not None and tuple(t.shape) != tuple(shape)), ERR_SHAPE, where)
    _refuse(not t.is_cuda or t.device != like.device, ERR_UNSUPPORTED, where)
    _refuse(t.dtype != dtype, ERR_DTYPE, where)
    _refuse(not t.is_contiguous(), ERR_STRIDE, where)


def route_backward(dweights: torch.Tensor, logits: torch.Tensor, experts: torch.Tensor, *, score: str = "softmax", renorm: bool = True, scale: float = 1.0,
                   out: torch.Tensor | None = None) -> torch.Tensor:
    """sp24_route_backward: the gradient of the logits [T, E] from that of route's weights [T, k], for the experts that it chose; score, renorm and scale as
    there.  out may be the logits."""
    done = _native.route_backward(_ROUTE_BACKWARD, dweights, logits, experts, score, renorm, scale, out)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_route_backward")
    return _route_backward(dweights, logits, experts, score, renorm, scale, out)


@_on_device_of("dweights")
def _route_backward(dweights, logits, experts, score, renorm, scale, out):
    where = "sp24_route_backward"
    t = _float_code(logits, where)
    ld = _matrix(logits, where)
    T, E = logits.shape
    _refuse(score not in SCORE, ERR_UNSUPPORTED, where)
    _slots(experts, where, logits, torch.int32)
    _refuse(experts.shape[0] != T, ERR_SHAPE, where)
    _slots(dweights, where, logits, torch.float32, experts.shape)
    dlogits = logits.new_empty((T, E)) if out is None else out
    ldd = _matrix(dlogits, where, logits, logits.shape, logits.dtype)
    _check(lib.sp24_route_backward(t, T, E, _ptr(dweights), _ptr(logits), ld, _ptr(experts), experts.shape[1], SCORE[score], 1 if renorm else 0, scale,
                                   _ptr(dlogits), ldd, _stream()), where)
    return dlogits


def expert_order(experts: torch.Tensor, E: int, *, align: int = 1) -> ExpertOrder:
    """sp24_expert_order: where each slot of experts [T, k] (int32; negative or not below E: none) lies when the rows of an expert lie together, in their own
    order.  Every expert's rows begin at a multiple of align: 1 for inference, 16 where expert_linear_backward is to follow."""
    done = _native.expert_order(_ORDER, _ROWS, _ORDER_BYTES, experts, E, align)
    if done is not None:
        return ExpertOrder(*done) if type(done) is not int else _check(done, "sp24_expert_order")
    return _expert_order(experts, E, align)


@_on_device_of("experts")
def _expert_order(experts, E, align):
    where = "sp24_expert_order"
    _slots(experts, where, experts, torch.int32)
    n = experts.numel()
    _refuse(not 1 <= E <= 1024 or not 1 <= align <= 256 or n >= 2 ** 31, ERR_SHAPE, where)
    order = ExpertOrder(experts.new_empty(E + 1), torch.empty_like(experts), experts.new_empty(lib.sp24_expert_rows(n, E, align)))
    size = lib.sp24_expert_order_workspace_bytes(n, E)
    scratch = experts.new_empty(size, dtype=torch.uint8) if size else None
    _check(lib.sp24_expert_order(n, E, align, _ptr(experts), _ptr(order.offsets), _ptr(order.position), _ptr(order.source), _ptr(scratch), size, _stream()), where)
    return order


def _check_order(order: ExpertOrder, T: int, where: str, like: torch.Tensor):
    _slots(order.position, where, like, torch.int32)
    _refuse(order.position.shape[0] != T or order.source.dim() != 1, ERR_SHAPE, where)
    _vector(order.source, order.source.shape[0], where, like, (torch.int32,))


def expert_gather(x: torch.Tensor, order: ExpertOrder, *, scale: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """sp24_expert_gather: (rows of x [T, K] in the order of the experts [rows, K], their scales [rows] or None without scale [T]); rows that no slot has are
    zeros.  x of any type with 1, 2 or 4 bytes, as rms_norm gives it with its scale."""
    done = _native.expert_gather(_GATHER, x, order.position, order.source, scale, out)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_expert_gather")
    return _expert_gather(x, order, scale, out)


@_on_device_of("x")
def _expert_gather(x, order, scale, out):
    where = "sp24_expert_gather"
    code = _FROM_TORCH.get(x.dtype)
    _refuse(code is None, ERR_DTYPE, where)
    ldx = _matrix(x, where)
    T, K = x.shape
    _check_order(order, T, where, x)
    rows = order.source.shape[0]
    _vector(scale, T, where, x)
    y = x.new_empty((rows, K)) if out is None else out
    ldy = _matrix(y, where, x, (rows, K), x.dtype)
    scales = None if scale is None else x.new_empty(rows, dtype=torch.float32)
    _check(lib.sp24_expert_gather(DTYPE_CODE[code], T, K, _ptr(x), ldx, _ptr(scale), order.position.shape[1], _ptr(order.position), rows, _ptr(order.source),
                                  _ptr(y), ldy, _ptr(scales), _stream()), where)
    return y, scales


def expert_combine(y: torch.Tensor, order: ExpertOrder, weights: torch.Tensor | None = None, *, residual: torch.Tensor | None = None,
                   out: torch.Tensor | None = None) -> torch.Tensor:
    """sp24_expert_combine: the sums [T, K] of each token's rows of y [rows, K] with route's weights [T, k] (None: ones, the gradient of expert_gather),
    plus the residual [T, K].  out may be the residual."""
    done = _native.expert_combine(_COMBINE, y, order.position, order.source, weights, residual, out)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_expert_combine")
    return _expert_combine(y, order, weights, residual, out)


@_on_device_of("y")
def _expert_combine(y, order, weights, residual, out):
    where = "sp24_expert_combine"
    t = _float_code(y, where)
    ldy = _matrix(y, where)
    rows, K = y.shape
    _slots(order.position, where, y, torch.int32)
    T, k = order.position.shape
    _check_order(order, T, where, y)
    _refuse(order.source.shape[0] != rows, ERR_SHAPE, where)
    if weights is not None:
        _slots(weights, where, y, torch.float32, (T, k))
    o = y.new_empty((T, K)) if out is None else out
    ldo = ldr = _matrix(o, where, y, (T, K), y.dtype)
    if residual is not None:
        ldr = _matrix(residual, where, y, (T, K), y.dtype)
    _check(lib.sp24_expert_combine(t, T, K, rows, _ptr(y), ldy, k, _ptr(order.position), _ptr(weights), _ptr(residual), ldr, _ptr(o), ldo, _stream()), where)
    return o


def expert_combine_backward(dout: torch.Tensor, y: torch.Tensor, order: ExpertOrder, weights: torch.Tensor, *, out: torch.Tensor | None = None):
    """sp24_expert_combine_backward: (dy [rows, K], dweights [T, k]) of expert_combine from the gradient of its result; the residual's is dout itself.  Rows of dy
    that no slot has are zeros.  out may be y."""
    done = _native.expert_combine_backward(_COMBINE_BACKWARD, dout, y, order.position, order.source, weights, out)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_expert_combine_backward")
    return _expert_combine_backward(dout, y, order, weights, out)


@_on_device_of("dout")
def _expert_combine_backward(dout, y, order, weights, out):
    where = "sp24_expert_combine_backward"
    t = _float_code(dout, where)
    lddo = _matrix(dout, where)
    T, K = dout.shape
    _check_order(order, T, where, dout)
    rows = order.source.shape[0]
    ldy = _matrix(y, where, dout, (rows, K), dout.dtype)
    _slots(weights, where, dout, torch.float32, order.position.shape)
    dy = dout.new_empty((rows, K)) if out is None else out
    lddy = _matrix(dy, where, dout, (rows, K), dout.dtype)
    dweights = torch.empty_like(weights)
    _check(lib.sp24_expert_combine_backward(t, T, K, rows, _ptr(dout), lddo, _ptr(y), ldy, order.position.shape[1], _ptr(order.position), _ptr(order.source),
                                            _ptr(weights), _ptr(dy), lddy, _ptr(dweights), _stream()), where)
    return dy, dweights


def _stack(t: torch.Tensor, where: str, like: torch.Tensor | None = None, shape=None, dtype=None) -> int:
    """The leading dimension of [E, M, columns]: E matrices with contiguous rows, one after the other."""
    _refuse(t.dim() != 3 or (shape is not None and tuple(t.shape) != tuple(shape)), ERR_SHAPE, where)
    _refuse(not t.is_cuda or (like is not None and t.device != like.device), ERR_UNSUPPORTED, where)
    _refuse(dtype is not None and t.dtype != dtype, ERR_DTYPE, where)
    E, M, n = t.shape
    ld = t.stride(1) if M > 1 else (t.stride(0) if E > 1 else max(1, n))
    _refuse((n > 1 and t.stride(2) != 1) or (E > 1 and M > 0 and t.stride(0) != M * ld), ERR_STRIDE, where)
    return ld


@_on_device_of("W")
def expert_compress(W: torch.Tensor):
    """sp24_compress of every expert's weights W [E, M, K]: (vals [E, M, K/2], meta [E, bytes]) as expert_linear takes them."""
    where = "sp24_compress"
    dt = _FROM_TORCH.get(W.dtype)
    _refuse(dt is None or dt in ("i32", "f32"), ERR_DTYPE, where)
    ld = _stack(W, where)
    E, M, K = W.shape
    vals, meta = W.new_empty((E, M, K // 2)), W.new_empty((E, meta_bytes(dt, M, K)), dtype=torch.uint8)
    # (the metadata of an expert is whole blocks of 128 rows)
    for first, n in ([(0, E * M)] if M % 128 == 0 else [(e, M) for e in range(E)]):
        _check(lib.sp24_compress(DTYPE_CODE[dt], n, K, _ptr(W[first] if E else W), ld, _ptr(vals[first] if E else vals), K // 2,
                                 _ptr(meta[first] if E else meta), META_TCGEN05, None, _stream()), where)
    return vals, meta


def expert_linear(A: torch.Tensor, meta: torch.Tensor | None, X: torch.Tensor, offsets: torch.Tensor, *, bias: torch.Tensor | None = None,
                  act: str | None = None, residual: torch.Tensor | None = None, row_scale: torch.Tensor | None = None,
                  col_scale: torch.Tensor | None = None, pre: bool | torch.Tensor = False, out: torch.Tensor | None = None, cd: str | None = None,
                  a_is_dense: bool = False, ws: torch.Tensor | None = None):
    """sp24_expert_linear: for the rows r of expert e, offsets[e] <= r < offsets[e + 1],
    D[r, i] = act(row_scale[e, i] * col_scale[r] * (A_e X[r])[i] + bias[e, i]) + residual[r, i].  A: vals [E, M, K/2] and meta [E, bytes] of expert_compress (or
    dense [E, M, K] with a_is_dense), X [rows, K], offsets [E + 1] int32 of expert_order, bias and row_scale [E, M], col_scale [rows] (8-bit operands),
    residual [rows, M] in D's type (it may be `out`).  Returns D [rows, M] of type cd (A's own, bf16 for 8-bit operands), or with pre=True (or a tensor
    for it) (D, what act was applied to).  Rows that belong to no expert are left as they are.  M and K are multiples of 16, with 8-bit operands of 32."""
    done = _native.expert_linear(_EXPERT_LINEAR, _workspaces, _META_BYTES, A, meta, X, offsets, bias, act, residual, row_scale, col_scale, pre, out, cd,
                                 a_is_dense, ws)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_expert_linear")
    return _expert_linear(A, meta, X, offsets, bias, act, residual, row_scale, col_scale, pre, out, cd, a_is_dense, ws)


@_on_device_of("A")
def _expert_linear(A, meta, X, offsets, bias, act, residual, row_scale, col_scale, pre, out, cd, a_is_dense, ws):
    where = "sp24_expert_linear"
    ab = _FROM_TORCH.get(A.dtype)
    _refuse(ab not in ("f16", "bf16") + _QUANT, ERR_DTYPE, where)
    lda, ldx = _stack(A, where), _matrix(X, where, A, None, A.dtype)
    E, M, K = A.shape[0], A.shape[1], A.shape[2] * (1 if a_is_dense else 2)
    rows = X.shape[0]
    _refuse(X.shape[1] != K, ERR_SHAPE, where)
    _vector(offsets, E + 1, where, A, (torch.int32,))
    if not a_is_dense:
        _refuse(meta is None, 1, where)
        _refuse(meta.dim() != 2, ERR_SHAPE, where)
        _slots(meta, where, A, torch.uint8, (E, meta_bytes(ab, M, K)))
    cd = cd or ("bf16" if ab in _QUANT else ab)
    _refuse(cd not in TORCH_DTYPE, ERR_DTYPE, where)
    shape, dtype = (rows, M), TORCH_DTYPE[cd]
    D = A.new_empty(shape, dtype=dtype) if out is None else out
    ldd = _matrix(D, where, A, shape, dtype)
    ld_residual = ld_pre = ldd
    if residual is not None:
        ld_residual = _matrix(residual, where, A, shape, dtype)
    for v in (bias, row_scale):
        if v is not None:
            _slots(v, where, A, torch.float32, (E, M))
    _vector(col_scale, rows, where, A)
    z = None
    if pre is not False and pre is not None:
        z = torch.empty_like(D) if pre is True else pre
        ld_pre = _matrix(z, where, A, shape, dtype)
    stream = _stream()
    ws = ws if ws is not None else workspace(A.device, stream)
    desc = ExpertDesc(DTYPE_CODE[ab], DTYPE_CODE[cd], E, M, K, rows, lda, ldx, ldd, ld_residual, ld_pre, 1 if a_is_dense else 0)
    epilogue = ExpertEpilogue(_ptr(row_scale), _ptr(col_scale), _ptr(bias), _act_code(act, where), _ptr(residual), _ptr(z))
    _check(lib.sp24_expert_linear(byref(desc), byref(epilogue), _ptr(A), _ptr(meta), _ptr(X), _ptr(offsets), _ptr(D), _ptr(ws), ws.numel(), stream), where)
    return D if z is None else (D, z)


def expert_linear_backward(dy: torch.Tensor, pre: torch.Tensor | None, X: torch.Tensor, W: torch.Tensor, offsets: torch.Tensor, *, act: str | None = None,
                           meta: torch.Tensor | None = None, bias: bool = True, ws: torch.Tensor | None = None):
    """Gradients of expert_linear (16-bit operands) from dy [rows, M], its `pre` (None without an activation), X [rows, K] and the pruned weights W [E, M, K]
    themselves: (dX [rows, K], dW [E, M, K], dbias [E, M] float32, or None with bias=False).  Every offset is a multiple of 16 (expert_order with align=16): the
    dW of an expert that is not so placed is NaN.  With meta [E, bytes] the entries of dW that the 2:4 pattern leaves out are zeros.  Rows of dX that belong to
    no expert are left as they are; an expert without rows has dW and dbias of zeros.  The residual's gradient is dy.  dz = dy act'(pre) is rounded to dy's type
    before the two products, dbias is not."""
    done = _native.expert_linear_backward(_EXPERT_ACT, _EXPERT_ACT_BYTES, _EXPERT_DX, _EXPERT_DW, _META_BYTES, _workspaces, dy, pre, X, W,
                                          offsets, act, meta, bias, ws)
    if done is not None:
        return done if type(done) is not int else _check(done, "sp24_expert_linear_backward")
    return _expert_linear_backward(dy, pre, X, W, offsets, act, meta, bias, ws)


@_on_device_of("dy")
def _expert_linear_backward(dy, pre, X, W, offsets, act, meta, bias, ws):
    where = "sp24_expert_linear_backward"
    code = _FROM_TORCH.get(dy.dtype)
    _refuse(code not in ("f16", "bf16"), ERR_DTYPE, where)
    lddy = _matrix(dy, where)
    ldw = _stack(W, where, dy, None, dy.dtype)
    E, M, K = W.shape
    rows = dy.shape[0]
    _refuse(dy.shape[1] != M, ERR_SHAPE, where)
    ldx = _matrix(X, where, dy, (rows, K), dy.dtype)
    _vector(offsets, E + 1, where, dy, (torch.int32,))
    a = _act_code(act, where)
    _refuse(M % 16 or K % 16, ERR_SHAPE, where)
    _refuse(bool(a) and pre is None, 1, where)
    ldz = _matrix(pre, where, dy, dy.shape, dy.dtype) if a else lddy
    if meta is not None:
        _slots(meta, where, dy, torch.uint8, (E, meta_bytes(code, M, K)))
    t, stream = DTYPE_CODE[code], _stream()
    ws = ws if ws is not None else workspace(dy.device, stream)
    # (without an activation dz is dy itself, where a product can take it)
    dz, lddz = dy, lddy
    if a or dy.data_ptr() % 16 or lddy * dy.element_size() % 16:
        dz, lddz = dy.new_empty((rows, M)), M
    dbias = scratch = None
    size = 0
    if bias:
        dbias = dy.new_empty((E, M), dtype=torch.float32)
        size = lib.sp24_expert_act_backward_workspace_bytes(E, M, rows)
        scratch = dy.new_empty(size, dtype=torch.uint8)
    _check(lib.sp24_expert_act_backward(t, a, E, M, rows, _ptr(dy), lddy, _ptr(pre) if a else None, ldz, _ptr(offsets), None if dz is dy else _ptr(dz), lddz,
                                        _ptr(dbias), _ptr(scratch), size, stream), where)
    dX, dW = dy.new_empty((rows, K)), dy.new_empty((E, M, K))
    desc = ExpertDesc(t, t, E, M, K, rows, ldw, K, lddz, 0, 0, 1)
    _check(lib.sp24_expert_linear_dx(byref(desc), _ptr(dz), _ptr(W), _ptr(offsets), _ptr(dX), _ptr(ws), ws.numel(), stream), where)
    desc = ExpertDesc(t, t, E, M, K, rows, K, ldx, lddz, 0, 0, 1)
    _check(lib.sp24_expert_linear_dw(byref(desc), _ptr(dz), _ptr(X), _ptr(offsets), _ptr(meta), _ptr(dW), _ptr(ws), ws.numel(), stream), where)
    return dX, dW, dbias
