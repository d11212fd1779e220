"""ctypes binding of ``libmx_b200.so`` (the C ABI declared in ``include/mx.h``).

Argument marshalling only: every function takes torch tensors (or raw
pointers), passes ``data_ptr()`` and the current CUDA stream to the C entry point
of the same name and raises :class:`MxError` on a nonzero status.  The norm, routing,
row-moving, grouped-product and cache calls, whose GPU time may be a few microseconds, are
marshalled in C++ (``csrc/py_call.cpp``; without that module they raise ImportError).  PyTorch owns
the memory; all arithmetic runs in the library's CUDA kernels.  If the shared
library is missing the import of this module fails -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from . import build as _build

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmx_b200.so")

# enums of include/mx.h
MX_E4M3, MX_E5M2, MX_E3M2, MX_E2M3, MX_E2M1, MX_INT8 = range(6)
FORMATS = {"e4m3": MX_E4M3, "e5m2": MX_E5M2, "e3m2": MX_E3M2, "e2m3": MX_E2M3,
           "e2m1": MX_E2M1, "int8": MX_INT8}
MX_RNE, MX_RHAZ = 0, 1
MX_F32, MX_BF16 = 0, 1
MX_SCALES_LINEAR, MX_SCALES_SWIZZLED = 0, 1
MX_SCORE_SOFTMAX, MX_SCORE_SIGMOID = 0, 1
SCORES = {"softmax": MX_SCORE_SOFTMAX, "sigmoid": MX_SCORE_SIGMOID}
MX_GROUP_MAX, MX_GROUP_TOP2 = 0, 1
MX_OK = 0
MX_ERR_NULL, MX_ERR_SHAPE, MX_ERR_FMT, MX_ERR_ALIGN = -1, -2, -3, -4
MX_ERR_UNSUPPORTED, MX_ERR_CUDA, MX_ERR_TIMEOUT, MX_ERR_WORKSPACE = -5, -6, -7, -8

EXPORTS = [
    "mx_fmt_bits", "mx_elems_bytes", "mx_scales_bytes", "mx_scale_offset", "mx_strerror",
    "mx_last_cuda_error", "mx_quantize", "mx_quantize_dual", "mx_dequantize", "mx_gemm",
    "mx_gemm_bf16", "mx_gemm_ex", "mx_gemm_batched", "mx_gemm_quantize", "mx_gemm_dense_workspace_bytes",
    "mx_gemm_dense", "mx_conv_out_h", "mx_conv_out_w", "mx_im2col", "mx_conv2d",
    "mx_quantize_host_async", "mx_dequantize_host_async", "mx_host_synchronize",
    "mx_quantize_host_workspace_bytes", "mx_quantize_host", "mx_quantize_host_static",
    "mx_dequantize_host_workspace_bytes", "mx_dequantize_host",
    "mx_gemm_host_workspace_bytes", "mx_gemm_host",
    "mx_rmsnorm_quantize", "mx_rmsnorm_backward_workspace_bytes", "mx_rmsnorm_backward", "mx_route",
    "mx_route_backward", "mx_moe_rows", "mx_moe_plan_workspace_bytes", "mx_moe_plan", "mx_moe_gather",
    "mx_moe_combine", "mx_moe_combine_backward", "mx_gemm_grouped", "mx_gemm_grouped_k",
    "mx_gemm_grouped_ex", "mx_gemm_grouped_k_ex",
    "mx_kv_elems_bytes", "mx_kv_scales_bytes", "mx_kv_append", "mx_kv_read", "mx_kv_attention_workspace_bytes",
    "mx_kv_attention",
]


class mx_opts_t(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("scale_layout", ctypes.c_int32),
                ("stream", ctypes.c_void_p), ("check_status", ctypes.c_int32),
                ("pad_k128", ctypes.c_int32)]


class mx_gemm_plan_t(ctypes.Structure):
    _fields_ = [("c_dtype", ctypes.c_int32), ("tile_n", ctypes.c_int32),
                ("few_rows_limit", ctypes.c_int32), ("drop_fill", ctypes.c_int32),
                ("wait_cycles", ctypes.c_int64)]


class mx_conv_t(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("H", ctypes.c_int64), ("W", ctypes.c_int64), ("C", ctypes.c_int64),
                ("kh", ctypes.c_int32), ("kw", ctypes.c_int32),
                ("stride_h", ctypes.c_int32), ("stride_w", ctypes.c_int32),
                ("pad_h", ctypes.c_int32), ("pad_w", ctypes.c_int32),
                ("dil_h", ctypes.c_int32), ("dil_w", ctypes.c_int32)]


class mx_route_t(ctypes.Structure):
    _fields_ = [("topk", ctypes.c_int32), ("score", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("topk_groups", ctypes.c_int32), ("group_score", ctypes.c_int32),
                ("renormalize", ctypes.c_int32), ("scale", ctypes.c_float)]


class mx_kv_t(ctypes.Structure):
    _fields_ = [("k_elems", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_elems", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int64),
                ("heads", ctypes.c_int64), ("dim", ctypes.c_int64), ("fmt", ctypes.c_int32)]


class mx_kv_attention_t(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("new_tokens", ctypes.c_int64), ("q_heads", ctypes.c_int64),
                ("max_pages", ctypes.c_int64), ("q_stride", ctypes.c_int64), ("window", ctypes.c_int64),
                ("scale", ctypes.c_float)]


class MxError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = _lib.mx_strerror(status).decode()
        if status in (MX_ERR_CUDA, MX_ERR_TIMEOUT):
            msg += ": " + _lib.mx_last_cuda_error().decode()
        super().__init__(f"{where}: {msg} ({status})")


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python paper_2310_10537_b200/build.py` "
            "(the library has no CPU or PyTorch fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64p, u8p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64), ctypes.c_void_p
    ci, i64, sz = ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    op = ctypes.POINTER(mx_opts_t)
    lib.mx_fmt_bits.argtypes = [ci]
    lib.mx_elems_bytes.argtypes = [i64p, ci, ci, ci]
    lib.mx_elems_bytes.restype = sz
    lib.mx_scales_bytes.argtypes = [i64p, ci, ci, ci]
    lib.mx_scales_bytes.restype = sz
    lib.mx_scale_offset.argtypes = [i64, i64, i64, i64, ci]
    lib.mx_scale_offset.restype = sz
    lib.mx_strerror.argtypes = [ci]
    lib.mx_strerror.restype = ctypes.c_char_p
    lib.mx_last_cuda_error.restype = ctypes.c_char_p
    lib.mx_quantize.argtypes = [vp, vp, u8p, i64p, ci, ci, ci, ci, op]
    lib.mx_quantize_dual.argtypes = [vp, vp, u8p, vp, u8p, i64, i64, ci, ci, op]
    lib.mx_dequantize.argtypes = [vp, u8p, vp, i64p, ci, ci, ci, op]
    lib.mx_gemm.argtypes = [vp, u8p, vp, u8p, vp, i64, i64, i64, ci, ci, op]
    lib.mx_gemm_bf16.argtypes = [vp, u8p, vp, u8p, vp, i64, i64, i64, ci, ci, op]
    lib.mx_gemm_ex.argtypes = [vp, u8p, vp, u8p, vp, i64, i64, i64, ci, ci, op, ctypes.POINTER(mx_gemm_plan_t)]
    lib.mx_gemm_quantize.argtypes = [vp, u8p, vp, u8p, vp, u8p, i64, i64, i64, ci, ci, ci, ci, op]
    lib.mx_gemm_dense_workspace_bytes.argtypes = [i64, i64, i64]
    lib.mx_gemm_dense_workspace_bytes.restype = sz
    lib.mx_gemm_dense.argtypes = [vp, u8p, vp, u8p, vp, ci, i64, i64, i64, ci, ci, op, vp, sz]
    cp = ctypes.POINTER(mx_conv_t)
    lib.mx_conv_out_h.argtypes = [cp]
    lib.mx_conv_out_h.restype = i64
    lib.mx_conv_out_w.argtypes = [cp]
    lib.mx_conv_out_w.restype = i64
    lib.mx_im2col.argtypes = [vp, u8p, vp, u8p, cp, ci, op]
    lib.mx_conv2d.argtypes = [vp, u8p, vp, u8p, vp, ci, cp, i64, ci, ci, op]
    lib.mx_gemm_batched.argtypes = [vp, u8p, vp, u8p, vp, ci, i64, i64, i64, i64, ci, ci, op]
    lib.mx_quantize_host_workspace_bytes.argtypes = [i64p, ci, ci, ci, op]
    lib.mx_quantize_host_workspace_bytes.restype = sz
    lib.mx_quantize_host.argtypes = [vp, vp, u8p, i64p, ci, ci, ci, ci, op, vp, sz]
    lib.mx_quantize_host_async.argtypes = [vp, vp, u8p, i64p, ci, ci, ci, ci, op, vp, sz]
    lib.mx_host_synchronize.argtypes = []
    lib.mx_quantize_host_static.argtypes = [vp, vp, u8p, i64p, ci, ci, ci, ci, op]
    lib.mx_dequantize_host_workspace_bytes.argtypes = [i64p, ci, ci, ci, op]
    lib.mx_dequantize_host_workspace_bytes.restype = sz
    lib.mx_dequantize_host.argtypes = [vp, u8p, vp, i64p, ci, ci, ci, op, vp, sz]
    lib.mx_dequantize_host_async.argtypes = [vp, u8p, vp, i64p, ci, ci, ci, op, vp, sz]
    lib.mx_gemm_host_workspace_bytes.argtypes = [i64, i64, i64, ci, ci]
    lib.mx_gemm_host_workspace_bytes.restype = sz
    lib.mx_gemm_host.argtypes = [vp, u8p, vp, u8p, vp, i64, i64, i64, ci, ci, op, vp, sz]
    cf, rp = ctypes.c_float, ctypes.POINTER(mx_route_t)
    lib.mx_rmsnorm_quantize.argtypes = [vp, vp, vp, ci, cf, i64, i64, vp, vp, vp, u8p, ci, ci, op]
    lib.mx_rmsnorm_backward_workspace_bytes.argtypes = [i64, i64]
    lib.mx_rmsnorm_backward_workspace_bytes.restype = sz
    lib.mx_rmsnorm_backward.argtypes = [vp, vp, vp, ci, cf, vp, i64, i64, vp, vp, op, vp, sz]
    lib.mx_route.argtypes = [vp, vp, i64, i64, rp, vp, vp, op]
    lib.mx_route_backward.argtypes = [vp, vp, vp, i64, i64, rp, vp, op]
    lib.mx_moe_rows.argtypes = [i64, i64, i64, i64]
    lib.mx_moe_rows.restype = i64
    lib.mx_moe_plan_workspace_bytes.argtypes = [i64, i64, i64]
    lib.mx_moe_plan_workspace_bytes.restype = sz
    lib.mx_moe_plan.argtypes = [vp, i64, i64, i64, i64, vp, vp, vp, vp, op, vp, sz]
    lib.mx_moe_gather.argtypes = [vp, u8p, i64, i64, i64, ci, vp, vp, vp, vp, i64, i64, vp, u8p, op]
    lib.mx_moe_combine.argtypes = [vp, vp, vp, i64, i64, i64, i64, vp, op]
    lib.mx_moe_combine_backward.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, vp, vp, op]
    lib.mx_gemm_grouped.argtypes = [vp, u8p, vp, u8p, vp, vp, ci, i64, i64, i64, i64, ci, ci, op]
    lib.mx_gemm_grouped_k.argtypes = [vp, u8p, vp, u8p, vp, vp, ci, i64, i64, i64, i64, ci, ci, op]
    lib.mx_gemm_grouped_ex.argtypes = lib.mx_gemm_grouped.argtypes + [i64, ctypes.c_int32]
    lib.mx_gemm_grouped_k_ex.argtypes = lib.mx_gemm_grouped_k.argtypes + [i64, ctypes.c_int32]
    kp, ap = ctypes.POINTER(mx_kv_t), ctypes.POINTER(mx_kv_attention_t)
    lib.mx_kv_elems_bytes.argtypes = [kp]
    lib.mx_kv_elems_bytes.restype = sz
    lib.mx_kv_scales_bytes.argtypes = [kp]
    lib.mx_kv_scales_bytes.restype = sz
    lib.mx_kv_append.argtypes = [kp, vp, vp, i64, i64, vp, i64, ci, op]
    lib.mx_kv_read.argtypes = [kp, vp, i64, vp, vp, op]
    lib.mx_kv_attention_workspace_bytes.argtypes = [kp, ap]
    lib.mx_kv_attention_workspace_bytes.restype = sz
    lib.mx_kv_attention.argtypes = [kp, ap, vp, vp, vp, vp, vp, op, vp, sz]
    return lib


_lib = _load()



class _NoPyCall:
    """Stands for the marshalling module where it cannot be used: the calls that need it raise, all others work."""

    def __init__(self, why: str):
        self._why = why

    def __getattr__(self, name: str):
        raise ImportError(f"{name} needs {os.path.join(os.path.dirname(LIB_PATH), '_py_call.so')}, {self._why}: build it with "
                          "`python paper_2310_10537_b200/build.py` (there is no fallback)")


def _load_py_call():
    """csrc/py_call.cpp (it links against the library loaded above, and against the C++ interfaces of one torch)."""
    try:
        from . import _py_call as module
    except ImportError as e:
        return _NoPyCall(f"which cannot be loaded ({e})")
    here = _build.py_call_for()
    if module.compiled_for != here:
        return _NoPyCall(f"which was compiled for {module.compiled_for}, not for {here}")
    module.set_error_type(MxError)
    return module


_py_call = _load_py_call()


def lib() -> ctypes.CDLL:
    """The loaded C library (for callers that pass raw pointers)."""
    return _lib


def _shape_arr(shape: Sequence[int]):
    return (ctypes.c_int64 * len(shape))(*[int(s) for s in shape])


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float32:
        return MX_F32
    if dt == torch.bfloat16:
        return MX_BF16
    raise TypeError(f"unsupported float dtype {dt}")


def _opts(dtype: int, layout: int, check: bool = False, stream: Optional[int] = None,
          pad_k128: bool = False) -> mx_opts_t:
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    return mx_opts_t(dtype, layout, ctypes.c_void_p(stream), 1 if check else 0, 1 if pad_k128 else 0)


def _check(status: int, where: str) -> None:
    if status != MX_OK:
        raise MxError(status, where)


def mx_fmt_bits(fmt: int) -> int:
    return _lib.mx_fmt_bits(fmt)


def mx_elems_bytes(shape: Sequence[int], axis: int, fmt: int) -> int:
    return int(_lib.mx_elems_bytes(_shape_arr(shape), len(shape), axis, fmt))


def mx_scales_bytes(shape: Sequence[int], axis: int, layout: int = MX_SCALES_SWIZZLED) -> int:
    return int(_lib.mx_scales_bytes(_shape_arr(shape), len(shape), axis, layout))


def mx_scale_offset(row: int, kblock: int, rows: int, kblocks: int,
                    layout: int = MX_SCALES_SWIZZLED) -> int:
    return int(_lib.mx_scale_offset(row, kblock, rows, kblocks, layout))


def mx_quantize(x: torch.Tensor, axis: int, fmt: int, rounding: int = MX_RNE,
                layout: int = MX_SCALES_SWIZZLED,
                out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
                pad_k128: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """Quantize a contiguous CUDA tensor along ``axis`` (Algorithm 1).

    Returns (elems, scales) as flat uint8 tensors; the packed tensor has the
    quantization axis innermost.  ``out`` lets the caller reuse buffers.  ``pad_k128``: the
    result is the MX tensor of x zero-extended along ``axis`` to a multiple of 128."""
    assert x.is_cuda and x.is_contiguous()
    axis %= x.dim()
    shape = list(x.shape)
    if out is None:
        stored = list(shape)
        if pad_k128:
            stored[axis] = (stored[axis] + 127) // 128 * 128
        elems = torch.empty(mx_elems_bytes(stored, axis, fmt), dtype=torch.uint8, device=x.device)
        scales = torch.empty(mx_scales_bytes(stored, axis, layout), dtype=torch.uint8, device=x.device)
    else:
        elems, scales = out
    o = _opts(_dtype_code(x.dtype), layout, pad_k128=pad_k128)
    _check(_lib.mx_quantize(x.data_ptr(), elems.data_ptr(), scales.data_ptr(), _shape_arr(shape),
                            len(shape), axis, fmt, rounding, ctypes.byref(o)), "mx_quantize")
    return elems, scales


def mx_quantize_dual(x: torch.Tensor, fmt: int, rounding: int = MX_RNE, layout: int = MX_SCALES_SWIZZLED,
                     out=None, check_status: bool = False):
    """Both MX tensors of a contiguous 2-D CUDA tensor in one pass: returns
    ((elems_row, scales_row), (elems_col, scales_col)) = (mx_quantize(x, 1), mx_quantize(x, 0)).
    ``check_status``: synchronise and raise if a device-side wait of the kernel gave up."""
    assert x.is_cuda and x.is_contiguous() and x.dim() == 2
    R, C = x.shape
    if out is None:
        u8 = dict(dtype=torch.uint8, device=x.device)
        er = torch.empty(mx_elems_bytes([R, C], 1, fmt), **u8)
        sr = torch.empty(mx_scales_bytes([R, C], 1, layout), **u8)
        ec = torch.empty(mx_elems_bytes([R, C], 0, fmt), **u8)
        sc = torch.empty(mx_scales_bytes([R, C], 0, layout), **u8)
    else:
        (er, sr), (ec, sc) = out
    o = _opts(_dtype_code(x.dtype), layout, check=check_status)
    _check(_lib.mx_quantize_dual(x.data_ptr(), er.data_ptr(), sr.data_ptr(), ec.data_ptr(), sc.data_ptr(),
                                 R, C, fmt, rounding, ctypes.byref(o)), "mx_quantize_dual")
    return (er, sr), (ec, sc)


def mx_dequantize(elems: torch.Tensor, scales: torch.Tensor, shape: Sequence[int], fmt: int,
                  dtype: torch.dtype = torch.float32, layout: int = MX_SCALES_SWIZZLED,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Dequantize a packed MX tensor of logical shape ``shape`` (blocks along the last axis)."""
    assert elems.is_cuda and scales.is_cuda
    shape = list(shape)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=elems.device)
    o = _opts(_dtype_code(out.dtype), layout)
    _check(_lib.mx_dequantize(elems.data_ptr(), scales.data_ptr(), out.data_ptr(),
                              _shape_arr(shape), len(shape), len(shape) - 1, fmt,
                              ctypes.byref(o)), "mx_dequantize")
    return out


def mx_gemm(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor,
            M: int, N: int, K: int, fmtA: int, fmtB: int,
            out: Optional[torch.Tensor] = None, check_status: bool = False,
            pad_k128: bool = False) -> torch.Tensor:
    """C[M,N] = A[M,K] . B[N,K]^T on MX operands (swizzled scales), FP32 output.  ``pad_k128``:
    both operands were written by mx_quantize with the same option (K % 32 == 0 then suffices)."""
    assert A.is_cuda and B.is_cuda and sA.is_cuda and sB.is_cuda
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
    o = _opts(MX_F32, MX_SCALES_SWIZZLED, check=check_status, pad_k128=pad_k128)
    _check(_lib.mx_gemm(A.data_ptr(), sA.data_ptr(), B.data_ptr(), sB.data_ptr(), out.data_ptr(),
                        M, N, K, fmtA, fmtB, ctypes.byref(o)), "mx_gemm")
    return out


def mx_gemm_bf16(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor,
                 M: int, N: int, K: int, fmtA: int, fmtB: int,
                 out: Optional[torch.Tensor] = None, check_status: bool = False,
                 pad_k128: bool = False) -> torch.Tensor:
    """mx_gemm with the FP32 accumulator rounded to nearest even into a BF16 output."""
    assert A.is_cuda and B.is_cuda and sA.is_cuda and sB.is_cuda
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    assert out.dtype == torch.bfloat16
    o = _opts(MX_F32, MX_SCALES_SWIZZLED, check=check_status, pad_k128=pad_k128)
    _check(_lib.mx_gemm_bf16(A.data_ptr(), sA.data_ptr(), B.data_ptr(), sB.data_ptr(),
                             out.data_ptr(), M, N, K, fmtA, fmtB, ctypes.byref(o)), "mx_gemm_bf16")
    return out


def mx_gemm_ex(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor,
               M: int, N: int, K: int, fmtA: int, fmtB: int, out: Optional[torch.Tensor] = None,
               out_dtype: torch.dtype = torch.float32, tile_n: int = 0, few_rows_limit: int = -1,
               wait_cycles: int = 0, drop_fill: int = -1, check_status: bool = False,
               pad_k128: bool = False) -> torch.Tensor:
    """mx_gemm / mx_gemm_bf16 with the kernel selection (tile_n, few_rows_limit) and the device-side
    wait budget (wait_cycles; drop_fill is the failure drill) in the caller's hands."""
    assert A.is_cuda and B.is_cuda and sA.is_cuda and sB.is_cuda
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=A.device)
    o = _opts(MX_F32, MX_SCALES_SWIZZLED, check=check_status, pad_k128=pad_k128)
    plan = mx_gemm_plan_t(_dtype_code(out.dtype), tile_n, few_rows_limit, drop_fill, wait_cycles)
    _check(_lib.mx_gemm_ex(A.data_ptr(), sA.data_ptr(), B.data_ptr(), sB.data_ptr(), out.data_ptr(),
                           M, N, K, fmtA, fmtB, ctypes.byref(o), ctypes.byref(plan)), "mx_gemm_ex")
    return out


def mx_gemm_batched(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor,
                    batch: int, M: int, N: int, K: int, fmtA: int, fmtB: int,
                    out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
                    check_status: bool = False) -> torch.Tensor:
    """C[b] = A[b] . B[b]^T for b < batch; operands are the MX tensors of [batch, M, K] and
    [batch, N, K] quantized along K (swizzled scales)."""
    assert A.is_cuda and B.is_cuda and sA.is_cuda and sB.is_cuda
    if out is None:
        out = torch.empty((batch, M, N), dtype=out_dtype, device=A.device)
    o = _opts(MX_F32, MX_SCALES_SWIZZLED, check=check_status)
    _check(_lib.mx_gemm_batched(A.data_ptr(), sA.data_ptr(), B.data_ptr(), sB.data_ptr(),
                                out.data_ptr(), _dtype_code(out.dtype), batch, M, N, K, fmtA, fmtB,
                                ctypes.byref(o)), "mx_gemm_batched")
    return out


def mx_gemm_quantize(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor,
                     M: int, N: int, K: int, fmtA: int, fmtB: int, fmtC: int, rounding: int = MX_RNE,
                     elems: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                     check_status: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """A . B^T quantized along N in the GEMM epilogue: the MX tensor (codes, swizzled scales)
    mx_quantize would produce from the FP32 result."""
    assert A.is_cuda and B.is_cuda and sA.is_cuda and sB.is_cuda
    if elems is None:
        elems = torch.empty(M * N * mx_fmt_bits(fmtC) // 8, dtype=torch.uint8, device=A.device)
    if scales is None:
        scales = torch.empty(mx_scales_bytes((M, N), 1, MX_SCALES_SWIZZLED), dtype=torch.uint8,
                             device=A.device)
    o = _opts(MX_F32, MX_SCALES_SWIZZLED, check=check_status)
    _check(_lib.mx_gemm_quantize(A.data_ptr(), sA.data_ptr(), B.data_ptr(), sB.data_ptr(),
                                 elems.data_ptr(), scales.data_ptr(), M, N, K, fmtA, fmtB, fmtC,
                                 rounding, ctypes.byref(o)), "mx_gemm_quantize")
    return elems, scales


def mx_gemm_dense_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(_lib.mx_gemm_dense_workspace_bytes(M, N, K))


def mx_gemm_dense(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor,
                  M: int, N: int, K: int, fmtA: int, fmtB: int,
                  workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  out_dtype: torch.dtype = torch.float32, check_status: bool = False) -> torch.Tensor:
    """A . B^T through BF16: dequantize both operands into ``workspace`` and run the dense BF16
    tensor-core GEMM (any format pair, MXINT8 included)."""
    assert A.is_cuda and B.is_cuda and sA.is_cuda and sB.is_cuda
    if workspace is None:
        workspace = torch.empty(mx_gemm_dense_workspace_bytes(M, N, K), dtype=torch.uint8, device=A.device)
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=A.device)
    o = _opts(MX_F32, MX_SCALES_SWIZZLED, check=check_status)
    _check(_lib.mx_gemm_dense(A.data_ptr(), sA.data_ptr(), B.data_ptr(), sB.data_ptr(), out.data_ptr(),
                              _dtype_code(out.dtype), M, N, K, fmtA, fmtB, ctypes.byref(o),
                              workspace.data_ptr(), workspace.numel()), "mx_gemm_dense")
    return out


def mx_conv_geometry(N: int, H: int, W: int, C: int, kh: int, kw: int, stride=(1, 1), pad=(0, 0),
                     dilation=(1, 1)) -> mx_conv_t:
    return mx_conv_t(N, H, W, C, kh, kw, stride[0], stride[1], pad[0], pad[1], dilation[0], dilation[1])


def mx_conv_out_hw(conv: mx_conv_t) -> Tuple[int, int]:
    return int(_lib.mx_conv_out_h(ctypes.byref(conv))), int(_lib.mx_conv_out_w(ctypes.byref(conv)))


def mx_im2col(elems: torch.Tensor, scales: torch.Tensor, conv: mx_conv_t, fmt: int,
              layout: int = MX_SCALES_SWIZZLED) -> Tuple[torch.Tensor, torch.Tensor]:
    """The MX tensor of x[N, H, W, C] (quantized along C) laid out as the K-major operand
    [N*Ho*Wo x kh*kw*C] of mx_gemm: (codes, swizzled scales)."""
    assert elems.is_cuda and scales.is_cuda
    Ho, Wo = mx_conv_out_hw(conv)
    M, K = conv.N * Ho * Wo, conv.kh * conv.kw * conv.C
    out_e = torch.empty(M * K * mx_fmt_bits(fmt) // 8, dtype=torch.uint8, device=elems.device)
    out_s = torch.empty(mx_scales_bytes((M, K), 1, MX_SCALES_SWIZZLED), dtype=torch.uint8, device=elems.device)
    o = _opts(MX_F32, layout)
    _check(_lib.mx_im2col(elems.data_ptr(), scales.data_ptr(), out_e.data_ptr(), out_s.data_ptr(),
                          ctypes.byref(conv), fmt, ctypes.byref(o)), "mx_im2col")
    return out_e, out_s


def mx_conv2d(x_elems: torch.Tensor, x_scales: torch.Tensor, w_elems: torch.Tensor, w_scales: torch.Tensor,
              conv: mx_conv_t, Cout: int, fmt_x: int, fmt_w: int, layout: int = MX_SCALES_SWIZZLED,
              out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
              check_status: bool = False) -> torch.Tensor:
    """y[N*Ho*Wo, Cout] = the convolution of the MX activation (quantized along C, 8-bit codes, scales
    in `layout`) with the MX filter [Cout x kh*kw*C], the im2col operand gathered inside the GEMM."""
    assert x_elems.is_cuda and x_scales.is_cuda and w_elems.is_cuda and w_scales.is_cuda
    Ho, Wo = mx_conv_out_hw(conv)
    M = conv.N * Ho * Wo
    if out is None:
        out = torch.empty((M, Cout), dtype=out_dtype, device=x_elems.device)
    o = _opts(MX_F32, layout, check=check_status)
    _check(_lib.mx_conv2d(x_elems.data_ptr(), x_scales.data_ptr(), w_elems.data_ptr(), w_scales.data_ptr(),
                          out.data_ptr(), _dtype_code(out.dtype), ctypes.byref(conv), Cout, fmt_x, fmt_w,
                          ctypes.byref(o)), "mx_conv2d")
    return out


# ---- RMS norm, routing, moving rows, the experts' products ----------------------------

# These calls stand in loops of a few microseconds per step, so csrc/py_call.cpp checks their tensors, allocates
# their results and calls the C entry point: the functions here name and document the arguments.

def mx_rmsnorm_quantize(x: torch.Tensor, weight: torch.Tensor, fmt: int, eps: float = 1e-6,
                        residual: Optional[torch.Tensor] = None, rounding: int = MX_RNE,
                        layout: int = MX_SCALES_SWIZZLED, y_out: Optional[torch.Tensor] = None,
                        h_out: Optional[torch.Tensor] = None,
                        out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                        ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """RMS norm of ``x + residual`` [rows, dim] as an MX tensor along the rows: (elems, scales, h).

    ``h`` is the new residual stream (None without a residual, unless ``h_out`` is given; ``h_out`` may
    be ``x`` or ``residual``).  ``y_out`` also receives the norm itself."""
    elems, scales = (None, None) if out is None else out
    return _py_call.rmsnorm_quantize(x, weight, fmt, eps, residual, rounding, layout, y_out, h_out, elems, scales)


def mx_rmsnorm_backward(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6,
                        dres: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Gradients of the norm: (dh [rows, dim], dweight FP32 [dim]).  ``dres`` is added to dh; ``out``
    receives dh and may be ``dy`` or ``dres``."""
    return _py_call.rmsnorm_backward(dy, h, weight, eps, dres, out, workspace)


def mx_route(logits: torch.Tensor, topk: int, score: int = MX_SCORE_SOFTMAX, bias: Optional[torch.Tensor] = None,
             groups: int = 1, topk_groups: int = 1, group_score: int = MX_GROUP_MAX, renormalize: bool = True,
             scale: float = 1.0) -> Tuple[torch.Tensor, torch.Tensor]:
    """Experts of every token of ``logits`` [tokens, experts] and their weights: (ids int32, weights
    FP32), both [tokens, topk], the best first."""
    return _py_call.route(logits, topk, score, bias, groups, topk_groups, group_score, renormalize, scale)


def mx_route_backward(dweights: torch.Tensor, logits: torch.Tensor, ids: torch.Tensor,
                      score: int = MX_SCORE_SOFTMAX, renormalize: bool = True, scale: float = 1.0) -> torch.Tensor:
    """Gradient of mx_route's weights with respect to the logits (the choice ``ids`` held fixed)."""
    return _py_call.route_backward(dweights, logits, ids, score, renormalize, scale)


class MoePlan(NamedTuple):
    """Where the rows of a batch go: group e holds rows offsets[e] .. offsets[e + 1], the first counts[e]
    of them choices; row_of [tokens, topk] is the row of a choice (-1: dropped); ``rows`` bounds
    offsets[-1] and is what row tensors are allocated with; src_of [rows] is the choice of a row (-1: none),
    which mx_moe_gather needs."""
    offsets: torch.Tensor
    counts: torch.Tensor
    row_of: torch.Tensor
    rows: int
    src_of: Optional[torch.Tensor] = None


def mx_moe_rows(tokens: int, topk: int, experts: int, align: int = 64) -> int:
    return int(_lib.mx_moe_rows(tokens, topk, experts, align))


def mx_moe_plan(ids: torch.Tensor, experts: int, align: int = 64,
                workspace: Optional[torch.Tensor] = None) -> MoePlan:
    """Sort the choices ``ids`` [tokens, topk] by expert, groups padded to ``align`` rows: a multiple of
    64 for mx_gemm_grouped, of 128 for mx_gemm_grouped_k."""
    return MoePlan._make(_py_call.moe_plan(ids, experts, align, workspace))


def mx_moe_gather(elems: torch.Tensor, scales: torch.Tensor, dim: int, fmt: int, plan: MoePlan,
                  layout: int = MX_SCALES_SWIZZLED,
                  out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The rows of an MX tensor [tokens, dim] in the order of ``plan``: (elems, scales) of an MX tensor
    [plan.rows, dim], rows without a choice zero."""
    out_elems, out_scales = (None, None) if out is None else out
    return _py_call.moe_gather(elems, scales, dim, fmt, plan, layout, out_elems, out_scales)


def mx_moe_combine(y: torch.Tensor, weights: Optional[torch.Tensor], plan: MoePlan,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """out[t] = sum over j of weights[t, j] * y[row_of[t, j]] (``weights`` None: all 1); y [plan.rows, dim]."""
    return _py_call.moe_combine(y, weights, plan, out)


def mx_moe_combine_backward(dout: torch.Tensor, y: Optional[torch.Tensor], weights: Optional[torch.Tensor],
                            plan: MoePlan) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Gradients of mx_moe_combine: (dy [plan.rows, dim], dweights FP32 [tokens, topk]).  Without ``y``
    only dy; without ``weights`` as well it is the gather of the rows of a float tensor."""
    return _py_call.moe_combine_backward(dout, y, weights, plan)


def mx_gemm_grouped(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor, offsets: torch.Tensor,
                    rows: int, N: int, K: int, fmtA: int, fmtB: int, out: Optional[torch.Tensor] = None,
                    out_dtype: torch.dtype = torch.float32, check_status: bool = False) -> torch.Tensor:
    """C[r] = A[r] . B[g]^T for the rows r of group g, offsets[g] .. offsets[g + 1] (int32, on the device,
    multiples of 64): A is the MX tensor [rows, K], B that of [groups, N, K]; rows in no group are not
    written."""
    return _py_call.gemm_grouped(A, sA, B, sB, offsets, rows, N, K, fmtA, fmtB, out, out_dtype, check_status)


def mx_gemm_grouped_k(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor, offsets: torch.Tensor,
                      M: int, N: int, rows: int, fmtA: int, fmtB: int, out: Optional[torch.Tensor] = None,
                      out_dtype: torch.dtype = torch.float32, check_status: bool = False) -> torch.Tensor:
    """C[g] = A[:, r0:r1] . B[:, r0:r1]^T with r0, r1 = offsets[g], offsets[g + 1] (multiples of 128, or `rows`): A is the
    MX tensor [M, rows], B [N, rows], both quantized along the rows; C [groups, M, N]."""
    return _py_call.gemm_grouped_k(A, sA, B, sB, offsets, M, N, rows, fmtA, fmtB, out, out_dtype, check_status)


def mx_gemm_grouped_ex(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor, offsets: torch.Tensor,
                       rows: int, N: int, K: int, fmtA: int, fmtB: int, out: Optional[torch.Tensor] = None,
                       out_dtype: torch.dtype = torch.float32, check_status: bool = False, wait_cycles: int = 0,
                       drop_fill: int = -1) -> torch.Tensor:
    """mx_gemm_grouped with the device-side wait budget (wait_cycles; drop_fill is the failure drill) in the caller's
    hands."""
    return _py_call.gemm_grouped_ex(A, sA, B, sB, offsets, rows, N, K, fmtA, fmtB, out, out_dtype, check_status,
                                    wait_cycles, drop_fill)


def mx_gemm_grouped_k_ex(A: torch.Tensor, sA: torch.Tensor, B: torch.Tensor, sB: torch.Tensor, offsets: torch.Tensor,
                         M: int, N: int, rows: int, fmtA: int, fmtB: int, out: Optional[torch.Tensor] = None,
                         out_dtype: torch.dtype = torch.float32, check_status: bool = False, wait_cycles: int = 0,
                         drop_fill: int = -1) -> torch.Tensor:
    """mx_gemm_grouped_k with the device-side wait budget in the caller's hands, as mx_gemm_grouped_ex."""
    return _py_call.gemm_grouped_k_ex(A, sA, B, sB, offsets, M, N, rows, fmtA, fmtB, out, out_dtype, check_status,
                                      wait_cycles, drop_fill)


# ---- paged key-value cache ------------------------------------------------------------

class KvCache(NamedTuple):
    """A paged cache of keys and values in MX format: codes [pages, heads, page_size, dim * bits / 8] and scale bytes
    [pages, heads, page_size, 4 * ceil(dim / 128)], uint8, keys and values alike.  Token ``offset`` of page p is slot
    p * page_size + offset."""
    k_elems: torch.Tensor
    k_scales: torch.Tensor
    v_elems: torch.Tensor
    v_scales: torch.Tensor
    dim: int
    fmt: int


def mx_kv_cache(pages: int, page_size: int, heads: int, dim: int, fmt: int, device="cuda") -> KvCache:
    """An empty cache (all bytes zero) for ``pages`` pages of ``page_size`` tokens: ``dim`` a multiple of 32, ``fmt`` of 8 or 4 bits.
    (:func:`mx_kv_attention` takes ``dim`` 64, 96, 128, 192 and 256.)"""
    desc = mx_kv_t(None, None, None, None, pages or 1, page_size, heads, dim, fmt)  # (none at all: what a page would have to be)
    if not _lib.mx_kv_elems_bytes(ctypes.byref(desc)):
        raise ValueError(f"no cache of {pages} pages x {heads} heads x {page_size} tokens x {dim} in format {fmt}")
    code, scale = dim * mx_fmt_bits(fmt) // 8, (dim + 127) // 128 * 4
    zeros = lambda n: torch.zeros((pages, heads, page_size, n), dtype=torch.uint8, device=device)  # noqa: E731
    return KvCache(zeros(code), zeros(scale), zeros(code), zeros(scale), dim, fmt)


def mx_kv_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, rounding: int = MX_RNE) -> None:
    """Quantize the rows ``k``, ``v`` [tokens, heads, dim] into the slots ``slots`` (int32 [tokens], all different; one
    outside the cache: not written).  Tokens may be evenly spaced parts of a wider tensor."""
    _py_call.kv_append(cache, k, v, slots, rounding)


def mx_kv_read(cache: KvCache, slots: torch.Tensor, dtype: torch.dtype = torch.float32,
               out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Keys and values of ``slots`` as numbers, (k, v) [tokens, heads, dim]; zeros for a slot outside the cache."""
    out_k, out_v = (None, None) if out is None else out
    return _py_call.kv_read(cache, slots, dtype, out_k, out_v)


def mx_kv_attention(q: torch.Tensor, cache: KvCache, table: torch.Tensor, lengths: torch.Tensor,
                    scale: Optional[float] = None, window: int = 0, return_lse: bool = False,
                    out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Attention of the newest tokens ``q`` [batch, heads, dim], or [batch, new tokens, heads, dim], over the cached
    tokens of their sequences: sequence b has ``lengths[b]`` tokens (the new ones included) in the pages ``table[b]``
    (int32 [batch, pages of a sequence]).  ``scale`` defaults to dim ** -0.5; ``window`` > 0: a query sees its last
    ``window`` tokens only.  Returns out, shaped as q, or (out, lse); an ``out`` given must not share memory with q."""
    return _py_call.kv_attention(q, cache, table, lengths, scale, window, return_lse, out, workspace)


# ---- host-buffer variants: tensors live in (pinned) host memory ----------------

def mx_quantize_host_workspace_bytes(shape, axis, fmt, dtype, layout=MX_SCALES_SWIZZLED) -> int:
    o = _opts(_dtype_code(dtype), layout, stream=0)
    return int(_lib.mx_quantize_host_workspace_bytes(_shape_arr(shape), len(shape), axis, fmt,
                                                     ctypes.byref(o)))


def mx_quantize_host(x: torch.Tensor, elems: torch.Tensor, scales: torch.Tensor, axis: int,
                     fmt: int, rounding: int, workspace: torch.Tensor,
                     layout: int = MX_SCALES_SWIZZLED, queue: bool = False) -> None:
    """Host tensors in and out.  ``queue=True`` uses the asynchronous entry point: the call only
    queues its work (own workspace per queued call) and ``mx_host_synchronize()`` waits for it."""
    assert not x.is_cuda and not elems.is_cuda and not scales.is_cuda and workspace.is_cuda
    shape = list(x.shape)
    o = _opts(_dtype_code(x.dtype), layout)
    fn = _lib.mx_quantize_host_async if queue else _lib.mx_quantize_host
    _check(fn(x.data_ptr(), elems.data_ptr(), scales.data_ptr(),
                                 _shape_arr(shape), len(shape), axis % len(shape), fmt, rounding,
                                 ctypes.byref(o), workspace.data_ptr(), workspace.numel()),
           "mx_quantize_host")


MX_STATIC_SCRATCH_BYTES = 16 * 1024 * 1024


def mx_quantize_host_static(x: torch.Tensor, elems: torch.Tensor, scales: torch.Tensor, axis: int,
                            fmt: int, rounding: int, layout: int = MX_SCALES_SWIZZLED) -> None:
    """mx_quantize_host for callers that may not allocate device memory: the staging area is a
    fixed array inside the library (MX_STATIC_SCRATCH_BYTES), so no workspace is passed.  Calls
    on one device share that array and must not overlap."""
    assert not x.is_cuda and not elems.is_cuda and not scales.is_cuda
    shape = list(x.shape)
    o = _opts(_dtype_code(x.dtype), layout)
    _check(_lib.mx_quantize_host_static(x.data_ptr(), elems.data_ptr(), scales.data_ptr(),
                                        _shape_arr(shape), len(shape), axis % len(shape), fmt,
                                        rounding, ctypes.byref(o)), "mx_quantize_host_static")


def mx_dequantize_host_workspace_bytes(shape, fmt, dtype, layout=MX_SCALES_SWIZZLED) -> int:
    o = _opts(_dtype_code(dtype), layout, stream=0)
    return int(_lib.mx_dequantize_host_workspace_bytes(_shape_arr(shape), len(shape),
                                                       len(shape) - 1, fmt, ctypes.byref(o)))


def mx_host_synchronize() -> None:
    """Waits for every queued host-buffer call on the current device."""
    _check(_lib.mx_host_synchronize(), "mx_host_synchronize")


def mx_dequantize_host(elems: torch.Tensor, scales: torch.Tensor, out: torch.Tensor, fmt: int,
                       workspace: torch.Tensor, layout: int = MX_SCALES_SWIZZLED, queue: bool = False) -> None:
    assert not elems.is_cuda and not scales.is_cuda and not out.is_cuda and workspace.is_cuda
    shape = list(out.shape)
    o = _opts(_dtype_code(out.dtype), layout)
    fn = _lib.mx_dequantize_host_async if queue else _lib.mx_dequantize_host
    _check(fn(elems.data_ptr(), scales.data_ptr(), out.data_ptr(),
                                   _shape_arr(shape), len(shape), len(shape) - 1, fmt,
                                   ctypes.byref(o), workspace.data_ptr(), workspace.numel()),
           "mx_dequantize_host")


def mx_gemm_host_workspace_bytes(M: int, N: int, K: int, fmtA: int, fmtB: int) -> int:
    return int(_lib.mx_gemm_host_workspace_bytes(M, N, K, fmtA, fmtB))


def mx_gemm_host(A, sA, B, sB, C, M: int, N: int, K: int, fmtA: int, fmtB: int,
                 workspace: torch.Tensor) -> None:
    assert not A.is_cuda and not C.is_cuda and workspace.is_cuda
    o = _opts(MX_F32, MX_SCALES_SWIZZLED)
    _check(_lib.mx_gemm_host(A.data_ptr(), sA.data_ptr(), B.data_ptr(), sB.data_ptr(),
                             C.data_ptr(), M, N, K, fmtA, fmtB, ctypes.byref(o),
                             workspace.data_ptr(), workspace.numel()), "mx_gemm_host")
