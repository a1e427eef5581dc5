"""Python binding of the fp8_b200 C ABI (include/fp8_b200.h).

Argument marshalling only: every function checks dtypes, takes `data_ptr()` of
torch CUDA tensors, passes torch's current stream and calls the entry point of
the same name in ``libfp8_b200.so``.  There is no fallback: if the library is
not built, or a call returns a non-zero status, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

from . import _build

E4M3, E5M2 = 0, 1            # fp8_format
F32, BF16 = 0, 1             # fp8_wide
SATURATE, NOSAT = 0, 1       # fp8_overflow
MAJOR_K, MAJOR_MN = 0, 1     # fp8_major
ACC_SPLIT, ACC_FAST = 0, 1    # fp8_accumulate: bounded error for any data (default) / one accumulator
STORE_F32, STORE_BF16, STORE_E4M3, STORE_E5M2 = 0, 1, 2, 3                       # fp8_store
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4            # fp8_activation

EXPORTS = ["fp8_amax", "fp8_scale_from_amax", "fp8_quantize", "fp8_quantize_current",
           "fp8_quantize_current_workspace_bytes", "fp8_quantize_current_static", "fp8_dequantize", "fp8_fake_quantize",
           "fp8_scale_pow2_from_amax", "fp8_gemm", "fp8_gemm_fp8out", "fp8_amax_channels", "fp8_scales_from_amax",
           "fp8_quantize_channels", "fp8_quantize_transpose", "fp8_gemm_channel_scales", "fp8_gemm_batched",
           "fp8_gemm_splitk", "fp8_gemm_splitk_workspace",
           "fp8_gemm_epilogue", "fp8_gemm_gated", "fp8_gemm_gated_backward",
           "fp8_epilogue_backward", "fp8_epilogue_backward_workspace_bytes",
           "fp8_clip_plan_size", "fp8_clip_plan_fill", "fp8_grad_norm", "fp8_grad_clip",
           "fp8_async_status", "fp8_self_test_expire_wait", "fp8_sm_clock_probe", "fp8_status_string", "fp8_launch_count"]


class Fp8Error(RuntimeError):
    pass


class GemmDesc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("fa", ctypes.c_int), ("fb", ctypes.c_int), ("ma", ctypes.c_int), ("mb", ctypes.c_int),
                ("lda", ctypes.c_int64), ("ldb", ctypes.c_int64), ("ldd", ctypes.c_int64), ("out", ctypes.c_int), ("acc", ctypes.c_int)]


# The structures of the fused products as bytes, in the header's native layout: packing one and passing it costs a third of
# making the ctypes structure below, and single-token calls are short enough for that to show.
_pack_desc = struct.Struct("qqqiiiiqqqii").pack
_pack_epilogue = struct.Struct("iiiiiiPPPPqq").pack
_pack_gated = struct.Struct("iiiiPPq").pack


class Epilogue(ctypes.Structure):
    _fields_ = [("act", ctypes.c_int), ("store", ctypes.c_int), ("overflow", ctypes.c_int), ("bias_t", ctypes.c_int),
                ("residual_t", ctypes.c_int), ("pre_t", ctypes.c_int), ("scale_inv_b_vec", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("residual", ctypes.c_void_p), ("pre", ctypes.c_void_p), ("ldr", ctypes.c_int64), ("ldp", ctypes.c_int64)]


class Gated(ctypes.Structure):
    _fields_ = [("act", ctypes.c_int), ("store", ctypes.c_int), ("overflow", ctypes.c_int), ("gate_t", ctypes.c_int),
                ("gate", ctypes.c_void_p), ("up", ctypes.c_void_p), ("ldg", ctypes.c_int64)]


class ClipItem(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("x_t", ctypes.c_int), ("out_t", ctypes.c_int)]


class ClipSizes(ctypes.Structure):
    """fp8_clip_plan of the header"""
    _fields_ = [("count", ctypes.c_int64), ("chunks", ctypes.c_int64), ("table_bytes", ctypes.c_size_t), ("workspace_bytes", ctypes.c_size_t)]


_lib = None


def library_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = True) -> ctypes.CDLL:
    """Loads libfp8_b200.so (building it with nvcc when it is missing or stale)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    if build_if_missing and _build.is_stale():
        try:
            _build.build_library()
        except Exception as e:
            if not os.path.exists(path):     # stale is tolerable, missing is not
                raise Fp8Error("libfp8_b200.so is missing and could not be built: %s" % e) from e
    if not os.path.exists(path):
        raise Fp8Error("libfp8_b200.so not found at %s; run `python -m paper_2209_05433_b200._build`" % path)
    lib = ctypes.CDLL(path)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    lib.fp8_amax.restype = i32
    lib.fp8_amax.argtypes = [vp, i32, sz, vp, vp]
    lib.fp8_scale_from_amax.restype = i32
    lib.fp8_scale_from_amax.argtypes = [vp, i32, vp, vp, vp]
    lib.fp8_quantize.restype = i32
    lib.fp8_quantize.argtypes = [vp, i32, sz, i32, i32, vp, vp, vp, vp]
    lib.fp8_quantize_current.restype = i32
    lib.fp8_quantize_current.argtypes = [vp, i32, sz, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.fp8_quantize_current_workspace_bytes.restype = sz
    lib.fp8_quantize_current_workspace_bytes.argtypes = []
    lib.fp8_quantize_current_static.restype = i32
    lib.fp8_quantize_current_static.argtypes = [vp, i32, sz, i32, i32, vp, vp, vp, vp, vp]
    lib.fp8_dequantize.restype = i32
    lib.fp8_dequantize.argtypes = [vp, sz, i32, vp, vp, i32, vp]
    lib.fp8_fake_quantize.restype = i32
    lib.fp8_fake_quantize.argtypes = [vp, i32, sz, i32, i32, vp, vp, vp, vp]
    lib.fp8_scale_pow2_from_amax.restype = i32
    lib.fp8_scale_pow2_from_amax.argtypes = [vp, i32, vp, vp, vp]
    lib.fp8_gemm.restype = i32
    lib.fp8_gemm.argtypes = [ctypes.POINTER(GemmDesc), vp, vp, vp, vp, vp, vp, vp]
    lib.fp8_gemm_fp8out.restype = i32
    lib.fp8_gemm_fp8out.argtypes = [ctypes.POINTER(GemmDesc), vp, vp, vp, i32, i32, vp, vp, vp, vp, vp]
    i64 = ctypes.c_int64
    lib.fp8_amax_channels.restype = i32
    lib.fp8_amax_channels.argtypes = [vp, i32, i64, i64, i64, i32, vp, vp]
    lib.fp8_scales_from_amax.restype = i32
    lib.fp8_scales_from_amax.argtypes = [vp, i64, i32, i32, vp, vp, vp]
    lib.fp8_quantize_channels.restype = i32
    lib.fp8_quantize_channels.argtypes = [vp, i32, i64, i64, i64, i32, i32, i32, vp, vp, i64, vp]
    lib.fp8_quantize_transpose.restype = i32
    lib.fp8_quantize_transpose.argtypes = [vp, i32, i64, i64, i64, i32, i32, vp, vp, i64, vp, i64, vp, vp]
    lib.fp8_gemm_channel_scales.restype = i32
    lib.fp8_gemm_channel_scales.argtypes = [ctypes.POINTER(GemmDesc), vp, vp, vp, vp, vp, vp, vp]
    lib.fp8_gemm_batched.restype = i32
    lib.fp8_gemm_batched.argtypes = [ctypes.POINTER(GemmDesc), i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp]
    lib.fp8_gemm_splitk_workspace.restype = i32
    lib.fp8_gemm_splitk_workspace.argtypes = [ctypes.POINTER(GemmDesc), ctypes.POINTER(ctypes.c_int), ctypes.POINTER(sz)]
    lib.fp8_gemm_splitk.restype = i32
    lib.fp8_gemm_splitk.argtypes = [ctypes.POINTER(GemmDesc), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.fp8_gemm_epilogue.restype = i32
    lib.fp8_gemm_epilogue.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.fp8_gemm_gated.restype = i32
    lib.fp8_gemm_gated.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.fp8_gemm_gated_backward.restype = i32
    lib.fp8_gemm_gated_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.fp8_epilogue_backward_workspace_bytes.restype = sz
    lib.fp8_epilogue_backward_workspace_bytes.argtypes = [i64, i64]
    lib.fp8_epilogue_backward.restype = i32
    lib.fp8_epilogue_backward.argtypes = [i64, i64, i32, vp, i32, i64, vp, i32, i64, i32, i32, vp, vp, i64, vp, vp, vp, sz, vp]
    lib.fp8_clip_plan_size.restype = i32
    lib.fp8_clip_plan_size.argtypes = [ctypes.POINTER(ClipItem), i64, ctypes.POINTER(ClipSizes)]
    lib.fp8_clip_plan_fill.restype = i32
    lib.fp8_clip_plan_fill.argtypes = [ctypes.POINTER(ClipItem), ctypes.POINTER(ClipSizes), vp]
    lib.fp8_grad_norm.restype = i32
    lib.fp8_grad_norm.argtypes = [ctypes.POINTER(ClipSizes), vp, vp, vp, vp]
    lib.fp8_grad_clip.restype = i32
    lib.fp8_grad_clip.argtypes = [ctypes.POINTER(ClipSizes), vp, vp, ctypes.c_float, vp, vp]
    lib.fp8_async_status.restype = i32
    lib.fp8_async_status.argtypes = [ctypes.POINTER(ctypes.c_uint32)]
    lib.fp8_self_test_expire_wait.restype = i32
    lib.fp8_self_test_expire_wait.argtypes = [i32, ctypes.c_uint64, vp]
    lib.fp8_sm_clock_probe.restype = i32
    lib.fp8_sm_clock_probe.argtypes = [vp, ctypes.c_uint32, vp]
    lib.fp8_status_string.restype = ctypes.c_char_p
    lib.fp8_status_string.argtypes = [i32]
    lib.fp8_launch_count.restype = ctypes.c_uint64
    lib.fp8_launch_count.argtypes = []
    _lib = lib
    return lib


def _check(status: int, what: str) -> None:
    if status != 0:
        raise Fp8Error("%s failed: %s (status %d)" % (what, load().fp8_status_string(status).decode(), status))


def _stream() -> int:
    """handle of torch's current stream on the current device (the raw form: no Stream object is made per call)"""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _wide_of(t: torch.Tensor) -> int:
    dtype = t.dtype
    if dtype is torch.bfloat16:
        return BF16
    if dtype is torch.float32:
        return F32
    raise TypeError("wide tensors must be float32 or bfloat16, got %s" % dtype)


def _dev(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


def _scalar(t: torch.Tensor, name: str) -> int:
    if t.dtype is not torch.float32 or t.numel() != 1:
        raise TypeError("%s must be a one-element float32 CUDA tensor" % name)
    if not t.is_cuda:                       # one element is always contiguous
        raise ValueError("%s must be a CUDA tensor" % name)
    return t.data_ptr()


def fp8_amax(x: torch.Tensor, amax_out: torch.Tensor) -> None:
    _check(load().fp8_amax(_dev(x, "x"), _wide_of(x), x.numel(), _scalar(amax_out, "amax_out"), _stream()), "fp8_amax")


def fp8_scale_from_amax(amax: torch.Tensor, fmt: int, scale_out: torch.Tensor, scale_inv_out: torch.Tensor) -> None:
    _check(load().fp8_scale_from_amax(_scalar(amax, "amax"), fmt, _scalar(scale_out, "scale_out"),
                                      _scalar(scale_inv_out, "scale_inv_out"), _stream()), "fp8_scale_from_amax")


def fp8_quantize(x: torch.Tensor, fmt: int, scale: torch.Tensor, out: torch.Tensor,
                 overflow: int = SATURATE, amax_out: torch.Tensor | None = None) -> None:
    if out.dtype != torch.uint8 or out.numel() != x.numel():
        raise TypeError("out must be a uint8 tensor with as many elements as x")
    _check(load().fp8_quantize(_dev(x, "x"), _wide_of(x), x.numel(), fmt, overflow, _scalar(scale, "scale"),
                               _dev(out, "out"), None if amax_out is None else _scalar(amax_out, "amax_out"),
                               _stream()), "fp8_quantize")


_workspaces: dict = {}


def current_scaling_workspace(device: torch.device) -> torch.Tensor:
    """A zeroed workspace for fp8_quantize_current on `device`, made once per (device, stream).  A graph keeps the workspace
    of the stream it is captured on: where its replays may overlap plain calls of that stream, or another such graph's, pass
    each a workspace of its own.  One that is first needed inside a capture belongs to the graph, whose replays clear it."""
    key = (device.index if device.index is not None else torch.cuda.current_device(), _stream())
    ws = _workspaces.get(key)
    if ws is None:
        nbytes = int(load().fp8_quantize_current_workspace_bytes())
        ws = torch.zeros(max(nbytes, 16), dtype=torch.uint8, device=device)
        if not torch.cuda.is_current_stream_capturing():
            _workspaces[key] = ws
    return ws


def fp8_quantize_current(x: torch.Tensor, fmt: int, out: torch.Tensor, amax_out: torch.Tensor, scale_out: torch.Tensor,
                         scale_inv_out: torch.Tensor, overflow: int = SATURATE, workspace: torch.Tensor | None = None) -> None:
    if out.dtype != torch.uint8 or out.numel() != x.numel():
        raise TypeError("out must be a uint8 tensor with as many elements as x")
    ws = current_scaling_workspace(x.device) if workspace is None else workspace
    _check(load().fp8_quantize_current(_dev(x, "x"), _wide_of(x), x.numel(), fmt, overflow, _dev(out, "out"),
                                       _scalar(amax_out, "amax_out"), _scalar(scale_out, "scale_out"),
                                       _scalar(scale_inv_out, "scale_inv_out"), _dev(ws, "workspace"), _stream()),
           "fp8_quantize_current")


STATIC_MAX_ELEMENTS = 1 << 32


def fp8_quantize_current_static(x: torch.Tensor, fmt: int, out: torch.Tensor, amax_out: torch.Tensor,
                                scale_out: torch.Tensor, scale_inv_out: torch.Tensor, overflow: int = SATURATE) -> None:
    """fp8_quantize_current for callers that cannot allocate a workspace: the kernel's control words
    live in a small array inside the library.  Calls that overlap on the GPU race on that array."""
    if out.dtype != torch.uint8 or out.numel() != x.numel():
        raise TypeError("out must be a uint8 tensor with as many elements as x")
    _check(load().fp8_quantize_current_static(_dev(x, "x"), _wide_of(x), x.numel(), fmt, overflow, _dev(out, "out"),
                                              _scalar(amax_out, "amax_out"), _scalar(scale_out, "scale_out"),
                                              _scalar(scale_inv_out, "scale_inv_out"), _stream()),
           "fp8_quantize_current_static")


def fp8_dequantize(codes: torch.Tensor, fmt: int, scale_inv: torch.Tensor, out: torch.Tensor) -> None:
    if codes.dtype != torch.uint8 or out.numel() != codes.numel():
        raise TypeError("codes must be uint8 and out must have as many elements")
    _check(load().fp8_dequantize(_dev(codes, "codes"), codes.numel(), fmt, _scalar(scale_inv, "scale_inv"),
                                 _dev(out, "out"), _wide_of(out), _stream()), "fp8_dequantize")


def fp8_fake_quantize(x: torch.Tensor, fmt: int, scale: torch.Tensor, scale_inv: torch.Tensor, out: torch.Tensor,
                      overflow: int = SATURATE) -> None:
    if out.dtype != x.dtype or out.numel() != x.numel():
        raise TypeError("out must have the dtype and size of x")
    _check(load().fp8_fake_quantize(_dev(x, "x"), _wide_of(x), x.numel(), fmt, overflow, _scalar(scale, "scale"),
                                    _scalar(scale_inv, "scale_inv"), _dev(out, "out"), _stream()), "fp8_fake_quantize")


def fp8_scale_pow2_from_amax(amax: torch.Tensor, fmt: int, scale_out: torch.Tensor, scale_inv_out: torch.Tensor) -> None:
    _check(load().fp8_scale_pow2_from_amax(_scalar(amax, "amax"), fmt, _scalar(scale_out, "scale_out"),
                                           _scalar(scale_inv_out, "scale_inv_out"), _stream()), "fp8_scale_pow2_from_amax")


def fp8_gemm(A: torch.Tensor, fa: int, ma: int, B: torch.Tensor, fb: int, mb: int, D: torch.Tensor,
             scale_inv_a: torch.Tensor, scale_inv_b: torch.Tensor, amax_out: torch.Tensor | None = None,
             acc: int = ACC_SPLIT) -> None:
    """D[M,N] = (A[M,K] . B[K,N]) * scale_inv_a * scale_inv_b.

    A is a 2-D uint8 tensor stored [M,K] when ``ma == MAJOR_K`` or [K,M] when
    ``ma == MAJOR_MN``; B is stored [N,K] when ``mb == MAJOR_K`` or [K,N] when
    ``mb == MAJOR_MN``.  Row pitches are taken from the tensors' strides.
    ``acc``: ACC_SPLIT (default) adds partial sums every 2048 of K in registers (tolerance met on any data at any
    K); ACC_FAST keeps one accumulator over all of K (a few per cent faster; for zero-mean operands)."""
    d = _gemm_desc_2d(A, ma, B, mb, D, fa, fb, acc)
    _check(load().fp8_gemm(ctypes.byref(d), A.data_ptr(), B.data_ptr(), D.data_ptr(),
                           _scalar(scale_inv_a, "scale_inv_a"), _scalar(scale_inv_b, "scale_inv_b"),
                           None if amax_out is None else _scalar(amax_out, "amax_out"), _stream()), "fp8_gemm")


def _gemm_desc_2d(A, ma, B, mb, D, fa, fb, acc, codes_out=False):
    """descriptor of a 2-D product from the tensors' shapes and strides; D is a wide tensor, or uint8 codes"""
    return GemmDesc(*_gemm_fields(A, ma, B, mb, D, fa, fb, acc, codes_out))


def _gemm_fields(A, ma, B, mb, D, fa, fb, acc, codes_out=False):
    """the fields of that descriptor, checked"""
    if A.dtype is not torch.uint8 or B.dtype is not torch.uint8 or A.dim() != 2 or B.dim() != 2 or D.dim() != 2 or (codes_out and D.dtype is not torch.uint8):
        raise TypeError("A and B must be 2-D uint8 tensors and D a 2-D %s tensor" % ("uint8" if codes_out else "float32 or bfloat16"))
    lda, ia = A.stride()
    ldb, ib = B.stride()
    ldd, idd = D.stride()
    if ia != 1 or ib != 1 or idd != 1 or not (A.is_cuda and B.is_cuda and D.is_cuda):
        for t, name in ((A, "A"), (B, "B"), (D, "D")):
            if not t.is_cuda or t.stride(1) != 1:
                raise ValueError("%s must be a CUDA tensor with unit inner stride" % name)
    if ma == MAJOR_K:
        M, K = A.shape
    else:
        K, M = A.shape
    if mb == MAJOR_K:
        N, Kb = B.shape
    else:
        Kb, N = B.shape
    rows, cols = D.shape
    if K != Kb or rows != M or cols != N:
        raise ValueError("shape mismatch: A gives M=%d K=%d, B gives K=%d N=%d, D is %s" % (M, K, Kb, N, tuple(D.shape)))
    return M, N, K, fa, fb, ma, mb, lda, ldb, ldd, BF16 if codes_out else _wide_of(D), acc


def fp8_gemm_splitk_workspace(M: int, N: int, K: int) -> tuple[int, int]:
    """(number of K-slices, workspace bytes) fp8_gemm_splitk uses for this shape on the current device"""
    d = GemmDesc(M, N, K, E4M3, E4M3, MAJOR_K, MAJOR_K, K, K, N, BF16, ACC_FAST)
    splits, nbytes = ctypes.c_int(0), ctypes.c_size_t(0)
    _check(load().fp8_gemm_splitk_workspace(ctypes.byref(d), ctypes.byref(splits), ctypes.byref(nbytes)), "fp8_gemm_splitk_workspace")
    return splits.value, nbytes.value


def fp8_gemm_splitk(A: torch.Tensor, fa: int, ma: int, B: torch.Tensor, fb: int, mb: int, D: torch.Tensor,
                    scale_inv_a: torch.Tensor, scale_inv_b: torch.Tensor, workspace: torch.Tensor | None,
                    amax_out: torch.Tensor | None = None, acc: int = ACC_SPLIT) -> None:
    """fp8_gemm with the contraction cut into slices when the problem has few output tiles; ``workspace`` is a
    CUDA tensor of at least fp8_gemm_splitk_workspace(M, N, K)[1] bytes (None when that is 0)."""
    d = _gemm_desc_2d(A, ma, B, mb, D, fa, fb, acc)
    ws_ptr, ws_bytes = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    _check(load().fp8_gemm_splitk(ctypes.byref(d), A.data_ptr(), B.data_ptr(), D.data_ptr(),
                                  _scalar(scale_inv_a, "scale_inv_a"), _scalar(scale_inv_b, "scale_inv_b"),
                                  None if amax_out is None else _scalar(amax_out, "amax_out"), ws_ptr, ws_bytes, _stream()),
           "fp8_gemm_splitk")


def fp8_gemm_fp8out(A: torch.Tensor, fa: int, ma: int, B: torch.Tensor, fb: int, mb: int, D: torch.Tensor, fd: int,
                    scale_inv_a: torch.Tensor, scale_inv_b: torch.Tensor, scale_d: torch.Tensor,
                    amax_out: torch.Tensor | None = None, overflow: int = SATURATE, acc: int = ACC_SPLIT) -> None:
    """D[M,N] (uint8 codes of format fd) = encode((A . B) * scale_inv_a * scale_inv_b * scale_d); amax_out
    receives the amax of the result before the output scale and conversion.  Layout rules as fp8_gemm."""
    d = _gemm_desc_2d(A, ma, B, mb, D, fa, fb, acc, codes_out=True)
    _check(load().fp8_gemm_fp8out(ctypes.byref(d), A.data_ptr(), B.data_ptr(), D.data_ptr(), fd, overflow,
                                  _scalar(scale_inv_a, "scale_inv_a"), _scalar(scale_inv_b, "scale_inv_b"),
                                  _scalar(scale_d, "scale_d"), None if amax_out is None else _scalar(amax_out, "amax_out"),
                                  _stream()), "fp8_gemm_fp8out")


def _vec(t: torch.Tensor, count: int, name: str) -> int:
    if t.dtype != torch.float32 or t.numel() != count:
        raise TypeError("%s must be a float32 CUDA tensor with %d elements" % (name, count))
    return _dev(t, name)


def _rows2d(t: torch.Tensor, name: str):
    if t.dim() != 2 or not t.is_cuda or t.stride(1) != 1:
        raise ValueError("%s must be a 2-D CUDA tensor with unit inner stride" % name)
    return t.shape[0], t.shape[1], t.stride(0)


def fp8_amax_channels(x: torch.Tensor, axis: int, amax_vec: torch.Tensor) -> None:
    rows, cols, ld = _rows2d(x, "x")
    _check(load().fp8_amax_channels(x.data_ptr(), _wide_of(x), rows, cols, ld, axis,
                                    _vec(amax_vec, cols if axis == 0 else rows, "amax_vec"), _stream()), "fp8_amax_channels")


def fp8_scales_from_amax(amax_vec: torch.Tensor, fmt: int, scale_vec: torch.Tensor, scale_inv_vec: torch.Tensor, pow2: bool = False) -> None:
    n = amax_vec.numel()
    _check(load().fp8_scales_from_amax(_vec(amax_vec, n, "amax_vec"), n, fmt, 1 if pow2 else 0, _vec(scale_vec, n, "scale_vec"),
                                       _vec(scale_inv_vec, n, "scale_inv_vec"), _stream()), "fp8_scales_from_amax")


def fp8_quantize_channels(x: torch.Tensor, axis: int, fmt: int, scale_vec: torch.Tensor, out: torch.Tensor, overflow: int = SATURATE) -> None:
    rows, cols, ld = _rows2d(x, "x")
    orows, ocols, ld_out = _rows2d(out, "out")
    if out.dtype != torch.uint8 or (orows, ocols) != (rows, cols):
        raise TypeError("out must be a uint8 tensor of the shape of x")
    _check(load().fp8_quantize_channels(x.data_ptr(), _wide_of(x), rows, cols, ld, axis, fmt, overflow,
                                        _vec(scale_vec, cols if axis == 0 else rows, "scale_vec"), out.data_ptr(), ld_out, _stream()),
           "fp8_quantize_channels")


def fp8_quantize_transpose(x: torch.Tensor, fmt: int, scale: torch.Tensor, out: torch.Tensor | None, out_t: torch.Tensor,
                           amax_out: torch.Tensor | None = None, overflow: int = SATURATE) -> None:
    """codes of the 2-D tensor x in both orientations from one pass: ``out`` [rows, cols] (or None) and
    ``out_t`` [cols, rows]; ``amax_out`` optionally receives amax of x."""
    rows, cols, ldx = _rows2d(x, "x")
    trows, tcols, ldt = _rows2d(out_t, "out_t")
    if out_t.dtype != torch.uint8 or (trows, tcols) != (cols, rows):
        raise TypeError("out_t must be a uint8 tensor of the transposed shape of x")
    ldo = 0
    if out is not None:
        orows, ocols, ldo = _rows2d(out, "out")
        if out.dtype != torch.uint8 or (orows, ocols) != (rows, cols):
            raise TypeError("out must be a uint8 tensor of the shape of x")
    _check(load().fp8_quantize_transpose(x.data_ptr(), _wide_of(x), rows, cols, ldx, fmt, overflow, _scalar(scale, "scale"),
                                         None if out is None else out.data_ptr(), ldo, out_t.data_ptr(), ldt,
                                         None if amax_out is None else _scalar(amax_out, "amax_out"), _stream()),
           "fp8_quantize_transpose")


def fp8_gemm_channel_scales(A: torch.Tensor, fa: int, ma: int, B: torch.Tensor, fb: int, mb: int, D: torch.Tensor,
                            scale_inv_a: torch.Tensor, scale_inv_b_vec: torch.Tensor, amax_out: torch.Tensor | None = None,
                            acc: int = ACC_SPLIT) -> None:
    """fp8_gemm with one inverse scale per column of B (per output channel)."""
    d = _gemm_desc_2d(A, ma, B, mb, D, fa, fb, acc)
    _check(load().fp8_gemm_channel_scales(ctypes.byref(d), A.data_ptr(), B.data_ptr(), D.data_ptr(),
                                          _scalar(scale_inv_a, "scale_inv_a"), _vec(scale_inv_b_vec, d.N, "scale_inv_b_vec"),
                                          None if amax_out is None else _scalar(amax_out, "amax_out"), _stream()),
           "fp8_gemm_channel_scales")


def fp8_gemm_batched(A: torch.Tensor, fa: int, ma: int, B: torch.Tensor, fb: int, mb: int, D: torch.Tensor,
                     scale_inv_a: torch.Tensor, scale_inv_b: torch.Tensor, amax_out: torch.Tensor | None = None,
                     acc: int = ACC_SPLIT) -> None:
    """Batched fp8_gemm: A, B are 3-D uint8 tensors [batch, rows, cols] (layouts per member as fp8_gemm), D is
    [batch, M, N]; the batch strides are taken from the tensors."""
    if A.dtype != torch.uint8 or B.dtype != torch.uint8 or A.dim() != 3 or B.dim() != 3 or D.dim() != 3:
        raise TypeError("A and B must be 3-D uint8 tensors and D a 3-D tensor")
    for t, name in ((A, "A"), (B, "B"), (D, "D")):
        if not t.is_cuda or t.stride(2) != 1:
            raise ValueError("%s must be a CUDA tensor with unit inner stride" % name)
    batch = A.shape[0]
    M, K = (A.shape[1], A.shape[2]) if ma == MAJOR_K else (A.shape[2], A.shape[1])
    Kb, N = (B.shape[2], B.shape[1]) if mb == MAJOR_K else (B.shape[1], B.shape[2])
    if K != Kb or B.shape[0] != batch or tuple(D.shape) != (batch, M, N):
        raise ValueError("shape mismatch")
    d = GemmDesc(M, N, K, fa, fb, ma, mb, A.stride(1), B.stride(1), D.stride(1), _wide_of(D), acc)
    _check(load().fp8_gemm_batched(ctypes.byref(d), batch, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0),
                                   D.data_ptr(), D.stride(0), _scalar(scale_inv_a, "scale_inv_a"), _scalar(scale_inv_b, "scale_inv_b"),
                                   None if amax_out is None else _scalar(amax_out, "amax_out"), _stream()), "fp8_gemm_batched")


def _wide2d(t: torch.Tensor, shape, name: str) -> int:
    """fp8_wide of a 2-D float32 or bfloat16 CUDA tensor of the given shape with unit inner stride"""
    if t.shape != shape:
        raise ValueError("%s must be a 2-D tensor of shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if not t.is_cuda or t.stride(1) != 1:
        raise ValueError("%s must be a CUDA tensor with unit inner stride" % name)
    return _wide_of(t)


_amax_workspaces: dict = {}


def _amax_args(amax_out: torch.Tensor | None) -> tuple:
    """(amax address, workspace address, stream) of a fused product: the workspace takes the place of a launch that would
    zero the amax, and is kept per (device, stream).  A captured call takes none: a graph may be replayed on any stream,
    beside plain calls on the stream it was captured on, and the two words must not be shared by calls that overlap."""
    stream = _stream()
    if amax_out is None:
        return None, None, stream
    ptr, key = _scalar(amax_out, "amax_out"), (amax_out.device.index, stream)
    if torch.cuda.is_current_stream_capturing():
        return ptr, None, stream
    ws = _amax_workspaces.get(key)
    if ws is None:
        ws = torch.zeros(16, dtype=torch.uint8, device=amax_out.device)
        _amax_workspaces[key] = ws
    return ptr, ws.data_ptr(), stream


def _store_of(D: torch.Tensor, fd: int | None, scale_d: torch.Tensor | None) -> tuple[int, int | None]:
    """(fp8_store, address of the output scale) of an output tensor: wide, or uint8 codes of format fd"""
    if D.dtype is torch.uint8:
        if fd is None or scale_d is None:
            raise TypeError("a uint8 output needs its format fd and its scale_d")
        if fd not in (E4M3, E5M2):
            raise Fp8Error("fd must be E4M3 or E5M2, got %r" % (fd,))
        return STORE_E4M3 + fd, _scalar(scale_d, "scale_d")
    if fd is not None or scale_d is not None:
        raise TypeError("fd and scale_d go with a uint8 output, not %s" % D.dtype)
    return _wide_of(D), None


def fp8_gemm_epilogue(A: torch.Tensor, fa: int, ma: int, B: torch.Tensor, fb: int, mb: int, D: torch.Tensor,
                      scale_inv_a: torch.Tensor, scale_inv_b: torch.Tensor, act: int = ACT_NONE, bias: torch.Tensor | None = None,
                      residual: torch.Tensor | None = None, pre: torch.Tensor | None = None, fd: int | None = None,
                      scale_d: torch.Tensor | None = None, amax_out: torch.Tensor | None = None, overflow: int = SATURATE,
                      acc: int = ACC_SPLIT) -> None:
    """D = act((A . B) * scale_inv_a * scale_inv_b + bias) + residual, one kernel.  Operands as fp8_gemm; ``scale_inv_b``
    has one element or one per column of B.  D is float32, bfloat16, or uint8 codes of format ``fd`` made with ``scale_d``.
    ``pre`` (wide) receives the value before the activation, which fp8_epilogue_backward reads."""
    fields = _gemm_fields(A, ma, B, mb, D, fa, fb, acc, D.dtype is torch.uint8)
    N = fields[1]
    store, scale_d_ptr = _store_of(D, fd, scale_d)
    bias_t = residual_t = pre_t = BF16
    bias_ptr = residual_ptr = pre_ptr = sb_vec = 0
    ldr = ldp = 0
    if scale_inv_b.numel() == 1:
        sb = _scalar(scale_inv_b, "scale_inv_b")
    else:
        sb, sb_vec = None, _vec(scale_inv_b, N, "scale_inv_b")
    if bias is not None:
        if bias.numel() != N:
            raise ValueError("bias must have %d elements" % N)
        bias_t, bias_ptr = _wide_of(bias), _dev(bias, "bias")
    if residual is not None:
        residual_t, residual_ptr, ldr = _wide2d(residual, D.shape, "residual"), residual.data_ptr(), residual.stride(0)
    if pre is not None:
        pre_t, pre_ptr, ldp = _wide2d(pre, D.shape, "pre"), pre.data_ptr(), pre.stride(0)
    e = _pack_epilogue(act, store, overflow, bias_t, residual_t, pre_t, sb_vec, bias_ptr, residual_ptr, pre_ptr, ldr, ldp)
    _check((_lib or load()).fp8_gemm_epilogue(_pack_desc(*fields), e, A.data_ptr(), B.data_ptr(), D.data_ptr(),
                                              _scalar(scale_inv_a, "scale_inv_a"), sb, scale_d_ptr, *_amax_args(amax_out)), "fp8_gemm_epilogue")


def _gate_of(gate, up, shape, act, store, overflow) -> bytes:
    if (gate is None) != (up is None):
        raise ValueError("gate and up go together")
    if gate is None:
        return _pack_gated(act, store, overflow, BF16, 0, 0, 0)
    gate_t, ldg = _wide2d(gate, shape, "gate"), gate.stride(0)
    if _wide2d(up, shape, "up") != gate_t or up.stride(0) != ldg:
        raise ValueError("gate and up must have one dtype and one row pitch")
    return _pack_gated(act, store, overflow, gate_t, gate.data_ptr(), up.data_ptr(), ldg)


def fp8_gemm_gated(A: torch.Tensor, fa: int, ma: int, Bg: torch.Tensor, Bu: torch.Tensor, fb: int, mb: int, H: torch.Tensor,
                   scale_inv_a: torch.Tensor, scale_inv_bg: torch.Tensor, scale_inv_bu: torch.Tensor, act: int = ACT_SILU,
                   gate: torch.Tensor | None = None, up: torch.Tensor | None = None, fd: int | None = None,
                   scale_d: torch.Tensor | None = None, amax_out: torch.Tensor | None = None, overflow: int = SATURATE,
                   acc: int = ACC_SPLIT) -> None:
    """H = act((A . Bg) * sa * sbg) * ((A . Bu) * sa * sbu), one kernel.  Bg and Bu have one shape, layout and row pitch
    (they may be the halves of one matrix); H as D of fp8_gemm_epilogue; ``gate`` and ``up`` (wide, optional) receive the
    two products for the backward pass."""
    if Bg.shape != Bu.shape or Bg.stride() != Bu.stride() or Bu.dtype != Bg.dtype or not Bu.is_cuda:
        raise ValueError("Bg and Bu must be CUDA tensors of one dtype, one shape and one row pitch")
    fields = _gemm_fields(A, ma, Bg, mb, H, fa, fb, acc, H.dtype is torch.uint8)
    store, scale_d_ptr = _store_of(H, fd, scale_d)
    w = _gate_of(gate, up, H.shape, act, store, overflow)
    _check((_lib or load()).fp8_gemm_gated(_pack_desc(*fields), w, A.data_ptr(), Bg.data_ptr(), Bu.data_ptr(), H.data_ptr(),
                                 _scalar(scale_inv_a, "scale_inv_a"), _scalar(scale_inv_bg, "scale_inv_bg"),
                                 _scalar(scale_inv_bu, "scale_inv_bu"), scale_d_ptr, *_amax_args(amax_out)), "fp8_gemm_gated")


def fp8_gemm_gated_backward(A: torch.Tensor, fa: int, ma: int, B: torch.Tensor, fb: int, mb: int, gate: torch.Tensor, up: torch.Tensor,
                            dG: torch.Tensor, dU: torch.Tensor, scale_inv_a: torch.Tensor, scale_inv_b: torch.Tensor,
                            act: int = ACT_SILU, fd: int | None = None, scale_d: torch.Tensor | None = None,
                            amax_out: torch.Tensor | None = None, overflow: int = SATURATE, acc: int = ACC_SPLIT) -> None:
    """dh = (A . B) * sa * sb with A the codes of dY and B the down weights seen as [d_model, inner];
    dG = dh * up * act'(gate), dU = dh * act(gate): two outputs of one dtype and row pitch (halves of one [M, 2 N] tensor),
    converted with one ``scale_d`` and covered by one ``amax_out``."""
    if dG.shape != dU.shape or dG.stride() != dU.stride() or dG.dtype != dU.dtype or not dU.is_cuda:
        raise ValueError("dG and dU must be CUDA tensors of one dtype, one shape and one row pitch")
    fields = _gemm_fields(A, ma, B, mb, dG, fa, fb, acc, dG.dtype is torch.uint8)
    store, scale_d_ptr = _store_of(dG, fd, scale_d)
    if gate is None or up is None:
        raise ValueError("gate and up are required")
    w = _gate_of(gate, up, dG.shape, act, store, overflow)
    _check((_lib or load()).fp8_gemm_gated_backward(_pack_desc(*fields), w, A.data_ptr(), B.data_ptr(), dG.data_ptr(), dU.data_ptr(),
                                          _scalar(scale_inv_a, "scale_inv_a"), _scalar(scale_inv_b, "scale_inv_b"), scale_d_ptr,
                                          *_amax_args(amax_out)), "fp8_gemm_gated_backward")


_backward_workspaces: dict = {}


def epilogue_backward_workspace(device: torch.device, M: int, N: int) -> torch.Tensor:
    """A workspace for fp8_epilogue_backward on `device`, kept per (device, stream) and grown as needed.  While a graph is
    captured it is a buffer of the graph's own, cleared by every replay: the kept one may be replaced by a larger one while
    the graph lives, and the graph may be replayed beside calls that use the kept one."""
    need = int(load().fp8_epilogue_backward_workspace_bytes(M, N))
    if torch.cuda.is_current_stream_capturing():
        ws = torch.empty(need, dtype=torch.uint8, device=device)
        ws[:int(load().fp8_epilogue_backward_workspace_bytes(0, 0))].zero_()     # the counters; partial sums are written before they are read
        return ws
    key = (device.index if device.index is not None else torch.cuda.current_device(), _stream())
    ws = _backward_workspaces.get(key)
    if ws is None or ws.numel() < need:
        ws = _backward_workspaces[key] = torch.zeros(need, dtype=torch.uint8, device=device)
    return ws


def fp8_epilogue_backward(dy: torch.Tensor, pre: torch.Tensor | None, out: torch.Tensor, act: int = ACT_NONE, fd: int | None = None,
                          scale_d: torch.Tensor | None = None, dbias: torch.Tensor | None = None, amax_out: torch.Tensor | None = None,
                          overflow: int = SATURATE, workspace: torch.Tensor | None = None) -> None:
    """out = dy * act'(pre), wide or as codes of format ``fd`` made with ``scale_d``; ``dbias`` (float32, one element per
    column) receives its column sums.  ``pre`` is what fp8_gemm_epilogue kept (None goes with ACT_NONE)."""
    if dy.dim() != 2 or out.dim() != 2:
        raise ValueError("dy and out must be 2-D tensors")
    M, N = dy.shape
    dy_t = _wide2d(dy, (M, N), "dy")
    if tuple(out.shape) != (M, N) or not out.is_cuda or out.stride(1) != 1:
        raise ValueError("out must be a CUDA tensor of the shape of dy with unit inner stride")
    store, scale_ptr = _store_of(out, fd, scale_d)
    pre_t, pre_ptr, ldp = (BF16, None, N) if pre is None else (_wide2d(pre, (M, N), "pre"), pre.data_ptr(), pre.stride(0))
    ws_ptr, ws_bytes, dbias_ptr = None, 0, None
    if dbias is not None:
        dbias_ptr = _vec(dbias, N, "dbias")
    if dbias is not None or (amax_out is not None and (workspace is not None or not torch.cuda.is_current_stream_capturing())):
        ws = epilogue_backward_workspace(dy.device, M, N) if workspace is None else workspace
        ws_ptr, ws_bytes = _dev(ws, "workspace"), ws.numel() * ws.element_size()
    _check(load().fp8_epilogue_backward(M, N, act, dy.data_ptr(), dy_t, dy.stride(0), pre_ptr, pre_t, ldp, store, overflow, scale_ptr,
                                        out.data_ptr(), out.stride(0), dbias_ptr,
                                        None if amax_out is None else _scalar(amax_out, "amax_out"), ws_ptr, ws_bytes, _stream()),
           "fp8_epilogue_backward")


class ClipPlan:
    """The tensors that fp8_grad_norm and fp8_grad_clip go over, laid out once: their table and workspace on the device.
    ``outs`` (same sizes, float32 or bfloat16 each) receive the clipped gradients; None clips in place.  The plan goes by the
    tensors' addresses and keeps them alive: gradients that live in other tensors after a step (``zero_grad`` drops them by
    default; ``set_to_none=False`` keeps them) need a new plan, whose making copies its table and waits for the stream (288
    tensors: 430 us, 12 of 67M elements: 80 us).  It must outlive the graphs that captured calls with it.  The norm is that of
    these tensors alone, not of other ranks'.  Calls that may overlap on the GPU need plans of their own."""

    def __init__(self, grads: list[torch.Tensor], outs: list[torch.Tensor] | None = None):
        self.grads, self.outs = list(grads), list(grads if outs is None else outs)
        if len(self.grads) != len(self.outs):
            raise ValueError("grads and outs must have one length")
        items = (ClipItem * max(1, len(self.grads)))()
        for it, x, o in zip(items, self.grads, self.outs):
            if x.numel() != o.numel() or x.device != o.device or x.device != self.grads[0].device:
                raise ValueError("each output must have the size of its gradient, and all tensors one device")
            it.x, it.x_t, it.n = _dev(x, "gradient"), _wide_of(x), x.numel()
            it.out, it.out_t = _dev(o, "output"), _wide_of(o)
        self.sizes = ClipSizes()
        _check(load().fp8_clip_plan_size(items, len(self.grads), ctypes.byref(self.sizes)), "fp8_clip_plan_size")
        device = self.grads[0].device if self.grads else torch.device("cuda", torch.cuda.current_device())
        host = torch.zeros(max(16, self.sizes.table_bytes), dtype=torch.uint8)
        _check(load().fp8_clip_plan_fill(items, ctypes.byref(self.sizes), host.data_ptr()), "fp8_clip_plan_fill")
        # the copy from pageable memory returns when the stream has done it, and with it the zeros: any stream may use the plan
        self.workspace = torch.zeros(self.sizes.workspace_bytes, dtype=torch.uint8, device=device)
        self.table = host.to(device)
        self._call = (ctypes.byref(self.sizes), self.table.data_ptr(), self.workspace.data_ptr())


def fp8_grad_norm(plan: ClipPlan, norm_out: torch.Tensor) -> None:
    """Global 2-norm of the plan's gradients."""
    _check(load().fp8_grad_norm(*plan._call, _scalar(norm_out, "norm_out"), _stream()), "fp8_grad_norm")


def fp8_grad_clip(plan: ClipPlan, max_norm: float, norm_out: torch.Tensor) -> None:
    """Global 2-norm of the plan's gradients, and outs = grads * min(1, max_norm / norm)."""
    _check(load().fp8_grad_clip(*plan._call, max_norm, _scalar(norm_out, "norm_out"), _stream()), "fp8_grad_clip")


TIMEOUT = 7                                   # FP8_ERR_TIMEOUT
WAIT_MBARRIER, WAIT_GRID_BARRIER = 0, 1       # fp8_wait_kind


def fp8_async_status() -> tuple[int, int]:
    """(status, detail) of the device-side error latch; synchronises the device.  After a time-out the cached
    workspaces are cleared again (the kernel leaves them zeroed; this costs nothing and does not
    rely on it)."""
    detail = ctypes.c_uint32(0)
    s = load().fp8_async_status(ctypes.byref(detail))
    if int(s) == TIMEOUT:
        for ws in (*_workspaces.values(), *_amax_workspaces.values(), *_backward_workspaces.values()):
            ws.zero_()
        torch.cuda.synchronize()
    return int(s), int(detail.value)


def fp8_self_test_expire_wait(which: int, limit_cycles: int = 2_000_000) -> None:
    """Makes one bounded device-side wait run out on purpose (about a millisecond by default); see the header."""
    _check(load().fp8_self_test_expire_wait(which, limit_cycles, _stream()), "fp8_self_test_expire_wait")


def fp8_sm_clock_probe(out: torch.Tensor, duration_us: int = 200) -> None:
    """Enqueues the one-warp clock probe on the current stream; `out` is a 2-element int64 CUDA tensor that receives
    (SM clocks, nanoseconds) of a window of `duration_us` microseconds."""
    if out.dtype != torch.int64 or out.numel() != 2:
        raise TypeError("out must be a 2-element int64 CUDA tensor")
    _check(load().fp8_sm_clock_probe(_dev(out, "out"), duration_us, _stream()), "fp8_sm_clock_probe")


def fp8_launch_count() -> int:
    return int(load().fp8_launch_count())
