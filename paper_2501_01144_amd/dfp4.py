"""Binding of libdfp4.so: the same calls as include/dfp4.h, taking torch tensors for device
memory and the current torch stream.  Argument marshalling only: every step of the path runs in
the HIP kernels.  Calls that allocate their result go through the native module _binding
(csrc/binding.cpp), which allocates and calls at once; calls into buffers of the caller's and the
rarer entry points go through ctypes.  There is no fallback; if a library is missing or a call
fails, an exception is raised.
"""
import ctypes
import os
from dataclasses import dataclass

import torch

BLOCK = 32
F32, BF16 = 0, 1
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdfp4.so")
_lib = None
_native = None                   # the module _binding, bound to the library


class Dfp4Error(RuntimeError):
    pass


class _CTensor(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("dialect", ctypes.c_void_p), ("exponent", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("K", ctypes.c_int64)]


class _CCache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("page_tokens", ctypes.c_int64),
                ("n_slots", ctypes.c_int64), ("kv_heads", ctypes.c_int64), ("head_dim", ctypes.c_int64), ("slot_chunks", ctypes.c_int64)]


class _CBatch(ctypes.Structure):
    _fields_ = [("cu_tokens", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("table", ctypes.c_void_p), ("slots", ctypes.c_void_p),
                ("batch", ctypes.c_int64), ("table_width", ctypes.c_int64), ("tokens", ctypes.c_int64), ("max_new", ctypes.c_int64),
                ("max_length", ctypes.c_int64)]


class _CPlan(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("tokens", ctypes.c_int64), ("k", ctypes.c_int64), ("experts", ctypes.c_int64)]


class _CExperts(ctypes.Structure):
    _fields_ = [("packed", ctypes.c_void_p), ("experts", ctypes.c_int64), ("rows", ctypes.c_int64), ("K", ctypes.c_int64), ("gated", ctypes.c_int)]


SYMBOLS = [
    "dfp4_quantize", "dfp4_quantize_b64", "dfp4_quantize_mse", "dfp4_quantize_t", "mxfp4_quantize_t", "dfp4_quantize_t_at", "dfp4_dequantize", "dfp4_gemm", "dfp4_gemm_batched", "dfp4_gemm_workspace_bytes", "dfp4_gemm_noalloc",
    "dfp4_quantize_block", "dfp4_dequantize_block", "dfp4_gemm_blocks",
    "dfp4_gemm_prepared_bytes", "dfp4_gemm_prepare", "mxfp4_gemm_prepare", "dfp4_gemm_prepared_workspace_bytes",
    "dfp4_gemm_prepared", "mxfp4_gemm_prepared", "dfp4_gemm_declined_tiles", "dfp4_gemm_path",
    "mxfp4_gemm_native", "dfp4_gemm_native", "dfp4_gemm_native_workspace_bytes", "dfp4_native_packed_bytes",
    "dfp4_quantize_native", "dfp4_native_pack", "mxfp4_native_pack", "dfp4_gemm_native_packed_w", "mxfp4_gemm_native_packed_w",
    "dfp4_gemm_native_packed", "mxfp4_gemm_native_packed", "dfp4_gemm_native_splitk_bytes",
    "dfp4_gemm_requant", "mxfp4_gemm_requant", "dfp4_gemm_requant_workspace_bytes", "dfp4_gemm_requant_batched",
    "mxfp4_quantize", "mxfp4_dequantize", "mxfp4_gemm", "dfp4_formatbook", "dfp4_strerror",
    "dfp4_paged_cell_bytes", "dfp4_paged_write", "dfp4_paged_read", "dfp4_paged_attention_workspace_bytes", "dfp4_paged_attention_rows", "dfp4_paged_attention",
    "dfp4_norm_rope",
    "dfp4_route", "dfp4_expert_plan_bytes", "dfp4_expert_plan", "dfp4_expert_weights_bytes", "dfp4_expert_weights", "dfp4_experts_workspace_bytes", "dfp4_experts_way",
    "dfp4_experts_up", "dfp4_experts_down", "dfp4_add_norm",
]


def lib_path():
    return _LIB_PATH


def load():
    """Load libdfp4.so (built by `python -m paper_2501_01144_amd.build`)."""
    global _lib, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise Dfp4Error(f"{_LIB_PATH} not found: build it with `python -m paper_2501_01144_amd.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    i64, vp, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    lib.dfp4_quantize.argtypes = [vp, i64, i64, i64, _CTensor, vp]
    lib.mxfp4_quantize.argtypes = [vp, i64, i64, i64, _CTensor, vp]
    lib.dfp4_quantize_mse.argtypes = [vp, i64, i64, i64, _CTensor, vp]
    lib.dfp4_quantize_b64.argtypes = [vp, i64, i64, i64, _CTensor, vp]
    lib.dfp4_quantize_t.argtypes = [vp, i64, i64, i64, _CTensor, vp]
    lib.mxfp4_quantize_t.argtypes = [vp, i64, i64, i64, _CTensor, vp]
    lib.dfp4_quantize_t_at.argtypes = [vp, i64, i64, i64, _CTensor, i64, vp]
    lib.dfp4_quantize_t_at.restype = ci
    lib.dfp4_dequantize.argtypes = [_CTensor, vp, ci, i64, vp]
    lib.mxfp4_dequantize.argtypes = [_CTensor, vp, ci, i64, vp]
    lib.dfp4_gemm.argtypes = [_CTensor, _CTensor, vp, ci, i64, vp, ctypes.c_size_t, vp]
    lib.mxfp4_gemm.argtypes = [_CTensor, _CTensor, vp, ci, i64, vp, ctypes.c_size_t, vp]
    lib.dfp4_gemm_batched.argtypes = [_CTensor, _CTensor, vp, ci, i64, i64, i64, i64, i64, vp,
                                      ctypes.c_size_t, vp]
    lib.dfp4_quantize_block.argtypes = [vp, i64, i64, i64, ci, _CTensor, vp]
    lib.dfp4_quantize_block.restype = ci
    lib.dfp4_dequantize_block.argtypes = [_CTensor, ci, vp, ci, i64, vp]
    lib.dfp4_dequantize_block.restype = ci
    lib.dfp4_gemm_blocks.argtypes = [_CTensor, ci, _CTensor, ci, vp, ci, i64, vp, ctypes.c_size_t, vp]
    lib.dfp4_gemm_blocks.restype = ci
    lib.dfp4_gemm_prepared_bytes.argtypes = [i64, i64, ci]
    lib.dfp4_gemm_prepared_bytes.restype = ctypes.c_size_t
    lib.dfp4_gemm_prepared_workspace_bytes.argtypes = [i64, i64, i64]
    lib.dfp4_gemm_prepared_workspace_bytes.restype = ctypes.c_size_t
    for name in ("dfp4_gemm_prepare", "mxfp4_gemm_prepare"):
        getattr(lib, name).argtypes = [_CTensor, ci, vp, ctypes.c_size_t, vp]
        getattr(lib, name).restype = ci
    for name in ("dfp4_gemm_prepared", "mxfp4_gemm_prepared"):
        getattr(lib, name).argtypes = [_CTensor, vp, _CTensor, vp, vp, ci, i64, vp, ctypes.c_size_t, vp]
        getattr(lib, name).restype = ci
    lib.dfp4_gemm_declined_tiles.argtypes = [vp, i64, i64, ctypes.POINTER(ctypes.c_uint32)]
    lib.dfp4_gemm_declined_tiles.restype = ci
    lib.dfp4_gemm_path.argtypes = [i64, i64, i64, i64, ci]
    lib.dfp4_gemm_path.restype = ci
    lib.dfp4_gemm_noalloc.argtypes = [_CTensor, _CTensor, vp, ci, i64, vp]
    lib.dfp4_gemm_noalloc.restype = ci
    lib.dfp4_gemm_workspace_bytes.argtypes = [i64, i64, i64]
    lib.dfp4_gemm_workspace_bytes.restype = ctypes.c_size_t
    lib.mxfp4_gemm_native.argtypes = [_CTensor, _CTensor, vp, ci, i64, vp, ctypes.c_size_t, vp]
    lib.mxfp4_gemm_native.restype = ci
    lib.dfp4_gemm_native.argtypes = [_CTensor, _CTensor, vp, ci, i64, vp, ctypes.c_size_t, vp]
    lib.dfp4_gemm_native.restype = ci
    lib.dfp4_gemm_native_workspace_bytes.argtypes = [i64, i64, i64]
    lib.dfp4_gemm_native_workspace_bytes.restype = ctypes.c_size_t
    lib.dfp4_native_packed_bytes.argtypes = [i64, i64]
    lib.dfp4_native_packed_bytes.restype = ctypes.c_size_t
    lib.dfp4_quantize_native.argtypes = [vp, i64, i64, i64, vp, ctypes.c_size_t, vp]
    lib.dfp4_quantize_native.restype = ci
    for name in ("dfp4_native_pack", "mxfp4_native_pack"):
        getattr(lib, name).argtypes = [_CTensor, vp, ctypes.c_size_t, vp]
        getattr(lib, name).restype = ci
    for name in ("dfp4_gemm_native_packed", "mxfp4_gemm_native_packed"):
        getattr(lib, name).argtypes = [vp, i64, vp, i64, i64, vp, ci, i64, vp, ctypes.c_size_t, vp]
        getattr(lib, name).restype = ci
    lib.dfp4_gemm_native_splitk_bytes.argtypes = [i64, i64, i64]
    lib.dfp4_gemm_native_splitk_bytes.restype = ctypes.c_size_t
    for name in ("dfp4_gemm_native_packed_w", "mxfp4_gemm_native_packed_w"):
        getattr(lib, name).argtypes = [_CTensor, vp, i64, vp, ci, i64, vp, ctypes.c_size_t, vp]
        getattr(lib, name).restype = ci
    lib.dfp4_gemm_requant.argtypes = [_CTensor, _CTensor, _CTensor, vp, ctypes.c_size_t, vp]
    lib.mxfp4_gemm_requant.argtypes = [_CTensor, _CTensor, _CTensor, vp, ctypes.c_size_t, vp]
    lib.dfp4_gemm_requant_batched.argtypes = [_CTensor, _CTensor, _CTensor, i64, i64, i64, vp, ctypes.c_size_t, vp]
    lib.dfp4_gemm_requant_batched.restype = ci
    lib.dfp4_gemm_requant.restype = ci
    lib.mxfp4_gemm_requant.restype = ci
    lib.dfp4_gemm_requant_workspace_bytes.argtypes = [i64, i64, i64]
    lib.dfp4_gemm_requant_workspace_bytes.restype = ctypes.c_size_t
    cf = ctypes.c_float
    lib.dfp4_paged_cell_bytes.argtypes = [i64]
    lib.dfp4_paged_cell_bytes.restype = ctypes.c_size_t
    lib.dfp4_paged_write.argtypes = [vp, i64, i64, vp, i64, i64, _CCache, _CBatch, vp]
    lib.dfp4_paged_write.restype = ci
    lib.dfp4_paged_read.argtypes = [_CCache, _CBatch, vp, vp, ci, vp]
    lib.dfp4_paged_read.restype = ci
    lib.dfp4_paged_attention_workspace_bytes.argtypes = [_CCache, _CBatch, i64, i64]
    lib.dfp4_paged_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.dfp4_paged_attention_rows.argtypes = [_CCache, _CBatch, i64, i64]
    lib.dfp4_paged_attention_rows.restype = ci
    lib.dfp4_paged_attention.argtypes = [vp, i64, i64, i64, _CCache, _CBatch, cf, cf, i64, vp, vp, i64, i64, vp, vp, ctypes.c_size_t, vp]
    lib.dfp4_paged_attention.restype = ci
    lib.dfp4_norm_rope.argtypes = [vp, i64, i64, i64, vp, i64, i64, i64, i64, i64, vp, vp, cf, vp, vp, i64, ci, vp, vp, vp]
    lib.dfp4_norm_rope.restype = ci
    lib.dfp4_route.argtypes = [vp, ci, i64, i64, i64, i64, ci, vp, i64, i64, i64, ci, cf, vp, vp, vp]
    lib.dfp4_route.restype = ci
    lib.dfp4_expert_plan_bytes.argtypes = [i64, i64, i64]
    lib.dfp4_expert_plan_bytes.restype = ctypes.c_size_t
    lib.dfp4_expert_plan.argtypes = [vp, _CPlan, vp]
    lib.dfp4_expert_plan.restype = ci
    lib.dfp4_expert_weights_bytes.argtypes = [i64, i64, i64, ci]
    lib.dfp4_expert_weights_bytes.restype = ctypes.c_size_t
    lib.dfp4_expert_weights.argtypes = [_CTensor, _CTensor, _CExperts, vp]
    lib.dfp4_expert_weights.restype = ci
    lib.dfp4_experts_workspace_bytes.argtypes = [_CPlan, _CExperts]
    lib.dfp4_experts_workspace_bytes.restype = ctypes.c_size_t
    lib.dfp4_experts_way.argtypes = [_CPlan, _CExperts, vp]
    lib.dfp4_experts_way.restype = ci
    lib.dfp4_experts_up.argtypes = [vp, i64, _CPlan, _CExperts, vp, vp, ctypes.c_size_t, vp]
    lib.dfp4_experts_up.restype = ci
    lib.dfp4_experts_down.argtypes = [vp, i64, _CPlan, _CExperts, vp, vp, ci, vp, ctypes.c_size_t, vp]
    lib.dfp4_experts_down.restype = ci
    lib.dfp4_add_norm.argtypes = [vp, i64, vp, i64, ci, vp, i64, i64, i64, vp, vp, cf, cf, vp, vp, vp]
    lib.dfp4_add_norm.restype = ci
    lib.dfp4_formatbook.argtypes = [vp]
    lib.dfp4_strerror.argtypes = [ci]
    lib.dfp4_strerror.restype = ctypes.c_char_p
    for name in ("dfp4_quantize", "dfp4_quantize_b64", "dfp4_quantize_mse", "dfp4_quantize_t", "mxfp4_quantize_t", "mxfp4_quantize", "dfp4_dequantize", "mxfp4_dequantize", "dfp4_gemm",
                 "mxfp4_gemm", "dfp4_gemm_batched", "dfp4_formatbook"):
        getattr(lib, name).restype = ci
    try:
        from . import _binding
    except ImportError as e:
        raise Dfp4Error(f"paper_2501_01144_amd/_binding.so: {e} (built by `python -m paper_2501_01144_amd.build`)") from e
    _binding.bind(_LIB_PATH, Dfp4Error)
    _lib, _native = lib, _binding
    return lib


def _calls():
    if _native is None:
        load()
    return _native


def _is_bf16(dtype):
    assert dtype in (torch.float32, torch.bfloat16)
    return dtype is torch.bfloat16


def _five(q):
    return q.codes, q.dialect, q.exponent, q.rows, q.K


def strerror(code):
    return load().dfp4_strerror(int(code)).decode()


def _check(rc, what):
    if rc != 0:
        raise Dfp4Error(f"{what} failed: {strerror(rc)} ({rc})")


def _stream():
    # the handle of torch.cuda.current_stream(), without the Python object around it (0.2 against 2.8 microseconds a call)
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr() if t is not None and t.numel() > 0 else 0) if t is not None \
        else ctypes.c_void_p(0)


def _steps(x):
    # strides of tokens and heads (a single one's is nobody's concern: torch leaves anything there)
    return tuple(x.stride(d) if x.shape[d] > 1 else 0 for d in (0, 1)) if x is not None else (0, 0)


@dataclass
class QTensor:
    """A quantized [rows, K] tensor on the device (layouts in include/dfp4.h)."""
    codes: torch.Tensor            # uint8 [rows, K/2]
    dialect: torch.Tensor          # uint8 [rows, K/32] or None (MXFP4)
    exponent: torch.Tensor         # uint8 [rows, K/32]
    rows: int
    K: int

    def c(self):
        return _CTensor(_ptr(self.codes).value, _ptr(self.dialect).value, _ptr(self.exponent).value,
                        self.rows, self.K)


def empty_qtensor(rows, K, device, mx=False):
    return QTensor(torch.empty((rows, K // 2), dtype=torch.uint8, device=device),
                   None if mx else torch.empty((rows, K // BLOCK), dtype=torch.uint8, device=device),
                   torch.empty((rows, K // BLOCK), dtype=torch.uint8, device=device), rows, K)


def _quantize(fn, what, x, out, mx):
    assert x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_cuda and x.stride(1) == 1
    rows, K = x.shape
    if out is None:
        out = empty_qtensor(rows, K, x.device, mx)
    ld = x.stride(0) if rows > 1 else K
    _check(fn(_ptr(x), rows, K, ld, out.c(), _stream()), what)
    return out


def quantize(x, out=None):
    """dfp4_quantize: bf16 [rows, K] (row stride allowed) -> QTensor."""
    if out is None:
        return QTensor(*_calls().quantize(x, 32, False))
    return _quantize(load().dfp4_quantize, "dfp4_quantize", x, out, False)


def quantize_b64(x, out=None):
    """dfp4_quantize_b64: blocks of 64 elements, output in the layout of the 32-element format."""
    return _quantize(load().dfp4_quantize_b64, "dfp4_quantize_b64", x, out, False)


def quantize_block(x, block, out=None):
    """dfp4_quantize_block: block size 16, 32 or 64.  Blocks of 16 carry dialect / exponent arrays [rows, K/16]."""
    if out is None:
        return QTensor(*_calls().quantize(x, block, False))
    assert x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_cuda and x.stride(1) == 1
    rows, K = x.shape
    ld = x.stride(0) if rows > 1 else K
    _check(load().dfp4_quantize_block(_ptr(x), rows, K, ld, block, out.c(), _stream()), "dfp4_quantize_block")
    return out


def dequantize_block(q, block, dtype=torch.float32, out=None):
    """dfp4_dequantize_block: the inverse of quantize_block for the same block size."""
    if out is None:
        out = torch.empty((q.rows, q.K), dtype=dtype, device=q.codes.device)
    ld = out.stride(0) if q.rows > 1 else q.K
    _check(load().dfp4_dequantize_block(q.c(), block, _ptr(out), F32 if out.dtype == torch.float32 else BF16, ld,
                                        _stream()), "dfp4_dequantize_block")
    return out


def gemm_blocks(a, block_a, w, block_w, dtype=torch.float32, out=None, workspace=None):
    """dfp4_gemm_blocks: product of operands quantized with block sizes block_a / block_w (16, 32 or 64)."""
    if out is None:
        out = torch.empty((a.rows, w.rows), dtype=dtype, device=a.codes.device)
    workspace, nbytes = _workspace(a.rows, w.rows, a.K, out.device, workspace)
    ldc = out.stride(0) if a.rows > 1 else w.rows
    _check(load().dfp4_gemm_blocks(a.c(), block_a, w.c(), block_w, _ptr(out), F32 if out.dtype == torch.float32 else BF16,
                                   ldc, _ptr(workspace), nbytes, _stream()), "dfp4_gemm_blocks")
    return out


def quantize_mse(x, out=None):
    """dfp4_quantize_mse: offline quantization, the dialect of each block chosen by squared error."""
    return _quantize(load().dfp4_quantize_mse, "dfp4_quantize_mse", x, out, False)


def _quantize_t(fn, what, x, out, mx):
    assert x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_cuda and x.stride(1) == 1
    rows, cols = x.shape
    if out is None:
        out = empty_qtensor(cols, rows, x.device, mx)
    ld = x.stride(0) if rows > 1 else cols
    _check(fn(_ptr(x), rows, cols, ld, out.c(), _stream()), what)
    return out


def quantize_t(x, out=None):
    """dfp4_quantize_t: bf16 [rows, cols] -> QTensor of x^T (blocks of 32 along the rows of x)."""
    return _quantize_t(load().dfp4_quantize_t, "dfp4_quantize_t", x, out, False)


def quantize_t_at(x, out, row_offset):
    """dfp4_quantize_t_at: quantize `x` [rows, cols] (rows a multiple of 32) along its rows into the
    quantized transpose `out` [cols, capacity] at token `row_offset`."""
    assert x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_cuda and x.stride(1) == 1
    rows, cols = x.shape
    ld = x.stride(0) if rows > 1 else cols
    _check(load().dfp4_quantize_t_at(_ptr(x), rows, cols, ld, out.c(), row_offset, _stream()), "dfp4_quantize_t_at")
    return out


def mxfp4_quantize_t(x, out=None):
    return _quantize_t(load().mxfp4_quantize_t, "mxfp4_quantize_t", x, out, True)


def mxfp4_quantize(x, out=None):
    if out is None:
        return QTensor(*_calls().quantize(x, 32, True))
    return _quantize(load().mxfp4_quantize, "mxfp4_quantize", x, out, True)


def _dequantize(fn, what, q, dtype, out):
    if out is None:
        out = torch.empty((q.rows, q.K), dtype=dtype, device=q.codes.device)
    assert out.dtype in (torch.float32, torch.bfloat16) and out.stride(1) == 1
    ld = out.stride(0) if q.rows > 1 else q.K
    _check(fn(q.c(), _ptr(out), F32 if out.dtype == torch.float32 else BF16, ld, _stream()), what)
    return out


def dequantize(q, dtype=torch.float32, out=None):
    if out is None:
        return _calls().dequantize(*_five(q), _is_bf16(dtype), False)
    return _dequantize(load().dfp4_dequantize, "dfp4_dequantize", q, dtype, out)


def mxfp4_dequantize(q, dtype=torch.float32, out=None):
    if out is None:
        return _calls().dequantize(*_five(q), _is_bf16(dtype), True)
    return _dequantize(load().mxfp4_dequantize, "mxfp4_dequantize", q, dtype, out)


def gemm_workspace_bytes(M, N, K):
    return int(load().dfp4_gemm_workspace_bytes(M, N, K))


def _workspace(M, N, K, device, workspace, batch=1):
    need = gemm_workspace_bytes(M, N, K) * batch
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, (workspace.numel() if workspace is not None else 0)


def _gemm(fn, what, a, w, dtype, out, workspace):
    if out is None:
        out = torch.empty((a.rows, w.rows), dtype=dtype, device=a.codes.device)
    assert out.dtype in (torch.float32, torch.bfloat16) and out.stride(1) == 1
    workspace, nbytes = _workspace(a.rows, w.rows, a.K, out.device, workspace)
    ldc = out.stride(0) if a.rows > 1 else w.rows
    _check(fn(a.c(), w.c(), _ptr(out), F32 if out.dtype == torch.float32 else BF16, ldc,
              _ptr(workspace), nbytes, _stream()), what)
    return out


def gemm(a, w, dtype=torch.float32, out=None, workspace=None):
    """dfp4_gemm: out[M, N] = A[M, K] * W[N, K]^T on quantized operands."""
    if out is None and workspace is None:
        return _calls().gemm(*_five(a), *_five(w), _is_bf16(dtype), False)
    return _gemm(load().dfp4_gemm, "dfp4_gemm", a, w, dtype, out, workspace)


@dataclass
class PreparedOperand:
    """A quantized tensor together with its prepared form (dfp4_gemm_prepare)."""
    q: "QTensor"
    buf: torch.Tensor              # uint8, private layout; None when nothing is prepared for this operand
    weight: bool
    mx: bool


def gemm_prepare(q, weight, mx=False, buf=None):
    """dfp4_gemm_prepare / mxfp4_gemm_prepare: the per-operand work of the GEMM, done once."""
    if buf is None:
        return PreparedOperand(q, _calls().gemm_prepare(*_five(q), bool(weight), bool(mx)), weight, mx)
    need = int(load().dfp4_gemm_prepared_bytes(q.rows, q.K, 1 if weight else 0))
    if need == 0:
        return PreparedOperand(q, None, weight, mx)
    fn = load().mxfp4_gemm_prepare if mx else load().dfp4_gemm_prepare
    _check(fn(q.c(), 1 if weight else 0, _ptr(buf), buf.numel(), _stream()), "gemm_prepare")
    return PreparedOperand(q, buf, weight, mx)


def gemm_prepared(a, w, dtype=torch.float32, out=None, workspace=None):
    """dfp4_gemm_prepared / mxfp4_gemm_prepared: a, w are PreparedOperands."""
    assert not a.weight and w.weight and a.mx == w.mx
    if out is None and workspace is None:
        return _calls().gemm_prepared(*_five(a.q), a.buf, *_five(w.q), w.buf, _is_bf16(dtype), bool(a.mx))
    if out is None:
        out = torch.empty((a.q.rows, w.q.rows), dtype=dtype, device=a.q.codes.device)
    assert out.dtype in (torch.float32, torch.bfloat16) and out.stride(1) == 1
    need = int(load().dfp4_gemm_prepared_workspace_bytes(a.q.rows, w.q.rows, a.q.K))
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=out.device)
    fn = load().mxfp4_gemm_prepared if a.mx else load().dfp4_gemm_prepared
    ldc = out.stride(0) if a.q.rows > 1 else w.q.rows
    _check(fn(a.q.c(), _ptr(a.buf), w.q.c(), _ptr(w.buf), _ptr(out), F32 if out.dtype == torch.float32 else BF16,
              ldc, _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream()), "gemm_prepared")
    return out


def gemm_declined_tiles(a):
    """dfp4_gemm_declined_tiles: tiles of products on this prepared A whose exponents spread beyond int32 sums (include/dfp4.h)."""
    n = ctypes.c_uint32(0)
    _check(load().dfp4_gemm_declined_tiles(_ptr(a.buf), a.q.rows, a.q.K, ctypes.byref(n)), "dfp4_gemm_declined_tiles")
    return int(n.value)


def gemm_path(M, N, K, batch=1, prepared=False):
    """dfp4_gemm_path: the kernel a product takes (0: the large kernel, 1..7: a shape of gemm_f8_kernel)."""
    return int(load().dfp4_gemm_path(M, N, K, batch, 1 if prepared else 0))


NOALLOC_SCRATCH_BYTES = 64 << 20


def gemm_noalloc(a, w, out):
    """dfp4_gemm_noalloc: dfp4_gemm on the library's own fixed scratch array; `out` must be given
    (nothing is allocated on either side of the boundary)."""
    assert out.dtype in (torch.float32, torch.bfloat16) and out.stride(1) == 1
    ldc = out.stride(0) if a.rows > 1 else w.rows
    _check(load().dfp4_gemm_noalloc(a.c(), w.c(), _ptr(out), F32 if out.dtype == torch.float32 else BF16, ldc,
                                    _stream()), "dfp4_gemm_noalloc")
    return out


def mxfp4_gemm(a, w, dtype=torch.float32, out=None, workspace=None):
    if out is None and workspace is None:
        return _calls().gemm(*_five(a), *_five(w), _is_bf16(dtype), True)
    return _gemm(load().mxfp4_gemm, "mxfp4_gemm", a, w, dtype, out, workspace)


def _gemm_requant(fn, what, a, w, out, workspace, mx):
    if out is None:
        out = empty_qtensor(a.rows, w.rows, a.codes.device, mx)
    need = int(load().dfp4_gemm_requant_workspace_bytes(a.rows, w.rows, a.K))
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=a.codes.device)
    _check(fn(a.c(), w.c(), out.c(), _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream()),
           what)
    return out


def gemm_requant(a, w, out=None, workspace=None):
    """dfp4_gemm_requant: quantize(bf16(A W^T)) in blocks of 32 along N -> QTensor [M, N]."""
    return _gemm_requant(load().dfp4_gemm_requant, "dfp4_gemm_requant", a, w, out, workspace, False)


def gemm_requant_batched(a, w, batch, M, N, out=None, workspace=None):
    """dfp4_gemm_requant_batched: a holds batch*M rows, w batch*N rows; returns the quantized [batch*M, N] result."""
    if out is None:
        out = empty_qtensor(batch * M, N, a.codes.device)
    need = int(load().dfp4_gemm_requant_workspace_bytes(M, N, a.K)) * batch
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=a.codes.device)
    ac, wc = a.c(), w.c()
    ac.rows, wc.rows = M, N
    _check(load().dfp4_gemm_requant_batched(ac, wc, out.c(), batch, M, N, _ptr(workspace), workspace.numel(), _stream()),
           "dfp4_gemm_requant_batched")
    return out


def mxfp4_gemm_requant(a, w, out=None, workspace=None):
    return _gemm_requant(load().mxfp4_gemm_requant, "mxfp4_gemm_requant", a, w, out, workspace, True)


def _gemm_native(fn, what, a, w, dtype, out, workspace):
    if out is None:
        out = torch.empty((a.rows, w.rows), dtype=dtype, device=a.codes.device)
    assert out.dtype in (torch.float32, torch.bfloat16) and out.stride(1) == 1
    need = int(load().dfp4_gemm_native_workspace_bytes(a.rows, w.rows, a.K))
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=out.device)
    ldc = out.stride(0) if a.rows > 1 else w.rows
    _check(fn(a.c(), w.c(), _ptr(out), F32 if out.dtype == torch.float32 else BF16, ldc, _ptr(workspace),
              workspace.numel() if workspace is not None else 0, _stream()), what)
    return out


def gemm_native(a, w, dtype=torch.float32, out=None, workspace=None):
    """dfp4_gemm_native: DialectFP4 product on the block-scaled matrix instruction (FP6 E2M3 operands)."""
    return _gemm_native(load().dfp4_gemm_native, "dfp4_gemm_native", a, w, dtype, out, workspace)


def mxfp4_gemm_native(a, w, dtype=torch.float32, out=None, workspace=None):
    """mxfp4_gemm_native: the MXFP4 product on the block-scaled matrix instruction (FP4 operands)."""
    return _gemm_native(load().mxfp4_gemm_native, "mxfp4_gemm_native", a, w, dtype, out, workspace)


@dataclass
class PackedWeights:
    """A quantized [rows, K] tensor in the matrix instruction's register order (dfp4_native_pack)."""
    buf: torch.Tensor
    rows: int
    K: int
    mx: bool


def native_pack(w, mx=False, buf=None):
    """dfp4_native_pack / mxfp4_native_pack: pack a quantized tensor (weights: once)."""
    if buf is None:
        return PackedWeights(_calls().native_pack(*_five(w), bool(mx)), w.rows, w.K, mx)
    fn = load().mxfp4_native_pack if mx else load().dfp4_native_pack
    _check(fn(w.c(), _ptr(buf), buf.numel(), _stream()), "native_pack")
    return PackedWeights(buf, w.rows, w.K, mx)


def quantize_native(x, buf=None):
    """dfp4_quantize_native: bf16 [rows, K] -> packed FP6 operand of the block-scaled matrix instruction."""
    if buf is None and x.numel() > 0:
        return PackedWeights(_calls().quantize_native(x), *x.shape, False)
    assert x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_cuda and x.stride(1) == 1
    rows, K = x.shape
    if buf is None:
        buf = torch.zeros(256, dtype=torch.uint8, device=x.device)
    ld = x.stride(0) if rows > 1 else K
    _check(load().dfp4_quantize_native(_ptr(x), rows, K, ld, _ptr(buf), buf.numel(), _stream()), "dfp4_quantize_native")
    return PackedWeights(buf, rows, K, False)


def gemm_native_packed_w(a, wp, dtype=torch.float32, out=None, workspace=None):
    """dfp4_gemm_native_packed_w / mxfp4_gemm_native_packed_w: A quantized, W packed beforehand."""
    if out is None:
        out = torch.empty((a.rows, wp.rows), dtype=dtype, device=a.codes.device)
    assert out.dtype in (torch.float32, torch.bfloat16) and out.stride(1) == 1 and a.K == wp.K
    need = int(load().dfp4_native_packed_bytes(a.rows, a.K)) + \
        int(load().dfp4_gemm_native_splitk_bytes(a.rows, wp.rows, a.K))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=out.device)
    fn = load().mxfp4_gemm_native_packed_w if wp.mx else load().dfp4_gemm_native_packed_w
    ldc = out.stride(0) if a.rows > 1 else wp.rows
    _check(fn(a.c(), _ptr(wp.buf), wp.rows, _ptr(out), F32 if out.dtype == torch.float32 else BF16, ldc,
              _ptr(workspace), workspace.numel(), _stream()), "gemm_native_packed_w")
    return out


def gemm_native_packed(ap, wp, dtype=torch.float32, out=None, workspace=None):
    """dfp4_gemm_native_packed / mxfp4_gemm_native_packed: both operands packed beforehand."""
    if out is None and workspace is None:
        assert ap.K == wp.K and ap.mx == wp.mx
        return _calls().gemm_native_packed(ap.buf, ap.rows, wp.buf, wp.rows, ap.K, _is_bf16(dtype), bool(wp.mx))
    if out is None:
        out = torch.empty((ap.rows, wp.rows), dtype=dtype, device=ap.buf.device)
    need = int(load().dfp4_gemm_native_splitk_bytes(ap.rows, wp.rows, ap.K))
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=out.device)
    assert out.dtype in (torch.float32, torch.bfloat16) and out.stride(1) == 1 and ap.K == wp.K and ap.mx == wp.mx
    fn = load().mxfp4_gemm_native_packed if wp.mx else load().dfp4_gemm_native_packed
    ldc = out.stride(0) if ap.rows > 1 else wp.rows
    _check(fn(_ptr(ap.buf), ap.rows, _ptr(wp.buf), wp.rows, ap.K, _ptr(out),
              F32 if out.dtype == torch.float32 else BF16, ldc, _ptr(workspace),
              workspace.numel() if workspace is not None else 0, _stream()), "gemm_native_packed")
    return out


def gemm_batched(a, w, batch, M, N, dtype=torch.float32, out=None, workspace=None):
    """dfp4_gemm_batched: a holds batch*M rows, w batch*N rows (problem after problem);
    out [batch, M, N]."""
    if out is None and workspace is None:
        return _calls().gemm_batched(*_five(a), *_five(w), batch, M, N, _is_bf16(dtype))
    if out is None:
        out = torch.empty((batch, M, N), dtype=dtype, device=a.codes.device)
    assert out.is_contiguous()
    ac, wc = a.c(), w.c()
    ac.rows, wc.rows = M, N
    workspace, nbytes = _workspace(M, N, a.K, out.device, workspace, batch)
    _check(load().dfp4_gemm_batched(ac, wc, _ptr(out), F32 if out.dtype == torch.float32 else BF16, N,
                                    batch, M, N, M * N, _ptr(workspace), nbytes, _stream()),
           "dfp4_gemm_batched")
    return out


def paged_write(k, v, cache, batch):
    """dfp4_paged_write: quantize the keys and values of the batch's new tokens, bf16 [tokens, kv_heads, head_dim] each (token and
    head strides allowed), into a kvcache.PagedCache; `batch` is a kvcache.PagedBatch."""
    _calls().paged_write(k, v, cache.at, batch.at)


def paged_read(cache, batch, tokens=None, dtype=torch.bfloat16):
    """dfp4_paged_read: the values that the cache stands for, k and v [tokens, kv_heads, head_dim], of the batch's tokens (`tokens`
    of them, by default batch.tokens, which waits for the device unless the batch was given the number)."""
    return _calls().paged_read(cache.at, batch.at, batch.tokens if tokens is None else tokens, _is_bf16(dtype), cache.pages)


def paged_attention(q, cache, batch, scale=None, softcap=0.0, window=0, slopes=None, return_lse=False, out=None, workspace=None):
    """dfp4_paged_attention: attention of the batch's new tokens, q bf16 [tokens, heads, head_dim], over the cached tokens of
    their sequences (these included: paged_write comes first).  scale: 1 / sqrt(head_dim) unless given; softcap, window: 0 is
    none; slopes: f32 [heads].  Returns out, bf16 like q, or (out, lse), lse f32 [tokens, heads]."""
    if scale is None:
        scale = cache.head_dim ** -0.5
    if out is None and workspace is None:
        return _calls().paged_attention(q, cache.at, batch.at, scale, softcap, window, slopes, bool(return_lse))
    tokens, heads, head_dim = q.shape
    if out is None:
        out = torch.empty((tokens, heads, head_dim), dtype=torch.bfloat16, device=q.device)
    for x in (q, out):
        assert x.dtype == torch.bfloat16 and x.is_cuda and x.stride(2) == 1 and x.shape == q.shape and head_dim == cache.head_dim
    assert slopes is None or (slopes.dtype == torch.float32 and slopes.is_cuda and slopes.is_contiguous() and slopes.numel() == heads)
    lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device) if return_lse else None
    b = batch.c(tokens)
    need = int(load().dfp4_paged_attention_workspace_bytes(cache.c, b, heads, window))
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    assert workspace is None or (workspace.is_cuda and workspace.is_contiguous())
    _check(load().dfp4_paged_attention(_ptr(q), *_steps(q), heads, cache.c, b, scale, softcap, window, _ptr(slopes), _ptr(out), *_steps(out),
                                       _ptr(lse), _ptr(workspace), workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                       _stream()),
           "dfp4_paged_attention")
    return (out, lse) if return_lse else out


def norm_rope(q, k, positions, inv_freq, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, out=None):
    """dfp4_norm_rope: norms of queries and keys per head (where a weight, f32 [head_dim], is given) and their rotation by
    position, in one pass.  q bf16 [tokens, heads, head_dim], k the same with its heads (or None); positions int32 [tokens];
    inv_freq f32 [rotary / 2] (None: no rotation, and positions may be None).  Returns q and k (out=(q, k): into these, which may be the inputs where those are contiguous)."""
    if out is None:
        return _calls().norm_rope(q, k, positions, inv_freq, q_weight, k_weight, eps, bool(interleaved))
    tokens, heads, head_dim = q.shape
    for w in (q_weight, k_weight):
        assert w is None or (w.dtype == torch.float32 and w.is_cuda and w.is_contiguous() and w.numel() == head_dim)
    assert positions is None or (positions.dtype == torch.int32 and positions.is_cuda and positions.is_contiguous() and positions.numel() == tokens)
    assert inv_freq is None or (inv_freq.dtype == torch.float32 and inv_freq.is_cuda and inv_freq.is_contiguous())
    q_out, k_out = out
    for x, y in ((q, q_out), (k, k_out)):
        assert (x is None and y is None) or (x.dtype == y.dtype == torch.bfloat16 and x.is_cuda and y.is_cuda and x.stride(2) == 1 and y.is_contiguous() and
                                             y.shape == x.shape and (x.shape[0], x.shape[2]) == (tokens, head_dim))
    _check(load().dfp4_norm_rope(_ptr(q), *_steps(q), heads, _ptr(k), *_steps(k), k.shape[1] if k is not None else 0, tokens, head_dim, _ptr(q_weight),
                                 _ptr(k_weight), eps, _ptr(positions), _ptr(inv_freq), 2 * inv_freq.numel() if inv_freq is not None else 0, 1 if interleaved else 0,
                                 _ptr(q_out), _ptr(k_out), _stream()), "dfp4_norm_rope")
    return q_out, k_out


def paged_attention_rows(cache, batch, tokens, heads, window=0):
    """dfp4_paged_attention_rows: the query rows a workgroup takes of a call with `tokens` new tokens, 16 or 256."""
    return int(load().dfp4_paged_attention_rows(cache.c, batch.c(tokens), heads, window))


def paged_cell_bytes(head_dim):
    return int(load().dfp4_paged_cell_bytes(head_dim))


def route(logits, k, score="softmax", bias=None, groups=1, kept=1, best=1, renormalize=True, scale=1.0):
    """dfp4_route: the k experts of every token and their weights, from logits f32 or bf16 [tokens, experts] (row stride allowed).
    score: "softmax" or "sigmoid"; bias: f32 [experts], added for the choice only; groups, kept, best: of `groups` groups of experts the
    `kept` with the largest sums of their `best` largest scores stay.  Returns ids int32 [tokens, k] and weights f32 [tokens, k]."""
    assert score in ("softmax", "sigmoid")
    return _calls().route(logits, k, score == "sigmoid", bias, groups, kept, best, bool(renormalize), scale)


class ExpertPlan:
    """The order of the experts' products (include/dfp4.h): offsets int32 [experts + 1], order and place int32 [tokens * k]."""
    __slots__ = ("data", "tokens", "k", "experts")

    def __init__(self, data, tokens, k, experts):
        self.data, self.tokens, self.k, self.experts = data, tokens, k, experts

    @property
    def offsets(self):
        return _calls().piece(self.data, 0, self.experts + 1)

    @property
    def order(self):
        return _calls().piece(self.data, self.experts + 1, self.tokens * self.k)

    @property
    def place(self):
        n = self.tokens * self.k
        return _calls().piece(self.data, self.experts + 1 + n, n)

    def c(self):
        return _CPlan(_ptr(self.data).value, self.tokens, self.k, self.experts)


def expert_plan(ids, experts):
    """dfp4_expert_plan: the pairs of tokens and experts, ids int32 [tokens, k], in the order of their experts.  Ids that are no
    expert (another GPU's) are absent."""
    return ExpertPlan(_calls().expert_plan(ids, experts), *ids.shape, experts)


@dataclass
class ExpertWeights:
    """The quantized matrices [rows, K] of `experts` experts in the matrix instruction's order (dfp4_expert_weights)."""
    buf: torch.Tensor
    experts: int
    rows: int
    K: int
    gated: bool

    def c(self):
        return _CExperts(_ptr(self.buf).value, self.experts, self.rows, self.K, 1 if self.gated else 0)


def expert_weights(w, experts, up=None, buf=None):
    """dfp4_expert_weights: lay out the weights of `experts` experts, w a QTensor [experts * rows, K], once; up: a second one of the
    same shape, w is then the gate (for experts_up)."""
    assert experts > 0 and w.rows % experts == 0 and (up is None or (up.rows, up.K) == (w.rows, w.K))
    rows = w.rows // experts
    need = int(load().dfp4_expert_weights_bytes(experts, rows, w.K, 0 if up is None else 1))
    if buf is None:
        buf = torch.empty(max(need, 256), dtype=torch.uint8, device=w.codes.device)
    assert buf.is_cuda and buf.is_contiguous()
    if buf.numel() * buf.element_size() < need:
        raise Dfp4Error(f"dfp4_expert_weights: {need} bytes are needed")
    out = ExpertWeights(buf, experts, rows, w.K, up is not None)
    _check(load().dfp4_expert_weights(w.c(), (w if up is None else up).c(), out.c(), _stream()), "dfp4_expert_weights")
    return out


def _product_workspace(plan, w, workspace, device):
    need = int(load().dfp4_experts_workspace_bytes(plan.c(), w.c()))
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    assert workspace is None or (workspace.is_cuda and workspace.is_contiguous())
    return workspace, workspace.numel() * workspace.element_size() if workspace is not None else 0


def experts_way(plan, w):
    """dfp4_experts_way: the rows that a workgroup of the product takes (1, 32, 64, 128 or 256), the waves that share K, and how rows are
    quantized (0 within, 1 before, 2 once a token)."""
    way = (ctypes.c_int32 * 3)()
    _check(load().dfp4_experts_way(plan.c(), w.c(), way), "dfp4_experts_way")
    return tuple(way)


def experts_up(x, plan, w, out=None, workspace=None):
    """dfp4_experts_up: h = silu(gate x) * (up x), bf16 [tokens * k, rows], for every pair of a token of x, bf16 [tokens, K] (row
    stride allowed), and one of its experts, in the plan's order.  Rows behind plan.offsets[-1] are not written."""
    if out is None and workspace is None:
        return _calls().experts_up(x, plan.data, plan.tokens, plan.k, plan.experts, w.buf, w.experts, w.rows, w.K, w.gated)
    if out is None:
        out = torch.empty((plan.tokens * plan.k, w.rows), dtype=torch.bfloat16, device=x.device)
    assert x.dtype == out.dtype == torch.bfloat16 and x.is_cuda and out.is_cuda and x.shape == (plan.tokens, w.K) and x.stride(1) == 1
    assert out.is_contiguous() and out.shape == (plan.tokens * plan.k, w.rows)
    workspace, n = _product_workspace(plan, w, workspace, x.device)
    _check(load().dfp4_experts_up(_ptr(x), x.stride(0) if plan.tokens > 1 else w.K, plan.c(), w.c(), _ptr(out), _ptr(workspace), n, _stream()), "dfp4_experts_up")
    return out


def experts_down(h, plan, w, weights, dtype=torch.bfloat16, out=None, workspace=None):
    """dfp4_experts_down: y [tokens, rows], the sum over a token's experts of the router's weights (f32 [tokens, k]) times W h, from
    h bf16 [tokens * k, K] in the plan's order (row stride allowed)."""
    if out is None and workspace is None:
        return _calls().experts_down(h, plan.data, plan.tokens, plan.k, plan.experts, w.buf, w.experts, w.rows, w.K, w.gated, weights, _is_bf16(dtype))
    if out is None:
        out = torch.empty((plan.tokens, w.rows), dtype=dtype, device=h.device)
    assert h.dtype == torch.bfloat16 and h.is_cuda and out.is_cuda and h.shape == (plan.tokens * plan.k, w.K) and h.stride(1) == 1
    assert out.is_contiguous() and out.shape == (plan.tokens, w.rows)
    assert weights.dtype == torch.float32 and weights.is_cuda and weights.is_contiguous() and weights.numel() == plan.tokens * plan.k
    workspace, n = _product_workspace(plan, w, workspace, h.device)
    _check(load().dfp4_experts_down(_ptr(h), h.stride(0) if h.shape[0] > 1 else w.K, plan.c(), w.c(), _ptr(weights), _ptr(out), BF16 if _is_bf16(out.dtype) else F32,
                                    _ptr(workspace), n, _stream()), "dfp4_experts_down")
    return out


def add_norm(y, residual, weight, post_weight=None, gate=None, scale=1.0, eps=1e-6, out=None):
    """dfp4_add_norm: r = residual + scale * gate * norm(y) and norm(r), in one pass.  y bf16 [tokens, dim], residual f32 or bf16 (row
    strides allowed); weight, post_weight f32 [dim] (post_weight None: y is not normalized); gate bf16 [dim] or [tokens, dim].
    Returns r, of the residual's type, and its norm, bf16 (out=(r, normed): into these, which may be residual and y where those are
    contiguous)."""
    if out is None:
        return _calls().add_norm(y, residual, weight, post_weight, gate, scale, eps)
    r_out, normed = out
    tokens, dim = y.shape
    assert y.dtype == normed.dtype == torch.bfloat16 and residual.dtype == r_out.dtype and residual.shape == r_out.shape == normed.shape == y.shape
    assert all(t.is_cuda and t.stride(1) == 1 for t in (y, residual)) and all(t.is_cuda and t.is_contiguous() for t in out)
    assert all(t is None or (t.dtype == torch.float32 and t.is_cuda and t.is_contiguous() and t.numel() == dim) for t in (weight, post_weight)) and weight is not None
    assert gate is None or (gate.dtype == torch.bfloat16 and gate.is_cuda and gate.stride(-1) == 1 and tuple(gate.shape) in ((dim,), (tokens, dim)))
    ld = lambda t: t.stride(0) if tokens > 1 else 0  # noqa: E731
    _check(load().dfp4_add_norm(_ptr(y), ld(y), _ptr(residual), ld(residual), BF16 if _is_bf16(residual.dtype) else F32, _ptr(gate),
                                0 if gate is None or gate.dim() == 1 else ld(gate), tokens, dim, _ptr(post_weight), _ptr(weight), scale, eps, _ptr(r_out), _ptr(normed),
                                _stream()), "dfp4_add_norm")
    return r_out, normed


def formatbook():
    """The library's formatbook as a 16 x 8 list of half-unit magnitudes."""
    buf = (ctypes.c_uint8 * 128)()
    _check(load().dfp4_formatbook(ctypes.cast(buf, ctypes.c_void_p)), "dfp4_formatbook")
    return [[int(buf[d * 8 + j]) for j in range(8)] for d in range(16)]
