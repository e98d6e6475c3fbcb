"""Binding of include/lora_mx.h: the multi-LoRA layer on a backbone in 4 bits, the root-mean-square norm with an output in 8
bits, and the conversions in and out of both formats.

The ``lora_*`` functions have the names of the C ABI and take descriptors (argument marshalling only); ``*_desc`` make those
from tensors; ``quantize``, ``dequantize``, ``rms_norm``, ``linear``, ``linear_multi`` and ``norm_linear_multi`` allocate what
they return and run on the current stream.  PyTorch is used for device memory and streams only: every step runs in the HIP
kernels of the shared library.

    W = mx.quantize(ctx, W0, "e2m1")                      # once, when the model is loaded
    pl = runtime.plan(ctx, ids, ntok, ranks)              # once per batch
    normed = mx.rms_norm(ctx, x, gamma, eps, residual=r, quantize=True)
    q, k, v = mx.linear_multi(ctx, pl, normed.y, [(Wq, tq), (Wk, tk), (Wv, tv)], Xq=normed.q)
"""
from __future__ import annotations

import ctypes as C
from typing import List, NamedTuple, Optional, Sequence

import torch

from . import binding as B
from .binding import lib as _layer_lib
from .runtime import AdapterTable, Context, Plan, _output, _stream, dtype_code

LORA_MX_E2M1 = 0
LORA_MX_E4M3 = 1
LORA_MX_BLOCK = 32
LORA_RMS_NORM_MAX_K = 65536

FORMATS = {"e2m1": LORA_MX_E2M1, "e4m3": LORA_MX_E4M3}

EXPORTS = ["lora_mx_quantize", "lora_mx_dequantize", "lora_rms_norm", "lora_mx_linear_workspace_bytes", "lora_mx_linear",
           "lora_mx_linear_multi"]


class lora_mx_rows_t(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("ld_codes", C.c_int64), ("scales", C.c_void_p), ("ld_scales", C.c_int64),
                ("format", C.c_int32), ("reserved", C.c_int32)]


class lora_mx_convert_desc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("K", C.c_int32), ("rows", C.c_int64), ("X", C.c_void_p), ("ldx", C.c_int64), ("q", lora_mx_rows_t)]


class lora_rms_norm_desc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("K", C.c_int32), ("rows", C.c_int64), ("eps", C.c_float), ("flags", C.c_int32),
                ("X", C.c_void_p), ("ldx", C.c_int64), ("R", C.c_void_p), ("ldr", C.c_int64), ("gamma", C.c_void_p),
                ("H", C.c_void_p), ("ldh", C.c_int64), ("Y", C.c_void_p), ("ldy", C.c_int64), ("q", lora_mx_rows_t)]


class lora_mx_linear_desc(C.Structure):
    _fields_ = [("K", C.c_int32), ("N", C.c_int32), ("flags", C.c_int32), ("reserved", C.c_int32), ("X", C.c_void_p), ("ldx", C.c_int64),
                ("Xq", lora_mx_rows_t), ("W", lora_mx_rows_t), ("Y", C.c_void_p), ("ldy", C.c_int64),
                ("tbl", C.POINTER(B.lora_adapter_table_t)), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


_ready = False


def lib():
    global _ready
    L = _layer_lib()
    if not _ready:
        for name in ("lora_mx_quantize", "lora_mx_dequantize"):
            getattr(L, name).argtypes = [C.c_void_p, C.POINTER(lora_mx_convert_desc), C.c_void_p]
        L.lora_rms_norm.argtypes = [C.c_void_p, C.POINTER(lora_rms_norm_desc), C.c_void_p]
        L.lora_mx_linear_workspace_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
        L.lora_mx_linear_workspace_bytes.restype = C.c_size_t
        L.lora_mx_linear.argtypes = [C.c_void_p, C.POINTER(B.lora_plan_t), C.POINTER(lora_mx_linear_desc), C.c_void_p]
        L.lora_mx_linear_multi.argtypes = [C.c_void_p, C.POINTER(B.lora_plan_t), C.POINTER(C.POINTER(lora_mx_linear_desc)), C.c_int32, C.c_void_p]
        _ready = True
    return L


def _done(status: int, name: str, raw: bool):
    if raw:
        return status
    if status != B.LORA_OK:
        raise B.LoraError(status, name)
    return None


def lora_mx_quantize(ctx, desc, stream: int, *, raw: bool = False):
    return _done(lib().lora_mx_quantize(ctx, C.byref(desc), stream), "lora_mx_quantize", raw)


def lora_mx_dequantize(ctx, desc, stream: int, *, raw: bool = False):
    return _done(lib().lora_mx_dequantize(ctx, C.byref(desc), stream), "lora_mx_dequantize", raw)


def lora_rms_norm(ctx, desc, stream: int, *, raw: bool = False):
    return _done(lib().lora_rms_norm(ctx, C.byref(desc), stream), "lora_rms_norm", raw)


def lora_mx_linear_workspace_bytes(T: int, K: int, N: int, r_max: int, with_xq: int) -> int:
    return int(lib().lora_mx_linear_workspace_bytes(int(T), int(K), int(N), int(r_max), int(with_xq)))


def lora_mx_linear(ctx, plan, desc, stream: int, *, raw: bool = False):
    return _done(lib().lora_mx_linear(ctx, C.byref(plan), C.byref(desc), stream), "lora_mx_linear", raw)


def lora_mx_linear_multi(ctx, plan, descs, stream: int, *, raw: bool = False):
    """descs: a sequence of lora_mx_linear_desc that share X, ldx, Xq and K."""
    n = len(descs)
    arr = (C.POINTER(lora_mx_linear_desc) * max(n, 1))(*[C.pointer(d) for d in descs])
    return _done(lib().lora_mx_linear_multi(ctx, C.byref(plan), arr, n, stream), "lora_mx_linear_multi", raw)


# ---- tensors ---------------------------------------------------------------------------------------------------------------

class MxTensor:
    """``rows`` x ``K`` values in a block-scaled format: ``codes`` (uint8, [rows, K] of e4m3 or [rows, K / 2] of e2m1, the even value
    in the low half) and ``scales`` (uint8, [rows, K / 32], 127 = 1).  Tensors are taken as they are where the kernels can read them: rows
    of codes at multiples of 16 bytes, rows of scales at multiples of 4.  Others are copied into such rows, which ``self.codes`` and
    ``self.scales`` then are, also for what an operator writes."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, fmt: str):
        self.format = fmt
        code = FORMATS[fmt]
        assert codes.dtype == torch.uint8 and scales.dtype == torch.uint8 and codes.dim() == 2 and scales.dim() == 2
        rows, K = codes.shape[0], codes.shape[1] * (2 if code == LORA_MX_E2M1 else 1)
        assert K % LORA_MX_BLOCK == 0 and tuple(scales.shape) == (rows, K // LORA_MX_BLOCK), (tuple(codes.shape), tuple(scales.shape))
        if codes.stride(1) != 1 or codes.stride(0) % 16 and rows > 1 or codes.data_ptr() % 16:
            codes = codes.contiguous().clone() if codes.data_ptr() % 16 else codes.contiguous()
        if not _scales_fit(scales):
            padded = _empty_scales(rows, scales.shape[1], scales.device)
            padded.copy_(scales)
            scales = padded
        self.codes, self.scales, self.shape = codes, scales, (rows, K)
        ld_codes = codes.stride(0) if rows > 1 else max(codes.shape[1], codes.stride(0) // 16 * 16)
        ld_scales = scales.stride(0) if rows > 1 else (scales.shape[1] + 3) // 4 * 4
        self.struct = lora_mx_rows_t(codes.data_ptr(), ld_codes, scales.data_ptr(), ld_scales, code, 0)


def _scales_fit(scales: torch.Tensor) -> bool:
    """Whether every row has whole 4-byte pieces of memory, which the kernels read."""
    rows, n = scales.shape
    if scales.stride(1) != 1 and n > 1 or scales.data_ptr() % 4 or rows > 1 and (scales.stride(0) % 4 or scales.stride(0) < n):
        return False
    end = scales.storage_offset() + (max(rows, 1) - 1) * scales.stride(0) + (n + 3) // 4 * 4 if rows > 1 else scales.storage_offset() + (n + 3) // 4 * 4
    return end <= scales.untyped_storage().nbytes()


def _empty_scales(rows: int, n: int, device) -> torch.Tensor:
    return torch.empty((rows, (n + 3) // 4 * 4), dtype=torch.uint8, device=device)[:, :n]


def empty(rows: int, K: int, fmt: str, device) -> MxTensor:
    """Room for ``rows`` x ``K`` values, uninitialised."""
    if K <= 0 or K % LORA_MX_BLOCK:
        raise B.LoraError(B.LORA_ERR_SHAPE, "mx.empty")
    codes = torch.empty((rows, K // 2 if FORMATS[fmt] == LORA_MX_E2M1 else K), dtype=torch.uint8, device=device)
    return MxTensor(codes, _empty_scales(rows, K // LORA_MX_BLOCK, device), fmt)


_NONE = lora_mx_rows_t(None, 0, None, 0, LORA_MX_E4M3, 0)


def _ld(t: torch.Tensor) -> int:
    assert t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1), "rows are contiguous"
    return t.stride(0) if t.shape[0] > 1 else (t.shape[1] + 7) // 8 * 8  # (the stride of a single row says nothing)


def quantize_desc(X: torch.Tensor, q: MxTensor) -> lora_mx_convert_desc:
    assert tuple(X.shape) == q.shape
    return lora_mx_convert_desc(dtype_code(X.dtype), X.shape[1], X.shape[0], X.data_ptr(), _ld(X), q.struct)


def dequantize_desc(q: MxTensor, X: torch.Tensor) -> lora_mx_convert_desc:
    return quantize_desc(X, q)


def norm_desc(X: torch.Tensor, gamma: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None,
              y: Optional[torch.Tensor] = None, q: Optional[MxTensor] = None) -> lora_rms_norm_desc:
    rows, K = X.shape
    assert gamma.shape == (K,) and gamma.is_contiguous()
    for t in (gamma, residual, h, y):
        assert t is None or t.dtype is X.dtype
    for t in (residual, h, y):
        assert t is None or t.shape == X.shape
    assert q is None or q.shape == (rows, K)
    ptr = lambda t: (t.data_ptr(), _ld(t)) if t is not None else (None, 0)  # noqa: E731
    return lora_rms_norm_desc(dtype_code(X.dtype), K, rows, eps, 0, *ptr(X), *ptr(residual), gamma.data_ptr(), *ptr(h), *ptr(y),
                              q.struct if q is not None else _NONE)


def linear_desc(pl: Plan, X: Optional[torch.Tensor], W: MxTensor, Y: torch.Tensor, table: Optional[AdapterTable], ws: torch.Tensor,
                Xq: Optional[MxTensor] = None) -> lora_mx_linear_desc:
    N, K = W.shape
    T = pl.T
    assert Y.dtype is torch.bfloat16 and tuple(Y.shape) == (T, N) and (X is not None or Xq is not None)
    assert X is None or X.dtype is torch.bfloat16 and tuple(X.shape) == (T, K)
    assert Xq is None or Xq.shape == (T, K)
    d = lora_mx_linear_desc(K, N, 0, 0, X.data_ptr() if X is not None else None, _ld(X) if X is not None else 0,
                            Xq.struct if Xq is not None else _NONE, W.struct, Y.data_ptr(), _ld(Y),
                            C.pointer(table.struct) if table is not None else None, ws.data_ptr(), ws.numel())
    d._keep = table
    return d


def workspace(T: int, K: int, N: int, r_max: int, device, x8: bool) -> torch.Tensor:
    nbytes = lora_mx_linear_workspace_bytes(T, K, N, r_max, int(x8))
    if nbytes == 0:
        raise B.LoraError(B.LORA_ERR_INVALID_ARG, "lora_mx_linear_workspace_bytes")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


# ---- operators -------------------------------------------------------------------------------------------------------------

def quantize(ctx: Context, X: torch.Tensor, fmt: str, out: Optional[MxTensor] = None) -> MxTensor:
    """``X`` (bf16 or fp32, [rows, K]) in ``fmt``: "e2m1" (4 bits) or "e4m3" (8 bits)."""
    q = out if out is not None else empty(X.shape[0], X.shape[1], fmt, X.device)
    assert q.format == fmt
    lora_mx_quantize(ctx.handle, quantize_desc(X, q), _stream())
    return q


def dequantize(ctx: Context, q: MxTensor, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    X = out if out is not None else torch.empty(q.shape, dtype=dtype, device=q.codes.device)
    lora_mx_dequantize(ctx.handle, dequantize_desc(q, X), _stream())
    return X


class Normed(NamedTuple):
    y: Optional[torch.Tensor]  # the normed rows
    h: Optional[torch.Tensor]  # X + residual (None without a residual)
    q: Optional[MxTensor]      # the normed rows in 8 bits (None unless asked for)


def rms_norm(ctx: Context, X: torch.Tensor, gamma: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
             quantize: bool = False, normed: bool = True) -> Normed:
    """Root-mean-square norm of ``X + residual`` along the rows; ``normed=False`` leaves ``y`` out (with ``quantize``)."""
    y = torch.empty(X.shape, dtype=X.dtype, device=X.device) if normed else None
    h = torch.empty(X.shape, dtype=X.dtype, device=X.device) if residual is not None else None
    q = empty(X.shape[0], X.shape[1], "e4m3", X.device) if quantize else None
    lora_rms_norm(ctx.handle, norm_desc(X, gamma, eps, residual, h, y, q), _stream())
    return Normed(y, h, q)


def linear(ctx: Context, pl: Plan, X: Optional[torch.Tensor], W: MxTensor, table: Optional[AdapterTable], Xq: Optional[MxTensor] = None,
           Y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """lora_mx_linear on the current stream; returns Y."""
    N, K = W.shape
    if Y is None:
        Y = _output(pl.T, N, X if X is not None else torch.empty(0, dtype=torch.bfloat16, device=W.codes.device))
    if ws is None:
        ws = workspace(pl.T, K, N, pl.r_max, W.codes.device, Xq is not None)
    lora_mx_linear(ctx.handle, pl.struct, linear_desc(pl, X, W, Y, table, ws, Xq), _stream())
    return Y


def linear_multi(ctx: Context, pl: Plan, X: Optional[torch.Tensor], projections: Sequence[tuple], Xq: Optional[MxTensor] = None) -> List[torch.Tensor]:
    """lora_mx_linear_multi on the current stream: ``projections`` is a list of (W, table) that share the activations."""
    descs, outs, keep = [], [], []
    for W, table in projections:
        N, K = W.shape
        Y = _output(pl.T, N, X if X is not None else torch.empty(0, dtype=torch.bfloat16, device=W.codes.device))
        ws = workspace(pl.T, K, N, pl.r_max, W.codes.device, Xq is not None)
        descs.append(linear_desc(pl, X, W, Y, table, ws, Xq))
        outs.append(Y)
        keep.append(ws)
    lora_mx_linear_multi(ctx.handle, pl.struct, descs, _stream())
    return outs


def norm_linear_multi(ctx: Context, pl: Plan, X: torch.Tensor, residual: Optional[torch.Tensor], gamma: torch.Tensor, eps: float,
                      projections: Sequence[tuple], x8: bool = True):
    """The front of a decoder layer's half: the residual's addition, the norm, and the projections that read it.  Returns (X +
    residual, list of outputs).  ``x8``: the base products read the normed rows in 8 bits; the adapters read them in bf16 either way."""
    bare = all(table is None for _, table in projections)
    n = rms_norm(ctx, X, gamma, eps, residual, quantize=x8, normed=not (x8 and bare))
    return n.h if residual is not None else X, linear_multi(ctx, pl, n.y, projections, Xq=n.q)
