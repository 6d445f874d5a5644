"""Binding of the 8-bit floating-point matrices of libtula_ags (include/tula_train.h).

    q = quantize(x)                       # E4M3, a scale for each 128 elements of a row
    q, qt = quantize(x, cols=True)        # and x's transpose, blocks along x's columns
    q = quantize(w, square=True)          # a scale for each 128 x 128 elements
    x8 = dequantize(q, torch.bfloat16)
    y = matmul(a, b)                      # A B^T
    y = linear(x, w)                      # x w^T, differentiable: both gradients are 8-bit products

Scales are powers of two.  Everything runs in the CUDA library, asynchronously on the current stream.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd.function import once_differentiable

from .mx import _forward_gradient, _i64, _on_gpu, _Quantised, _type
from .mx import _call as _mx_call
from .tula_ags import _check, _stream_ptr, c_int, c_size_t, c_void_p, lib

CODES = {torch.float8_e4m3fn: 0, torch.float8_e5m2: 1}  # TULA_FP8_*
_fns = None  # the library's functions, their types declared


def _lib():
    global _fns
    if _fns is None:
        L = lib()
        L.tula_fp8_size.argtypes = [_i64, _i64, ctypes.POINTER(c_size_t), ctypes.POINTER(c_size_t)]
        L.tula_fp8_quantize.argtypes = [c_void_p, c_int, _i64, _i64, _i64, c_int, c_int] + [c_void_p] * 5
        L.tula_fp8_dequantize.argtypes = [c_void_p, c_void_p, _i64, _i64, c_int, c_void_p, c_int, c_void_p]
        L.tula_fp8_matmul.argtypes = [c_void_p, c_void_p, c_int] * 2 + [_i64] * 3 + [c_void_p, c_int, c_void_p]
        operand = ctypes.POINTER(tula_fp8_operand)
        L.tula_fp8_linear.argtypes = [operand, operand, _i64, _i64, _i64, c_int, c_int, c_int] + [c_void_p] * 4
        L.tula_fp8_linear_backward.argtypes = [operand, _i64, _i64, _i64, c_int, c_int, c_void_p, c_void_p, c_void_p, c_int,
                                               c_void_p, c_int, c_int, c_int, c_void_p]
        L.tula_fp8_error.argtypes = [c_void_p, ctypes.POINTER(c_int)]
        L.tula_fp8_check_wait_timeout.argtypes = [c_void_p]
        _fns = L
    return _fns


def _call(name, dev, *args):
    if _fns is None:
        _lib()
    _mx_call(name, dev, *args)


def _code(dtype, what):
    code = CODES.get(dtype)
    if code is None:
        raise TypeError(f"{what}: float8_e4m3fn or float8_e5m2 is wanted, got {dtype}")
    return code


class FP8Matrix(_Quantised):
    """A rows x cols matrix of 8-bit codes (``dtype``: torch.float8_e4m3fn or torch.float8_e5m2):
    ``codes`` uint8 [rows, P] and ``scales`` uint8 [ceil(rows / 128), ceil(P / 512), 32, 4, 4], P = cols
    rounded up to a multiple of 128; of any shapes of those sizes, contiguous, on one GPU.  Its memory
    and its use on other streams are as MXMatrix's."""

    __slots__ = ("dtype", "code")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int, dtype=torch.float8_e4m3fn):
        super().__init__(codes, scales, rows, cols)
        self.dtype, self.code = dtype, _code(dtype, "FP8Matrix")

    @staticmethod
    def _sizes(rows, cols):
        """Bytes of the scales and of the codes."""
        return (rows + 127) // 128 * ((cols + 511) // 512) * 512, rows * ((cols + 127) // 128) * 128

    @staticmethod
    def _shapes(rows, cols):
        return ((rows + 127) // 128, (cols + 511) // 512, 32, 4, 4), (rows, (cols + 127) // 128 * 128)

    def _of(self, dtype):
        self.dtype, self.code = dtype, CODES[dtype]
        return self


def tula_fp8_size(rows: int, cols: int) -> tuple[int, int]:
    """Bytes of the codes and of the scales."""
    a, b = c_size_t(0), c_size_t(0)
    _check(_lib().tula_fp8_size(rows, cols, ctypes.byref(a), ctypes.byref(b)), "tula_fp8_size")
    return a.value, b.value


def tula_fp8_check_wait_timeout(stream=None) -> None:
    """Makes a bounded wait of these kernels run out (about two seconds on the GPU): afterwards
    tula_fp8_error reports bit 0."""
    _check(_lib().tula_fp8_check_wait_timeout(_stream_ptr(stream)), "tula_fp8_check_wait_timeout")


def tula_fp8_error(stream=None) -> int:
    """Reads and clears the products' error word after the work on `stream` (synchronous): 0 =
    every wait inside the kernels completed."""
    out = c_int(0)
    _check(_lib().tula_fp8_error(_stream_ptr(stream), ctypes.byref(out)), "tula_fp8_error")
    return out.value


def _quantize_into(x, dev, kind, square, q, t):
    """A matrix into q, its transpose into t; either may be None."""
    r, c = x.shape
    stride, step = x.stride()
    if step != 1 and stride == 1 and r > 1 and step >= r:
        # a transposed matrix lies in memory as its transpose does: each form is the other's of that
        return _quantize_into(x.t(), dev, kind, square, t, q)
    # a row of one element, or the only row, may have any stride
    if c > 1 and step != 1 or r > 1 and stride < c:
        x = x.contiguous()
        stride = c
    if r <= 1:
        stride = c
    a, b = (q.code_ptr, q.scale_ptr) if q else (None, None)
    a_t, b_t = (t.code_ptr, t.scale_ptr) if t else (None, None)
    _call("tula_fp8_quantize", dev, x.data_ptr(), kind, r, c, stride, (q or t).code, square, a, b, a_t, b_t)


def quantize(x: torch.Tensor, rows: bool = True, cols: bool = False, square: bool = False,
             dtype=torch.float8_e4m3fn):
    """x (2-D; its rows may lie apart) as an FP8Matrix (rows), its transpose as one (cols), or both
    as a pair from one reading of x.  Blocks that share a scale are 128 elements of a row (of the
    transpose: of a column of x), or 128 x 128 (square)."""
    dev = x.get_device()
    if dev < 0:
        raise TypeError(f"quantize: a tensor on a GPU is wanted, got {x.device}")
    kind = _type(x.dtype, "quantize")
    _code(dtype, "quantize")
    if x.dim() != 2 or not (rows or cols):
        raise ValueError("quantize: a matrix, and at least one of rows and cols, are wanted")
    r, c = x.shape
    q = FP8Matrix.empty(r, c, x.device)._of(dtype) if rows else None
    t = FP8Matrix.empty(c, r, x.device)._of(dtype) if cols else None
    _quantize_into(x, dev, kind, bool(square), q, t)
    return (q, t) if rows and cols else q or t


def dequantize(q: FP8Matrix, dtype=torch.bfloat16) -> torch.Tensor:
    """The values that q stands for."""
    kind = _type(dtype, "dequantize")
    q._reads()
    out = torch.empty((q.rows, q.cols), dtype=dtype, device=q.device)
    _call("tula_fp8_dequantize", q.dev, q.code_ptr, q.scale_ptr, q.rows, q.cols, q.code, out.data_ptr(), kind)
    return out


def matmul(a: FP8Matrix, b: FP8Matrix, dtype=torch.bfloat16) -> torch.Tensor:
    """A B^T for a of M x K and b of N x K, of either code each, as an M x N tensor of dtype."""
    if a.cols != b.cols or a.dev != b.dev:
        raise ValueError(f"matmul: {a.cols} columns on GPU {a.dev} and {b.cols} on GPU {b.dev}")
    kind = _type(dtype, "matmul")
    a._reads()
    b._reads()
    out = torch.empty((a.rows, b.rows), dtype=dtype, device=a.device)
    _call("tula_fp8_matmul", a.dev, a.code_ptr, a.scale_ptr, a.code, b.code_ptr, b.scale_ptr, b.code, a.rows, b.rows,
          a.cols, out.data_ptr(), kind)
    return out


class tula_fp8_operand(ctypes.Structure):
    """Mirror of the C struct tula_fp8_operand."""
    _fields_ = [("data", c_void_p), ("stride", _i64), ("type", c_int), ("transposed", c_int)]


def _operand(x, what):
    """A matrix as the library takes it, and what has to live until the call."""
    kind = _type(x.dtype, what)
    (r, c), (stride, step) = x.shape, x.stride()
    if step != 1 and stride == 1 and r > 1 and step >= r:  # it lies in memory as its transpose does
        return tula_fp8_operand(x.data_ptr(), step, kind, 1), x
    # a row of one element, or the only row, may have any stride
    if c > 1 and step != 1 or r > 1 and stride < c:
        x = x.contiguous()
        stride = c
    return tula_fp8_operand(x.data_ptr(), stride if r > 1 else c, kind, 0), x


_bytes = FP8Matrix._bytes


def _forward(x, w, dtype, need_x, need_w):
    """x w^T, and what the backward pass multiplies by: x^T for dw, then w^T for dx, in 8 bits."""
    (m, k), n, dev = x.shape, w.shape[0], _on_gpu(x, w)
    (ox, x), (ow, w) = _operand(x, "linear"), _operand(w, "linear")
    device = x.device
    end = (_bytes(k, m) if need_w else 0) + (_bytes(k, n) if need_x else 0)
    kept = torch.empty(end, dtype=torch.uint8, device=device)
    temp = torch.empty(_bytes(m, k) + _bytes(n, k), dtype=torch.uint8, device=device)
    y = torch.empty((m, n), dtype=x.dtype, device=device)
    _call("tula_fp8_linear", dev, ox, ow, m, n, k, CODES[dtype], need_x, need_w, kept.data_ptr(), temp.data_ptr(), y.data_ptr())
    return y, kept


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, dtype, grad_dtype):
        need_x, need_w = ctx.needs_input_grad[:2]
        y, kept = _forward(x, w, dtype, need_x, need_w)
        ctx.types, ctx.sizes, ctx.codes = (x.dtype, w.dtype), (x.shape[0], *w.shape), (CODES[dtype], CODES[grad_dtype])
        ctx.end, ctx.device = kept.numel(), x.device
        ctx.save_for_backward(kept)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        kept, = ctx.saved_tensors
        device = ctx.device
        if _forward_gradient(dy):
            raise NotImplementedError("linear: no forward-mode derivative of the gradients")
        if kept.dtype != torch.uint8 or kept.numel() != ctx.end or kept.device != device or not kept.is_contiguous():
            raise RuntimeError("linear: a hook on saved tensors gave back another tensor than it was given")
        (m, n, k), (need_x, need_w), (x_type, w_type) = ctx.sizes, ctx.needs_input_grad[:2], ctx.types
        dev = _on_gpu(dy, kept)
        od, dy = _operand(dy, "linear")
        temp = torch.empty((_bytes(m, n) if need_x else 0) + (_bytes(n, m) if need_w else 0), dtype=torch.uint8, device=device)
        dx = torch.empty((m, k), dtype=x_type, device=device) if need_x else None
        dw = torch.empty((n, k), dtype=w_type, device=device) if need_w else None
        _call("tula_fp8_linear_backward", dev, od, m, n, k, *ctx.codes, kept.data_ptr(), temp.data_ptr(),
              dx.data_ptr() if need_x else None, _type(x_type, "linear"), dw.data_ptr() if need_w else None,
              _type(w_type, "linear"), need_x, need_w)
        return dx, dw, None, None


def linear(x: torch.Tensor, w: torch.Tensor, dtype=torch.float8_e4m3fn, grad_dtype=torch.float8_e4m3fn) -> torch.Tensor:
    """y = x w^T with x [..., K] and w [N, K] quantised to 8 bits (`dtype`), x with a scale for each 128
    elements along K, w for each 128 x 128, in x's type.  Its gradients are products of 8-bit matrices
    too, dy quantised to `grad_dtype` along the dimension that each sums over: dx = dy w in x's type
    (w's codes are those of the forward pass), dw = dy^T x in w's type (blocks along the rows of x)."""
    if x.shape[-1] != w.shape[-1] or w.dim() != 2:
        raise ValueError(f"linear: x {tuple(x.shape)} and w {tuple(w.shape)}")
    _code(dtype, "linear")
    _code(grad_dtype, "linear")
    # (the rows are counted here: reshape cannot infer them where x has no columns)
    rows = x if x.dim() == 2 else x.reshape(x.shape[:-1].numel(), x.shape[-1])
    if torch.is_grad_enabled() and (x.requires_grad or w.requires_grad):
        y = _Linear.apply(rows, w, dtype, grad_dtype)
    elif _forward_gradient(rows, w):
        raise NotImplementedError("linear: no forward-mode derivative")
    else:
        y = _forward(rows, w, dtype, False, False)[0]
    return y if x.dim() == 2 else y.view(*x.shape[:-1], w.shape[0])
