"""Binding of layer norm of libtula_ags (include/tula_train.h).

    y = layer_norm(x, weight, bias)       # over the last dimension of x, differentiable

Everything runs in the CUDA library, asynchronously on the current stream.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd.function import once_differentiable

from .mx import _call as _mx_call
from .mx import _forward_gradient, _i64, _on_gpu, _type
from .optim import TYPES
from .tula_ags import _check, _stream_ptr, c_float, c_int, c_size_t, c_void_p, lib

_fns = None  # the library's functions, their types declared


def _lib():
    global _fns
    if _fns is None:
        L = lib()
        L.tula_layer_norm.argtypes = [c_void_p, c_int, _i64, _i64, _i64, c_void_p, c_void_p, c_int, c_float, c_void_p,
                                      c_void_p, c_void_p]
        L.tula_layer_norm_workspace_size.argtypes = [_i64, _i64, ctypes.POINTER(c_size_t)]
        L.tula_layer_norm_backward.argtypes = [c_void_p, _i64, c_void_p, _i64, c_int, _i64, _i64, c_void_p, c_int,
                                               c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
        L.tula_layer_norm_error.argtypes = [c_void_p, ctypes.POINTER(c_int)]
        L.tula_layer_norm_check_wait_timeout.argtypes = [c_void_p]
        _fns = L
    return _fns


def _call(name, dev, *args):
    if _fns is None:
        _lib()
    _mx_call(name, dev, *args)


def tula_layer_norm_workspace_size(rows: int, cols: int) -> int:
    out = c_size_t(0)
    _check(_lib().tula_layer_norm_workspace_size(rows, cols, ctypes.byref(out)), "tula_layer_norm_workspace_size")
    return out.value


def tula_layer_norm_check_wait_timeout(stream=None) -> None:
    """Makes a bounded wait of these kernels run out (about two seconds on the GPU): afterwards
    tula_layer_norm_error reports bit 0."""
    _check(_lib().tula_layer_norm_check_wait_timeout(_stream_ptr(stream)), "tula_layer_norm_check_wait_timeout")


def tula_layer_norm_error(stream=None) -> int:
    """Reads and clears the kernels' error word after the work on `stream` (synchronous): 0 = every wait
    inside them completed."""
    out = c_int(0)
    _check(_lib().tula_layer_norm_error(_stream_ptr(stream), ctypes.byref(out)), "tula_layer_norm_error")
    return out.value


def _rows_of(t, cols):
    """t as a matrix of `cols` columns whose rows may lie apart, and its stride."""
    # (the rows are counted here: reshape cannot infer them where t has no columns)
    t = t if t.dim() == 2 else t.reshape(t.shape[:-1].numel(), cols)
    stride, step = t.stride()
    if cols > 1 and step != 1 or t.shape[0] > 1 and stride < cols:
        t = t.contiguous()
        stride = cols
    return t, stride if t.shape[0] > 1 else cols


def _forward(x, weight, bias, eps, keep):
    """The output, and what the backward pass wants of it."""
    cols = x.shape[-1]
    dev, kind, param_kind = x.get_device(), TYPES.get(x.dtype), 0
    at = [None, None]
    for i, p in enumerate((weight, bias)):
        if p is not None:
            if p.get_device() != dev:
                _on_gpu(x, p)
            if not p.is_contiguous():
                p = p.contiguous()
                at.append(p)  # (lives until the call)
            param_kind = _type(p.dtype, "layer_norm")
            at[i] = p.data_ptr()
    if dev < 0 or kind is None:
        _on_gpu(x)
        _type(x.dtype, "layer_norm")
    if x.dim() == 2 and x.is_contiguous():
        rows, n, stride = x, x.shape[0], cols
    else:
        rows, stride = _rows_of(x, cols)
        n = rows.shape[0]
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    stats = torch.empty((n, 2), dtype=torch.float32, device=x.device) if keep else None
    _call("tula_layer_norm", dev, rows.data_ptr(), kind, n, cols, stride, at[0], at[1], param_kind, eps, y.data_ptr(),
          stats.data_ptr() if keep else None)
    return y, stats


def _kept(*tensors):
    return [t if t is None else (t.dtype, t.shape, t.device) for t in tensors]


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, stats = _forward(x, weight, bias, eps, True)
        ctx.save_for_backward(x, weight, stats)
        ctx.param_type = next((p.dtype for p in (weight, bias) if p is not None), torch.float32)
        ctx.kept = _kept(x, weight, stats)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, stats = ctx.saved_tensors
        if _forward_gradient(dy):
            raise NotImplementedError("layer_norm: no forward-mode derivative of the gradients")
        if _kept(x, weight, stats) != ctx.kept or not stats.is_contiguous():
            raise RuntimeError("layer_norm: a hook on saved tensors gave back another tensor than it was given")
        need_x, need_w, need_b, _ = ctx.needs_input_grad
        cols, dev = x.shape[-1], _on_gpu(x, dy, stats)
        rows, stride = _rows_of(x, cols)
        grads, dy_stride = _rows_of(dy, cols)
        weight = None if weight is None else weight.contiguous()

        def empty(shape, dtype):
            return torch.empty(shape, dtype=dtype, device=x.device)

        dx = empty(x.shape, x.dtype) if need_x else None
        dw = empty((cols,), ctx.param_type) if need_w else None
        db = empty((cols,), ctx.param_type) if need_b else None
        n = tula_layer_norm_workspace_size(rows.shape[0], cols) if need_w or need_b else 0
        space = empty((n,), torch.uint8) if n else None
        _call("tula_layer_norm_backward", dev, grads.data_ptr(), dy_stride, rows.data_ptr(), stride, _type(x.dtype, "layer_norm"),
              rows.shape[0], cols, None if weight is None else weight.data_ptr(), _type(ctx.param_type, "layer_norm"),
              stats.data_ptr(), *(None if t is None else t.data_ptr() for t in (dx, dw, db, space)), n)
        return dx, dw, db, None


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
               eps: float = 1e-5) -> torch.Tensor:
    """(x - mean) / sqrt(var + eps) * weight + bias over the last dimension of x, in fp32, in x's type (fp32,
    bf16 or fp16).  weight and bias: [cols], of one type of these, or None."""
    last = x.shape[-1:]
    if (weight is not None and weight.shape != last) or (bias is not None and bias.shape != last):
        raise ValueError(f"layer_norm: x {tuple(x.shape)} and parameters "
                         f"{[None if p is None else tuple(p.shape) for p in (weight, bias)]}")
    if not last or weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise TypeError(f"layer_norm: x of {x.dim()} dimensions, weight and bias "
                        f"{[None if p is None else p.dtype for p in (weight, bias)]}: one dimension or more and one type are wanted")
    if torch.is_grad_enabled() and (x.requires_grad or weight is not None and weight.requires_grad
                                    or bias is not None and bias.requires_grad):
        return _LayerNorm.apply(x, weight, bias, eps)
    if _forward_gradient(x, weight, bias):
        raise NotImplementedError("layer_norm: no forward-mode derivative")
    return _forward(x, weight, bias, eps, False)[0]
