"""Binding of the MXFP4 matrices of libtula_ags (include/tula_train.h).

    q = quantize(x)                       # blocks of 32 along the rows of x
    q, qt = quantize(x, cols=True)        # and x's transpose, blocks along x's columns
    x4 = dequantize(q, torch.bfloat16)
    y = matmul(a, b)                      # A B^T
    y = linear(x, w)                      # x w^T, differentiable: both gradients are MXFP4 products

Everything runs in the CUDA library, asynchronously on the current stream.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd.function import once_differentiable

from .optim import TYPES
from .tula_ags import _check, _stream_ptr, c_int, c_size_t, c_void_p, lib

_i64 = ctypes.c_int64
_fns = None  # the library's functions, their types declared


def _lib():
    global _fns
    if _fns is None:
        L = lib()
        L.tula_mx_size.argtypes = [_i64, _i64, ctypes.POINTER(c_size_t), ctypes.POINTER(c_size_t)]
        L.tula_mx_quantize.argtypes = [c_void_p, c_int, _i64, _i64, _i64] + [c_void_p] * 5
        L.tula_mx_dequantize.argtypes = [c_void_p, c_void_p, _i64, _i64, c_void_p, c_int, c_void_p]
        L.tula_mx_matmul.argtypes = [c_void_p] * 4 + [_i64] * 3 + [c_void_p, c_int, c_void_p]
        L.tula_mx_error.argtypes = [c_void_p, ctypes.POINTER(c_int)]
        L.tula_mx_check_wait_timeout.argtypes = [c_void_p]
        _fns = L
    return _fns


_raw_stream, _get_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


_raw_delete = torch._C._cuda_cudaCachingAllocator_raw_delete
_unfreed: list = []  # blocks that were dropped while another stream may read them


def _stream(handle, device):
    return torch.cuda.ExternalStream(handle, device) if handle else torch.cuda.default_stream(device)


def _under_capture(stream):
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


def _wait_for_readers(device, own, readers):
    """Has the stream that a block's memory goes back to wait for those that read it; False under capture."""
    own, *readers = [_stream(s, device) for s in (own, *readers)]
    if any(map(_under_capture, (own, *readers))):
        return False
    for s in readers:
        own.wait_stream(s)
    return True


def _free_after_readers(delete):
    """Gives such blocks back once their own streams, whose next allocations may get them, wait for the
    readers.  Streams under capture cannot wait so; their blocks stay for the next call, which the next
    block's making is at the latest.  A block is the caller's alone from the moment it is taken out of the
    list: other threads, and the collector in the middle of this, may be here too."""
    held = []
    try:
        while _unfreed:
            try:
                block = _unfreed.pop()
            except IndexError:  # another took the last
                break
            ptr, *where = block
            try:
                waits = _wait_for_readers(*where)
            except RuntimeError:
                # a stream that is no more, as one of another library may be: nothing says when its work
                # ends, so the memory stays taken, and the blocks after it are not held up
                continue
            if waits:
                delete(ptr)
            else:
                held.append(block)
    finally:
        _unfreed.extend(held)


class _Block:
    """Device memory from torch's allocator, for the current device and stream, without a tensor around
    it: with torch.empty ahead of it a launch takes the host 7.5 us on a GB300 machine, with this 3.5."""

    __slots__ = ("ptr", "size", "device", "stream", "_noted")

    def __init__(self, size: int, device: int, _alloc=torch._C._cuda_cudaCachingAllocator_raw_alloc):
        self.ptr, self.size, self.device, self._noted = 0, size, device, set()
        self.stream = stream = _raw_stream(device)
        if _unfreed and not torch.cuda.is_current_stream_capturing():
            _free_after_readers(_raw_delete)
        if size and device == _get_device():
            self.ptr = _alloc(size, stream)
        elif size:
            with torch.cuda.device(device):
                self.ptr = _alloc(size, stream)

    def read_elsewhere(self, stream: int):
        """The device's current stream, which is not the block's own, is about to read the block.  Under
        capture that is noted where the block may be of the same capture, so that its memory is not handed
        out again within it.  (What a graph reads of before it has to live as long as the graph: its
        streams hold no work to wait for.)"""
        if stream in self._noted:
            return
        with torch.cuda.device(self.device):
            if torch.cuda.is_current_stream_capturing() and not (
                    self.stream and _under_capture(_stream(self.stream, self.device))):
                return
        self._noted.add(stream)  # (one step: other threads may be noting theirs)

    @property
    def readers(self):
        """The other streams that have read it, or None."""
        return self._noted or None

    def __del__(self, _delete=_raw_delete):
        if not self.ptr:
            return
        if not self._noted:
            _delete(self.ptr)
        else:
            _unfreed.append((self.ptr, self.device, self.stream, self._noted))
            _free_after_readers(_delete)

    @property
    def __cuda_array_interface__(self):
        return {"shape": (self.size,), "typestr": "|u1", "data": (self.ptr, False), "version": 3}


def _bytes(rows, cols):
    """Of a matrix's scales and codes, which follow them."""
    return (rows + 127) // 128 * ((cols + 127) // 128) * 512 + rows * ((cols + 127) // 128) * 64


class MXMatrix:
    """A rows x cols matrix in MXFP4: ``codes`` uint8 [rows, P / 2] and ``scales`` uint8
    [ceil(rows / 128), P / 128, 32, 4, 4], P = cols rounded up to a multiple of 128; of any shapes
    of those sizes, contiguous, on one GPU.  Not to be changed once made.  Its memory belongs to the
    stream it was made on, as a tensor's does; products and readings on other streams are waited for
    before it is used again, once they are ordered after its making.  (Tensors taken from ``codes`` and
    ``scales`` keep it alive, but what other operations read of them on other streams is not noted.)"""

    __slots__ = ("rows", "cols", "device", "dev", "code_ptr", "scale_ptr", "_codes", "_scales", "_block")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int):
        tiles = (cols + 127) // 128
        if (codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or not codes.is_contiguous()
                or not scales.is_contiguous() or rows < 0 or cols < 0 or codes.numel() != rows * tiles * 64
                or scales.numel() != (rows + 127) // 128 * tiles * 512):
            raise ValueError(f"not the codes and scales of a {rows} x {cols} matrix")
        self.rows, self.cols, self._codes, self._scales, self._block = rows, cols, codes, scales, None
        self.dev, self.device = _on_gpu(codes, scales), codes.device
        self.code_ptr, self.scale_ptr = codes.data_ptr(), scales.data_ptr()

    @classmethod
    def empty(cls, rows: int, cols: int, device: torch.device) -> "MXMatrix":
        """One to quantise into, in one allocation."""
        self = cls.__new__(cls)
        tiles = (cols + 127) // 128
        n = (rows + 127) // 128 * tiles * 512
        self.rows, self.cols, self.dev, self.device = rows, cols, device.index, device
        self._block = block = _Block(n + rows * tiles * 64, device.index)
        self._codes = self._scales = None
        self.scale_ptr = block.ptr
        self.code_ptr = block.ptr + n
        return self

    @classmethod
    def _within(cls, memory: torch.Tensor, at: int, rows: int, cols: int) -> "MXMatrix":
        """One to quantise into, or quantised there before, `at` bytes into a uint8 tensor that outlives it."""
        self = cls.__new__(cls)
        self.rows, self.cols, self.dev, self.device = rows, cols, memory.get_device(), memory.device
        self._codes = self._scales = self._block = None
        self.scale_ptr = memory.data_ptr() + at
        self.code_ptr = self.scale_ptr + (rows + 127) // 128 * ((cols + 127) // 128) * 512
        return self

    def _reads(self):
        """The current stream is about to read it."""
        block = self._block
        if block is not None and block.stream != _raw_stream(self.dev):  # (a caller's tensors are the caller's)
            block.read_elsewhere(_raw_stream(self.dev))

    def _split(self):
        n, tiles = self.code_ptr - self.scale_ptr, (self.cols + 127) // 128
        all_ = (torch.as_tensor(self._block, device=self.device) if self._block.size
                else torch.empty(0, dtype=torch.uint8, device=self.device))
        self._scales = all_[:n].view((self.rows + 127) // 128, tiles, 32, 4, 4)
        self._codes = all_[n:].view(self.rows, tiles * 64)

    @property
    def codes(self) -> torch.Tensor:
        if self._codes is None:
            self._split()
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            self._split()
        return self._scales


def tula_mx_size(rows: int, cols: int) -> tuple[int, int]:
    """Bytes of the codes and of the scales."""
    a, b = c_size_t(0), c_size_t(0)
    _check(_lib().tula_mx_size(rows, cols, ctypes.byref(a), ctypes.byref(b)), "tula_mx_size")
    return a.value, b.value


def _on_gpu(*tensors):
    """The index of the one GPU that the tensors are on."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t.get_device() != dev or dev < 0:
            raise TypeError(f"tensors on one GPU are wanted, got {[str(t.device) for t in tensors]}")
    return dev


def _call(name, dev, *args):
    """The library's `name` with these arguments and the current stream, with the tensors' GPU
    current; switching to it costs some microseconds, so only where it is not."""
    fn = getattr(_fns or _lib(), name)
    if dev == _get_device():
        rc = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc:
        _check(rc, name)


def _type(dtype, what):
    kind = TYPES.get(dtype)
    if kind is None:
        raise TypeError(f"{what}: float32, bfloat16 or float16 is wanted, got {dtype}")
    return kind


def _quantize_into(x, dev, kind, q, t):
    """A matrix into q, its transpose into t; either may be None."""
    r, c = x.shape
    stride, step = x.stride()
    if step != 1 and stride == 1 and r > 1 and step >= r:
        # a transposed matrix lies in memory as its transpose does: each form is the other's of that
        return _quantize_into(x.t(), dev, kind, t, q)
    # a row of one element, or the only row, may have any stride
    if c > 1 and step != 1 or r > 1 and stride < c:
        x = x.contiguous()
        stride = c
    if r <= 1:
        stride = c
    a, b = (q.code_ptr, q.scale_ptr) if q else (None, None)
    a_t, b_t = (t.code_ptr, t.scale_ptr) if t else (None, None)
    _call("tula_mx_quantize", dev, x.data_ptr(), kind, r, c, stride, a, b, a_t, b_t)


def quantize(x: torch.Tensor, rows: bool = True, cols: bool = False):
    """x (2-D; its rows may lie apart) as an MXMatrix (rows), its transpose as one (cols), or both
    as a pair from one reading of x."""
    dev = x.get_device()
    if dev < 0:
        raise TypeError(f"quantize: a tensor on a GPU is wanted, got {x.device}")
    kind = _type(x.dtype, "quantize")
    shape, device = x.shape, x.device
    if len(shape) != 2 or not (rows or cols):
        raise ValueError("quantize: a matrix, and at least one of rows and cols, are wanted")
    r, c = shape
    q = MXMatrix.empty(r, c, device) if rows else None
    if not cols:
        _quantize_into(x, dev, kind, q, None)
        return q
    t = MXMatrix.empty(c, r, device)
    _quantize_into(x, dev, kind, q, t)
    return (q, t) if rows else t


def dequantize(q: MXMatrix, dtype=torch.bfloat16) -> torch.Tensor:
    """The values that q stands for."""
    kind = _type(dtype, "dequantize")
    q._reads()
    out = torch.empty((q.rows, q.cols), dtype=dtype, device=q.device)
    _call("tula_mx_dequantize", q.dev, q.code_ptr, q.scale_ptr, q.rows, q.cols, out.data_ptr(), kind)
    return out


def matmul(a: MXMatrix, b: MXMatrix, dtype=torch.bfloat16) -> torch.Tensor:
    """A B^T for a of M x K and b of N x K, as an M x N tensor of dtype."""
    if a.cols != b.cols or a.dev != b.dev:
        raise ValueError(f"matmul: {a.cols} columns on GPU {a.dev} and {b.cols} on GPU {b.dev}")
    kind = _type(dtype, "matmul")
    a._reads()
    b._reads()
    out = torch.empty((a.rows, b.rows), dtype=dtype, device=a.device)
    _call("tula_mx_matmul", a.dev, a.code_ptr, a.scale_ptr, b.code_ptr, b.scale_ptr, a.rows, b.rows, a.cols,
          out.data_ptr(), kind)
    return out


def tula_mx_check_wait_timeout(stream=None) -> None:
    """Makes a bounded wait of the kernels run out (about two seconds on the GPU): afterwards
    tula_mx_error reports bit 0."""
    _check(_lib().tula_mx_check_wait_timeout(_stream_ptr(stream)), "tula_mx_check_wait_timeout")


def tula_mx_error(stream=None) -> int:
    """Reads and clears the products' error word after the work on `stream` (synchronous): 0 =
    every wait inside the kernels completed."""
    out = c_int(0)
    _check(_lib().tula_mx_error(_stream_ptr(stream), ctypes.byref(out)), "tula_mx_error")
    return out.value


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, recorded):
        # (needs_input_grad follows requires_grad, also where no gradient is recorded)
        need_x, need_w = (n and recorded for n in ctx.needs_input_grad[:2])
        (m, k), n = x.shape, w.shape[0]
        dev, x_kind, w_kind = _on_gpu(x, w), _type(x.dtype, "linear"), _type(w.dtype, "linear")
        # what the backward pass multiplies by is kept in 4 bits: x^T for dw, then w^T for dx
        ctx.types, ctx.sizes, ctx.device = (x.dtype, w.dtype), (m, n, k), x.device
        ctx.at = at = _bytes(k, m) if need_w else 0
        ctx.end = end = at + (_bytes(k, n) if need_x else 0)
        xt = wt = None
        if need_x or need_w:
            kept = torch.empty(end, dtype=torch.uint8, device=x.device)
            xt = MXMatrix._within(kept, 0, k, m) if need_w else None
            wt = MXMatrix._within(kept, at, k, n) if need_x else None
        qx, qw = MXMatrix.empty(m, k, x.device), MXMatrix.empty(n, k, w.device)
        _quantize_into(x, dev, x_kind, qx, xt)
        _quantize_into(w, dev, w_kind, qw, wt)
        if need_x or need_w:
            ctx.save_for_backward(kept)
        return matmul(qx, qw, x.dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        kept, = ctx.saved_tensors
        if kept.dtype != torch.uint8 or kept.numel() != ctx.end or kept.device != ctx.device or not kept.is_contiguous():
            raise RuntimeError("linear: a hook on saved tensors gave back another tensor than it was given")
        (m, n, k), (need_x, need_w, _) = ctx.sizes, ctx.needs_input_grad
        dx = dw = None
        q = quantize(dy, rows=need_x, cols=need_w)
        rows, cols = q if need_x and need_w else (q, q)
        if need_x:  # dy [M, N] (w^T [K, N])^T
            dx = matmul(rows, MXMatrix._within(kept, ctx.at, k, n), ctx.types[0])
        if need_w:  # dy^T [N, M] (x^T [K, M])^T
            dw = matmul(cols, MXMatrix._within(kept, 0, k, m), ctx.types[1])
        return dx, dw, None


def linear(x: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
    """y = x w^T with x [..., K] and w [N, K] quantised to MXFP4 along K, in x's type.  Its
    gradients are products of MXFP4 matrices too, quantised along the dimension that each sums
    over: dx = dy w in x's type (blocks along N), dw = dy^T x in w's type (blocks along the rows
    of x)."""
    if x.shape[-1] != w.shape[-1] or w.dim() != 2:
        raise ValueError(f"linear: x {tuple(x.shape)} and w {tuple(w.shape)}")
    recorded = torch.is_grad_enabled()
    if x.dim() == 2:
        return _Linear.apply(x, w, recorded)
    # (the rows are counted here: reshape cannot infer them where x has no columns)
    rows = x.reshape(x.shape[:-1].numel(), x.shape[-1])
    return _Linear.apply(rows, w, recorded).view(*x.shape[:-1], w.shape[0])
