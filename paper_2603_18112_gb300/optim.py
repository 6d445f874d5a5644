"""Binding of the gradient norm, clipping, AdamW and Muon of libtula_ags (include/tula_train.h).

    clip = GradClipper(grads)                 # a list of fp32, bf16 or fp16 CUDA tensors
    record = clip.clip_(1.0)                  # [|G|, coefficient, finite, -] on the GPU

    step = AdamWStep(params, grads, exp_avgs, exp_avg_sqs, copies=bf16_weights, max_norm=1.0)
    step(1e-3, (0.9, 0.95), 1e-8, 0.1)        # asynchronous on the current stream

    step = MuonStep(matrices, grads, momenta, copies=bf16_weights)
    step(2e-4, 0.95, 0.1, record=record)
    o = orthogonalize(u)                      # a matrix, or a batch of them

The first three lay their tensors out in a plan once; a call then passes scalars only.  The tensors must stay
where they are (zero gradients in place).  As in ``tula_ags``, everything runs in the CUDA library.
"""
from __future__ import annotations

import ctypes
from operator import attrgetter

import torch

from .tula_ags import (_check, _host_array, _stream_ptr, c_float, c_int, c_size_t, c_void_p, lib)

TULA_TYPE_F32, TULA_TYPE_BF16, TULA_TYPE_F16 = 0, 1, 2
TULA_RECORD_NORM, TULA_RECORD_COEF, TULA_RECORD_FINITE = range(3)
TULA_RECORD_LEN = 4
TYPES = {torch.float32: TULA_TYPE_F32, torch.bfloat16: TULA_TYPE_BF16, torch.float16: TULA_TYPE_F16}


class tula_train_tensors(ctypes.Structure):
    """Mirror of the C struct tula_train_tensors."""
    _fields_ = [("n_tensors", c_int), ("numels", c_void_p), ("grad_ptrs", c_void_p),
                ("grad_types", c_void_p), ("param_ptrs", c_void_p), ("exp_avg_ptrs", c_void_p),
                ("exp_avg_sq_ptrs", c_void_p), ("copy_ptrs", c_void_p), ("copy_types", c_void_p)]


class tula_adamw_hparams(ctypes.Structure):
    """Mirror of the C struct tula_adamw_hparams."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("grad_scale", ctypes.c_double), ("max_norm", ctypes.c_double),
                ("skip_nonfinite", c_int), ("record", c_void_p), ("steps", c_void_p)]


class tula_muon_matrices(ctypes.Structure):
    """Mirror of the C struct tula_muon_matrices."""
    _fields_ = [("n_matrices", c_int), ("rows", c_void_p), ("cols", c_void_p), ("grad_ptrs", c_void_p),
                ("grad_types", c_void_p), ("param_ptrs", c_void_p), ("momentum_ptrs", c_void_p),
                ("copy_ptrs", c_void_p), ("copy_types", c_void_p)]


class tula_muon_hparams(ctypes.Structure):
    """Mirror of the C struct tula_muon_hparams."""
    _fields_ = [("lr", ctypes.c_double), ("momentum", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("grad_scale", ctypes.c_double), ("nesterov", c_int), ("ns_steps", c_int), ("scale", c_int),
                ("record", c_void_p)]


MUON_SCALES = {"rms": 0, "aspect": 1}  # TULA_MUON_SCALE_*

_typed = False


def _lib():
    global _typed
    L = lib()
    if not _typed:
        i64p = ctypes.POINTER(ctypes.c_int64)
        L.tula_train_workspace_size.argtypes = [i64p, c_int, ctypes.POINTER(c_size_t)]
        L.tula_train_plan_create.argtypes = [ctypes.POINTER(tula_train_tensors), c_void_p, c_size_t,
                                             c_void_p, ctypes.POINTER(c_void_p)]
        L.tula_train_plan_destroy.argtypes = [c_void_p]
        L.tula_grad_norm.argtypes = [c_void_p, c_float, c_float, c_void_p, c_void_p]
        L.tula_grad_clip.argtypes = [c_void_p, c_float, c_void_p, c_void_p]
        L.tula_adamw_default_hparams.argtypes = [ctypes.POINTER(tula_adamw_hparams)]
        L.tula_adamw_default_hparams.restype = None
        L.tula_adamw_step.argtypes = [c_void_p, ctypes.POINTER(tula_adamw_hparams), c_void_p]
        L.tula_muon_workspace_size.argtypes = [i64p, i64p, c_int, ctypes.POINTER(c_size_t)]
        L.tula_muon_plan_create.argtypes = [ctypes.POINTER(tula_muon_matrices), c_void_p, c_size_t,
                                            c_void_p, ctypes.POINTER(c_void_p)]
        L.tula_muon_plan_destroy.argtypes = [c_void_p]
        L.tula_muon_default_hparams.argtypes = [ctypes.POINTER(tula_muon_hparams)]
        L.tula_muon_default_hparams.restype = None
        L.tula_muon_step.argtypes = [c_void_p, ctypes.POINTER(tula_muon_hparams), c_void_p]
        L.tula_muon_error.argtypes = [c_void_p, ctypes.POINTER(c_int)]
        L.tula_muon_check_wait_timeout.argtypes = [c_void_p]
        i64 = ctypes.c_int64
        L.tula_orthogonalize_workspace_size.argtypes = [i64, i64, i64, ctypes.POINTER(c_size_t)]
        L.tula_orthogonalize.argtypes = [c_void_p, c_int, i64, i64, i64, i64, i64, c_int, c_void_p, c_int,
                                         c_void_p, c_size_t, c_void_p]
        _typed = True
    return L


def tula_train_workspace_size(numels) -> int:
    arr = _host_array(ctypes.c_int64, "q", map(int, numels))
    out = c_size_t(0)
    _check(_lib().tula_train_workspace_size(arr, len(numels), ctypes.byref(out)),
           "tula_train_workspace_size")
    return out.value


_dtype, _contiguous, _numel = attrgetter("dtype"), torch.Tensor.is_contiguous, torch.Tensor.numel
_data_ptr, _device = torch.Tensor.data_ptr, torch.Tensor.get_device


def _ptrs(tensors, allowed, numels, index, what):
    """The tensors' addresses, after checking them (loops in C: a plan over 1024 tensors and five
    roles checks 5120)."""
    if not set(map(_dtype, tensors)) <= allowed or not all(map(_contiguous, tensors)) or \
            set(map(_device, tensors)) != {index}:
        bad = next(t for t in tensors if t.dtype not in allowed or not t.is_contiguous() or t.get_device() != index)
        raise TypeError(f"{what}: contiguous tensors of {sorted(map(str, allowed))} on GPU {index} are wanted, got "
                        f"{bad.dtype} on {bad.device}, strides {bad.stride()} of {tuple(bad.shape)}")
    if list(map(_numel, tensors)) != numels:
        raise ValueError(f"{what}: other numbers of elements than the gradients have")
    return _host_array(c_void_p, "Q", map(_data_ptr, tensors))


_get_device = torch._C._cuda_getDevice


class _Planned:
    """What plans over fixed tensors have in common: a handle, and memory of their own."""

    def call(self, name, stream, *args):
        """The library's `name` for this plan and these arguments, on `stream` or the current one of the plan's GPU,
        which is made current for the call where it is not."""
        index = self.device.index
        if isinstance(stream, torch.cuda.Stream) and stream.device.index != index:
            raise ValueError(f"{name}: tensors on GPU {index}, a stream of {stream.device}")
        if index != _get_device():
            with torch.cuda.device(index):
                return self.call(name, stream, *args)
        s = _stream_ptr(stream)
        _check(getattr(_lib(), name)(self.handle, *args, s), name)
        if s.value != self.last:
            self.ran_on(s)

    def ran_on(self, stream):
        """A call went to this stream, not the one of the call before.  Kernels read the tiles' rows from the
        workspace, so what is the plan's own goes back to the allocator only after its work."""
        self.last, index = stream.value, self.device.index
        s = torch.cuda.ExternalStream(stream.value, index) if stream.value else torch.cuda.default_stream(index)
        for t in self.memory:
            t.record_stream(s)

    def __del__(self):
        if getattr(self, "handle", None):
            self._destroy(self.handle)
            self.handle = None


class _Plan(_Planned):
    """A tula_train_plan over fixed tensors, with its workspace."""

    def __init__(self, grads, params=None, exp_avgs=None, exp_avg_sqs=None, copies=None):
        grads = list(grads)
        if not grads:
            raise ValueError("no gradients")
        self.device = dev = grads[0].device
        if dev.type != "cuda":
            raise TypeError(f"CUDA tensors are wanted, got {dev}")
        numels = list(map(_numel, grads))
        self._tensors = [grads]
        roles = {}
        for name, ts, allowed in (("params", params, {torch.float32}),
                                  ("exp_avgs", exp_avgs, {torch.float32}),
                                  ("exp_avg_sqs", exp_avg_sqs, {torch.float32}),
                                  ("copies", copies, {torch.bfloat16, torch.float16})):
            if ts is None:
                continue
            ts = list(ts)
            if len(ts) != len(grads):
                raise ValueError(f"{len(ts)} {name} for {len(grads)} gradients")
            self._tensors.append(ts)  # must outlive the plan
            roles[name] = (ts, _ptrs(ts, allowed, numels, dev.index, name))
        g = _ptrs(grads, set(TYPES), numels, dev.index, "grads")
        gt = _host_array(c_int, "i", [TYPES[d] for d in map(_dtype, grads)])
        ct = (_host_array(c_int, "i", [TYPES[d] for d in map(_dtype, roles["copies"][0])])
              if copies is not None else None)
        n = _host_array(ctypes.c_int64, "q", numels)

        def at(a):
            return ctypes.cast(a, c_void_p) if a is not None else None

        desc = tula_train_tensors(len(grads), at(n), at(g), at(gt),
                                  *(at(roles[k][1]) if k in roles else None
                                    for k in ("params", "exp_avgs", "exp_avg_sqs", "copies")), at(ct))
        self.workspace = torch.empty(tula_train_workspace_size(numels), dtype=torch.uint8, device=dev)
        self.handle = c_void_p()
        with torch.cuda.device(dev):
            _check(_lib().tula_train_plan_create(ctypes.byref(desc), c_void_p(self.workspace.data_ptr()),
                                                 self.workspace.numel(), _stream_ptr(None),
                                                 ctypes.byref(self.handle)), "tula_train_plan_create")
        self._destroy = _lib().tula_train_plan_destroy  # kept for __del__ at shutdown
        self.memory, self.last = [self.workspace], ()


class GradClipper:
    """The global norm over a fixed list of gradients, and clipping by it.  ``record`` holds what
    the last call left (TULA_RECORD_*), on the GPU.  The tensors are those it was made with: a gradient
    that is replaced, as by zero_grad's default, is not seen."""

    def __init__(self, grads):
        self._plan = _Plan(grads)
        self.record = torch.zeros(TULA_RECORD_LEN, dtype=torch.float32, device=self._plan.device)
        self._record = c_void_p(self.record.data_ptr())
        self._plan.memory.append(self.record)
        # The fill above ran on the current stream; calls may be issued on any other.
        torch.cuda.synchronize(self._plan.device)

    def norm(self, grad_scale=1.0, max_norm=0.0, stream=None) -> torch.Tensor:
        """|G| / grad_scale, and the coefficient that max_norm would ask for; gradients are read
        only.  Returns the record."""
        self._plan.call("tula_grad_norm", stream, grad_scale, max_norm, self._record)
        return self.record

    def clip_(self, max_norm, stream=None) -> torch.Tensor:
        """Scales the gradients in place to a norm of at most max_norm.  Returns the record, whose
        norm is that before clipping."""
        self._plan.call("tula_grad_clip", stream, max_norm, self._record)
        return self.record


class AdamWStep:
    """AdamW on fp32 weights and moments, from gradients of any of the types; copies: bf16 or fp16
    tensors that receive the weights.

    max_norm > 0 clips by the global norm (the gradients stay as they are); skip_nonfinite leaves a
    step out whose norm is not finite.  ``steps`` is int64 [taken, left out] and ``record`` as in
    GradClipper, both on the GPU; exp_avgs and exp_avg_sqs are zero-filled before the first step.  The
    tensors, gradients among them, are those it was made with, as in GradClipper."""

    def __init__(self, params, grads, exp_avgs, exp_avg_sqs, copies=None, *, max_norm=0.0,
                 skip_nonfinite=False, steps=None):
        self._plan = _Plan(grads, params, exp_avgs, exp_avg_sqs, copies)
        dev = self._plan.device
        if steps is None:
            steps = torch.zeros(2, dtype=torch.int64, device=dev)
        if steps.dtype != torch.int64 or steps.numel() != 2 or steps.device != dev or not steps.is_contiguous():
            raise TypeError(f"steps: two int64 on {dev} are wanted")
        self.steps = steps
        self.record = torch.zeros(TULA_RECORD_LEN, dtype=torch.float32, device=dev)
        self._plan.memory += [steps, self.record]
        self.hp = tula_adamw_hparams()
        _lib().tula_adamw_default_hparams(ctypes.byref(self.hp))
        self.hp.max_norm = max_norm
        self.hp.skip_nonfinite = 1 if skip_nonfinite else 0
        self.hp.record = self.record.data_ptr()
        self.hp.steps = self.steps.data_ptr()
        self._hp = ctypes.byref(self.hp)
        torch.cuda.synchronize(dev)

    def step(self, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=1.0, stream=None) -> None:
        hp = self.hp
        hp.lr, hp.eps, hp.weight_decay, hp.grad_scale = lr, eps, weight_decay, grad_scale
        hp.beta1, hp.beta2 = betas
        self._plan.call("tula_adamw_step", stream, self._hp)

    __call__ = step


class _MuonPlan(_Planned):
    """A tula_muon_plan over fixed matrices, with its workspace."""

    def __init__(self, params, grads, momenta, copies):
        params = list(params)
        if not params:
            raise ValueError("no matrices")
        self.device = dev = params[0].device
        if dev.type != "cuda":
            raise TypeError(f"CUDA tensors are wanted, got {dev}")
        if any(t.dim() != 2 for t in params):
            raise ValueError(f"matrices are wanted, got {next(tuple(t.shape) for t in params if t.dim() != 2)}")
        numels, shapes = list(map(_numel, params)), [t.shape for t in params]
        self._tensors, ptrs, types = [], [], []
        for name, ts, allowed in (("grads", grads, set(TYPES)), ("params", params, {torch.float32}),
                                  ("momenta", momenta, {torch.float32}),
                                  ("copies", copies, {torch.bfloat16, torch.float16})):
            if ts is None:
                ptrs.append(None)
                types.append(None)
                continue
            ts = list(ts)
            if len(ts) != len(params):
                raise ValueError(f"{len(ts)} {name} for {len(params)} matrices")
            if [t.shape for t in ts] != shapes:
                raise ValueError(f"{name}: other shapes than the matrices have")
            self._tensors.append(ts)  # must outlive the plan
            ptrs.append(_ptrs(ts, allowed, numels, dev.index, name))
            types.append(_host_array(c_int, "i", [TYPES[t.dtype] for t in ts]))
        rows, cols = (_host_array(ctypes.c_int64, "q", [t.shape[k] for t in params]) for k in (0, 1))

        def at(a):
            return ctypes.cast(a, c_void_p) if a is not None else None

        desc = tula_muon_matrices(len(params), at(rows), at(cols), at(ptrs[0]), at(types[0]), at(ptrs[1]), at(ptrs[2]),
                                  at(ptrs[3]), at(types[3]))
        need = c_size_t(0)
        _check(_lib().tula_muon_workspace_size(rows, cols, len(params), ctypes.byref(need)), "tula_muon_workspace_size")
        self.workspace = torch.empty(need.value, dtype=torch.uint8, device=dev)
        self.handle = c_void_p()
        with torch.cuda.device(dev):
            _check(_lib().tula_muon_plan_create(ctypes.byref(desc), c_void_p(self.workspace.data_ptr()),
                                                self.workspace.numel(), _stream_ptr(None), ctypes.byref(self.handle)),
                   "tula_muon_plan_create")
        self._destroy = _lib().tula_muon_plan_destroy  # kept for __del__ at shutdown
        self.memory, self.last = [self.workspace], ()


class MuonStep:
    """Muon on fp32 matrices and momenta, from gradients of any of the types; copies: bf16 or fp16
    tensors that receive the weights.  Updates are orthogonalised from fp16 operands, as ``orthogonalize`` says.

    momenta are zero-filled before the first step.  scale: what an update is multiplied by beside lr,
    "rms" (0.2 sqrt(max(rows, cols)), updates as large as AdamW's) or "aspect" (sqrt(max(1, rows / cols))).
    The tensors, gradients among them, are those it was made with, as in GradClipper."""

    def __init__(self, params, grads, momenta, copies=None, *, nesterov=True, ns_steps=5, scale="rms"):
        if scale not in MUON_SCALES:
            raise ValueError(f"scale: one of {sorted(MUON_SCALES)} is wanted, got {scale!r}")
        self._plan = _MuonPlan(params, grads, momenta, copies)
        self.hp = tula_muon_hparams()
        _lib().tula_muon_default_hparams(ctypes.byref(self.hp))
        self.hp.nesterov, self.hp.ns_steps, self.hp.scale = 1 if nesterov else 0, ns_steps, MUON_SCALES[scale]
        self._hp = ctypes.byref(self.hp)
        torch.cuda.synchronize(self._plan.device)

    def step(self, lr, momentum=0.95, weight_decay=0.0, grad_scale=1.0, record=None, stream=None) -> None:
        """record: as GradClipper.norm leaves it (with this grad_scale), for clipping by the norm that it
        was taken over and for leaving a step out whose norm is not finite."""
        hp, plan = self.hp, self._plan
        hp.lr, hp.momentum, hp.weight_decay, hp.grad_scale = lr, momentum, weight_decay, grad_scale
        if record is None:
            hp.record = None
        else:
            if (record.dtype != torch.float32 or record.numel() != TULA_RECORD_LEN or record.device != plan.device
                    or not record.is_contiguous()):
                raise TypeError(f"record: {TULA_RECORD_LEN} float32 on {plan.device} are wanted")
            hp.record = record.data_ptr()
        plan.call("tula_muon_step", stream, self._hp)

    __call__ = step


def orthogonalize(x: torch.Tensor, steps: int = 5, dtype=torch.bfloat16) -> torch.Tensor:
    """The matrix x, or each matrix of a batch [..., rows, cols] (fp32, bf16 or fp16), with its singular
    values brought near 1 by Muon's Newton-Schulz steps, as bf16 or fp16, on the current stream.  No
    gradient is recorded.

    X, A = X X^T and the polynomial of A are held in fp16.  The result is 0.5 to 2e-3 off the formula's, relative to
    its norm, where most singular values are within 20 of the largest; up to 1e-2 where the smaller side is 2 to 7;
    more where many lie far below the largest (2e-2 where they fall off like 1 / k^2, as those of momenta in training
    may), as rounding x to bf16 moves it more still."""
    if x.dim() < 2:
        raise ValueError(f"orthogonalize: a matrix or a batch of them is wanted, got {tuple(x.shape)}")
    if x.dtype not in TYPES or dtype not in (torch.bfloat16, torch.float16) or not x.is_cuda:
        raise TypeError(f"orthogonalize: float32, bfloat16 or float16 on a GPU to bfloat16 or float16 is wanted, got {x.dtype} "
                        f"on {x.device} to {dtype}")
    x = x.detach()
    rows, cols = x.shape[-2:]
    out = torch.empty(x.shape, dtype=dtype, device=x.device)
    if not out.numel():
        return out
    batch = out.numel() // (rows * cols)
    if x.dim() != 3:
        x = x.reshape(batch, rows, cols)
    apart, stride, step = x.stride()
    if step != 1 and cols > 1 or stride < cols and rows > 1 or apart < 0:
        x = x.contiguous()
        apart, stride, step = x.stride()
    need = c_size_t(0)
    _check(_lib().tula_orthogonalize_workspace_size(batch, rows, cols, ctypes.byref(need)), "tula_orthogonalize_workspace_size")
    with torch.cuda.device(x.device):
        space = torch.empty(need.value, dtype=torch.uint8, device=x.device)
        _check(_lib().tula_orthogonalize(x.data_ptr(), TYPES[x.dtype], batch, rows, cols, max(stride, cols),
                                         apart, steps, out.data_ptr(), TYPES[dtype], space.data_ptr(), need.value,
                                         _stream_ptr(None)), "tula_orthogonalize")
    return out


def tula_muon_check_wait_timeout(stream=None) -> None:
    """Makes a bounded wait of these kernels run out (about two seconds on the GPU): afterwards
    tula_muon_error reports bit 0."""
    _check(_lib().tula_muon_check_wait_timeout(_stream_ptr(stream)), "tula_muon_check_wait_timeout")


def tula_muon_error(stream=None) -> int:
    """Reads and clears the error word of Muon's products after the work on `stream` (synchronous): 0 =
    every wait inside the kernels completed."""
    out = c_int(0)
    _check(_lib().tula_muon_error(_stream_ptr(stream), ctypes.byref(out)), "tula_muon_error")
    return out.value
