"""The operators of training in reduced precision that speed is measured on: the global gradient
norm and clipping, AdamW on fp32 master weights with copies in the model's type, and microscaled
4-bit matrices (MXFP4): quantisation, reading back, products and a linear layer with its gradients.

A case is a dict of plain values.

op "clip": the norm over all gradients, and the gradients scaled where it exceeds the threshold
op "adamw": one AdamW step
  set       "log": `tensors` 1-D tensors with sizes log-uniform in [64, hi], odd ones among them;
            "layers": `layers` blocks of width `d` (four d x d matrices, two d x ff, two vectors)
            behind an embedding of `vocab` rows
  type      of the gradients: "f32", "bf16", "f16"; "mixed": matrices bf16 and vectors f32 ("log":
            every other tensor)
  packed    every role back to back in one flat buffer (most tensors off 16-byte boundaries), or
            every tensor at a 256-byte boundary
  clip      adamw: by the global norm
  copy      adamw: type of the weights' copies for the model, or ""
  scale     adamw: the loss scale, a factor in the gradients
  overflow  adamw: with one infinite gradient, for which the step is left out
op "quant": a matrix quantised to MXFP4 and read back
  rows, cols, type, stride (elements from row to row)
  forms     "rows": blocks of 32 along the rows; "both": also the transposed matrix, with blocks
            along the columns
op "product": A B^T of two MXFP4 matrices, M x K and N x K; out "bf16" or "f32"
op "linear": y = x w^T in MXFP4 and its gradients dx and dw; x and dy bf16, w fp32
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

LR, BETA1, BETA2, EPS, WD = 1e-3, 0.9, 0.95, 1e-8, 0.1
MAX_NORM = 1.0
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _adamw(**kw):
    case = {"op": "adamw", "type": "f32", "packed": False, "clip": True, "copy": "", "scale": 1.0,
            "overflow": False}
    case.update(kw)
    return case


def listed():
    return [
        # A small model's gradients (the count and the largest tensor of a CIFAR ResNet-20): a few
        # microseconds of work, launches are what counts.
        {"name": "clip_small", "op": "clip", "set": "log", "tensors": 65, "hi": 36864,
         "type": "f32", "packed": False},
        # A language model of ordinary size as it is trained: matrices in bf16, norms in fp32.
        {"name": "clip_layers", "op": "clip", "set": "layers", "layers": 12, "d": 1024, "ff": 4096,
         "vocab": 32000, "type": "mixed", "packed": False},
        # Thousands of tensors of very unequal sizes as views into one bucket, half precision.
        {"name": "clip_buckets", "op": "clip", "set": "log", "tensors": 4096, "hi": 1 << 20,
         "type": "f16", "packed": True},
        # The smallest step: no clipping, no copies.
        _adamw(name="adamw_small", set="log", tensors=65, hi=36864, clip=False),
        # The step of the language model above: bf16 gradients, clipped, bf16 weights written.
        _adamw(name="adamw_layers", set="layers", layers=12, d=1024, ff=4096, vocab=32000,
               type="bf16", copy="bf16"),
        # Half-precision gradients with a loss scale, odd sizes back to back.
        _adamw(name="adamw_buckets", set="log", tensors=1024, hi=1 << 20, type="f16", copy="f16",
               packed=True, scale=1024.0),
        # One token's activations, before a product.
        {"name": "quant_token", "op": "quant", "rows": 1, "cols": 4096, "stride": 4096,
         "type": "bf16", "forms": "rows"},
        # A batch's activations for the forward product and for the weight gradient.
        {"name": "quant_batch", "op": "quant", "rows": 8192, "cols": 4096, "stride": 4096,
         "type": "bf16", "forms": "both"},
        # Master weights of odd sizes, a view into a wider matrix.
        {"name": "quant_weights", "op": "quant", "rows": 4999, "cols": 2047, "stride": 2050,
         "type": "f32", "forms": "both"},
        # One token through the largest layer of VGG-16: the weights are what is read.
        {"name": "product_token", "op": "product", "M": 1, "N": 4096, "K": 25088, "out": "bf16"},
        # A large square product.
        {"name": "product_square", "op": "product", "M": 8192, "N": 8192, "K": 8192, "out": "bf16"},
        # A layer in training, forward and backward: six quantisations and three products.
        {"name": "linear_train", "op": "linear", "M": 8192, "N": 8192, "K": 4096},
    ]


MOST_BYTES = 5e9   # of a drawn case over many tensors
MOST_FLOPS = 6e11  # of a drawn product; the largest listed case has 1.6e12


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(("clip", "adamw", "quant", "product", "product", "linear"))
    if op in ("clip", "adamw"):
        while True:
            case = {"op": op, "type": rng.choice(("f32", "bf16", "f16", "mixed")),
                    "packed": rng.random() < 0.3}
            if op == "adamw":
                case = _adamw(**case)
                case["clip"] = rng.random() < 0.7
                case["copy"] = rng.choice(("", "bf16", "bf16", "f16"))
                case["scale"] = rng.choice((1.0, 1.0, 1024.0))
                case["overflow"] = case["clip"] and rng.random() < 0.15
            if rng.random() < 0.4:
                case["set"] = "layers"
                case["layers"] = rng.randint(1, 24)
                case["d"] = 8 * _log(rng, 4, 200)
                case["ff"] = 4 * case["d"] + 8
                case["vocab"] = _log(rng, 256, 50000)
                if case["d"] == 3072 or case["ff"] == 3072:
                    continue
            else:
                case["set"] = "log"
                case["tensors"] = _log(rng, 1, 4096)
                case["hi"] = _log(rng, 100, 1 << 24)
            if work(case)["bytes"] <= MOST_BYTES:
                return case
    if op == "quant":
        while True:
            case = {"op": op, "rows": _log(rng, 1, 1 << 15), "cols": _log(rng, 1, 1 << 15),
                    "type": rng.choice(("f32", "bf16", "f16")),
                    "forms": rng.choice(("rows", "both"))}
            case["stride"] = case["cols"] + rng.choice((0, 0, 0, 1, 8, 64))
            if case["rows"] * case["cols"] <= 1 << 27:
                return case
    while True:
        case = {"op": op, "M": _log(rng, 1, 1 << 14), "N": _log(rng, 16, 1 << 15),
                "K": _log(rng, 16, 1 << 15)}
        if rng.random() < 0.5:
            case["N"], case["K"] = -(-case["N"] // 64) * 64, -(-case["K"] // 64) * 64
            case["N"], case["K"] = (n + 64 if n == 3072 else n for n in (case["N"], case["K"]))
        if op == "product":
            case["out"] = rng.choice(("bf16", "f32"))
        if work(case)["flops"] <= MOST_FLOPS and work(case)["bytes"] <= MOST_BYTES / 4:
            return case


# --------------------------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------------------------

def _shapes(case):
    if case["set"] == "layers":
        d, ff = case["d"], case["ff"]
        block = [(d,), (d, d), (d, d), (d, d), (d, d), (d,), (ff, d), (d, ff)]
        return [(case["vocab"], d)] + block * case["layers"] + [(d,)]
    n, hi = case["tensors"], case["hi"]
    rng = np.random.default_rng([n, hi])
    sizes = np.rint(np.exp(rng.uniform(math.log(64), math.log(hi), size=n))).astype(np.int64)
    return [(int(s) + (int(s) == 3072),) for s in sizes]


def _groups(case):
    """The tensors by the type of their gradients: (type, shapes), every group a flat buffer a role."""
    shapes = _shapes(case)
    if case["type"] != "mixed":
        return [(case["type"], shapes)]
    first = [len(s) > 1 if case["set"] == "layers" else i % 2 == 0 for i, s in enumerate(shapes)]
    both = [("bf16", [s for s, b in zip(shapes, first) if b]),
            ("f32", [s for s, b in zip(shapes, first) if not b])]
    return [(t, s) for t, s in both if s]


class _Group:
    """One group's roles, flat, zero between the tensors, and the tensors as views into them."""

    def __init__(self, case, kind, shapes, sd, gen, factors):
        self.type, self.shapes = TYPES[kind], shapes
        numels = np.array([math.prod(s) for s in shapes], np.int64)
        room = numels if case["packed"] else (numels + 63) // 64 * 64
        ends = np.cumsum(room)
        self.off, self.numels, self.n = (ends - room).tolist(), numels.tolist(), int(ends[-1])
        both, counts = np.zeros((len(shapes), 2), np.float32), np.zeros((len(shapes), 2), np.int64)
        both[:, 0] = factors
        counts[:, 0], counts[:, 1] = numels, room - numels
        # a factor for each tensor's elements, 0 in the padding after it
        self.factor = torch.repeat_interleave(
            torch.from_numpy(both.ravel()).cuda(), torch.from_numpy(counts.ravel()).cuda(),
            output_size=self.n).mul_(sd)
        self.gen = gen
        self.grad = (self.normal() * (self.factor * case.get("scale", 1.0))).to(self.type)

    def normal(self):
        return torch.randn(self.n, generator=self.gen, device="cuda")

    def state(self, case):
        """Weights and moments of a run some hundred steps old."""
        self.w = self.normal().mul_(0.02).mul_(self.factor != 0)
        self.m = self.normal().mul_(0.3).mul_(self.factor)
        self.v = torch.rand(self.n, generator=self.gen, device="cuda").add_(0.1).mul_(self.factor.square())
        self.copy = self.w.to(TYPES[case["copy"]]) if case["copy"] else None

    def views(self, flat):
        return [flat[o:o + n].view(s) for o, n, s in zip(self.off, self.numels, self.shapes)]


def _tensors(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1 + int(seed))
    host = np.random.default_rng([int(seed), 3])
    groups = _groups(case)
    total = sum(math.prod(s) for _, shapes in groups for s in shapes)
    # gradients of a norm of several units, of which clipping leaves one; factors as they differ
    # from layer to layer
    sd = 2.0 / math.sqrt(total)
    made = []
    for kind, shapes in groups:
        factors = np.exp(host.uniform(math.log(0.3), math.log(10.0), len(shapes)))
        made.append(_Group(case, kind, shapes, sd, gen, factors))
    if case.get("overflow"):
        made[0].grad[made[0].off[-1]] = math.inf
    return made


def _join(groups, role):
    return [t for g in groups for t in g.views(getattr(g, role))]


def _matrix(gen, rows, cols, spread=True):
    """N(0, 1) times a factor for each column, with a few large columns, as activations have."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    if spread:
        f = torch.exp(torch.randn(cols, generator=gen, device="cuda") * 0.7)
        x.mul_(f)
    return x


def _tiles(scales):
    """E8M0 scales [rows, blocks] as they lie in memory: tiles of 128 rows by 4 blocks, 512 bytes
    each, byte (row % 32) * 16 + (row % 128) // 32 * 4 + block % 4; zero beyond the matrix."""
    r, c = scales.shape
    full = torch.zeros(-(-r // 128) * 128, -(-c // 4) * 4, dtype=torch.uint8, device=scales.device)
    full[:r, :c] = scales
    return full.view(full.shape[0] // 128, 4, 32, full.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()


def _untiled(tiles, rows, blocks):
    r, c = tiles.shape[:2]
    return tiles.permute(0, 3, 2, 1, 4).reshape(r * 128, c * 4)[:rows, :blocks]


def _packed(code):
    """E2M1 codes [rows, cols], two a byte, the even column in the low half; rows of a multiple of
    64 bytes, zero beyond the matrix."""
    r, c = code.shape
    full = torch.zeros(r, -(-c // 128) * 128, dtype=torch.uint8, device=code.device)
    full[:, :c] = code
    return full[:, 0::2] | full[:, 1::2] << 4


def prepare(case, seed):
    st = {"case": case}
    if case["op"] in ("clip", "adamw"):
        groups = st["groups"] = _tensors(case, seed)
        st["grads"] = _join(groups, "grad")
        if case["op"] == "clip":
            st["max_norm"] = MAX_NORM
            if own:
                from paper_2603_18112_gb300 import optim
                st["clipper"] = optim.GradClipper(st["grads"])
            return st
        for g in groups:
            g.state(case)
        st["params"], st["m"], st["v"] = (_join(groups, r) for r in ("w", "m", "v"))
        st["copies"] = _join(groups, "copy") if case["copy"] else None
        st["steps"] = torch.tensor([100, 0], dtype=torch.int64, device="cuda")
        if own:
            from paper_2603_18112_gb300 import optim
            st["step"] = optim.AdamWStep(
                st["params"], st["grads"], st["m"], st["v"], copies=st["copies"],
                max_norm=MAX_NORM if case["clip"] else 0.0, skip_nonfinite=case["clip"],
                steps=st["steps"])
        return st
    gen = torch.Generator(device="cuda").manual_seed(1 + int(seed))
    if case["op"] == "quant":
        x = _matrix(gen, case["rows"], case["stride"]).to(TYPES[case["type"]])
        st["x"] = x[:, :case["cols"]]
    elif case["op"] == "product":
        for name, rows in (("a", case["M"]), ("b", case["N"])):
            code, scale = _quantised(_matrix(gen, rows, case["K"]))
            st[name] = (_packed(code), _tiles(scale))
    else:
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = _matrix(gen, M, K).to(torch.bfloat16).requires_grad_()
        st["w"] = _matrix(gen, N, K, False).mul_(1 / math.sqrt(K)).requires_grad_()
        st["dy"] = _matrix(gen, M, N).mul_(1e-3).to(torch.bfloat16)
    return st


# --------------------------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------------------------

def _quantised(x):
    """MXFP4 codes [rows, cols] and scales [rows, blocks of 32] of an fp32 matrix: the scale
    2^(floor(log2 max|x|) - 2), elements to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the
    even code), at most 6.  A block with an infinity or NaN gets the scale NaN (255)."""
    r, c = x.shape
    nb = -(-c // 32)
    y = torch.nn.functional.pad(x, (0, nb * 32 - c)).view(r, nb, 32)
    top = y.abs().amax(2)
    e = torch.frexp(top)[1] - 3
    e = torch.where(top == 0, -127, e).clamp(-127, 127)
    a = y * (127 - e << 23).view(torch.float32)[..., None]
    sign = torch.signbit(a)
    a = a.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5.0)) | (sign.to(torch.uint8) << 3)
    scale = torch.where(torch.isfinite(top), e + 127, 255).to(torch.uint8)
    return code.view(r, nb * 32)[:, :c], scale


def _values(code, scale):
    """The matrix that codes and scales stand for."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    s = scale.int()
    s = torch.where(s == 0, 1 << 22, s << 23).view(torch.float32)  # 2^(scale - 127), by its bits
    s = torch.where(scale == 255, math.nan, s)
    r, c = code.shape
    return table[code.int()] * s.repeat_interleave(32, 1)[:, :c]


def _rounded(x):
    return _values(*_quantised(x))


def _unpacked(packed, tiles, rows, cols):
    code = torch.stack((packed & 15, packed >> 4), 2).view(rows, -1)[:, :cols]
    return _values(code, _untiled(tiles, rows, -(-cols // 32)))


def _plain_norm(groups, scale):
    return sum([(g.grad.float() / scale).square().sum() for g in groups]).sqrt()


def _plain_adamw(g, case, mult, t, go):
    """One group's step, left out where `go` is false."""
    grad = g.grad.float() * mult
    m = BETA1 * g.m + (1 - BETA1) * grad
    v = BETA2 * g.v + (1 - BETA2) * grad.square()
    c1, c2 = -torch.expm1(t * math.log(BETA1)), -torch.expm1(t * math.log(BETA2))
    w = g.w * (1 - LR * WD) - LR / c1 * m / (v.sqrt() / c2.sqrt() + EPS)
    g.w.copy_(torch.where(go, w, g.w))
    g.m.copy_(torch.where(go, m, g.m))
    g.v.copy_(torch.where(go, v, g.v))
    if g.copy is not None:
        g.copy.copy_(g.w)
    return {"w": g.w, "m": g.m, "v": g.v, "copy": g.copy}


def _run_clip(state):
    """The threshold falls a little from pass to pass: gradients that one pass has clipped are
    clipped by the next again, as the new gradients of a training loop would be."""
    top = state["max_norm"]
    state["max_norm"] *= 0.9999
    if own:
        record = state["clipper"].clip_(top)
        return {"norm": record[0], "grads": [g.grad for g in state["groups"]]}
    norm = _plain_norm(state["groups"], 1.0)
    coef = (top / (norm + 1e-6)).clamp(max=1.0)
    return {"norm": norm, "grads": [g.grad.copy_(g.grad.float() * coef) for g in state["groups"]]}


def _run_adamw(state):
    case, groups = state["case"], state["groups"]
    if own:
        step = state["step"]
        step.step(LR, (BETA1, BETA2), EPS, WD, grad_scale=case["scale"])
        out = {"steps": state["steps"],
               "groups": [{"w": g.w, "m": g.m, "v": g.v, "copy": g.copy} for g in groups]}
        return out | {"norm": step.record[0]} if case["clip"] else out
    mult, go = torch.full((), 1 / case["scale"], device="cuda"), torch.ones((), dtype=torch.bool, device="cuda")
    out = {"steps": state["steps"]}
    if case["clip"]:
        norm = out["norm"] = _plain_norm(groups, case["scale"])
        mult, go = mult * (MAX_NORM / (norm + 1e-6)).clamp(max=1.0), torch.isfinite(norm)
    state["steps"].add_(torch.stack((go, ~go)))
    t = state["steps"][0].float()
    return out | {"groups": [_plain_adamw(g, case, mult, t, go) for g in groups]}


def _run_quant(state):
    case, x = state["case"], state["x"]
    both = case["forms"] == "both"
    if own:
        from paper_2603_18112_gb300 import mx
        got = mx.quantize(x, cols=both)
        return [mx.dequantize(q, x.dtype) for q in (got if both else (got,))]
    y = x.float()
    return [_rounded(q).to(x.dtype) for q in ((y, y.t().contiguous()) if both else (y,))]


def _run_product(state):
    case = state["case"]
    M, N, K, kind = case["M"], case["N"], case["K"], TYPES[case["out"]]
    if own:
        from paper_2603_18112_gb300 import mx
        return mx.matmul(mx.MXMatrix(*state["a"], M, K), mx.MXMatrix(*state["b"], N, K), kind)
    return (_unpacked(*state["a"], M, K) @ _unpacked(*state["b"], N, K).t()).to(kind)


def _run_linear(state):
    x, w, dy = state["x"], state["w"], state["dy"]
    if own:
        from paper_2603_18112_gb300 import mx
        y = mx.linear(x, w)
        return (y.detach(), *torch.autograd.grad(y, (x, w), dy))
    with torch.no_grad():
        a, b, c = x.float(), w, dy.float()
        y = _rounded(a) @ _rounded(b).t()
        dx = _rounded(c) @ _rounded(b.t().contiguous()).t()
        dw = _rounded(c.t().contiguous()) @ _rounded(a.t().contiguous()).t()
        return y.to(x.dtype), dx.to(x.dtype), dw


def run(state):
    return {"clip": _run_clip, "adamw": _run_adamw, "quant": _run_quant, "product": _run_product,
            "linear": _run_linear}[state["case"]["op"]](state)


def work(case):
    op = case["op"]
    if op in ("clip", "adamw"):
        sizes = [({"f32": 4, "bf16": 2, "f16": 2}[t], sum(math.prod(s) for s in shapes))
                 for t, shapes in _groups(case)]
        n = sum(k for _, k in sizes)
        grads = sum(b * k for b, k in sizes)
        if op == "clip":
            return {"bytes": 2.0 * grads, "flops": 3.0 * n}
        return {"bytes": grads + 24.0 * n + (2.0 * n if case["copy"] else 0.0), "flops": 17.0 * n}
    if op == "quant":
        n = case["rows"] * case["cols"]
        forms = 2 if case["forms"] == "both" else 1
        size = 4 if case["type"] == "f32" else 2
        # the matrix read, a half byte and a 32nd written for each form, and its values
        return {"bytes": n * (size + forms * (17 / 32 + size)), "flops": 4.0 * forms * n}
    M, N, K = case["M"], case["N"], case["K"]
    if op == "product":
        return {"bytes": (M + N) * K * 17 / 32 + M * N * (4 if case["out"] == "f32" else 2),
                "flops": 2.0 * M * N * K}
    # x, w, dy read, y, dx, dw written
    return {"bytes": 2.0 * (2 * M * K + 2 * M * N) + 8.0 * N * K, "flops": 6.0 * M * N * K}


# --------------------------------------------------------------------------------------------
# The same in 64 bits
# --------------------------------------------------------------------------------------------

def _power64(k):
    """2^k in fp64, by its bits: a library's powers may be off in the last place."""
    return (k.long() + 1023 << 52).view(torch.float64)


def _near64(x):
    """x (fp64) with each block of 32 along the rows rounded to MXFP4: elements lie on a grid of
    a quarter of the largest's binade at least, an eighth below it, and so on."""
    r, c = x.shape
    y = torch.zeros(r, -(-c // 32) * 32, dtype=torch.float64, device=x.device)
    y[:, :c] = x
    y = y.view(r, -1, 32)
    top = y.abs().max(2, keepdim=True).values
    unit = torch.where(top > 0, _power64(torch.frexp(top)[1] - 3), 1.0).clamp(min=2.0 ** -127)
    a = y / unit
    # steps of 0.5 up to 2, of 1 up to 4, of 2 beyond
    grid = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0)).double()
    a = torch.round(a / grid) * grid
    return (a.clamp(-6, 6) * unit).view(r, -1)[:, :c]


def exact(case, seed):
    op = case["op"]
    if op in ("clip", "adamw"):
        groups = _tensors(case, seed)
        scale = case.get("scale", 1.0)
        norm = math.sqrt(sum(float((g.grad.double() / scale).square().sum()) for g in groups))
        coef = min(1.0, MAX_NORM / (norm + 1e-6))
        if op == "clip":
            return {"norm": torch.tensor(norm, dtype=torch.float64),
                    "grads": [g.grad.double() * coef for g in groups]}
        mult = (coef if case["clip"] else 1.0) / scale
        out = {"steps": None, "groups": []}
        if case["clip"]:
            out["norm"] = torch.tensor(norm, dtype=torch.float64)
        for g in groups:
            g.state(case)
            w, m, v = g.w.double(), g.m.double(), g.v.double()
            if not case["overflow"]:
                d = g.grad.double() * mult
                m = BETA1 * m + (1 - BETA1) * d
                v = BETA2 * v + (1 - BETA2) * d * d
                hat, var = m / (1 - BETA1 ** 101), v / (1 - BETA2 ** 101)
                w = w - LR * WD * w - LR * hat / (torch.sqrt(var) + EPS)
            out["groups"].append({"w": w, "m": m, "v": v, "copy": w if case["copy"] else None})
        return out
    st = prepare(case, seed)
    if op == "quant":
        x = st["x"].double()
        return [_near64(q) for q in ((x, x.t()) if case["forms"] == "both" else (x,))]
    if op == "product":
        a, b = (_decoded64(*st[n], rows, case["K"]) for n, rows in (("a", case["M"]), ("b", case["N"])))
        return a @ b.t()
    x, w, dy = (st[n].detach().double() for n in ("x", "w", "dy"))
    return (_near64(x) @ _near64(w).t(), _near64(dy) @ _near64(w.t()).t(),
            _near64(dy.t()) @ _near64(x.t()).t())



def _decoded64(packed, tiles, rows, cols):
    """Codes and tiled scales to fp64, by their bits: sign, two of exponent, one of mantissa."""
    code = torch.empty(rows, packed.shape[1] * 2, dtype=torch.int64, device=packed.device)
    code[:, 0::2], code[:, 1::2] = packed % 16, packed // 16
    e, man = code // 2 % 4, code % 2
    mag = torch.where(e > 0, (1 + 0.5 * man) * _power64(e - 1), 0.5 * man)
    value = torch.where(code >= 8, -mag, mag)
    r = torch.arange(rows, device=packed.device)[:, None]
    b = torch.arange(packed.shape[1] * 2, device=packed.device)[None] // 32
    flat = tiles.reshape(-1).long()
    at = ((r // 128) * tiles.shape[1] + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4
    return (value * _power64(flat[at] - 127))[:, :cols]
