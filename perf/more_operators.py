"""More operators of training that speed is measured on: orthogonalised updates (Muon), 8-bit
floating-point matrices with a scale for each block of 128, and layer norm.

A case is a dict of plain values.

op "orth": `batch` matrices, rows x cols, orthogonalised by five Newton-Schulz steps
  type, out  of the matrices and of what comes out: "f32", "bf16", "f16"
op "muon": one Muon step over a list of matrices: momentum, Newton-Schulz, weights and copies
  set       "layers": `layers` blocks of width `d` (four d x d matrices, ff x d and d x ff); "odd":
            `shapes` shapes, two matrices each, sides log-uniform in [lo, hi]
  type      of the gradients
  copy      type of the weights' copies for the model, or ""
  nesterov  the momentum looks ahead
  clip      by the global norm, and a loss scale in the gradients; the step is left out with an
            infinite one
op "quant8": a matrix quantised to 8 bits and read back
  rows, cols, type, stride (elements from row to row)
  code      "e4m3" or "e5m2"
  forms     "rows": blocks along the rows; "both": also the transposed matrix, with blocks along
            the columns
  square    blocks of 128 x 128 (weights) instead of 1 x 128 (activations)
op "product8": A B^T of two such matrices, M x K (blocks 1 x 128) and N x K (128 x 128); out "bf16"
  or "f32"
op "linear8": y = x w^T on 8-bit operands and its gradients dx and dw; x and dy of `type`, w of
  `wtype`; code: of dy
op "norm": layer norm over rows of cols elements; x of `type`, weight and bias of `wtype`
  dir       "fwd": the output alone; "both": its three gradients too
  bias      with a bias, or a weight alone
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "": 0}
CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
NS = (3.4445, -4.7750, 2.0315)  # the quintic that Muon's Newton-Schulz steps apply to singular values
NS_STEPS = 5
LR, MU, WD = 2e-4, 0.95, 0.1
MAX_NORM, LOSS_SCALE = 1.0, 1024.0
EPS = 1e-5


def _muon(**kw):
    case = {"op": "muon", "type": "bf16", "copy": "bf16", "nesterov": True, "clip": False}
    case.update(kw)
    return case


def listed():
    return [
        # The smallest call: one convolution of a CIFAR ResNet-20's last stage, its kernels as rows.
        {"name": "orth_one", "op": "orth", "batch": 1, "rows": 64, "cols": 576, "type": "f32",
         "out": "bf16"},
        # Tall matrices of odd sizes, as of an expert layer, whose update another optimiser applies.
        {"name": "orth_batch", "op": "orth", "batch": 6, "rows": 4099, "cols": 1502, "type": "bf16",
         "out": "f16"},
        # The hidden layers of an ordinary language model in training.
        _muon(name="muon_layers", set="layers", layers=12, d=1024, ff=4096),
        # Small matrices of unequal odd sizes, half precision with a loss scale, clipped.
        _muon(name="muon_odd", set="odd", shapes=8, lo=17, hi=700, type="f16", copy="f16", clip=True),
        # A batch's activations for the forward product and for the weight gradient.
        {"name": "quant8_batch", "op": "quant8", "rows": 8192, "cols": 4096, "stride": 4096,
         "type": "bf16", "code": "e4m3", "forms": "both", "square": False},
        # Master weights of odd sizes, a view into a wider matrix.
        {"name": "quant8_weights", "op": "quant8", "rows": 4999, "cols": 2047, "stride": 2050,
         "type": "f32", "code": "e4m3", "forms": "both", "square": True},
        # One token through the largest layer of VGG-16: the weights are what is read.
        {"name": "product8_token", "op": "product8", "M": 1, "N": 4096, "K": 25088, "out": "bf16"},
        # A large square product.
        {"name": "product8_square", "op": "product8", "M": 8192, "N": 8192, "K": 8192, "out": "bf16"},
        # A layer in training, forward and backward.
        {"name": "linear8_train", "op": "linear8", "M": 8192, "N": 8192, "K": 4096, "type": "bf16",
         "wtype": "f32", "code": "e4m3"},
        # A narrow layer of odd sizes, its gradients in the code of wider range.
        {"name": "linear8_odd", "op": "linear8", "M": 1003, "N": 1234, "K": 777, "type": "f16",
         "wtype": "bf16", "code": "e5m2"},
        # One token on its way through a served model.
        {"name": "norm_token", "op": "norm", "rows": 1, "cols": 4096, "type": "bf16",
         "wtype": "bf16", "dir": "fwd", "bias": True},
        # A batch's tokens in training, forward and backward.
        {"name": "norm_train", "op": "norm", "rows": 16384, "cols": 4096, "type": "bf16",
         "wtype": "f32", "dir": "both", "bias": True},
    ]


MOST_FLOPS = 6e11  # of a drawn case; the largest listed ones have 1.6e12 and more
MOST_ELEMS = 1 << 26  # of a drawn matrix; the largest listed one has 2^26


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("orth", "muon", "quant8", "product8", "linear8", "norm"))
    types = ("f32", "bf16", "f16")
    while True:
        case = {"op": op}
        if op == "orth":
            case |= {"batch": _log(rng, 1, 24), "rows": _log(rng, 16, 5000), "cols": _log(rng, 16, 5000),
                     "type": rng.choice(types), "out": rng.choice(("bf16", "f16"))}
        elif op == "muon":
            case = _muon(type=rng.choice(types), copy=rng.choice(("", "bf16", "f16")),
                         nesterov=rng.random() < 0.7, clip=rng.random() < 0.4)
            if rng.random() < 0.4:
                case |= {"set": "layers", "layers": rng.randint(1, 16), "d": 8 * _log(rng, 4, 200)}
                case["ff"] = 4 * case["d"] + rng.choice((0, 8))
            else:
                case |= {"set": "odd", "shapes": rng.randint(1, 16), "lo": _log(rng, 1, 200)}
                case["hi"] = _log(rng, case["lo"] + 1, 2500)
        elif op == "quant8":
            case |= {"rows": _log(rng, 1, 1 << 15), "cols": _log(rng, 1, 1 << 15),
                     "type": rng.choice(types), "code": rng.choice(("e4m3", "e4m3", "e5m2")),
                     "forms": rng.choice(("rows", "both")), "square": rng.random() < 0.4}
            case["stride"] = case["cols"] + rng.choice((0, 0, 0, 1, 8, 64))
        elif op == "norm":
            case |= {"rows": _log(rng, 1, 1 << 17), "cols": _log(rng, 16, 1 << 15), "type": rng.choice(types),
                     "dir": rng.choice(("fwd", "both", "both")), "bias": rng.random() < 0.7}
            case["wtype"] = rng.choice(("f32", case["type"]))
        else:
            case |= {"M": _log(rng, 1, 1 << 14), "N": _log(rng, 16, 1 << 14), "K": _log(rng, 16, 1 << 14)}
            if rng.random() < 0.5:
                case["N"], case["K"] = -(-case["N"] // 64) * 64, -(-case["K"] // 64) * 64
            if op == "product8":
                case["out"] = rng.choice(("bf16", "f32"))
            else:
                case |= {"type": rng.choice(("bf16", "f16")), "wtype": rng.choice(("f32", "bf16")),
                         "code": rng.choice(("e4m3", "e5m2"))}
        elems = (case.get("stride") or case.get("cols", 1)) * case.get("rows", 1) * case.get("batch", 1)
        if work(case)["flops"] <= MOST_FLOPS and elems <= MOST_ELEMS:
            return case


# --------------------------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------------------------

def _shapes(case):
    """The list's shapes as [(count, rows, cols)]."""
    if case["set"] == "layers":
        n, d, ff = case["layers"], case["d"], case["ff"]
        return [(4 * n, d, d), (n, ff, d), (n, d, ff)]
    rng = random.Random(f"{case['shapes']} {case['lo']} {case['hi']}")
    return [(2, _log(rng, case["lo"], case["hi"]), _log(rng, case["lo"], case["hi"]))
            for _ in range(case["shapes"])]


def _updates(gen, n, rows, cols):
    """Matrices as gradients are: rows and columns of unequal size, and a few directions that many
    samples share."""
    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    x = normal(n, rows, cols)
    x.mul_(torch.exp(0.5 * normal(n, 1, cols)))
    x.add_(torch.bmm(normal(n, rows, 4), normal(n, 4, cols)), alpha=0.25)
    return x


def _matrix(gen, rows, cols, spread=0.7):
    """N(0, 1) times a factor for each column, with a few large columns, as activations have."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    return x.mul_(torch.exp(torch.randn(cols, generator=gen, device="cuda") * spread))


def _tiles(scales):
    """E8M0 scales [rows, blocks] as they lie in memory: tiles of 128 rows by 4 blocks, 512 bytes
    each, byte (row % 32) * 16 + (row % 128) // 32 * 4 + block % 4; zero beyond the matrix."""
    r, c = scales.shape
    full = torch.zeros(-(-r // 128) * 128, -(-c // 4) * 4, dtype=torch.uint8, device=scales.device)
    full[:r, :c] = scales
    return full.view(full.shape[0] // 128, 4, 32, full.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()


def _coded(x, square):
    """Codes (uint8, rows of a multiple of 128, zero beyond the matrix) and tiles of scales of an
    fp32 matrix."""
    value, scale = _quantised(x, "e4m3", square)
    codes = torch.zeros(x.shape[0], -(-x.shape[1] // 128) * 128, dtype=torch.uint8, device=x.device)
    codes[:, :x.shape[1]] = value.to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, _tiles(scale)


def prepare(case, seed):
    st = {"case": case}
    op = case["op"]
    gen = torch.Generator(device="cuda").manual_seed(1 + int(seed))
    if op == "orth":
        st["x"] = (_updates(gen, case["batch"], case["rows"], case["cols"]) * 1e-3).to(TYPES[case["type"]])
    elif op == "muon":
        groups = st["groups"] = []
        total = sum(n * r * c for n, r, c in _shapes(case))
        # gradients of a norm of some units, weights and a momentum of a run some hundred steps old
        scale = 2.0 / math.sqrt(total) * (LOSS_SCALE if case["clip"] else 1.0)
        for n, r, c in _shapes(case):
            g = {"g": (_updates(gen, n, r, c) * scale).to(TYPES[case["type"]]),
                 "w": torch.randn(n, r, c, generator=gen, device="cuda").mul_(0.02),
                 "m": _updates(gen, n, r, c).mul_(6.0 / math.sqrt(total))}
            g["copy"] = g["w"].to(TYPES[case["copy"]]) if case["copy"] else None
            groups.append(g)
        if own:
            from paper_2603_18112_gb300 import optim

            def each(role):
                return [m for g in groups for m in g[role].unbind(0)]

            st["clipper"] = optim.GradClipper(each("g")) if case["clip"] else None
            st["step"] = optim.MuonStep(each("w"), each("g"), each("m"),
                                        copies=each("copy") if case["copy"] else None,
                                        nesterov=case["nesterov"], ns_steps=NS_STEPS, scale="rms")
    elif op == "quant8":
        st["x"] = _matrix(gen, case["rows"], case["stride"]).to(TYPES[case["type"]])[:, :case["cols"]]
    elif op == "product8":
        st["a"] = _coded(_matrix(gen, case["M"], case["K"]), False)
        st["b"] = _coded(_matrix(gen, case["N"], case["K"], 0.3), True)
    elif op == "linear8":
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = _matrix(gen, M, K).to(TYPES[case["type"]]).requires_grad_()
        st["w"] = _matrix(gen, N, K, 0.3).mul_(1 / math.sqrt(K)).to(TYPES[case["wtype"]]).requires_grad_()
        st["dy"] = _matrix(gen, M, N).mul_(1e-2).to(TYPES[case["type"]])
    else:
        r, c = case["rows"], case["cols"]
        train = case["dir"] == "both"
        # a residual stream: columns of unequal size, rows off the mean
        x = _matrix(gen, r, c, 0.5).add_(torch.randn(r, 1, generator=gen, device="cuda"))
        st["x"] = x.to(TYPES[case["type"]]).requires_grad_(train)
        wtype = TYPES[case["wtype"]]
        st["w"] = torch.randn(c, generator=gen, device="cuda").mul_(0.2).add_(1).to(wtype).requires_grad_(train)
        st["b"] = (torch.randn(c, generator=gen, device="cuda").mul_(0.1).to(wtype).requires_grad_(train)
                   if case["bias"] else None)
        st["dy"] = _matrix(gen, r, c, 0.3).mul_(1e-2).to(TYPES[case["type"]]) if train else None
    return st


# --------------------------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------------------------

def _orthogonalised(u):
    """Five Newton-Schulz steps on a batch of fp32 matrices of Frobenius norm 1."""
    a, b, c = NS
    u = u / u.square().sum((1, 2), keepdim=True).sqrt()
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    for _ in range(NS_STEPS):
        gram = torch.bmm(x, x.transpose(1, 2))
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return x.transpose(1, 2) if tall else x


def _run_orth(state):
    case, x = state["case"], state["x"]
    if own:
        from paper_2603_18112_gb300 import optim
        return optim.orthogonalize(x, steps=NS_STEPS, dtype=TYPES[case["out"]])
    return _orthogonalised(x.float()).to(TYPES[case["out"]])


def _plain_muon(g, case, mult, go):
    """The step of one shape's matrices, left out where `go` is false."""
    d = g["g"].float() * mult
    m = MU * g["m"] + d
    x = _orthogonalised(d + MU * m if case["nesterov"] else m)
    w = g["w"] * (1 - LR * WD) - LR * 0.2 * math.sqrt(max(x.shape[1:])) * x
    g["m"].copy_(torch.where(go, m, g["m"]))
    g["w"].copy_(torch.where(go, w, g["w"]))
    if g["copy"] is not None:
        g["copy"].copy_(g["w"])
    return {"w": g["w"], "m": g["m"], "copy": g["copy"]}


def _run_muon(state):
    case, groups = state["case"], state["groups"]
    if own:
        record = state["clipper"].norm(LOSS_SCALE, MAX_NORM) if case["clip"] else None
        state["step"].step(LR, MU, WD, grad_scale=LOSS_SCALE if case["clip"] else 1.0, record=record)
        return [{"w": g["w"], "m": g["m"], "copy": g["copy"]} for g in groups]
    mult = torch.ones((), device="cuda")
    go = torch.ones((), dtype=torch.bool, device="cuda")
    if case["clip"]:
        norm = sum([(g["g"].float() / LOSS_SCALE).square().sum() for g in groups]).sqrt()
        mult, go = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0) / LOSS_SCALE, torch.isfinite(norm)
    return [_plain_muon(g, case, mult, go) for g in groups]


def _quantised(x, code, square):
    """The 8-bit values [rows, cols] and scale bytes [rows, blocks of 128] of an fp32 matrix.  A
    block's scale is the least power of two that brings it within the code's largest value; one with
    an infinity or NaN gets the scale NaN (255)."""
    most, least, bits = {"e4m3": (8, -6, 3), "e5m2": (15, -14, 2)}[code]
    r, c = x.shape
    nb = -(-c // 128)
    y = torch.nn.functional.pad(x, (0, nb * 128 - c)).view(r, nb, 128)
    top = y.abs().amax(2)
    if square:
        nr = -(-r // 128)
        top = torch.nn.functional.pad(top, (0, 0, 0, nr * 128 - r)).view(nr, 128, nb).amax(1)
        top = top.repeat_interleave(128, 0)[:r]
    man, e = torch.frexp(top)
    s = torch.where(top == 0, 0, e + 127 - 1 - most + (man > 0.875)).clamp(0, 254)
    a = y * (254 - s << 23).view(torch.float32)[..., None]
    step = ((torch.frexp(a)[1] - 1).clamp(min=least) - bits + 127 << 23).view(torch.float32)  # by its bits
    a = torch.round(a / step) * step
    finite = torch.isfinite(top)
    a = torch.where(finite[..., None], a, 0.0)
    return a.view(r, nb * 128)[:, :c], torch.where(finite, s, 255).to(torch.uint8)


def _scaled(value, scale):
    """The matrix that values and scale bytes stand for."""
    s = scale.int()
    s = torch.where(s == 0, 1 << 22, s << 23).view(torch.float32)  # 2^(scale - 127), by its bits
    s = torch.where(scale == 255, math.nan, s)
    return value * s.repeat_interleave(128, 1)[:, :value.shape[1]]


def _rounded(x, code="e4m3", square=False):
    return _scaled(*_quantised(x, code, square))


def _unpacked(codes, tiles, rows, cols):
    r, c = tiles.shape[:2]
    scale = tiles.permute(0, 3, 2, 1, 4).reshape(r * 128, c * 4)[:rows, :-(-cols // 128)]
    return _scaled(codes[:, :cols].view(torch.float8_e4m3fn).float(), scale)


def _run_quant8(state):
    case, x = state["case"], state["x"]
    both = case["forms"] == "both"
    if own:
        from paper_2603_18112_gb300 import fp8
        got = fp8.quantize(x, cols=both, square=case["square"], dtype=CODES[case["code"]])
        return [fp8.dequantize(q, x.dtype) for q in (got if both else (got,))]
    y = x.float()
    return [_rounded(q, case["code"], case["square"]).to(x.dtype)
            for q in ((y, y.t().contiguous()) if both else (y,))]


def _run_product8(state):
    case = state["case"]
    M, N, K, kind = case["M"], case["N"], case["K"], TYPES[case["out"]]
    if own:
        from paper_2603_18112_gb300 import fp8
        return fp8.matmul(fp8.FP8Matrix(*state["a"], M, K), fp8.FP8Matrix(*state["b"], N, K), kind)
    return (_unpacked(*state["a"], M, K) @ _unpacked(*state["b"], N, K).t()).to(kind)


def _run_linear8(state):
    case, x, w, dy = state["case"], state["x"], state["w"], state["dy"]
    if own:
        from paper_2603_18112_gb300 import fp8
        y = fp8.linear(x, w, grad_dtype=CODES[case["code"]])
        return (y.detach(), *torch.autograd.grad(y, (x, w), dy))
    with torch.no_grad():
        a, b, c = x.float(), _rounded(w.float(), square=True), dy.float()
        y = _rounded(a) @ b.t()
        dx = _rounded(c, case["code"]) @ b
        dw = _rounded(c.t().contiguous(), case["code"]) @ _rounded(a.t().contiguous()).t()
        return y.to(x.dtype), dx.to(x.dtype), dw.to(w.dtype)


def _run_norm(state):
    case, x, w, b, dy = state["case"], state["x"], state["w"], state["b"], state["dy"]
    train = case["dir"] == "both"
    if own:
        from paper_2603_18112_gb300 import norm
        y = norm.layer_norm(x, w, b, EPS)
        leaves = [t for t in (x, w, b) if t is not None]
        return [y.detach(), *(torch.autograd.grad(y, leaves, dy) if train else ())]
    with torch.no_grad():
        c = x.float() - x.float().mean(1, keepdim=True)
        r = 1 / (c.square().mean(1, keepdim=True) + EPS).sqrt()
        n = c * r
        y = n * w.float()
        out = [(y + b.float() if b is not None else y).to(x.dtype)]
        if train:
            d = dy.float()
            g = d * w.float()
            dx = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
            out += [dx.to(x.dtype), (d * n).sum(0).to(w.dtype)]
            out += [d.sum(0).to(w.dtype)] if b is not None else []
        return out


def run(state):
    return {"orth": _run_orth, "muon": _run_muon, "quant8": _run_quant8, "product8": _run_product8,
            "linear8": _run_linear8, "norm": _run_norm}[state["case"]["op"]](state)


def work(case):
    op = case["op"]
    if op in ("orth", "muon"):
        sets = [(case["batch"], case["rows"], case["cols"])] if op == "orth" else _shapes(case)
        elems = sum(n * r * c for n, r, c in sets)
        # of a symmetric product half the elements: two of them, n x n, and one n x m a step
        flops = sum(NS_STEPS * k * (3.0 * min(r, c) * r * c + 1.0 * min(r, c) ** 3) for k, r, c in sets)
        each = SIZE[case["type"]] + (SIZE[case["out"]] if op == "orth" else 16 + SIZE[case["copy"]])
        return {"bytes": 1.0 * elems * each, "flops": flops}
    if op == "quant8":
        n = case["rows"] * case["cols"]
        forms, size = (2 if case["forms"] == "both" else 1), SIZE[case["type"]]
        # the matrix read, a byte and a 128th of one written for each form, and its values
        return {"bytes": n * (size + forms * (129 / 128 + size)), "flops": 4.0 * forms * n}
    if op == "norm":
        n = case["rows"] * case["cols"]
        both = case["dir"] == "both"
        # x read and y written, dy read and dx written
        return {"bytes": n * SIZE[case["type"]] * (4.0 if both else 2.0) + 4.0 * case["cols"] * SIZE[case["wtype"]],
                "flops": n * (19.0 if both else 8.0)}
    M, N, K = case["M"], case["N"], case["K"]
    if op == "product8":
        return {"bytes": (M + N) * K * 129 / 128 + M * N * SIZE[case["out"]], "flops": 2.0 * M * N * K}
    # x, w, dy read, y, dx, dw written
    return {"bytes": 2.0 * SIZE[case["type"]] * (M * K + M * N) + 2.0 * SIZE[case["wtype"]] * N * K,
            "flops": 6.0 * M * N * K}


# --------------------------------------------------------------------------------------------
# The same in 64 bits
# --------------------------------------------------------------------------------------------

def _orth64(u):
    """Horner's form of the polynomial, along the rows as they are or the columns."""
    a, b, c = NS
    x = u / torch.linalg.vector_norm(u, dim=(1, 2), keepdim=True)
    for _ in range(NS_STEPS):
        if x.shape[1] <= x.shape[2]:
            gram = x @ x.mT
            p = c * gram
            p.diagonal(dim1=1, dim2=2).add_(b)
            p = p @ gram
            p.diagonal(dim1=1, dim2=2).add_(a)
            x = p @ x
        else:
            gram = x.mT @ x
            p = c * gram
            p.diagonal(dim1=1, dim2=2).add_(b)
            p = gram @ p
            p.diagonal(dim1=1, dim2=2).add_(a)
            x = x @ p
    return x


def _power64(k):
    """2^k in fp64, by its bits: a library's powers may be off in the last place."""
    return (k.long() + 1023 << 52).view(torch.float64)


def _near64(x, code="e4m3", square=False):
    """x (fp64) with each block rounded to 8 bits: the largest magnitude of a block lies in the
    code's top binades, steps are an 8th (e4m3) or a 4th (e5m2) of an element's own binade."""
    parts, top_e, low_e = (8, 8, -6) if code == "e4m3" else (4, 15, -14)
    r, c = x.shape
    rows = 128 if square else 1
    y = torch.zeros(-(-r // rows) * rows, -(-c // 128) * 128, dtype=torch.float64, device=x.device)
    y[:r, :c] = x
    y = y.view(y.shape[0] // rows, rows, y.shape[1] // 128, 128)
    top = y.abs().amax((1, 3), keepdim=True)
    t = torch.frexp(top)[1] - 1 - top_e
    t = t + (top > 1.75 * _power64(t + top_e))
    unit = _power64(torch.where(top > 0, t, 0).clamp(min=-127))
    a = y / unit
    grid = _power64((torch.frexp(a)[1] - 1).clamp(min=low_e)) / parts
    return (torch.round(a / grid) * grid * unit).view(-1, y.shape[2] * 128)[:r, :c]


def _decoded64(codes, tiles, rows, cols):
    """E4M3 codes and tiled scales to fp64, by their bits: sign, four of exponent, three of mantissa."""
    code = codes.long()
    e, man = code // 8 % 16, code % 8
    mag = torch.where(e > 0, (8 + man) * _power64(e - 10), man * _power64(e - 9))
    r = torch.arange(rows, device=codes.device)[:, None]
    b = torch.arange(codes.shape[1], device=codes.device)[None] // 128
    flat = tiles.reshape(-1).long()
    at = ((r // 128) * tiles.shape[1] + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4
    return (torch.where(code >= 128, -mag, mag) * _power64(flat[at] - 127))[:, :cols]


def exact(case, seed):
    op = case["op"]
    st = prepare(case, seed)
    if op == "orth":
        return _orth64(st["x"].double())
    if op == "muon":
        coef = 1.0
        if case["clip"]:
            norm = math.sqrt(sum(float((g["g"].double() / LOSS_SCALE).square().sum()) for g in st["groups"]))
            coef = min(1.0, MAX_NORM / (norm + 1e-6)) / LOSS_SCALE
        out = []
        for g in st["groups"]:
            d = g["g"].double() * coef
            m = g["m"].double() * MU + d
            x = _orth64(d + m * MU if case["nesterov"] else m)
            w = g["w"].double()
            w = w - LR * (WD * w + 0.2 * max(w.shape[1:]) ** 0.5 * x)
            out.append({"w": w, "m": m, "copy": w if case["copy"] else None})
        return out
    if op == "quant8":
        x = st["x"].double()
        return [_near64(q, case["code"], case["square"])
                for q in ((x, x.t()) if case["forms"] == "both" else (x,))]
    if op == "product8":
        return _decoded64(*st["a"], case["M"], case["K"]) @ _decoded64(*st["b"], case["N"], case["K"]).t()
    if op == "linear8":
        x, w, dy = (st[n].detach().double() for n in ("x", "w", "dy"))
        q = _near64(w, square=True)
        return (_near64(x) @ q.t(), _near64(dy, case["code"]) @ q,
                _near64(dy.t(), case["code"]) @ _near64(x.t()).t())
    # by autograd through the definition
    x, w = (st[n].detach().double().requires_grad_() for n in ("x", "w"))
    b = st["b"].detach().double().requires_grad_() if case["bias"] else None
    var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
    y = (x - mean) / torch.sqrt(var + EPS) * w
    y = y + b if case["bias"] else y
    leaves = [x, w] + ([b] if case["bias"] else [])
    grads = torch.autograd.grad(y, leaves, st["dy"].double()) if case["dir"] == "both" else ()
    return [y.detach(), *grads]
