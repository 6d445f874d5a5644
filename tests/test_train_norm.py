"""Layer norm and its gradients (tula_layer_norm*): refusals on the CPU; outputs and gradients against the
formulas in 64 bits, and against differences, on a GPU."""
import ctypes

import pytest
import torch

from paper_2603_18112_gb300 import norm
from paper_2603_18112_gb300.tula_ags import TulaError

TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUND = {t: torch.finfo(t).eps / 2 for t in TYPES}  # a rounding is off by at most half a step
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
U = 2.0 ** -24  # fp32's rounding


def test_refusals_of_the_library():
    L, n = norm._lib(), None
    p = ctypes.c_void_p(256)

    def forward(x=p, kind=0, rows=4, cols=8, stride=8, w=p, b=p, wkind=0, eps=1e-5, y=p, stats=p):
        return L.tula_layer_norm(x, kind, rows, cols, stride, w, b, wkind, eps, y, stats, n)

    odd = ctypes.c_void_p(258)
    for bad in ({"kind": 3}, {"wkind": -1}, {"rows": -1}, {"cols": -1}, {"cols": 1 << 25}, {"rows": 1 << 41}, {"stride": 7},
                {"eps": -1.0}, {"eps": float("nan")}, {"x": n}, {"y": n}, {"x": odd}, {"y": odd}, {"w": odd}, {"b": odd},
                {"stats": ctypes.c_void_p(260)}):
        assert forward(**bad) == -1, bad
    assert forward(rows=0, x=n) == 0 and forward(cols=0, stride=0, x=n) == 0

    def backward(dy=p, dstride=8, x=p, stride=8, kind=0, rows=4, cols=8, wkind=0, stats=p, dx=p, dw=n, space=n, size=0):
        return L.tula_layer_norm_backward(dy, dstride, x, stride, kind, rows, cols, p, wkind, stats, dx, dw, n, space, size, n)

    for bad in ({"kind": 3}, {"wkind": 3}, {"rows": -1}, {"stride": 7}, {"dstride": 7}, {"dy": n}, {"x": n}, {"stats": n}, {"dx": odd},
                {"dy": odd}, {"dw": odd}):
        assert backward(**bad) == -1, bad
    need = norm.tula_layer_norm_workspace_size(4, 8)
    short = L.tula_layer_norm_backward(p, 8, p, 8, 0, 4, 8, p, 0, p, p, p, n, p, need - 1, n)
    assert short == backward(dw=p) == -2
    assert L.tula_layer_norm_error(n, n) == -1
    with pytest.raises(TulaError):
        norm.tula_layer_norm_workspace_size(-1, 8)


def test_refusals_of_the_binding():
    x, w = torch.zeros(4, 8), torch.zeros(8)
    with pytest.raises(TypeError):
        norm.layer_norm(x, w)
    with pytest.raises(ValueError):
        norm.layer_norm(x, torch.zeros(7))
    with pytest.raises(ValueError):
        norm.layer_norm(x, w, torch.zeros(1))
    with pytest.raises(TypeError):
        norm.layer_norm(x, w, w.half())
    with pytest.raises(TypeError):
        norm.layer_norm(torch.zeros(()))


def _exact(x, w, b, dy, eps):
    """Output, gradients and how far each may be off before its last rounding."""
    x, dy = x.detach().double(), dy.detach().double()
    cols = x.shape[1]
    w64 = torch.ones(cols, dtype=torch.float64, device=x.device) if w is None else w.detach().double()
    b64 = torch.zeros_like(w64) if b is None else b.detach().double()
    mean = x.mean(1, keepdim=True)
    r = 1 / ((x - mean).square().mean(1, keepdim=True) + eps).sqrt()
    n, g = (x - mean) * r, dy * w64
    y = n * w64 + b64
    dx = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    dw, db = (dy * n).sum(0), dy.sum(0)
    # Sums over a row are trees of at most 8 + 5 + 5 + 8 additions in registers, exchanges, warps and
    # CTAs (wide rows: one of cols / 1024 + 10): the mean is off by `depth` roundings of the row's mean
    # magnitude, n by that and by some roundings (the variance's sum, the division, the root) of its own.
    depth = 28 if cols <= 65536 else cols // 1024 + 12
    off_n = U * (depth * x.abs().mean(1, keepdim=True) * r + (depth + 6) * n.abs())
    off_y = off_n * w64.abs() + 2 * U * (n * w64).abs() + 2 * U * b64.abs()
    ga, gn = g.abs().mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    off_dx = r * (U * (depth + 8) * (g.abs() + ga + 2 * n.abs() * gn) + off_n * gn + n.abs() * (g.abs() * off_n).mean(1, keepdim=True))
    off_dx = off_dx + dx.abs() * U * (depth + 6) + r * off_n.mean(1, keepdim=True) * ga
    # a column's sum: chains of at most 200 additions (a CTA's rows, its groups, the CTAs)
    off_dw = (dy.abs() * (off_n + 200 * U * n.abs())).sum(0)
    off_db = 200 * U * dy.abs().sum(0)
    return (y, dx, dw, db), (off_y, off_dx, off_dw, off_db)


def _inputs(rows, cols, dtype, wtype, seed, bias=True):
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen)

    x = (normal(rows, cols) * torch.exp(0.5 * normal(cols)) + normal(rows, 1)).to(dtype).cuda().requires_grad_()
    w = (1 + 0.3 * normal(cols)).to(wtype).cuda().requires_grad_()
    b = (0.2 * normal(cols)).to(wtype).cuda().requires_grad_() if bias else None
    return x, w, b, normal(rows, cols).to(dtype).cuda()


def _check(x, w, b, dy, eps=1e-5):
    y = norm.layer_norm(x, w, b, eps)
    leaves = [t for t in (x, w, b) if t is not None]
    grads = torch.autograd.grad(y, leaves, dy)
    want, off = _exact(x, w, b, dy, eps)
    keep = [True, True, w is not None, b is not None]
    want, off = ([t for t, k in zip(ts, keep) if k] for ts in (want, off))
    for got, ref, tol, like in zip((y, *grads), want, off, (x, *leaves)):
        assert got.dtype == like.dtype and got.shape == like.shape
        tol = tol + 1.01 * ROUND[got.dtype] * ref.abs() + TINY[got.dtype]
        bad = (got.detach().double() - ref).abs() - tol
        assert bool((bad <= 0).all()), (got.dtype, float(bad.max()))
    with torch.no_grad():
        assert torch.equal(norm.layer_norm(x, w, b, eps), y)
    return (y.detach(), *grads)


SIZES = [(1, 16), (1, 4096), (3, 8), (5, 17), (7, 33), (1000, 24), (33, 100), (64, 250), (129, 256), (65, 257), (40, 512), (300, 770),
         (77, 1023), (1001, 1024), (5000, 1001), (31, 2050), (700, 4096), (17, 8192), (9, 8193), (200, 12000), (3, 16386), (5, 40000),
         (2, 65536), (3, 65537), (70, 70000)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_layer_norm(rows, cols, dtype):
    for wtype in {torch.float32, dtype}:
        first = _check(*_inputs(rows, cols, dtype, wtype, rows + cols))
        again = _check(*_inputs(rows, cols, dtype, wtype, rows + cols))
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    assert norm.tula_layer_norm_error() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_without_parameters(dtype):
    x, w, b, dy = _inputs(50, 300, dtype, torch.float32, 1)
    _check(x, None, None, dy)
    _check(x, w, None, dy)
    _check(x, None, b, dy)
    y = norm.layer_norm(x.detach(), w, b)  # the parameters' gradients alone, and each by itself
    dw, db = torch.autograd.grad(y, (w, b), dy)
    full = torch.autograd.grad(norm.layer_norm(x, w, b), (x, w, b), dy)
    assert torch.equal(dw, full[1]) and torch.equal(db, full[2])
    assert torch.equal(torch.autograd.grad(norm.layer_norm(x.detach(), w, b), b, dy)[0], db)
    assert torch.equal(torch.autograd.grad(norm.layer_norm(x, w.detach(), b.detach()), x, dy)[0], full[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_views(dtype):
    """Rows apart, off 16-byte boundaries, transposed, repeated; more dimensions; gradients that are views."""
    x, w, b, dy = _inputs(120, 260, dtype, torch.float32, 2)
    for cut in (slice(0, 256), slice(3, 259), slice(1, 257), slice(8, 136)):
        a, g = x.detach()[:, cut].requires_grad_(), dy[:, cut]
        _check(a, w.detach()[cut].requires_grad_(), b.detach()[cut].requires_grad_(), g)
    _check(x.detach()[:, ::2].requires_grad_(), w.detach()[::2].requires_grad_(), None, dy[:, ::2])
    _check(x.detach().t().requires_grad_(), w.detach()[:120].requires_grad_(), None, dy.t())
    _check(x.detach()[:1].expand(40, 260).requires_grad_(), w, b, dy[:1].expand(40, 260))
    x3 = x.detach().view(4, 30, 260).transpose(0, 1).requires_grad_()
    y = norm.layer_norm(x3, w, b)
    assert y.shape == (30, 4, 260)
    flat = norm.layer_norm(x, w, b)
    assert torch.equal(y, flat.view(4, 30, 260).transpose(0, 1))
    ones = torch.autograd.grad(y.sum(), (x3, w, b))  # a gradient of strides 0
    ref = torch.autograd.grad(flat, (x, w, b), torch.ones_like(flat))
    assert torch.equal(ones[0], ref[0].view(4, 30, 260).transpose(0, 1))
    assert norm.layer_norm(x.detach()[0], w, b).shape == (260,)


@pytest.mark.gpu
def test_rows_of_zeros_equal_values_infinities_and_nan():
    x, w, b, dy = _inputs(40, 130, torch.float32, torch.float32, 3)
    x.data[2], x.data[3], x.data[4, 7], x.data[5, 9] = 0.0, 5.0, float("inf"), float("nan")
    y = norm.layer_norm(x, w, b)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    assert torch.equal(y[2], b) and torch.equal(y[3], b)
    assert bool(torch.isnan(y[4:6]).all()) and bool(torch.isfinite(y[6:]).all()) and bool(torch.isnan(dx[4:6]).all())
    assert bool(torch.isnan(dw).all())
    ok = [i for i in range(40) if i not in (4, 5)]
    _check(x.detach()[ok].requires_grad_(), w, b, dy[ok])
    big = x.detach()[6:].mul(1e15).requires_grad_()  # large and small rows
    _check(big, w, b, dy[6:])
    _check(x.detach()[6:].mul(1e-12).requires_grad_(), w, b, dy[6:])
    _check(x.detach()[6:].mul(1e-12).requires_grad_(), w, b, dy[6:], eps=0.0)


@pytest.mark.gpu
def test_empty():
    x, w = torch.zeros(0, 16, device="cuda", requires_grad=True), torch.ones(16, device="cuda", requires_grad=True)
    y = norm.layer_norm(x, w, w)
    dx, dw = torch.autograd.grad(y.sum(), (x, w))
    assert y.shape == dx.shape == (0, 16) and torch.equal(dw, torch.zeros(16, device="cuda"))
    e = torch.zeros(4, 0, device="cuda", requires_grad=True)
    v = torch.zeros(0, device="cuda", requires_grad=True)
    y = norm.layer_norm(e, v, v)
    assert y.shape == (4, 0) and torch.autograd.grad(y.sum(), (e, v))[0].shape == (4, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(6, 40), (4, 300), (2, 9000)])
def test_gradients_against_differences(rows, cols):
    """Along a random direction of all inputs, with central differences of the output in 64 bits."""
    x, w, b, dy = _inputs(rows, cols, torch.float32, torch.float32, 4)
    grads = torch.autograd.grad(norm.layer_norm(x, w, b), (x, w, b), dy)
    gen = torch.Generator(device="cuda").manual_seed(5)
    dirs = [torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64) for t in (x, w, b)]
    h = 1e-4

    def f(s):
        u, v, c = (t.detach().double() + s * h * d for t, d in zip((x, w, b), dirs))
        n = (u - u.mean(1, keepdim=True)) / (u.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
        return float(((n * v + c) * dy.double()).sum())

    slope = (f(1) - f(-1)) / (2 * h)
    own = sum(float((g.double() * d).sum()) for g, d in zip(grads, dirs))
    size = sum(float((g.double() * d).abs().sum()) for g, d in zip(grads, dirs))
    # the differences' own error is h^2 times a third derivative of the size of the sum; fp32's some roundings
    assert abs(own - slope) <= (20 * h * h + 60 * U) * size


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    x, w, b, dy = _inputs(500, 768, torch.bfloat16, torch.float32, 6)
    xs, ws, bs, ds = x.detach().clone().requires_grad_(), w.detach().clone().requires_grad_(), b.detach().clone().requires_grad_(), dy.clone()
    eager = norm.layer_norm(x, w, b)  # an eager graph lives meanwhile
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(norm.layer_norm(xs, ws, bs), (xs, ws, bs), ds)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = norm.layer_norm(xs, ws, bs)
        got = (y, *torch.autograd.grad(y, (xs, ws, bs), ds))
    for seed in (7, 8):
        x2, w2, b2, d2 = _inputs(500, 768, torch.bfloat16, torch.float32, seed)
        for s, t in ((xs, x2), (ws, w2), (bs, b2), (ds, d2)):
            s.detach().copy_(t.detach())
        graph.replay()
        y2 = norm.layer_norm(x2, w2, b2)
        want = (y2, *torch.autograd.grad(y2, (x2, w2, b2), d2))
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    want = torch.autograd.grad(eager, (x, w, b), dy)
    with torch.cuda.stream(side):
        y = norm.layer_norm(x, w, b)
        got = torch.autograd.grad(y, (x, w, b), dy)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.gpu
def test_hooks_on_saved_tensors():
    x, w, b, dy = _inputs(20, 64, torch.float32, torch.float32, 9)
    want = torch.autograd.grad(norm.layer_norm(x, w, b), (x, w, b), dy)
    with torch.autograd.graph.save_on_cpu():
        y = norm.layer_norm(x, w, b)
    assert all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(y, (x, w, b), dy), want))
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t[..., :1]):
        y = norm.layer_norm(x, w, b)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y, (x, w, b), dy)


@pytest.mark.gpu
def test_more_than_2_to_the_31_elements():
    rows, cols = (1 << 19) + 5, 4112
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[:, ::2] = 1.0
    x[-1] = torch.randn(cols, device="cuda")
    w = torch.full((cols,), 2.0, device="cuda", requires_grad=True)
    tail = x[-3:].clone()
    x.requires_grad_()
    y = norm.layer_norm(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), y.detach())
    short = tail.requires_grad_()
    ys = norm.layer_norm(short, w)
    dxs, _ = torch.autograd.grad(ys, (short, w), ys.detach())
    assert torch.equal(y[-3:], ys) and torch.equal(dx[-3:], dxs) and bool((y[:-1] == y[0]).all())
