"""8-bit matrices with a scale for each block of 128 (tula_fp8_*): the host's side on the CPU; codes and
scales bit for bit against a plain quantiser in 64 bits, products and layers against 64-bit products of
what the codes stand for, on a GPU."""
import ctypes
import math

import pytest
import torch

from paper_2603_18112_gb300 import fp8
from paper_2603_18112_gb300.tula_ags import TulaError

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
MOST = {E4: 448.0, E5: 57344.0}
# a rounding is off by at most half a step
ROUND = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # below the normal range


# --------------------------------------------------------------------------------------------
# In 64 bits, on the CPU
# --------------------------------------------------------------------------------------------

def quantised64(x, code=E4, square=False):
    """Values (before the scale) [r, c] in fp64 and scale bytes [r, ceil(c / 128)]."""
    x = x.detach().double().cpu()
    r, c = x.shape
    values, scales = torch.zeros(r, c, dtype=torch.float64), torch.zeros(r, -(-c // 128), dtype=torch.int64)
    least, bits = (-6, 3) if code == E4 else (-14, 2)
    rows = 128 if square else 1
    for i in range(0, r, rows):
        for j in range(0, c, 128):
            block = x[i:i + rows, j:j + 128]
            if not bool(torch.isfinite(block).all()):
                scales[i:i + rows, j // 128] = 255
                continue
            top = float(block.abs().max())
            t = -127
            while top > MOST[code] * 2.0 ** t:
                t += 1
            scales[i:i + rows, j // 128] = t + 127
            a = block / 2.0 ** t
            e = torch.frexp(a)[1] - 1
            step = 2.0 ** (e.clamp(min=least) - bits).double()
            values[i:i + rows, j:j + 128] = torch.round(a / step) * step
    return values, scales


def values64(values, scales):
    s = 2.0 ** (scales.double() - 127)
    s[scales == 255] = math.nan
    return values * s.repeat_interleave(128, 1)[:, :values.shape[1]]


def unpacked(q):
    """A matrix's values (before the scale) and scale bytes, after checking that what lies beyond the
    matrix is zero."""
    codes, tiles = q.codes.cpu(), q.scales.cpu()
    p = -(-q.cols // 128) * 128
    assert codes.shape == (q.rows, p) and not codes[:, q.cols:].any()
    flat = tiles.permute(0, 3, 2, 1, 4).reshape(tiles.shape[0] * 128, tiles.shape[1] * 4)
    nb = p // 128
    assert not flat[q.rows:].any() and not flat[:, nb:].any()
    return codes[:, :q.cols].view(q.dtype).double(), flat[:q.rows, :nb].long()


def _matrix(r, c, dtype, seed, spread=3.0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(r, c, generator=gen) * torch.exp(spread * torch.randn(1, c, generator=gen))
    return (x * torch.exp(spread * torch.randn(r, 1, generator=gen))).to(dtype)


# --------------------------------------------------------------------------------------------
# On the CPU
# --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("r,c", [(0, 0), (1, 1), (128, 512), (129, 513), (5, 4096)])
def test_sizes(r, c):
    codes, scales = fp8.tula_fp8_size(r, c)
    assert codes == r * -(-c // 128) * 128 and scales == -(-r // 128) * -(-c // 512) * 512
    assert fp8.FP8Matrix._sizes(r, c) == (scales, codes)


def test_refusals_of_the_library():
    L, n, big = fp8._lib(), None, 1 << 40
    p = ctypes.c_void_p(256)

    def quant(x=p, kind=0, r=4, c=4, stride=4, code=0, codes=p, scales=p, codes_t=n, scales_t=n):
        return L.tula_fp8_quantize(x, kind, r, c, stride, code, 0, codes, scales, codes_t, scales_t, n)

    for bad in ({"kind": 3}, {"kind": -1}, {"code": 2}, {"code": -1}, {"r": -1}, {"c": -1}, {"r": big}, {"stride": 3}, {"x": n},
                {"codes": n}, {"scales": n}, {"codes_t": p}, {"codes": n, "scales": n}, {"codes": ctypes.c_void_p(8)},
                {"x": ctypes.c_void_p(2)}, {"codes_t": p, "scales_t": ctypes.c_void_p(24)}):
        assert quant(**bad) == -1, bad

    def product(ac=0, bc=0, m=4, k=4, a=p, out=p, kind=0):
        return L.tula_fp8_matmul(a, p, ac, p, p, bc, m, 4, k, out, kind, n)

    for bad in ({"ac": 2}, {"bc": -1}, {"m": -1}, {"k": big}, {"a": n}, {"out": n}, {"kind": 5}, {"out": ctypes.c_void_p(2)},
                {"a": ctypes.c_void_p(8)}):
        assert product(**bad) == -1, bad
    assert L.tula_fp8_dequantize(p, p, 4, 4, 2, p, 0, n) == -1 and L.tula_fp8_dequantize(n, p, 4, 4, 0, p, 0, n) == -1
    assert L.tula_fp8_error(n, n) == -1

    def layer(data=256, stride=128, kind=0, transposed=0, m=4, k=128, code=0, kept=p, temp=p, y=p):
        x = fp8.tula_fp8_operand(data, stride, kind, transposed)
        return L.tula_fp8_linear(x, fp8.tula_fp8_operand(256, 128, 0, 0), m, 4, k, code, 1, 1, kept, temp, y, n)

    def back(data=256, stride=8, kind=0, transposed=0, code=0, grad_code=1, kept=p, temp=p, dx=p, dxt=0, dw=p, dwt=0):
        dy = fp8.tula_fp8_operand(data, stride, kind, transposed)
        return L.tula_fp8_linear_backward(dy, 4, 8, 128, code, grad_code, kept, temp, dx, dxt, dw, dwt, 1, 1, n)

    for bad in ({"data": None}, {"data": 258}, {"stride": 127}, {"kind": 3}, {"transposed": 1, "stride": 3}, {"m": -1}, {"k": big}, {"code": 2}, {"y": n},
                {"kept": ctypes.c_void_p(8)}, {"temp": ctypes.c_void_p(8)}, {"y": ctypes.c_void_p(258)}):
        assert layer(**bad) == -1, bad
    for bad in ({"data": None}, {"stride": 7}, {"kind": -1}, {"transposed": 1, "stride": 3}, {"code": -1}, {"grad_code": 2}, {"dx": n}, {"dw": n},
                {"dxt": 3}, {"dwt": -1}, {"dw": ctypes.c_void_p(258)}, {"temp": ctypes.c_void_p(8)}):
        assert back(**bad) == -1, bad
    w = fp8.tula_fp8_operand(258, 128, 0, 0)  # (found before anything is enqueued)
    assert L.tula_fp8_linear(fp8.tula_fp8_operand(256, 128, 0, 0), w, 4, 4, 128, 0, 1, 1, p, p, p, n) == -1
    assert layer(kept=n) == layer(temp=n) == back(kept=n) == back(temp=n) == -2
    with pytest.raises(TulaError):
        fp8.tula_fp8_size(-1, 4)


def test_refusals_of_the_binding():
    x = torch.zeros(4, 4)
    with pytest.raises(TypeError):
        fp8.quantize(x)
    with pytest.raises(TypeError):
        fp8.linear(x, x)
    with pytest.raises(TypeError):
        fp8.linear(x, x, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        fp8.linear(x, torch.zeros(4, 5))
    with pytest.raises(ValueError):
        fp8.FP8Matrix(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 4, 100)
    with pytest.raises(TypeError):  # of the right sizes, but on the CPU
        fp8.FP8Matrix(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 4, 100)


# --------------------------------------------------------------------------------------------
# On a GPU
# --------------------------------------------------------------------------------------------

def _check_quantised(x, code, square, rows=True, cols=True):
    got = fp8.quantize(x, rows=rows, cols=cols, square=square, dtype=code)
    got = got if rows and cols else (got,)
    for q, src in zip(got, ([x] if rows else []) + ([x.t()] if cols else [])):
        values, scales = quantised64(src, code, square)
        v, s = unpacked(q)
        assert (q.rows, q.cols, q.dtype) == (*src.shape, code)
        assert torch.equal(s, scales) and torch.equal(v, values)
        for dtype in (torch.float32, torch.bfloat16, torch.float16):
            want = values64(values, scales)
            back = fp8.dequantize(q, dtype).cpu()
            nan = torch.isnan(want)
            assert torch.equal(torch.isnan(back), nan) and torch.equal(back[~nan], want.to(dtype)[~nan])


SHAPES = [(1, 1), (1, 128), (128, 1), (3, 129), (127, 127), (128, 128), (130, 384), (257, 513), (40, 1031), (515, 70)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("r,c", SHAPES)
def test_quantise(r, c, square, dtype):
    x = _matrix(r, c, torch.float32, 1 + r + c).clamp(-60000, 60000).to(dtype).cuda()
    for code in (E4, E5):
        _check_quantised(x, code, square)
    _check_quantised(x, E4, square, cols=False)
    _check_quantised(x, E5, square, rows=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("square", [False, True])
def test_quantise_views(dtype, square):
    """Rows apart, at odd starts, transposed, repeated."""
    base = _matrix(300, 410, dtype, 5).cuda()
    for x in (base[:, :384], base[3:290, 5:400], base[:, 1:2], base[7:8, 3:399], base.t(), base.t()[5:200, 1:130],
              base[::2, ::3], base[:1].expand(200, 410)):
        _check_quantised(x, E4, square)


@pytest.mark.gpu
@pytest.mark.parametrize("square", [False, True])
def test_quantise_extremes(square):
    """Zeros, denormal and the largest values, infinities and NaN; sums at a code's largest value and
    just above it."""
    x = torch.zeros(300, 300)
    x[1, 5], x[130, 40], x[260, 299] = math.inf, -math.inf, math.nan
    x[2, 130:140] = 1e-45
    x[3, 260:] = 3.4e38
    x[4, :128] = 448.0
    x[5, 0] = 448.0000305
    x[6, 130] = 57344.0
    x[7, 131] = 57344.004
    x[8, 260:] = -1e-40
    x[9, 140] = 1.1754944e-38
    x[290, ::7] = -0.0
    for code in (E4, E5):
        _check_quantised(x.cuda(), code, square)
        # finite, so that the squares too are looked at
        _check_quantised(torch.nan_to_num(x, 3.0, 3.0, -3.0).cuda(), code, square)


@pytest.mark.gpu
@pytest.mark.parametrize("code", [E4, E5])
@pytest.mark.parametrize("cols", [1, 120, 128, 130, 513, 520])
def test_every_code_at_every_scale_is_read_back(code, cols):
    r = 256
    codes = torch.zeros(r, -(-cols // 128) * 128, dtype=torch.uint8)
    codes[:, :cols] = (torch.arange(r)[:, None] + 3 * torch.arange(cols)[None]) % 256
    nb = -(-cols // 128)
    scale = (torch.arange(r)[:, None] * 5 + torch.arange(nb)[None]) % 256
    tiles = torch.zeros(2, -(-nb // 4), 512, dtype=torch.uint8)
    row, block = torch.arange(r)[:, None], torch.arange(nb)[None]
    tiles[row // 128, block // 4, row % 32 * 16 + row % 128 // 32 * 4 + block % 4] = scale.to(torch.uint8)
    q = fp8.FP8Matrix(codes.cuda(), tiles.cuda(), r, cols, code)
    want = values64(codes[:, :cols].view(code).double(), scale)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        got, ref = fp8.dequantize(q, dtype).cpu(), want.to(dtype)
        nan = torch.isnan(ref)
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], ref[~nan])


def _check_product(a, b, dtype):
    """The tensor cores add 32 products to a running sum at a time.  Taken that each of an addition's
    parts is held to 2^-23 of its largest at worst: K / 32 additions to sums of at most `size`, and in
    each 32 parts of at most its own largest product, which together are `size` at most; then one
    rounding."""
    out = fp8.matmul(a, b, dtype)
    x, y = fp8.dequantize(a, torch.float32).double(), fp8.dequantize(b, torch.float32).double()
    want, size = x @ y.t(), x.abs() @ y.abs().t()
    tol = 1.01 * ROUND[dtype] * want.abs() + (a.cols // 32 + 34) * 2.0 ** -23 * size + TINY[dtype]
    assert out.shape == want.shape and out.dtype == dtype
    assert bool(((out.double() - want).abs() <= tol).all())
    return out


MNK = [(1, 1, 1), (1, 40, 130), (3, 4096, 700), (17, 100, 2050), (40, 33, 128), (64, 300, 1000), (65, 129, 385), (128, 512, 513),
       (129, 127, 640), (200, 1000, 96), (300, 200, 5000), (257, 2049, 260), (2048, 1024, 640), (1300, 1801, 333)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K", MNK)
def test_products(M, N, K, dtype):
    a, b = _matrix(M, K, torch.float32, 3, 0.7).cuda(), _matrix(N, K, torch.float32, 4, 0.7).cuda()
    if dtype == torch.float16:
        a, b = a * 2.0 ** -6, b * 2.0 ** -6
    for ca, cb, sq in ((E4, E4, True), (E5, E4, False), (E4, E5, False), (E5, E5, True)):
        out = _check_product(fp8.quantize(a, dtype=ca), fp8.quantize(b, dtype=cb, square=sq), dtype)
    again = fp8.matmul(fp8.quantize(a, dtype=ca), fp8.quantize(b, dtype=cb, square=sq), dtype)
    assert torch.equal(out, again) and fp8.tula_fp8_error() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", [(1, 300), (40, 50), (100, 129), (300, 300), (2048, 1100)])
def test_products_of_every_block(M, N):
    """Each block of 128 columns has its own power of two, so that a scale taken for another shows."""
    K = 128 * 9
    s = 2.0 ** (torch.arange(K) // 128 * 5 - 20.0)
    rows = 2.0 ** (torch.arange(M) % 7).float()[:, None]
    a = (torch.randint(-8, 9, (M, K)) * s * rows).cuda()
    b = (torch.randint(-8, 9, (N, K)) / s * 2.0 ** (torch.arange(N) % 5).float()[:, None]).cuda()
    got = fp8.matmul(fp8.quantize(a), fp8.quantize(b), torch.float32)
    assert torch.equal(got.double(), a.double() @ b.double().t())


@pytest.mark.gpu
def test_products_of_empty_and_nan_rows():
    a = _matrix(70, 300, torch.float32, 1, 0.5).cuda()
    b = _matrix(50, 300, torch.float32, 2, 0.5).cuda()
    a[3, 200], b[7, 10] = math.nan, math.inf
    out = fp8.matmul(fp8.quantize(a), fp8.quantize(b))
    want = torch.zeros(70, 50, dtype=torch.bool, device="cuda")
    want[3], want[:, 7] = True, True
    assert torch.equal(torch.isnan(out), want)
    none = fp8.quantize(torch.zeros(5, 0, device="cuda"))
    assert torch.equal(fp8.matmul(none, fp8.quantize(torch.zeros(6, 0, device="cuda"))), torch.zeros(5, 6, device="cuda", dtype=torch.bfloat16))
    assert fp8.matmul(fp8.quantize(a[:0]), fp8.quantize(b)).shape == (0, 50)
    assert fp8.dequantize(none).shape == (5, 0) and fp8.quantize(a[:0], cols=True)[1].cols == 0
    with pytest.raises(ValueError):
        fp8.matmul(fp8.quantize(a), fp8.quantize(b[:, :299]))
    with pytest.raises(TypeError):
        fp8.quantize(a.double())
    with pytest.raises(ValueError):
        fp8.quantize(a, rows=False)
    with pytest.raises(TypeError):
        fp8.quantize(a, dtype=torch.float8_e4m3fnuz)


@pytest.mark.gpu
@pytest.mark.parametrize("xt,wt,grad", [(torch.bfloat16, torch.float32, E4), (torch.float16, torch.bfloat16, E5),
                                        (torch.float32, torch.float32, E4)])
@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (37, 100, 130), (260, 300, 513), (600, 2100, 300)])
def test_linear(M, N, K, xt, wt, grad):
    x = _matrix(M, K, torch.float32, 20, 0.5).to(xt).cuda().requires_grad_()
    w = (_matrix(N, K, torch.float32, 21, 0.3) / K ** 0.5).to(wt).cuda().requires_grad_()
    dy = _matrix(M, N, torch.float32, 22, 0.5).to(xt).cuda()
    y = fp8.linear(x, w, grad_dtype=grad)
    dx, dw = torch.autograd.grad(y, (x, w), dy)

    def near(t, code=E4, square=False):
        return values64(*quantised64(t, code, square))

    xd, wd = x.detach(), w.detach()
    q = near(wd, square=True)
    assert torch.equal(near(wd.t(), square=True).t(), q)
    for got, a, b in ((y.detach(), near(xd), q), (dx, near(dy, grad), q.t()), (dw, near(dy.t(), grad), near(xd.t()))):
        want, size = a @ b.t(), a.abs() @ b.abs().t()
        tol = 1.01 * ROUND[got.dtype] * want.abs() + (a.shape[1] // 32 + 34) * 2.0 ** -23 * size + TINY[got.dtype]
        assert bool(((got.double().cpu() - want).abs() <= tol).all())
    assert (y.dtype, dx.dtype, dw.dtype) == (xt, xt, wt)


@pytest.mark.gpu
def test_linear_forms():
    """More dimensions, one gradient wanted, none recorded, empty ones; hooks, twice through a graph."""
    w = torch.randn(70, 200, device="cuda", requires_grad=True)
    x = torch.randn(2, 3, 5, 200, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    y = fp8.linear(x, w)
    assert y.shape == (2, 3, 5, 70) and torch.equal(y.view(30, 70), fp8.linear(x.view(30, 200), w))
    dx, = torch.autograd.grad(y.sum(), (x,))
    dw, = torch.autograd.grad(fp8.linear(x.detach(), w).sum(), (w,))
    both = torch.autograd.grad(fp8.linear(x, w).sum(), (x, w))
    assert torch.equal(dx, both[0]) and torch.equal(dw, both[1])
    with torch.no_grad():
        assert torch.equal(fp8.linear(x, w), y) and not fp8.linear(x, w).requires_grad
    assert fp8.linear(x[:0], w).shape == (0, 3, 5, 70)
    e = fp8.linear(torch.zeros(4, 0, device="cuda", requires_grad=True), torch.zeros(6, 0, device="cuda", requires_grad=True))
    assert torch.equal(e, torch.zeros(4, 6, device="cuda"))
    with pytest.raises(RuntimeError):  # no second derivative
        g, = torch.autograd.grad(fp8.linear(x, w).sum(), (x,), create_graph=True)
        g.sum().backward()


@pytest.mark.gpu
def test_linear_of_views():
    """Operands that lie transposed or apart, gradients of strides 0, another than the current device's order."""
    x = torch.randn(260, 150, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(300, 150, device="cuda")
    dy = torch.randn(260, 300, device="cuda", dtype=torch.bfloat16)

    def run(x, w, dy):
        x, w = x.detach().requires_grad_(), w.detach().requires_grad_()
        y = fp8.linear(x, w)
        return (y.detach(), *torch.autograd.grad(y, (x, w), dy))

    want = run(x, w, dy)
    wide = torch.randn(260, 190, device="cuda", dtype=torch.bfloat16)
    wide[:, 11:161] = x
    for forms in ((x.t().contiguous().t(), w.t().contiguous().t(), dy.t().contiguous().t()), (wide[:, 11:161], w, dy),
                  (x.repeat_interleave(2, 1)[:, ::2], w, dy)):
        assert all(torch.equal(a, b) for a, b in zip(run(*forms), want))
    ones = torch.ones(260, 300, device="cuda", dtype=torch.bfloat16)
    assert all(torch.equal(a, b) for a, b in zip(run(x, w, torch.ones((), device="cuda", dtype=torch.bfloat16).expand(260, 300)), run(x, w, ones)))
    col = run(x[:, :1], w[:, :1], dy)  # of one column, one row, one output
    assert torch.equal(col[0], run(x[:, :1].contiguous(), w[:, :1].contiguous(), dy)[0])
    assert torch.equal(run(x[:1], w, dy[:1])[0], fp8.linear(x[:1].contiguous(), w))
    assert run(x, w[:1], dy[:, :1])[2].shape == (1, 150)


@pytest.mark.gpu
def test_captured_layer():
    """Forward and backward in a graph, replayed on other inputs, beside an eager graph of other leaves."""
    x = torch.randn(300, 256, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(130, 256, device="cuda")
    dy = torch.randn(300, 130, device="cuda", dtype=torch.bfloat16)
    xs, ws, ds = x.clone().requires_grad_(), w.clone().requires_grad_(), dy.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(fp8.linear(xs, ws), (xs, ws), ds)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = fp8.linear(xs, ws)
        dx, dw = torch.autograd.grad(y, (xs, ws), ds)
    for seed in (1, 2):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for s in (xs, ws, ds):
            s.detach().copy_(torch.randn(s.shape, generator=gen, device="cuda"))
        graph.replay()
        xe, we = xs.detach().clone().requires_grad_(), ws.detach().clone().requires_grad_()
        ye = fp8.linear(xe, we)
        want = (ye, *torch.autograd.grad(ye, (xe, we), ds))
        torch.cuda.synchronize()
        for got, ref in zip((y, dx, dw), want):
            assert torch.equal(got, ref)


@pytest.mark.gpu
def test_other_streams():
    """A matrix made on one stream and read on another is not overwritten by what its own stream makes next."""
    side = torch.cuda.Stream()
    a, b = torch.randn(512, 4096, device="cuda"), torch.randn(640, 4096, device="cuda")
    want = fp8.matmul(fp8.quantize(a), fp8.quantize(b))
    for _ in range(10):
        qa, qb = fp8.quantize(a), fp8.quantize(b)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)
            got = fp8.matmul(qa, qb)
        del qa, qb
        fp8.quantize(-a), fp8.quantize(-b)
        side.synchronize()
        assert torch.equal(got, want)
