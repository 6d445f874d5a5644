"""MXFP4 matrices (include/tula_train.h) against the format's definition, and products and
gradients against fp64."""
import ctypes
import math

import pytest
import torch

from paper_2603_18112_gb300 import build as B
from paper_2603_18112_gb300 import mx
from paper_2603_18112_gb300 import tula_ags as T


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    T.lib()


# ---------------------------------------------------------------------------------------------
# Refusals and sizes (no GPU)
# ---------------------------------------------------------------------------------------------

def test_sizes():
    assert mx.tula_mx_size(1, 1) == (64, 512)
    assert mx.tula_mx_size(128, 128) == (128 * 64, 512)
    assert mx.tula_mx_size(129, 129) == (129 * 128, 4 * 512)
    assert mx.tula_mx_size(0, 5) == (0, 0)
    for bad in ((-1, 5), (5, -1), (1 << 31, 1 << 31)):
        with pytest.raises(T.TulaError):
            mx.tula_mx_size(*bad)


def test_refusals():
    L, P = mx._lib(), 0x10000
    A = T.TULA_ERR_ARG
    quant = L.tula_mx_quantize
    assert quant(P, 3, 4, 4, 4, P, P, None, None, None) == A           # type
    assert quant(P, 0, -1, 4, 4, P, P, None, None, None) == A
    assert quant(P, 0, 4, 4, 3, P, P, None, None, None) == A           # stride below cols
    assert quant(P, 0, 4, 4, 4, None, None, None, None, None) == A     # nothing to write
    assert quant(P, 0, 4, 4, 4, P, None, None, None, None) == A        # codes without scales
    assert quant(P, 0, 4, 4, 4, None, None, None, P, None) == A
    assert quant(None, 0, 4, 4, 4, P, P, None, None, None) == A
    assert quant(P + 2, 0, 4, 4, 4, P, P, None, None, None) == A       # fp32 off 4 bytes
    assert quant(P, 0, 4, 4, 4, P + 8, P, None, None, None) == A       # codes off 16 bytes
    assert quant(P, 0, 0, 4, 4, P, P, None, None, None) == 0           # nothing to do
    deq = L.tula_mx_dequantize
    assert deq(P, P, 4, 4, P, 7, None) == A
    assert deq(P, P, 4, 4, None, 0, None) == A
    assert deq(P, P + 4, 4, 4, P, 0, None) == A
    assert deq(P, P, 4, 4, P + 1, 1, None) == A
    mm = L.tula_mx_matmul
    assert mm(P, P, P, P, 4, 4, -1, P, 0, None) == A
    assert mm(P, P, P, P, 4, 4, 4, P, 9, None) == A
    assert mm(P, P, P, P, 4, 4, 4, None, 0, None) == A
    assert mm(P, P, P, P, 4, 4, 4, P + 2, 0, None) == A
    assert mm(None, P, P, P, 4, 4, 4, P, 0, None) == A
    assert mm(P, P, P, P + 8, 4, 4, 4, P, 0, None) == A
    assert mm(P, P, P, P, 0, 4, 4, P, 0, None) == 0
    assert L.tula_mx_error(None, None) == A


def test_binding_refusals():
    with pytest.raises(TypeError):
        mx.quantize(torch.zeros(4, 4))
    with pytest.raises(ValueError):
        mx.MXMatrix(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 5, 4)
    with pytest.raises(TypeError):
        mx.MXMatrix(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 4, 4)
    with pytest.raises(ValueError):
        mx.linear(torch.zeros(3, 4), torch.zeros(5, 6))


# ---------------------------------------------------------------------------------------------
# The format, in fp64
# ---------------------------------------------------------------------------------------------

VALUES = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def quantised64(x):
    """(codes [r, c], scale bytes [r, blocks]) by the definition: nearest of VALUES, ties to the
    even code, element by element in fp64."""
    x = x.double().cpu()
    r, c = x.shape
    nb = -(-c // 32)
    y = torch.zeros(r, nb * 32, dtype=torch.float64)
    y[:, :c] = x
    y = y.view(r, nb, 32)
    top = y.abs().amax(2)
    bad = ~torch.isfinite(y).all(2)
    e = torch.frexp(torch.where(bad, 1.0, top))[1].double() - 1          # floor(log2), of 0: -1
    e = torch.where(top == 0, -math.inf, e)
    s = (e - 2 + 127).clamp(min=0)
    a = y / torch.ldexp(torch.ones(()).double(), (s - 127).int())[..., None]
    a = torch.where(bad[..., None], 0.0, a)
    dist = (a.abs()[..., None] - VALUES).abs()
    best = dist.amin(-1, keepdim=True)
    near = dist == best
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])                       # even codes first
    code = order[near[..., order].double().argmax(-1)]
    code = code | (torch.signbit(a).long() << 3)
    code = torch.where(bad[..., None], 0, code).view(r, nb * 32)[:, :c]
    return code, torch.where(bad, 255, s.long())


def values64(code, s):
    sign = torch.where(code >= 8, -1.0, 1.0).double()
    scale = torch.ldexp(torch.ones(()).double(), (s - 127).int())
    scale = torch.where(s == 255, math.nan, scale)
    return sign * VALUES[code & 7] * scale.repeat_interleave(32, 1)[:, :code.shape[1]]


def unpacked(q):
    """codes and scale bytes of an MXMatrix, element by element; checks that what lies beyond the
    matrix is zero."""
    codes, scales = q.codes.cpu().long(), q.scales.cpu().long()
    full = torch.stack((codes & 15, codes >> 4), 2).view(q.rows, -1)
    assert not full[:, q.cols:].any()
    blocks, tiles = -(-q.cols // 32), scales.view(-(-q.rows // 128), -(-q.cols // 128), 512)
    rows = torch.arange(tiles.shape[0] * 128)[:, None]
    cols = torch.arange(tiles.shape[1] * 4)[None]
    s = tiles[rows // 128, cols // 4, rows % 32 * 16 + rows % 128 // 32 * 4 + cols % 4]
    assert not s[q.rows:].any() and not s[:, blocks:].any()
    return full[:, :q.cols], s[:q.rows, :blocks]


def _matrix(rows, cols, dtype, seed, stride=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, stride or cols, generator=gen, device="cuda")
    x *= torch.exp(2 * torch.randn(1, stride or cols, generator=gen, device="cuda"))
    return x.to(dtype)[:, :cols]


SHAPES = [(1, 1), (1, 31), (1, 4096), (2, 32), (3, 33), (31, 64), (127, 129), (128, 128), (129, 257),
          (200, 1000), (33, 4097), (1000, 7)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("extra", [0, 1, 2, 8])
def test_quantize(rows, cols, dtype, extra):
    """Codes and scales of both forms equal the definition's bit for bit, and so do the values."""
    x = _matrix(rows, cols, dtype, 1, cols + extra)
    q, t = mx.quantize(x, cols=True)
    only_q, only_t = mx.quantize(x), mx.quantize(x, rows=False, cols=True)
    assert torch.equal(q.codes, only_q.codes) and torch.equal(q.scales, only_q.scales)
    assert torch.equal(t.codes, only_t.codes) and torch.equal(t.scales, only_t.scales)
    for got, src in ((q, x), (t, x.t())):
        code, s = quantised64(src)
        c, r = unpacked(got)
        assert torch.equal(r, s)
        assert torch.equal(c, code)
        for kind in (torch.float32, torch.bfloat16, torch.float16):
            want = values64(code, s).to(kind)
            back = mx.dequantize(got, kind).cpu()
            assert torch.equal(back, want), kind


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_every_code_boundary(dtype):
    """Ties between neighbouring codes, and the values beside them, for all scales of the type."""
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.5], dtype=torch.float64)
    lo, hi = (-14, 12) if dtype == torch.float16 else (-126, 124)
    rows = []
    for k in range(lo, hi):
        row = torch.zeros(64, dtype=torch.float64)
        row[0], row[32] = 4.0, 7.5                                       # so that the scale is 2^k
        row[1:11], row[11:21] = ties, -ties
        row[33:43] = ties * (1 + 2.0 ** -7)
        row[43:53] = -ties * (1 - 2.0 ** -7)
        rows.append(row * 2.0 ** k)
    x = torch.stack(rows).to(dtype).cuda()
    q, t = mx.quantize(x, cols=True)
    for got, src in ((q, x), (t, x.t())):
        code, s = quantised64(src)
        c, r = unpacked(got)
        assert torch.equal(r, s) and torch.equal(c, code)


@pytest.mark.gpu
def test_zeros_denormals_infinities_and_nans():
    x = torch.zeros(40, 100, device="cuda")
    x[1, 5], x[1, 40], x[1, 70] = math.inf, -math.inf, math.nan
    x[2, :32] = 1e-45
    x[2, 3] = -1e-40
    x[3, :] = 3.4e38
    x[4, ::2] = -0.0
    x[5, 7] = 1.1754944e-38
    for y in (x, x.bfloat16()):
        q, t = mx.quantize(y, cols=True)
        for got, src in ((q, y), (t, y.t())):
            code, s = quantised64(src)
            c, r = unpacked(got)
            assert torch.equal(r, s) and torch.equal(c, code)
            back = mx.dequantize(got, torch.float32).double().cpu()
            assert torch.equal(torch.nan_to_num(back, 7.0), torch.nan_to_num(values64(code, s), 7.0))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,stride", [(3000, 4101, 4104), (5000, 2500, 2504), (1, 100000, 100000), (129, 80000, 80000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_large_matrices_equal_their_slabs(rows, cols, stride, dtype):
    """Large matrices go another way than small ones: each slab of 128 rows has to come out as by
    itself, and is checked against the definition in one place."""
    x = _matrix(rows, cols, dtype, 50, stride)
    x[rows // 2, cols // 3] = math.nan
    q, t = mx.quantize(x, cols=True)
    only_q, only_t = mx.quantize(x), mx.quantize(x, rows=False, cols=True)
    assert torch.equal(q.codes, only_q.codes) and torch.equal(q.scales, only_q.scales)
    assert torch.equal(t.codes, only_t.codes) and torch.equal(t.scales, only_t.scales)
    for k in range(-(-rows // 128)):
        a, b = 128 * k, min(rows, 128 * k + 128)
        sq, st = mx.quantize(x[a:b], cols=True)
        assert torch.equal(sq.codes, q.codes[a:b]) and torch.equal(sq.scales[0], q.scales[k])
        assert torch.equal(st.codes, t.codes[:, 64 * k:64 * k + 64]) and torch.equal(st.scales[:, 0], t.scales[:, k])
    a = 128 * (rows // 256)
    part = x[a:a + 128, :3000]
    code, s = quantised64(part)
    c, r = unpacked(mx.quantize(part))
    assert torch.equal(c, code) and torch.equal(r, s)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(3, 5), (40, 33), (300, 1001), (7, 4096), (1000, 130)])
@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_dequantize_into_any_alignment(rows, cols, kind, off):
    """The C call writes the matrix and nothing beside it, wherever out starts."""
    dtype = [torch.float32, torch.bfloat16, torch.float16][kind]
    q = mx.quantize(_matrix(rows, cols, torch.float32, 51))
    room = torch.full((rows * cols + 64,), 7.0, dtype=dtype, device="cuda")
    out = room[16 + off:16 + off + rows * cols]
    rc = mx._lib().tula_mx_dequantize(q.codes.data_ptr(), q.scales.data_ptr(), rows, cols, out.data_ptr(), kind,
                                      torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    assert torch.equal(out.view(rows, cols).cpu(), values64(*unpacked(q)).to(dtype))
    assert bool((room[:16 + off] == 7).all()) and bool((room[16 + off + rows * cols:] == 7).all())


@pytest.mark.gpu
def test_empty_matrices_and_odd_layouts():
    for shape in ((0, 5), (5, 0), (0, 0)):
        q, t = mx.quantize(torch.zeros(shape, device="cuda"), cols=True)
        assert mx.dequantize(q).shape == shape and mx.dequantize(t).shape == shape[::-1]
    x = _matrix(70, 50, torch.float32, 2)
    a, b = mx.quantize(x.t(), cols=True), mx.quantize(x.t().contiguous(), cols=True)  # a transposed view
    assert all(torch.equal(u.codes, v.codes) and torch.equal(u.scales, v.scales) for u, v in zip(a, b))
    y = x.expand(70, 50)[3:4]
    assert torch.equal(mx.quantize(y).codes, mx.quantize(y.contiguous()).codes)


# ---------------------------------------------------------------------------------------------
# Products
# ---------------------------------------------------------------------------------------------

def _exact(a, b):
    """A B^T in fp64 and the sum of its terms' magnitudes."""
    x, y = (mx.dequantize(q, torch.float32).double() for q in (a, b))
    return x @ y.t(), x.abs() @ y.abs().t()


ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _check_product(a, b, dtype):
    out = mx.matmul(a, b, dtype)
    want, size = _exact(a, b)
    K = a.cols
    # An fp32 sum of K / 32 exact parts, each addition within 2^-23 (rounding or truncation) of
    # the sum of magnitudes so far.
    tol = 1.01 * ROUND[dtype] * want.abs() + (K // 32 + 2) * 2.0 ** -23 * size
    if dtype == torch.float16:
        tol = tol + 2.0 ** -24
    assert out.dtype == dtype and out.shape == want.shape
    bad = (out.double() - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())
    assert torch.equal(out, mx.matmul(a, b, dtype))                      # bit for bit
    return out


MNK = [(1, 1, 1), (1, 16, 32), (1, 4096, 4096), (3, 5, 7), (16, 128, 256), (17, 100, 300), (33, 130, 128),
       (64, 257, 512), (65, 300, 384), (128, 128, 128), (128, 1000, 2048), (129, 128, 640), (200, 1, 1000),
       (300, 70, 96), (256, 256, 256), (257, 511, 1025), (1000, 999, 4097), (2048, 1024, 512), (4096, 2, 64),
       (130, 8200, 160), (513, 1536, 8192),
       # pairs of CTAs, for short and for long sums, rows at every alignment
       (2100, 2304, 100), (2049, 2561, 1024), (3000, 2500, 640), (2048, 2504, 1152), (1100, 3001, 2050),
       (2500, 2306, 1500), (5000, 136, 4100)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", MNK)
def test_matmul(M, N, K):
    a, b = mx.quantize(_matrix(M, K, torch.float32, 3)), mx.quantize(_matrix(N, K, torch.bfloat16, 4))
    for dtype in (torch.float32, torch.bfloat16):
        _check_product(a, b, dtype)
    assert mx.tula_mx_error() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(5, 40, 96), (128, 384, 256), (300, 260, 1100), (2050, 2400, 512), (2050, 2400, 2000)])
def test_matmul_exact(M, N, K):
    """Small integers: every sum is exact, so the product has to be, in every place."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    x, y = (torch.randint(-3, 4, (n, K), generator=gen, device="cuda").float() for n in (M, N))
    x[:, ::32], y[:, ::32] = 4.0, 4.0                                     # every scale is 1
    out = mx.matmul(mx.quantize(x), mx.quantize(y), torch.float32)
    assert torch.equal(out.double(), x.double() @ y.double().t())


@pytest.mark.gpu
def test_every_row_and_block_has_its_own_scale():
    """Scales that differ by row and by block, from 2^-20 to 2^20: a scale taken from another row
    or block shows."""
    M, N, K = 300, 400, 1100
    gen = torch.Generator(device="cuda").manual_seed(10)
    def spread(n):
        e = torch.randint(-20, 21, (n, -(-K // 32)), generator=gen, device="cuda").float()
        x = torch.randn(n, K, generator=gen, device="cuda")
        return x * torch.exp2(e).repeat_interleave(32, 1)[:, :K]
    _check_product(mx.quantize(spread(M)), mx.quantize(spread(N)), torch.float32)
    _check_product(mx.quantize(spread(7)), mx.quantize(spread(N)), torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 300])
def test_nan_blocks_and_empty_sums(M):
    x, y = _matrix(M, 200, torch.float32, 5), _matrix(150, 200, torch.float32, 6)
    x[1, 77] = math.inf
    out = mx.matmul(mx.quantize(x), mx.quantize(y), torch.float32)
    assert torch.isnan(out[1]).all() and torch.isfinite(out[0]).all() and torch.isfinite(out[2:]).all()
    zero = mx.matmul(mx.quantize(x[:, :0]), mx.quantize(y[:, :0]), torch.float32)
    assert zero.shape == (M, 150) and not zero.any()
    assert mx.matmul(mx.quantize(x[:0]), mx.quantize(y)).shape == (0, 150)
    assert mx.matmul(mx.quantize(x), mx.quantize(y[:0])).shape == (M, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", [(1, 128), (20, 300), (60, 128), (100, 200), (200, 100)])
@pytest.mark.parametrize("stages", [9, 17, 18, 33, 34, 35, 41])
def test_shares_of_a_sum_that_some_ctas_have_nothing_of(M, N, stages):
    """Sums whose stages of 256 columns do not divide among the CTAs of a cluster: the last ones have
    fewer or none.  Again and again, so that a CTA's barriers lie where another's did before."""
    K = 256 * stages - 100
    a, b = mx.quantize(_matrix(M, K, torch.float32, 70)), mx.quantize(_matrix(N, K, torch.float32, 71))
    want = _check_product(a, b, torch.float32)
    empty = mx.quantize(torch.zeros(M, 0, device="cuda")), mx.quantize(torch.zeros(N, 0, device="cuda"))
    for _ in range(20):
        zero = mx.matmul(*empty, torch.float32)
        assert torch.equal(mx.matmul(a, b, torch.float32), want) and not zero.any()
    assert mx.tula_mx_error() == 0


@pytest.mark.gpu
def test_calls_from_a_thread_that_has_made_none():
    """The first CUDA call of a thread is a product, a transpose's quantisation, a clipping."""
    import threading
    x = _matrix(600, 256, torch.float32, 61)
    a = mx.quantize(x)
    want = [mx.matmul(a, a), mx.quantize(x, rows=False, cols=True).codes]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def run(i, fn):
        try:
            got[i] = fn()
            torch.cuda.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    for i, fn in enumerate((lambda: mx.matmul(a, a), lambda: mx.quantize(x, rows=False, cols=True).codes)):
        t = threading.Thread(target=run, args=(i, fn))
        t.start()
        t.join()
    assert not errors
    assert all(torch.equal(u, v) for u, v in zip(want, got))


@pytest.mark.gpu
def test_matmul_refusals():
    a, b = mx.quantize(_matrix(4, 64, torch.float32, 7)), mx.quantize(_matrix(4, 96, torch.float32, 8))
    with pytest.raises(ValueError):
        mx.matmul(a, b)
    with pytest.raises(TypeError):
        mx.matmul(a, a, torch.float64)
    with pytest.raises(ValueError):
        mx.MXMatrix(a.codes, a.scales, 5, 64)
    same = mx.MXMatrix(a.codes, a.scales, 4, 64)
    assert torch.equal(mx.matmul(same, a), mx.matmul(a, a))


# ---------------------------------------------------------------------------------------------
# The linear layer
# ---------------------------------------------------------------------------------------------

def _rounded(x):
    return values64(*quantised64(x))


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (37, 100, 130), (260, 300, 513)])
@pytest.mark.parametrize("xtype", [torch.float32, torch.bfloat16])
def test_linear(M, N, K, xtype):
    """y and both gradients against the formulas in fp64 on the rounded operands."""
    x = _matrix(M, K, xtype, 20).requires_grad_()
    w = _matrix(N, K, torch.float32, 21).requires_grad_()
    dy = _matrix(M, N, xtype, 22)
    y = mx.linear(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    xd, wd, dyd = x.detach(), w.detach(), dy
    for got, a, b in ((y.detach(), _rounded(xd), _rounded(wd)), (dx, _rounded(dyd), _rounded(wd.t())),
                      (dw, _rounded(dyd.t()), _rounded(xd.t()))):
        want, size = a @ b.t(), a.abs() @ b.abs().t()
        tol = 1.01 * ROUND[got.dtype] * want.abs() + (a.shape[1] // 32 + 2) * 2.0 ** -23 * size
        assert bool(((got.double().cpu() - want).abs() <= tol).all())
    assert y.dtype == xtype and dx.dtype == xtype and dw.dtype == torch.float32
    only = torch.autograd.grad(mx.linear(xd, w), w, dy)[0]
    assert torch.equal(only, dw)
    assert torch.equal(torch.autograd.grad(mx.linear(x, wd), x, dy)[0], dx)


@pytest.mark.gpu
def test_linear_gradients_against_differences():
    """Integers that MXFP4 holds exactly, in x, w and dy: y is linear in each, so a difference
    quotient is exact up to fp32's rounding of the sums."""
    M, N, K = 8, 40, 64
    gen = torch.Generator(device="cuda").manual_seed(30)

    def ints(r, c):
        x = torch.randint(-2, 3, (r, c), generator=gen, device="cuda").float()
        return x

    x, w, dy = ints(M, K), ints(N, K), ints(M, N)
    x[:, ::32] = w[:, ::32] = dy[:, ::32] = 4.0
    x[0, :], w[0, :], dy[0, :] = 4.0, 4.0, 4.0
    x, w = x.requires_grad_(), w.requires_grad_()
    y = mx.linear(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy)

    def loss(a, b):
        return (mx.linear(a, b).double() * dy.double()).sum().item()

    base = loss(x.detach(), w.detach())
    for i, j in ((0, 5), (3, 63), (7, 1)):
        z = x.detach().clone()
        z[i, j] = 3.0 if z[i, j] != 3.0 else 2.0
        assert (loss(z, w.detach()) - base) == (z[i, j] - x.detach()[i, j]).item() * dx[i, j].item()
    for i, j in ((0, 5), (39, 63), (20, 2)):
        z = w.detach().clone()
        z[i, j] = 3.0 if z[i, j] != 3.0 else 2.0
        assert (loss(x.detach(), z) - base) == (z[i, j] - w.detach()[i, j]).item() * dw[i, j].item()


@pytest.mark.gpu
def test_linear_of_broadcast_gradients_and_views():
    """A gradient that is one value broadcast (that of a sum), a weight that is a transposed view, and
    a second differentiation, which is refused."""
    x, v = _matrix(70, 96, torch.bfloat16, 42).requires_grad_(), _matrix(96, 50, torch.float32, 43).requires_grad_()
    mx.linear(x, v.t()).sum().backward()
    ones = torch.ones(70, 50, dtype=torch.bfloat16, device="cuda")
    dx, dw = torch.autograd.grad(mx.linear(x, v.t().contiguous()), (x, v), ones)
    assert torch.equal(x.grad, dx) and torch.equal(v.grad, dw)
    dx = torch.autograd.grad(mx.linear(x, v.t()).square().sum(), x, create_graph=True)[0]
    with pytest.raises(RuntimeError):
        dx.sum().backward()


@pytest.mark.gpu
def test_a_wait_that_runs_out_is_reported():
    """Failure detection without a fault: the check's wait runs out (about two seconds), the word
    reports it once, and products go on."""
    assert mx.tula_mx_error() == 0
    mx.tula_mx_check_wait_timeout()
    a = mx.quantize(_matrix(5, 64, torch.float32, 44))
    out = mx.matmul(a, a, torch.float32)
    assert mx.tula_mx_error() == 1 and mx.tula_mx_error() == 0
    assert torch.equal(out, mx.matmul(a, a, torch.float32))


@pytest.mark.gpu
def test_linear_of_more_dimensions_and_on_another_stream():
    x, w = _matrix(6 * 35, 96, torch.bfloat16, 40).view(6, 35, 96), _matrix(50, 96, torch.float32, 41)
    want = mx.linear(x.view(-1, 96), w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = mx.linear(x, w)
    side.synchronize()
    assert torch.equal(got.view(-1, 50), want)


@pytest.mark.gpu
def test_memory_waits_for_readers_on_other_streams():
    x = torch.randn(512, 512, device="cuda", generator=torch.Generator("cuda").manual_seed(31)).bfloat16()
    expect, ones = mx.dequantize(mx.quantize(x)), torch.ones_like(x)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()  # no holes of other tests in the streams' pools
    own, other = torch.cuda.Stream(), torch.cuda.Stream()
    for stream in (own, other):
        stream.wait_stream(torch.cuda.current_stream())
    for read in (lambda q: mx.dequantize(q), lambda q: mx.matmul(q, q, torch.float32)):
        with torch.cuda.stream(own):
            q = mx.quantize(x)
            right = read(q)
        other.wait_stream(own)
        with torch.cuda.stream(other):
            torch.cuda._sleep(20_000_000)  # some 10 ms, in which q is dropped
            got = read(q)
        at = q.scale_ptr
        del q
        with torch.cuda.stream(own):  # takes the same memory
            again = [mx.quantize(ones)]
            while len(again) < 64 and not abs(again[-1].scale_ptr - at) < 512 * 256:
                again.append(mx.quantize(ones))
            assert len(again) < 64
        torch.cuda.synchronize()
        assert torch.equal(got, right)
        del again
    assert torch.equal(expect, mx.dequantize(mx.quantize(x)))
    assert mx.tula_mx_error() == 0 and not mx._unfreed
    # read in a graph, on the stream that captures it: nothing is noted, and dropping it there is harmless
    q = mx.quantize(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mx.dequantize(q)
    graph.replay()
    torch.cuda.synchronize()
    assert q._block.readers is None and torch.equal(out, expect)


@pytest.mark.gpu
def test_threads_on_streams_of_their_own_read_one_matrix():
    """All of their streams are noted, and none of their products sees other contents."""
    import threading
    a = mx.quantize(_matrix(40, 512, torch.float32, 90))
    for _ in range(5):
        q = mx.quantize(_matrix(300, 512, torch.float32, 91))
        want = mx.matmul(a, q)
        streams = [torch.cuda.Stream() for _ in range(6)]
        torch.cuda.synchronize()
        start, got, errors = threading.Barrier(len(streams)), [], []

        def serve(stream, q=q, want=want):
            try:
                with torch.cuda.stream(stream):
                    start.wait(60)
                    outs = [mx.matmul(a, q) for _ in range(10)]
                    same = torch.stack([(o == want).all() for o in outs]).all()
                    stream.synchronize()
                    got.append(bool(same))
            except Exception as e:  # noqa: BLE001
                errors.append(e)

        threads = [threading.Thread(target=serve, args=(s,)) for s in streams]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not errors and got == [True] * len(streams)
        assert q._block.readers == {s.cuda_stream for s in streams}


@pytest.mark.gpu
def test_a_matrix_dropped_under_capture_goes_back_after_it():
    x = _matrix(512, 512, torch.bfloat16, 92)
    own, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(own):
        q = mx.quantize(x)
    other.wait_stream(own)
    with torch.cuda.stream(other):
        out = mx.dequantize(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        twice = out + out
        del q
    assert len(mx._unfreed) == 1
    again = mx.dequantize(mx.quantize(x))
    graph.replay()
    torch.cuda.synchronize()
    assert not mx._unfreed and torch.equal(again, out) and torch.equal(twice, out + out)


@pytest.mark.gpu
def test_matrices_of_a_capture_read_on_its_second_stream():
    """A branch of a graph reads a matrix that the capture made and dropped: what the other branch makes
    after it lies elsewhere."""
    x = _matrix(512, 512, torch.bfloat16, 93)
    ones, want = torch.ones_like(x), mx.dequantize(mx.quantize(x))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q = mx.quantize(x)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            out = mx.dequantize(q)
        at = q.scale_ptr
        del q
        later = [mx.quantize(ones) for _ in range(4)]
        assert all(abs(m.scale_ptr - at) >= 512 * 256 for m in later)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    del later
    mx.quantize(x)
    assert not mx._unfreed


def _layer(M, N, K, xtype=torch.bfloat16, seed=80):
    x = _matrix(M, K, xtype, seed).requires_grad_()
    w = _matrix(N, K, torch.float32, seed + 1).requires_grad_()
    return x, w, _matrix(M, N, xtype, seed + 2)


@pytest.mark.gpu
def test_what_the_backward_pass_reads_goes_with_it():
    """The 4-bit operands are freed by the backward pass, not with y; a second one is refused, unless
    they were asked to stay."""
    x, w, dy = _layer(2048, 1024, 4096)
    torch.autograd.grad(mx.linear(x, w), (x, w), dy)
    before = torch.cuda.memory_allocated()
    y = mx.linear(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    results = sum(t.numel() * t.element_size() for t in (y, dx, dw))
    # (the allocator hands out multiples of 512 bytes)
    assert torch.cuda.memory_allocated() - before <= results + 4 * 512
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y, (x, w), dy)
    y = mx.linear(x, w)
    for keep in (True, False):
        again = torch.autograd.grad(y, (x, w), dy, retain_graph=keep)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.gpu
def test_hooks_on_saved_tensors_and_checkpoints():
    """What is kept for the backward pass goes through saved-tensor hooks (here to the host and back), and
    a checkpointed layer keeps nothing."""
    from torch.utils.checkpoint import checkpoint
    x, w, dy = _layer(300, 260, 520)
    want = torch.autograd.grad(mx.linear(x, w), (x, w), dy)
    packed = []

    def pack(t):
        packed.append(t.numel() * t.element_size())
        return t.cpu()

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
        y = mx.linear(x, w)
    got = torch.autograd.grad(y, (x, w), dy)
    assert sum(packed) == sum(sum(mx.tula_mx_size(r, c)) for r, c in ((520, 300), (520, 260)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    y = checkpoint(mx.linear, x, w, use_reentrant=False)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, (x, w), dy), want))
    checkpoint(mx.linear, x, w, use_reentrant=True).backward(dy)
    assert torch.equal(x.grad, want[0]) and torch.equal(w.grad, want[1])
    for wrong in (lambda t: t.cpu(), lambda t: t[:-16], lambda t: t.int()):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, wrong):
            y = mx.linear(x, w)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(y, (x, w), dy)


@pytest.mark.gpu
def test_linear_without_gradients_quantises_one_form(monkeypatch):
    """Where no gradient is recorded, or none is asked for, no transpose is quantised."""
    x, w, dy = _layer(70, 50, 96)
    want = mx.linear(x, w).detach()
    forms, call = [], mx._call

    def noted(name, dev, *args):
        if name == "tula_mx_quantize":
            forms.append((args[5] is not None, args[7] is not None))
        return call(name, dev, *args)

    monkeypatch.setattr(mx, "_call", noted)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            y = mx.linear(x, w)
        assert torch.equal(y, want) and not y.requires_grad
        assert forms == [(True, False)] * 2
        forms.clear()
    mx.linear(x.detach(), w.detach())
    assert forms == [(True, False)] * 2
    forms.clear()
    dw = torch.autograd.grad(mx.linear(x.detach(), w), w, dy)[0]        # dw reads x^T and dy^T alone
    assert forms == [(True, True), (True, False), (False, True)] and dw.shape == w.shape


@pytest.mark.gpu
@pytest.mark.parametrize("shape,N", [((2, 3, 0), 5), ((0,), 4), ((0, 3, 8), 5), ((2, 0, 0), 3), ((2, 3, 8), 0)])
def test_linear_of_empty_dimensions(shape, N):
    """Ones and a sum over nothing among them: each sum counts its terms."""
    x = torch.ones(shape, device="cuda", requires_grad=True)
    w = torch.ones(N, shape[-1], device="cuda", requires_grad=True)
    y = mx.linear(x, w)
    assert y.shape == (*shape[:-1], N) and bool((y == shape[-1]).all())
    dx, dw = torch.autograd.grad(y, (x, w), torch.ones_like(y))
    assert dx.shape == x.shape and dw.shape == w.shape and bool((dw == x.shape[:-1].numel()).all())
