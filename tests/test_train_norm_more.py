"""Layer norm where its sums and copies can go wrong: rows far from zero, and what follows below."""
import pytest
import torch

from paper_2603_18112_gb300 import norm

TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUND = {t: torch.finfo(t).eps / 2 for t in TYPES}  # a rounding is off by at most half a step
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
U = 2.0 ** -24  # fp32's rounding

# --------------------------------------------------------------------------------------------
# Rows far from zero
# --------------------------------------------------------------------------------------------

# one to some warps to a row, several CTAs, and rows that registers do not hold
WIDTHS = [24, 1000, 1001, 4099, 7168, 12000, 65540]


def _depth(cols):
    """Additions one after the other in a row's sum: of a thread's 16 elements, 5 exchanges, 6 of a CTA's warps and
    8 of a cluster's CTAs; of wide rows cols / 512 and those of the warp and the CTA."""
    return 36 if cols <= 65536 else cols // 512 + 14


def _forward_exact(x, w, b, eps):
    """The output in 64 bits and how far it may be off before its last rounding, without a term of the row's
    size: the mean is near + rest, near off by `depth` roundings of the row's mean magnitude and known exactly
    from then on, the differences c to it by a rounding each, the rest by depth + 2 roundings of their mean
    magnitude; the variance by depth + 6 of the mean square of c."""
    x, w, b = x.double(), w.double(), b.double()
    cols = x.shape[1]
    depth = _depth(cols)
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    r = 1 / (var + eps).sqrt()
    n = (x - mean) * r
    shift = depth * U * x.abs().mean(1, keepdim=True)  # of near
    c = (x - mean).abs() + shift
    off_n = r * U * ((depth + 2) * c.mean(1, keepdim=True) + 2 * c)
    off_n = off_n + n.abs() * U * ((depth + 6) * (1 + shift.square() * r.square()) + 8)
    return n * w + b, off_n * w.abs() + 2 * U * (n * w).abs() + 2 * U * b.abs()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_rows_far_from_zero(cols, dtype):
    """Equal values, and values about a large offset, through all kernels and with rows off 16-byte boundaries."""
    gen = torch.Generator().manual_seed(cols)
    offsets = torch.tensor([0.0, 1.0, 1000.0, 3000.0, -1000.0, 0.1, 60000.0, 1e-3]).repeat(8)[:, None]
    spread = torch.tensor([0.0, 1.0, 1e-2, 30.0]).repeat_interleave(16)[:, None]
    x = (offsets + spread * torch.randn(64, cols, generator=gen)).clamp(-65504, 65504).to(dtype).cuda()
    w, b = (1 + 0.3 * torch.randn(cols, generator=gen)).cuda(), (0.2 * torch.randn(cols, generator=gen)).cuda()
    apart = torch.zeros(64, cols + 3, dtype=dtype, device="cuda")
    apart[:, 1:cols + 1] = x
    want, off = _forward_exact(x, w, b, 1e-5)
    tol = off + 1.01 * ROUND[dtype] * want.abs() + TINY[dtype]
    for rows in (x, apart[:, 1:cols + 1]):
        y = norm.layer_norm(rows, w, b)
        bad = (y.double() - want).abs() - tol
        assert bool((bad <= 0).all()), [(i, float(v)) for i, v in enumerate(bad.max(1).values) if v > 0][:8]
    assert norm.tula_layer_norm_error() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("cols", WIDTHS)
def test_mean_of_rows_of_equal_values(cols):
    """What the backward pass is given: the mean of whole numbers is the number itself."""
    x = torch.tensor([1000.0, 3000.0, -7.0, 60000.0, 5.0, 333.0], device="cuda")[:, None].expand(6, cols).contiguous()
    y, stats = norm._forward(x, None, None, 1e-5, True)
    assert torch.equal(stats[:, 0], x[:, 0])
    # near is off by depth roundings of the value, the rest that is taken out by depth + 4 of that
    depth = _depth(cols)
    assert bool((y.double().abs().amax(1) <= (depth + 4) * U * depth * U * x[:, 0].double().abs() * 1e-5 ** -0.5).all())


# --------------------------------------------------------------------------------------------
# Narrow rows off 16-byte boundaries
# --------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 255, 256, 257, 513, 769])
def test_narrow_rows(rows, dtype):
    """Rows of a few bytes, the matrix and its gradient anywhere within 16 bytes and ending where their memory does."""
    gen = torch.Generator().manual_seed(rows)
    for cols in range(1, 8):
        for start, dstart, more in ((0, 0, 0), (1, 3, 0), (7, 2, 0), (5, 5, 3)):
            stride = cols + more
            size = (rows - 1) * stride + cols

            def made(first):
                flat = torch.randn(first + size, generator=gen).to(dtype).cuda()
                return flat.as_strided((rows, cols), (stride, 1), first)

            x, dy = made(start), made(dstart)
            w, b = torch.randn(cols, generator=gen).cuda(), torch.randn(cols, generator=gen).cuda()
            leaves = [t.requires_grad_() for t in (x.detach(), w, b)]
            y = norm.layer_norm(leaves[0], w, b, 0.5)
            grads = torch.autograd.grad(y, leaves, dy)
            x64, w64, g64 = x.double(), w.detach().double(), dy.double()
            mean = x64.mean(1, keepdim=True)
            r = 1 / ((x64 - mean).square().mean(1, keepdim=True) + 0.5).sqrt()
            n, g = (x64 - mean) * r, g64 * w64
            dx = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
            want = (n * w64 + b.detach().double(), dx, (g64 * n).sum(0), g64.sum(0))
            # r is below 1.5 and n below 3 (sqrt(7)): some 10 roundings of what is added up, of columns `rows` of it
            sizes = ((n * w64).abs() + b.detach().abs() + w64.abs(), r * (g.abs() + g.abs().mean(1, keepdim=True) * (1 + 3 * n.abs())),
                     (g64.abs() * (n.abs() + 1)).sum(0), g64.abs().sum(0))
            chain = 30 + min(rows, 16 + 256)
            for got, ref, size_of, c in zip((y, *grads), want, sizes, (20, 20, chain, chain)):
                tol = c * U * size_of + 1.01 * ROUND[got.dtype] * ref.abs() + TINY[got.dtype]
                assert bool(((got.detach().double() - ref).abs() <= tol).all()), (cols, start)
    assert norm.tula_layer_norm_error() == 0


# --------------------------------------------------------------------------------------------
# Long sums
# --------------------------------------------------------------------------------------------

def _backward_sums(t, cols, stats, dw, db):
    """dweight and dbias alone, of dy = x = t."""
    rows = t.shape[0]
    n = norm.tula_layer_norm_workspace_size(rows, cols)
    space = torch.empty(n, dtype=torch.uint8, device="cuda")
    norm._call("tula_layer_norm_backward", 0, t.data_ptr(), cols, t.data_ptr(), cols, 0, rows, cols, None, 0, stats.data_ptr(), None,
               dw.data_ptr(), db.data_ptr(), space.data_ptr(), n)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1 << 18, 4112), (1 << 16, 65540), ((1 << 22) + 3, 200)])
def test_gradients_of_parameters_over_many_rows(rows, cols):
    """Equal rows of 1 + 2^-14 or so: a single chain of additions rounds the same way again and again once its sum
    is large.  A part takes 256 rounds of rows (128 wide rows), its threads' sums are added up, then the parts, by 32."""
    value = 1.0 + 0.49 * 2.0 ** (-13 if cols == 4112 else -14)
    t = torch.full((rows, cols), value, device="cuda")
    stats = torch.tensor([0.0, 0.75], device="cuda").repeat(rows, 1)  # n = 0.75 t
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    _backward_sums(t, cols, stats, dw, db)
    v = float(t[0, 0])
    per = max(1, 256 * 16 // cols)
    parts = max(512, rows // per // 128)
    chain = (256 if cols < 65537 else 128) + per + min(128, parts // 32) + parts // 4096 + 10
    assert bool((db.double() / (rows * v) - 1).abs().max() <= chain * U)
    assert bool((dw.double() / (rows * v * (0.75 * v)) - 1).abs().max() <= (chain + 2) * U)
    assert norm.tula_layer_norm_error() == 0


@pytest.mark.gpu
def test_rows_of_2_to_the_24_columns():
    """The squares' sums of values that each round the same way."""
    cols = 1 << 24
    x = torch.full((2, cols), (1.0 + 0.49 * 2.0 ** -9) ** 0.5, device="cuda")
    x[:, ::2] *= -1
    dy = x.abs()
    leaf = x.requires_grad_()
    y = norm.layer_norm(leaf, None, None)
    dx, = torch.autograd.grad(y, leaf, dy)
    v = float(dy[0, 0])
    r = (v * v + 1e-5) ** -0.5
    chain = 128 + 256 + 10  # of a thread's 32768 columns by 128, and the CTA's threads
    tol = (chain + 8) * U
    assert bool((y.detach().double() / (x.detach().double() * r) - 1).abs().max() <= tol)
    # dy is constant: dx = r (dy - mean(dy) - n mean(dy n)), both of its terms sums that cancel; each off by that
    assert float(dx.double().abs().max()) <= 3 * tol * r * v
