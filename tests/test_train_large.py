"""Operands of more than 2^31 elements in Muon's updates and the 8-bit matrices: what lies at
the far end against the same by itself."""
import pytest
import torch

from paper_2603_18112_gb300 import fp8, mx
from paper_2603_18112_gb300 import optim as O
from test_train_fp8 import E4, E5
from test_train_muon import U, _near, _off, _updates

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory_given_back():
    yield
    torch.cuda.empty_cache()


def _corners(rows, cols, dtype, seed):
    """Zeros but for a block in the first rows and columns and one in the last ones; and the two alone."""
    small = torch.zeros(190, 270, device="cuda")
    small[:90, :130], small[90:, 130:] = _updates(1, 90, 130, seed)[0], _updates(1, 100, 140, seed + 1)[0]
    small = small.to(dtype)
    x = torch.zeros(rows, cols, dtype=dtype, device="cuda")
    x[:90, :130], x[-100:, -140:] = small[:90, :130], small[90:, 130:]
    return x, small


def _alone(x):
    """What _corners put together, out of a large matrix, after checking that the rest is zero."""
    out = torch.zeros(190, 270, dtype=x.dtype, device="cuda")
    out[:90, :130], out[90:, 130:] = x[:90, :130], x[-100:, -140:]
    assert int(torch.count_nonzero(x)) == int(torch.count_nonzero(out))
    return out


@pytest.mark.parametrize("rows,cols", [(50001, 43008), (43009, 50000), (50000, 43009)])
def test_orthogonalize(rows, cols):
    """Both orders of sides, and rows that move eight, eight and one at a time.  Steps on blocks are the blocks'
    steps, and the norm is of both."""
    x, small = _corners(rows, cols, torch.bfloat16, 1)
    assert x.numel() > 1 << 31
    got = O.orthogonalize(x, steps=2, dtype=torch.float16)
    _near(_alone(got), *_off(small, 2), torch.float16)
    assert O.tula_muon_error() == 0


def test_muon_step():
    rows, cols, lr, wd = 50000, 43008, 0.5, 0.25
    g, small = _corners(rows, cols, torch.bfloat16, 3)
    w, m, c = torch.ones(rows, cols, device="cuda"), torch.zeros(rows, cols, device="cuda"), torch.empty_like(g)
    O.MuonStep([w], [g], [m], copies=[c], ns_steps=2, scale="aspect")(lr, 0.0, wd)
    # the whole weights (1 - lr wd) exactly but where the gradient is not zero; s = sqrt(rows / cols)
    base, s = 1 - lr * wd, lr * (rows / cols) ** 0.5
    w.sub_(base)
    moved = _alone(w)
    want, off, most = _off(small, 2)
    d = (moved.double() + s * want).abs() - 8 * U
    assert float(d.clamp(min=0).norm()) <= s * off and float(d.max()) <= s * most
    assert torch.equal(_alone(m), small.float())
    assert torch.equal(c[-100:, -140:], w[-100:, -140:].add(base).bfloat16()) and bool((c[200:300] == base).all())
    assert O.tula_muon_error() == 0


def test_a_batch():
    x = torch.zeros(300000, 90, 90, dtype=torch.bfloat16, device="cuda")
    ends = _updates(4, 90, 90, 5, torch.bfloat16)
    x[0], x[150000], x[265146], x[-1] = ends  # (the third one's first element is beyond 2^31)
    got = O.orthogonalize(x, dtype=torch.float16)
    for k, u in zip((0, 150000, 265146, -1), ends):
        _near(got[k], *_off(u, 5), torch.float16)
    assert int(torch.count_nonzero(got)) == sum(int(torch.count_nonzero(got[k])) for k in (0, 150000, 265146, -1))
    assert O.tula_muon_error() == 0


def _tail(q, rows, cols):
    """The codes and scales of a matrix from a multiple of 128 rows and of 512 columns on."""
    return q.codes[rows:, cols:], q.scales[rows // 128:, cols // 512:]


@pytest.mark.parametrize("square", [False, True])
def test_quantisation(square):
    rows, cols = 70001, 32003
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda", dtype=torch.bfloat16)
    assert x.numel() > 1 << 31
    q, t = fp8.quantize(x, cols=True, square=square)
    r0, c0 = rows // 512 * 512, cols // 512 * 512  # both of its forms begin with whole tiles of scales there
    end_q, end_t = fp8.quantize(x[r0:, c0:], cols=True, square=square)
    for whole, end, at in ((q, end_q, (r0, c0)), (t, end_t, (c0, r0))):
        assert all(torch.equal(a, b) for a, b in zip(_tail(whole, *at), (end.codes, end.scales)))
    for dtype in (torch.bfloat16, torch.float32):
        back = fp8.dequantize(q, dtype)
        assert torch.equal(back[r0:, c0:], fp8.dequantize(end_q, dtype)) and torch.equal(back[:500], fp8.dequantize(fp8.quantize(
            x[:512], square=square), dtype)[:500])
        del back


def test_products_of_large_operands():
    rows, cols = 70001, 32003
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda", dtype=torch.bfloat16)
    few = torch.randn(40, cols, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda")
    q, p = fp8.quantize(x, dtype=E5), fp8.quantize(few, dtype=E4)
    r0 = rows // 128 * 128
    end = fp8.quantize(x[r0:].contiguous(), dtype=E5)
    del x
    # codes of more than 2^31 bytes on either side: exact products, added in an order of K's alone up to how the
    # columns are shared out, to fp32's roundings of some thousand instructions
    for a, b, ea, eb, cut in ((q, p, end, p, lambda y: y[r0:]), (p, q, p, end, lambda y: y[:, r0:])):
        got, alone = cut(fp8.matmul(a, b, torch.float32)).double(), fp8.matmul(ea, eb, torch.float32).double()
        assert float((got - alone).norm()) <= 2.0 ** -14 * float(alone.norm())


def test_products_of_many_outputs():
    gen = torch.Generator(device="cuda").manual_seed(10)
    a, b = (fp8.quantize(torch.randint(-3, 4, (n, 130), generator=gen, device="cuda").float()) for n in (70001, 32003))
    y = fp8.matmul(a, b, torch.bfloat16)  # whole numbers: exact but for the rounding to bf16
    assert y.numel() > 1 << 31
    x64, w64 = (fp8.dequantize(t, torch.float32).double() for t in (a, b))
    for rows in (slice(0, 200), slice(35000, 35100), slice(69800, 70001)):
        assert torch.equal(y[rows], (x64[rows] @ w64.t()).bfloat16())
    assert fp8.tula_fp8_error() == 0


@pytest.mark.parametrize("m,n", [(1, 64), (64, 64), (2048, 4096)])
@pytest.mark.parametrize("module,lost", [(fp8, 2.0 ** -28), (mx, 2.0 ** -29)])
def test_sums_of_one_sign_over_2_to_the_19_columns(module, lost, m, n):
    """What the tensor cores cut off: a unit in fp32's last place, 2^-23, with every instruction of 32 columns (4
    bits: 64); and the last rounding."""
    k = 1 << 19
    gen = torch.Generator(device="cuda").manual_seed(11)

    def made(rows):
        x = torch.rand(rows, k, generator=gen, device="cuda") + 0.5
        x *= torch.exp2(torch.randint(-3, 4, (1, k // 128), generator=gen, device="cuda").float()).repeat_interleave(128, 1)
        return module.quantize(x)

    a, b = made(m), made(n)
    got = module.matmul(a, b, torch.float32).double()
    x, w = module.dequantize(a, torch.float32), module.dequantize(b, torch.float32)
    want = sum(x[:, c:c + 8192].double() @ w[:, c:c + 8192].double().t() for c in range(0, k, 8192))
    assert float((got / want - 1).abs().max()) <= k * lost + U
