"""Forms of the training operators beside those of their own files: products and layers in fp16, every
scale byte read back in every type, lists of several types, a captured training step."""
import math

import pytest
import torch

from paper_2603_18112_gb300 import mx
from paper_2603_18112_gb300 import optim as O
from test_train_mx import MNK, ROUND, _built, _check_product, _matrix, _rounded, quantised64, unpacked, values64  # noqa: F401
from test_train_optim import NORM_TOL, _adam64, _adam_state, _norm64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", MNK)
def test_products_in_fp16(M, N, K):
    """Inputs whose sums lie within fp16's range: the powers of two move scales only."""
    a, b = (mx.quantize(_matrix(n, K, torch.float32, seed) * 2.0 ** -10) for n, seed in ((M, 3), (N, 4)))
    out = _check_product(a, b, torch.float16)
    assert bool(torch.isfinite(out).all()) and bool(out.any())
    assert mx.tula_mx_error() == 0


@pytest.mark.parametrize("M,N", [(1, 40), (20, 300), (50, 129), (100, 200), (200, 20), (300, 60), (200, 300), (2100, 2304), (2100, 2305)])
def test_fp16_sums_beyond_its_range(M, N):
    """4064 products of 16 are 65024, fp16's last multiple of 512; 4096 round to an infinity."""
    x, y = torch.full((M, 4096), 4.0, device="cuda"), torch.full((N, 4096), 4.0, device="cuda")
    y[1::3] *= -1
    want = torch.full((N,), math.inf, device="cuda")
    want[1::3] = -math.inf
    out = mx.matmul(mx.quantize(x), mx.quantize(y), torch.float16)
    assert bool((out.float() == want).all())
    out = mx.matmul(mx.quantize(x[:, :4064]), mx.quantize(y[:, :4064]), torch.float16)
    assert bool((out.float() == 65024.0 * want.sign()).all())
    x[0, 7] = math.nan
    out = mx.matmul(mx.quantize(x), mx.quantize(y), torch.float16)
    assert bool(torch.isnan(out[0]).all()) and not bool(torch.isnan(out[1:]).any())


@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (37, 100, 130), (260, 300, 513), (600, 2100, 300)])
def test_linear_in_fp16(M, N, K):
    x = (_matrix(M, K, torch.float32, 20) * 2.0 ** -9).half().requires_grad_()
    w = (_matrix(N, K, torch.float32, 21) * 2.0 ** -9).requires_grad_()
    dy = (_matrix(M, N, torch.float32, 22) * 2.0 ** -9).half()
    y = mx.linear(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    xd, wd = x.detach(), w.detach()
    for got, a, b in ((y.detach(), _rounded(xd), _rounded(wd)), (dx, _rounded(dy), _rounded(wd.t())),
                      (dw, _rounded(dy.t()), _rounded(xd.t()))):
        want, size = a @ b.t(), a.abs() @ b.abs().t()
        assert want.abs().max() < 60000
        # an fp32 sum of K / 32 exact parts, rounded once; below fp16's normal range to its grid
        tol = 1.01 * ROUND[got.dtype] * want.abs() + (a.shape[1] // 32 + 2) * 2.0 ** -23 * size
        tol = tol + (2.0 ** -24 if got.dtype == torch.float16 else 0.0)
        assert bool(((got.double().cpu() - want).abs() <= tol).all())
    assert y.dtype == dx.dtype == torch.float16 and dw.dtype == torch.float32


def _by_hand(code, scale):
    """An MXMatrix of these codes [r, c] and scale bytes [r, blocks], on the GPU."""
    r, c = code.shape
    tiles_r, tiles_c = -(-r // 128), -(-c // 128)
    codes = torch.zeros(r, tiles_c * 128, dtype=torch.uint8)
    codes[:, :c] = code
    scales = torch.zeros(tiles_r, tiles_c, 512, dtype=torch.uint8)
    row, block = torch.arange(r)[:, None], torch.arange(scale.shape[1])[None]
    scales[row // 128, block // 4, row % 32 * 16 + row % 128 // 32 * 4 + block % 4] = scale.to(torch.uint8)
    return mx.MXMatrix((codes[:, 0::2] | codes[:, 1::2] << 4).contiguous().cuda(), scales.cuda(), r, c)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cols", [1, 16, 31, 32, 160, 161])
def test_every_code_at_every_scale_is_read_back(dtype, cols):
    """All 16 codes at all 256 scale bytes, also those of denormal values, of values beyond the type and of
    NaN; signs of zeros too."""
    code = (torch.arange(256)[:, None] // 7 + torch.arange(cols)[None]) % 16
    scale = (torch.arange(256)[:, None] + 3 * torch.arange(-(-cols // 32))[None]) % 256
    want = values64(code, scale)
    got = mx.dequantize(_by_hand(code, scale), dtype).cpu()
    rounded = want.to(dtype)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan], rounded[~nan]) and torch.equal(torch.signbit(got)[~nan], torch.signbit(rounded)[~nan])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_zeros_denormals_infinities_and_nans_in_16_bits(dtype):
    x = torch.zeros(40, 100, device="cuda")
    x[1, 5], x[1, 40], x[1, 70] = math.inf, -math.inf, math.nan
    x[2, :32] = 1e-45
    x[2, 3] = -1e-40
    x[3, :] = 3.4e38
    x[4, ::2] = -0.0
    x[5, 7] = 1.1754944e-38
    x[6, :] = 6e-8
    y = x.to(dtype)  # what is not in its range becomes an infinity or zero
    for got, src in zip(mx.quantize(y, cols=True), (y, y.t())):
        code, s = quantised64(src)
        c, r = unpacked(got)
        assert torch.equal(r, s) and torch.equal(c, code)
        back, want = mx.dequantize(got, dtype).cpu(), values64(code, s).to(dtype)
        assert torch.equal(torch.isnan(back), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(back.float(), 7.0), torch.nan_to_num(want.float(), 7.0))


@pytest.mark.parametrize("sizes", [[1, 2047, 2048, 5000, 33, 9000], [700_001, 5, 900_000, 64, 1_000_003, 31]])
@pytest.mark.parametrize("layout", ["padded", "shifted"])
@pytest.mark.parametrize("max_norm", [0.0, 0.3])
def test_adamw_of_gradients_and_copies_of_several_types(sizes, layout, max_norm):
    types = [torch.float32, torch.bfloat16, torch.float16]
    made = {t: _adam_state(sizes, t, layout, c, 31) for t, c in
            zip(types, (torch.bfloat16, torch.float16, torch.bfloat16))}
    w, g, m, v, c = ([made[types[i % 3]][role][i] for i in range(len(sizes))] for role in range(5))
    lr, b1, b2, eps, wd, scale = 3e-3, 0.9, 0.98, 1e-8, 0.1, 64.0
    steps = torch.tensor([4, 0], dtype=torch.int64, device="cuda")
    step = O.AdamWStep(w, g, m, v, copies=c, max_norm=max_norm, steps=steps)
    norm = _norm64(g, scale)
    coef = min(1.0, max_norm / (norm + 1e-6)) if max_norm else 1.0
    want = [_adam64(*x, 5, coef / scale, lr, b1, b2, eps, wd) for x in zip(w, g, m, v)]
    step(lr, (b1, b2), eps, wd, grad_scale=scale)
    if max_norm:
        assert step.record[0].item() == pytest.approx(norm, rel=NORM_TOL)
    for i, (ref, tol) in enumerate(want):
        for role, x, r, e in zip("wmv", (w[i], m[i], v[i]), ref, tol):
            assert bool(((x.double() - r).abs() <= e).all()), (i, role)
        assert torch.equal(c[i], w[i].to(c[i].dtype))


def test_a_captured_training_step_replays_as_it_runs():
    """Two layers forward and backward, clipping and AdamW in one graph, replayed over new inputs."""
    gen = torch.Generator(device="cuda").manual_seed(50)
    data = [(torch.randn(300, 256, generator=gen, device="cuda").bfloat16(), torch.randn(300, 130, generator=gen, device="cuda"))
            for _ in range(6)]

    def fresh():
        gen = torch.Generator(device="cuda").manual_seed(51)
        w = [torch.randn(s, generator=gen, device="cuda").mul_(0.05).requires_grad_() for s in ((512, 256), (130, 512))]
        for p in w:
            p.grad = torch.zeros_like(p)
        zeros = [[torch.zeros_like(p) for p in w] for _ in range(2)]
        step = O.AdamWStep([p.detach() for p in w], [p.grad for p in w], *zeros, max_norm=1.0, skip_nonfinite=True)
        x, y, loss = (torch.zeros_like(t) for t in (*data[0], data[0][1].new_zeros(())))

        def once():
            for p in w:
                p.grad.zero_()
            out = mx.linear(torch.relu(mx.linear(x, w[0])), w[1])
            now = (out.float() - y).square().mean()
            now.backward()
            step(1e-3)
            loss.copy_(now.detach())

        return w, step, x, y, loss, once

    def run(captured):
        w, step, x, y, loss, once = fresh()
        go = once
        if captured:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                once()  # what is set up once, before the capture; its step is taken back
            torch.cuda.synchronize()
            start = fresh()[0]
            for p, q in zip(w, start):
                p.detach().copy_(q.detach())
            for t in (*step._plan._tensors[2], *step._plan._tensors[3], step.steps):
                t.zero_()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                once()
            go = graph.replay
        losses = []
        for a, b in data:
            x.copy_(a)
            y.copy_(b)
            go()
            losses.append(loss.clone())
        torch.cuda.synchronize()
        return [torch.stack(losses), *(p.detach().clone() for p in w), step.steps.clone(), step.record.clone()]

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)
    assert mx.tula_mx_error() == 0 and not mx._unfreed
