"""GPU tests of the order of calls: inputs that a kernel of the caller's own still writes when the call is
made, calls that follow one another without a wait, and sizes beyond 32-bit indexes."""
import ctypes
import subprocess

import pytest
import torch

from paper_2603_18112_gb300 import build as B
from paper_2603_18112_gb300 import mx, optim
from paper_2603_18112_gb300 import tula_ags as T
from test_gpu_callers import _LATE_WRITER

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def write_late(tmp_path_factory):
    """A kernel that lets its dependents start at once and copies src to dst some 300 us later."""
    B.build()
    d = tmp_path_factory.mktemp("late_writer")
    (d / "late_writer.cu").write_text(_LATE_WRITER)
    nvcc = B.nvcc_path()
    subprocess.run([nvcc, *B.ARCH, "-O2", "-shared", "-Xcompiler", "-fPIC", "-cudart", "shared", "-Xlinker",
                    f"-rpath={B.cuda_lib_dir(nvcc)}", str(d / "late_writer.cu"), "-o", str(d / "late.so")], check=True)
    fn = ctypes.CDLL(str(d / "late.so")).write_late
    fn.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_longlong, ctypes.c_void_p]

    def write(dst, src):
        assert dst.dtype == torch.float32 and dst.numel() == src.numel()
        assert fn(dst.data_ptr(), src.data_ptr(), dst.numel(), torch.cuda.current_stream().cuda_stream) == 0

    return write


def _randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("n", [3000, 4_000_000])
@pytest.mark.parametrize("shift", [0, 1])
def test_gradients_written_late(write_late, n, shift):
    good, bad = _randn(1, n), _randn(2, n) * 100
    # what L1 may hold of the buffers from before is the other values
    flat = torch.zeros(n + 8, device="cuda")
    g = flat[shift:shift + n]
    clip = optim.GradClipper([g])
    w, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    step = optim.AdamWStep([w], [g], [m], [v], max_norm=1.0)

    def run(late):
        outs = []
        g.copy_(bad)
        outs.append(clip.norm().clone())
        (write_late if late else torch.Tensor.copy_)(g, good)
        outs.append(clip.norm().clone())
        g.copy_(bad)
        outs.append(clip.norm().clone())
        (write_late if late else torch.Tensor.copy_)(g, good)
        clip.clip_(0.5)
        outs.append(g.clone())
        for t in (w, m, v, step.steps):
            t.zero_()
        (write_late if late else torch.Tensor.copy_)(g, bad)
        step(1e-2)
        (write_late if late else torch.Tensor.copy_)(g, good)
        step(1e-2)
        torch.cuda.synchronize()
        return outs + [w.clone(), m.clone(), v.clone()]

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("rows,cols", [(1, 4096), (300, 1001), (4096, 4096)])
def test_matrices_written_late(write_late, rows, cols):
    x, old = _randn(3, rows, cols), _randn(4, rows, cols) * 50
    other = mx.quantize(_randn(5, 256, cols))

    def run(late):
        z = old.clone()
        first = mx.quantize(z, cols=True)
        (write_late if late else torch.Tensor.copy_)(z, x)
        q, t = mx.quantize(z, cols=True)
        outs = [mx.dequantize(q, torch.float32), mx.dequantize(t, torch.float32), mx.matmul(q, other, torch.float32)]
        torch.cuda.synchronize()
        return outs + [q.codes.clone(), t.codes.clone(), mx.dequantize(first[0])]

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)


def test_a_chain_without_a_wait_repeats_itself():
    """Quantise, multiply, clip, step, again and again on one stream, twice from the same start."""
    def run():
        w = _randn(6, 700, 512) * 0.05
        g, m, v = torch.zeros_like(w), torch.zeros_like(w), torch.zeros_like(w)
        step = optim.AdamWStep([w], [g], [m], [v], max_norm=1.0, skip_nonfinite=True)
        x, y = _randn(7, 384, 512).bfloat16(), _randn(8, 384, 700)
        losses = []
        for _ in range(12):
            wr = w.detach().requires_grad_()
            out = mx.linear(x, wr).float()
            loss = (out - y).square().mean()
            g.copy_(torch.autograd.grad(loss, wr)[0])
            step(1e-2)
            losses.append(loss.detach())
        torch.cuda.synchronize()
        return torch.stack(losses), w

    (a, wa), (b, wb) = run(), run()
    assert torch.equal(a, b) and torch.equal(wa, wb)
    assert a[-1] < a[0] and mx.tula_mx_error() == 0


def test_beyond_32_bit_indexes():
    """A matrix of more than 2^32 elements: slabs at both ends and around that mark come out as by
    themselves, and so do the values read back."""
    rows, cols = 70200, 61448
    assert rows * cols > 1 << 32
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(9)
    for r in range(0, rows, 7020):
        x[r:r + 7020] = torch.randn(7020, cols, generator=gen, device="cuda")
    q, t = mx.quantize(x, cols=True)
    back = mx.dequantize(q)
    last = (rows - 1) // 128 * 128
    mark = (1 << 32) // cols // 128 * 128
    for a in (0, 35072, mark - 128, mark, mark + 128, last):
        b = min(rows, a + 128)
        sq, st = mx.quantize(x[a:b], cols=True)
        assert torch.equal(sq.codes, q.codes[a:b]) and torch.equal(sq.scales[0], q.scales[a // 128])
        assert torch.equal(st.codes, t.codes[:, a // 2:a // 2 + 64]) and torch.equal(st.scales[:, 0], t.scales[:, a // 128])
        assert torch.equal(back[a:b], mx.dequantize(sq))
    one = mx.quantize(_randn(10, 3, cols))
    out = mx.matmul(one, q, torch.float32)
    for a in (0, mark, last):
        b = min(rows, a + 128)
        part = mx.matmul(one, mx.quantize(x[a:b]), torch.float32)
        want = mx.dequantize(one, torch.float32).double() @ mx.dequantize(mx.quantize(x[a:b]), torch.float32).double().t()
        # both sums err by no more than cols / 32 additions of parts no larger than what they add
        size = mx.dequantize(one, torch.float32).double().abs() @ mx.dequantize(mx.quantize(x[a:b]), torch.float32).double().abs().t()
        tol = (cols // 32 + 2) * 2.0 ** -23 * size
        assert bool(((out[:, a:b].double() - want).abs() <= tol).all()) and bool(((part.double() - want).abs() <= tol).all())
    del x, q, t, back, out
    # a list of more than 2^32 gradients in one tensor
    g = torch.full(((1 << 32) + 4099,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    clip = optim.GradClipper([g])
    want = (g.numel() * 2.0 ** -20) ** 0.5
    assert clip.norm()[0].item() == pytest.approx(want, rel=1e-6)
    clip.clip_(want / 2)
    assert g[0].item() == g[-1].item() == g[1 << 32].item() == 2.0 ** -11
    assert g.float().sum(dtype=torch.float64).item() == g.numel() * 2.0 ** -11
