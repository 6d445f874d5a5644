"""A training step of layer norm, 8-bit layers, clipping, Muon and AdamW as they are used together: against the
formulas in 64 bits, call by call, and captured into a graph against eager steps."""
import pytest
import torch

from paper_2603_18112_gb300 import fp8, norm
from paper_2603_18112_gb300 import optim as O
from test_train_fp8 import E4, E5, quantised64, values64
from test_train_muon import ns64

pytestmark = pytest.mark.gpu

ROWS, WIDTH, HIDDEN, LR, MU, WD = 200, 160, 320, 1e-2, 0.9, 0.1
BF16 = 2.0 ** -9  # of a value in bf16: half a step, 2^-8 / 2


class Block:
    """x + down(relu(up(layer_norm(x)))), with its optimizers: Muon for the matrices, AdamW for the vectors."""

    def __init__(self, seed):
        gen = torch.Generator().manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(*shape, generator=gen) * scale).cuda()

        self.x = normal(ROWS, WIDTH, scale=1.0).bfloat16()
        self.dy = normal(ROWS, WIDTH, scale=1e-2).bfloat16()
        self.w = [normal(HIDDEN, WIDTH, scale=WIDTH ** -0.5), normal(WIDTH, HIDDEN, scale=HIDDEN ** -0.5)]
        self.v = [1 + normal(WIDTH, scale=0.1), normal(WIDTH, scale=0.1)]
        self.leaves = [t.requires_grad_() for t in (*self.w, *self.v)]
        self.grads = [torch.zeros_like(t) for t in self.leaves]
        self.moms = [torch.zeros_like(t) for t in self.w]
        self.copies = [t.detach().bfloat16() for t in self.w]
        self.m, self.s = [torch.zeros_like(t) for t in self.v], [torch.zeros_like(t) for t in self.v]
        self.clip = O.GradClipper(self.grads)
        self.muon = O.MuonStep([t.detach() for t in self.w], self.grads[:2], self.moms, copies=self.copies)
        self.adam = O.AdamWStep([t.detach() for t in self.v], self.grads[2:], self.m, self.s)

    def forward(self):
        h = norm.layer_norm(self.x, self.v[0], self.v[1])
        return self.x + fp8.linear(torch.relu(fp8.linear(h, self.w[0], grad_dtype=E5)), self.w[1], grad_dtype=E5)

    def step(self):
        y = self.forward()
        for g, new in zip(self.grads, torch.autograd.grad(y, self.leaves, self.dy)):
            g.copy_(new)
        record = self.clip.norm(1.0, 0.05)
        self.muon(LR, MU, WD, record=record)
        self.adam(LR, (0.9, 0.99), 1e-8, WD)
        return y.detach()

    def state(self):
        return [t.detach() for t in (*self.leaves, *self.grads, *self.moms, *self.copies, *self.m, *self.s, self.clip.record)]


def _near(t, code=E4, square=False):
    """What a matrix's codes stand for, on the CPU in 64 bits."""
    return values64(*quantised64(t, code, square))


def _close(got, want, rel):
    assert float((got.double().cpu() - want).norm()) <= rel * float(want.norm()), float((got.double().cpu() - want).norm() / want.norm())


def test_a_step_against_the_formulas():
    """Each call's result from the one before it as that was, in 64 bits: roundings to bf16 of its output
    and fp32's of its sums (far below) are what is left; the gradients through bf16 values too."""
    b = Block(1)
    before = [t.detach().double().cpu() for t in b.leaves]
    x, dy = b.x.double().cpu(), b.dy.double().cpu()
    h = norm.layer_norm(b.x, *b.v).detach()
    n = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    _close(h, n * before[2] + before[3], BF16)
    up = fp8.linear(h, b.w[0].detach())
    _close(up, _near(h) @ _near(b.w[0], square=True).t(), BF16 + 1e-5)
    a = torch.relu(up)
    y = b.step()
    _close(y, x + (_near(a) @ _near(before[1], square=True).t()).bfloat16().double(), 2 * BF16)
    # the gradients; ds and dh pass through bf16 on their way
    w_up, w_down = _near(before[0], square=True), _near(before[1], square=True)
    da = (_near(b.dy, E5) @ w_down).bfloat16()
    d_up = da * (up.cpu() > 0)
    dh = (_near(d_up, E5) @ w_up).bfloat16().double()
    want = [_near(d_up.t(), E5) @ _near(h.t()).t(), _near(b.dy.t(), E5) @ _near(a.t()).t(), (dh * n).sum(0), dh.sum(0)]
    # a value of da or dh that falls on the other side of a rounding to bf16, or of one to a code, moves by a
    # step: 2^-8 and 2^-2 of it.  Sums in fp32 are off by 1e-6 of their size, so that it is few of them.
    for got, ref in zip(b.grads, want):
        _close(got, ref, 2e-3)
    size = sum(float(g.double().square().sum()) for g in b.grads) ** 0.5
    coef = min(1.0, 0.05 / (size + 1e-6))
    assert coef < 1 and float(b.clip.record[O.TULA_RECORD_COEF]) == pytest.approx(coef, rel=1e-5)
    for i in range(2):
        d = b.grads[i].double().cpu() * coef
        _close(b.moms[i], d, 1e-6)
        u = d + MU * d
        o, off = ns64(u), ns64(u, half=True)
        scale = LR * 0.2 * max(u.shape) ** 0.5
        moved = (b.w[i].detach().double().cpu() - before[i] * (1 - LR * WD)) / -scale
        assert float((moved - o).norm()) <= 2 * float((off - o).norm()) + 2e-3 * float(o.norm())
        assert torch.equal(b.copies[i], b.w[i].detach().bfloat16())
    for i in range(2):  # AdamW's first step moves each weight by lr, after the decay
        moved = (before[2 + i] * (1 - LR * WD) - b.v[i].detach().double().cpu()) / LR
        assert bool(((moved - torch.sign(b.grads[2 + i].double().cpu())).abs() <= 1e-4).all())


def test_captured_steps_are_eager_ones():
    eager, graphed = Block(2), Block(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.step()
    torch.cuda.current_stream().wait_stream(side)
    eager.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = graphed.step()
    for seed in range(4):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for t in ("x", "dy"):
            new = torch.randn(ROWS, WIDTH, generator=gen, device="cuda") * (1e-2 if t == "dy" else 1.0)
            getattr(eager, t).copy_(new)
            getattr(graphed, t).copy_(new)
        graph.replay()
        want = eager.step()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        for p, q in zip(graphed.state(), eager.state()):
            assert torch.equal(p, q)
    assert fp8.tula_fp8_error() == 0 and O.tula_muon_error() == 0
