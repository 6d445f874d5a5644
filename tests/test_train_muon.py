"""Orthogonalised updates (tula_orthogonalize, tula_muon_*): refusals and the workspace's tiles on the CPU;
against Newton-Schulz steps in 64 bits on a GPU."""
import ctypes
import math

import pytest
import torch

from paper_2603_18112_gb300 import optim as O
from paper_2603_18112_gb300.tula_ags import TulaError

NS = (3.4445, -4.7750, 2.0315)
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUND = {t: torch.finfo(t).eps / 2 for t in TYPES}  # a rounding is off by at most half a step
U = 2.0 ** -24


# --------------------------------------------------------------------------------------------
# In 64 bits, and with the operands' roundings
# --------------------------------------------------------------------------------------------

def ns64(x, steps=5, half=False):
    """Newton-Schulz steps on x / |x| in fp64; half: what the products take and give is rounded to fp16
    where the kernels hold it so (their sums, in fp32, are off by far less)."""
    a, b, c = NS
    x = x.double()
    norm = x.norm()
    if not bool(norm > 0):
        return x * norm
    x = x / norm

    def held(t):
        return t.half().double() if half else t

    k = 2.0 ** min(15, math.floor(math.log2(math.sqrt(x.numel())))) if half and steps else 1.0
    tall = x.shape[0] > x.shape[1]
    x = held((x.t() if tall else x) * k)
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for _ in range(steps):
        gram = held(x @ x.t() / k ** 2)
        x = held(held(a * eye + b * gram + c * gram @ gram) @ x / k)
        k = 1.0
    return x.t() if tall else x


def _off(u, steps):
    """How far O(u) may be off in its norm and in an element: the same roundings of operands give errors of
    the same size, but where a sum in fp32 falls on the other side of a rounding they differ, by a step of
    2^-11 at most, here and there: twice that error, and a few steps besides."""
    want, held = ns64(u, steps), ns64(u, steps, True)
    d = held - want
    return want, 2 * float(d.norm()) + 2.0 ** -10 * float(want.norm()), 3 * float(d.abs().max()) + 2.0 ** -9 * float(want.abs().max())


def _near(got, want, off, most, dtype):
    d = (got.double() - want).abs() - 1.01 * ROUND[dtype] * want.abs() - 2.0 ** -24
    assert float(d.clamp(min=0).norm()) <= off and float(d.max()) <= most, (float(d.norm()), off, float(d.max()), most)


def _updates(n, rows, cols, seed, dtype=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(n, rows, cols, generator=gen) * torch.exp(0.5 * torch.randn(n, 1, cols, generator=gen))
    return (x + 0.25 * torch.randn(n, rows, 3, generator=gen) @ torch.randn(n, 3, cols, generator=gen)).to(dtype).cuda()


# --------------------------------------------------------------------------------------------
# On the CPU
# --------------------------------------------------------------------------------------------

def _size(rows, cols):
    r, c = ((ctypes.c_int64 * len(v))(*v) for v in (rows, cols))
    out = ctypes.c_size_t(0)
    return O._lib().tula_muon_workspace_size(r, c, len(rows), ctypes.byref(out)), out.value


def test_workspace_sizes():
    # tiles of 128 x 64 elements, twice each of X and of the two products of its smaller side (none for a list
    # of matrices that CTAs hold); parts of a norm and rows of a table by whole 256 bytes
    def of(r, c):
        n = min(r, c)
        x, a = -(-r // 128) * -(-c // 64), -(-n // 128) * -(-n // 64)
        return x, 2 * (x + a) * 16384

    for shapes in ([(1, 1)], [(64, 576)], [(4096, 1024), (1024, 4096), (4096, 1024)], [(0, 5), (129, 65)], [(64, 64)] * 500,
                   [(64, 64), (300, 200)], [(128, 769)], [(1536, 64)], [(1537, 64)]):
        full = [s for s in shapes if s[0]]
        tiles, space = sum(of(*s)[0] for s in full), sum(of(*s)[1] for s in full)
        if all(min(s) <= 128 and -(-s[0] // 128) * -(-s[1] // 64) <= 12 for s in full):
            tiles = space = 0
        want = -(-48 * len(full) // 256) * 256 + -(-8 * tiles // 256) * 256 + space
        assert _size(*zip(*shapes)) == (0, max(want, 256))
    assert _size([0], [7])[0] == 0 and _size([-1], [7])[0] == -1 and _size([1 << 21], [1])[0] == -1
    assert _size([1 << 20], [1 << 20])[0] == -1  # beyond 256 GB


def test_refusals_of_the_library():
    L, n, p = O._lib(), None, ctypes.c_void_p(256)

    def orth(x=p, kind=0, batch=1, rows=4, cols=8, stride=8, apart=32, steps=5, out=p, okind=1, space=p, size=1 << 20):
        return L.tula_orthogonalize(x, kind, batch, rows, cols, stride, apart, steps, out, okind, space, size, n)

    for bad in ({"kind": 3}, {"okind": 0}, {"okind": 3}, {"batch": -1}, {"rows": -1}, {"cols": 1 << 21}, {"stride": 7}, {"apart": -1},
                {"steps": -1}, {"steps": 101}, {"x": n}, {"out": n}, {"x": ctypes.c_void_p(258)}, {"out": ctypes.c_void_p(257)}):
        assert orth(**bad) == -1, bad
    assert orth(space=n) == orth(size=255) == orth(space=ctypes.c_void_p(128)) == -2
    assert orth(rows=300, cols=300, stride=300, size=1000) == -2
    assert orth(batch=0, x=n) == orth(rows=0, x=n) == 0
    assert L.tula_orthogonalize_workspace_size(1, 4, 4, n) == -1

    hp = O.tula_muon_hparams()
    L.tula_muon_default_hparams(ctypes.byref(hp))
    assert (hp.lr, hp.momentum, hp.weight_decay, hp.grad_scale, hp.nesterov, hp.ns_steps, hp.scale, hp.record) == \
        (1e-3, 0.95, 0.0, 1.0, 1, 5, 0, None)
    assert L.tula_muon_step(n, ctypes.byref(hp), n) == -1
    plan = ctypes.c_void_p()
    assert L.tula_muon_plan_create(n, p, 1 << 20, n, ctypes.byref(plan)) == -1 and not plan

    def create(**kw):
        one = {"rows": 4, "cols": 8, "g": 256, "w": 1024, "m": 2048, "gt": 0, "c": 4096, "ct": 1, "space": p, "size": 1 << 20} | kw
        arr = {k: (ctypes.c_int64 if k in ("rows", "cols") else ctypes.c_int if k in ("gt", "ct") else ctypes.c_void_p)
               for k in ("rows", "cols", "g", "w", "m", "gt", "c", "ct")}
        a = {k: (t * 1)(one[k]) for k, t in arr.items()}
        at = {k: ctypes.cast(v, ctypes.c_void_p) for k, v in a.items()}
        d = O.tula_muon_matrices(1, at["rows"], at["cols"], at["g"], at["gt"], at["w"], at["m"], at["c"], at["ct"])
        return L.tula_muon_plan_create(ctypes.byref(d), one["space"], one["size"], n, ctypes.byref(plan))

    for bad in ({"rows": -1}, {"cols": 1 << 21}, {"g": 0}, {"w": 0}, {"m": 0}, {"c": 0}, {"gt": 3}, {"ct": 0}, {"g": 258}, {"w": 258},
                {"m": 258}, {"c": 257}, {"w": 2048}, {"c": 1024}):
        assert create(**bad) == -1, bad
    assert create(size=255) == create(rows=300, cols=300, size=1000) == create(space=n) == create(space=ctypes.c_void_p(128)) == -2
    assert not plan and L.tula_muon_plan_destroy(n) == 0 and L.tula_muon_error(n, n) == -1
    # an empty list wants no GPU: its plan refuses hyperparameters that are out of range
    assert create(rows=0) == 0 and plan
    assert L.tula_muon_step(plan, ctypes.byref(hp), n) == 0
    for name, values in {"lr": (-1, math.nan, math.inf), "momentum": (-0.1, 1.0, math.nan), "weight_decay": (-1, math.inf),
                         "grad_scale": (0, 2.0 ** 101, math.nan), "ns_steps": (-1, 101), "scale": (2, -1)}.items():
        for v in values:
            bad = O.tula_muon_hparams.from_buffer_copy(hp)
            setattr(bad, name, v)
            assert L.tula_muon_step(plan, ctypes.byref(bad), n) == -1, (name, v)
    assert L.tula_muon_plan_destroy(plan) == 0


def test_refusals_of_the_binding():
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        O.orthogonalize(x)
    with pytest.raises(ValueError):
        O.orthogonalize(x[0])
    with pytest.raises(TypeError):
        O.MuonStep([x], [x], [x])
    with pytest.raises(ValueError):
        O.MuonStep([], [], [])
    with pytest.raises(ValueError):
        O.MuonStep([x], [x], [x], scale="none")


# --------------------------------------------------------------------------------------------
# On a GPU
# --------------------------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 1, 40), (2, 50, 1), (3, 2, 3), (1, 64, 64), (2, 65, 63), (1, 64, 576), (1, 576, 64), (3, 127, 129), (2, 128, 128),
          (1, 128, 256), (2, 129, 130), (5, 200, 333), (2, 333, 200), (1, 257, 640), (1, 1000, 257), (1, 1025, 1030), (2, 700, 2051),
          (1, 2051, 300), (9, 512, 512), (2, 128, 768), (2, 128, 769), (1, 65, 700), (1, 64, 512), (2, 1536, 64), (1, 1537, 64),
          (2, 768, 128), (1, 769, 128), (3, 1100, 50), (400, 90, 200), (300, 200, 30)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,rows,cols", SHAPES)
def test_orthogonalize(n, rows, cols):
    for dtype, out in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float16), (torch.float16, torch.float16)):
        x = _updates(n, rows, cols, rows + cols, dtype)
        got = O.orthogonalize(x, dtype=out)
        assert got.shape == x.shape and got.dtype == out
        for u, o in zip(x, got):
            _near(o, *_off(u, 5), out)
        assert torch.equal(got, O.orthogonalize(x, dtype=out))
        assert torch.equal(got[-1], O.orthogonalize(x[-1], dtype=out)) or n > 1  # (a batch may be shared out otherwise)
    assert O.tula_muon_error() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n,rows,cols", [(40, 512, 1024), (30, 1024, 512), (80, 300, 300), (1, 4096, 2048), (1, 2000, 4100)])
def test_many_and_large(n, rows, cols):
    """Enough blocks for pairs of CTAs to take several each."""
    x = _updates(n, rows, cols, 3)
    got = O.orthogonalize(x, dtype=torch.float16)
    for k in range(0, n, max(1, n // 5)):
        _near(got[k], *_off(x[k], 5), torch.float16)
    # each matrix by itself takes the same products in other blocks: sums of the same order
    for k in (0, n - 1):
        assert float((got[k].double() - O.orthogonalize(x[k], dtype=torch.float16).double()).norm()) <= 2.0 ** -9 * float(got[k].double().norm())
    assert O.tula_muon_error() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [0, 1, 2, 4, 7])
def test_steps(steps):
    for rows, cols in ((130, 70), (70, 130)):
        x = _updates(2, rows, cols, 9)
        got = O.orthogonalize(x, steps=steps, dtype=torch.float16)
        for u, o in zip(x, got):
            _near(o, *_off(u, steps), torch.float16)


@pytest.mark.gpu
def test_views_and_ranges():
    base = _updates(4, 150, 260, 5)
    for x in (base[:, :, :256], base[:, 3:140, 5:200], base[::2], base.transpose(1, 2), base[:, ::2, ::3], base[0, :1], base[1, :, 7:8],
              base[:1].expand(3, 150, 260), base.view(2, 2, 150, 260), base.transpose(0, 1)):
        got = O.orthogonalize(x, dtype=torch.float16)
        assert torch.equal(got.reshape(-1), O.orthogonalize(x.contiguous(), dtype=torch.float16).reshape(-1)) or \
            float((got.double() - O.orthogonalize(x.contiguous(), dtype=torch.float16).double()).norm()) <= 2.0 ** -10 * float(got.double().norm())
        u, o = x.reshape(-1, *x.shape[-2:])[-1], got.reshape(-1, *x.shape[-2:])[-1]
        _near(o, *_off(u, 5), torch.float16)
    # the norm holds over fp32's whole range, and a power of two changes nothing
    want = O.orthogonalize(base)
    for k in (-100, -60, 30, 100):
        assert torch.equal(O.orthogonalize(base * 2.0 ** k), want)
    tiny = torch.zeros(20, 30, device="cuda")
    tiny[3, 4], tiny[5, 6] = 1e-45, -1e-44
    _near(O.orthogonalize(tiny, dtype=torch.float16), *_off(tiny, 5), torch.float16)
    huge = torch.full((20, 30), 3.0e38, device="cuda")
    huge[::2] *= -1
    _near(O.orthogonalize(huge, dtype=torch.float16), *_off(huge, 5), torch.float16)


@pytest.mark.gpu
def test_zeros_infinities_nan_and_rank():
    x = _updates(6, 140, 200, 6)
    x[1] = 0.0
    x[2, 130, 199] = math.nan
    x[3, 0, 0] = math.inf
    x[4] = x[4][:, :1] * x[4][:1]  # of rank one
    x[5, 3:, :] = 0.0
    got = O.orthogonalize(x, dtype=torch.float16)
    assert not got[1].any() and bool(torch.isnan(got[2:4]).all())
    for k in (0, 4, 5):
        _near(got[k], *_off(x[k], 5), torch.float16)
    assert O.orthogonalize(x[:0]).shape == (0, 140, 200) and O.orthogonalize(x[:, :0]).shape == (6, 0, 200)
    # the workspace that NaN went through serves the next call
    assert bool(torch.isfinite(O.orthogonalize(x[[0, 0, 0, 0, 0, 0]])).all())


def _state(shapes, gtype, ctype, seed, offset=0):
    gen = torch.Generator().manual_seed(seed)

    def made(scale, dtype):
        """Views into one flat buffer, back to back from an offset."""
        flat = torch.randn(offset + sum(r * c for r, c in shapes), generator=gen).mul_(scale).to(dtype).cuda()
        out, at = [], offset
        for r, c in shapes:
            out.append(flat[at:at + r * c].view(r, c))
            at += r * c
        return out

    w, g, m = made(0.02, torch.float32), made(0.1, gtype), made(0.3, torch.float32)
    return w, g, m, ([t.to(ctype) for t in w] if ctype else None)


def _check_step(w, g, m, c, step, record=None, **kw):
    lr, mu, wd = kw.get("lr", 2e-3), kw.get("momentum", 0.95), kw.get("weight_decay", 0.1)
    scale, nesterov = kw.pop("grad_scale", 1.0), kw.pop("nesterov", True)
    kind = kw.pop("kind", "rms")
    coef = float(record[O.TULA_RECORD_COEF]) if record is not None else 1.0
    before = [(x.clone(), y.clone()) for x, y in zip(w, m)]
    grads = [t.clone() for t in g]
    step(lr, mu, wd, grad_scale=scale, record=record)
    for i, (w0, m0) in enumerate(before):
        if not w0.numel():
            continue
        d = g[i].double() * (coef / scale)
        m1 = m0.double() * mu + d
        off_m = 6 * U * (mu * m0.double().abs() + d.abs()) + 2.0 ** -149
        assert torch.equal(g[i], grads[i])
        assert bool(((m[i].double() - m1).abs() <= off_m).all())
        want, off, most = _off(d + mu * m1 if nesterov else m1, 5)
        r, q = w0.shape
        s = lr * (0.2 * math.sqrt(max(r, q)) if kind == "rms" else math.sqrt(max(1.0, r / q)))
        w1 = w0.double() * (1 - lr * wd) - s * want
        # the weights' own roundings, and the update's error
        d = (w[i].double() - w1).abs() - 4 * U * (w0.double().abs() + s * want.abs())
        assert float(d.clamp(min=0).norm()) <= s * off and float(d.max()) <= s * most
        if c is not None:
            assert torch.equal(c[i], w[i].to(c[i].dtype))
    assert O.tula_muon_error() == 0


LISTS = [[(1, 1)], [(64, 576), (16, 16), (64, 576)], [(100 + k % 30, 8 * (k % 7 + 1)) for k in range(310)], [(130, 70), (70, 130), (0, 5), (130, 70), (1, 300), (257, 257)],
         [(256, 64)] * 3 + [(64, 256)] * 2 + [(512, 512)] * 4, [(17 + 3 * k, 20 + 5 * k) for k in range(40)]]


@pytest.mark.gpu
@pytest.mark.parametrize("gtype,ctype", [(torch.float32, torch.bfloat16), (torch.bfloat16, None), (torch.float16, torch.float16)])
@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("shapes", LISTS)
def test_muon_step(shapes, gtype, ctype, offset):
    w, g, m, c = _state(shapes, gtype, ctype, 11, offset)
    step = O.MuonStep(w, g, m, c)
    for k in range(2):  # momentum and weights go on
        _check_step(w, g, m, c, step, grad_scale=4.0)
    w, g, m, c = _state(shapes, gtype, ctype, 12, offset)
    _check_step(w, g, m, c, O.MuonStep(w, g, m, c, nesterov=False, scale="aspect"), nesterov=False, kind="aspect", momentum=0.5)


@pytest.mark.gpu
def test_muon_of_several_types_clipped_and_left_out():
    """With the norm over these and other gradients, as a training step has it."""
    shapes = [(100, 64), (64, 100), (100, 64), (33, 33)]
    parts = [_state(shapes, t, c, 20 + i) for i, (t, c) in enumerate(zip(TYPES, (torch.bfloat16, torch.float16, torch.bfloat16)))]
    w, g, m, c = ([parts[i % 3][role][i] for i in range(4)] for role in range(4))
    other = torch.randn(1000, device="cuda")
    clip = O.GradClipper(g + [other])
    step = O.MuonStep(w, g, m, c)
    record = clip.norm(8.0, 0.5)
    assert float(record[O.TULA_RECORD_COEF]) < 1
    _check_step(w, g, m, c, step, record=record, grad_scale=8.0)
    for bad in (math.inf, math.nan):
        other[7] = bad
        before = [[t.clone() for t in ts] for ts in (w, m, c)]
        step(1e-3, 0.9, 0.1, grad_scale=8.0, record=clip.norm(8.0, 0.5))
        for ts, olds in zip((w, m, c), before):
            assert all(torch.equal(t, old) for t, old in zip(ts, olds))
    other[7] = 0.0
    _check_step(w, g, m, c, step, record=clip.norm(8.0, 0.5), grad_scale=8.0)


@pytest.mark.gpu
def test_muon_captured():
    """Two steps and the norm in a graph, replayed with new gradients, as two eager steps do it."""
    shapes = [(300, 200), (200, 300), (64, 64), (300, 200)]
    w, g, m, c = _state(shapes, torch.bfloat16, torch.bfloat16, 30)
    w2, g2, m2, c2 = ([t.clone() for t in ts] for ts in (w, g, m, c))
    clip, step = O.GradClipper(g), O.MuonStep(w, g, m, c)
    clip2, step2 = O.GradClipper(g2), O.MuonStep(w2, g2, m2, c2)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            for _ in range(2):
                step(1e-3, 0.9, 0.1, record=clip.norm(1.0, 1.0))
    torch.cuda.current_stream().wait_stream(side)
    for seed in (1, 2, 3):
        for a, b in zip(g, g2):
            a.copy_(torch.randn(a.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
            b.copy_(a)
        graph.replay()
        for _ in range(2):
            step2(1e-3, 0.9, 0.1, record=clip2.norm(1.0, 1.0))
        torch.cuda.synchronize()
        for a, b in zip((*w, *m, *c), (*w2, *m2, *c2)):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_orthogonalize_captured_and_on_another_stream():
    x = _updates(2, 200, 300, 40)
    xs, side = x.clone(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = O.orthogonalize(xs)
        b = O.orthogonalize(xs.transpose(1, 2))
    for seed in (41, 42):
        xs.copy_(_updates(2, 200, 300, seed))
        graph.replay()
        assert torch.equal(a, O.orthogonalize(xs)) and torch.equal(b, O.orthogonalize(xs.transpose(1, 2).contiguous()))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [O.orthogonalize(x) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(t, O.orthogonalize(x)) for t in got)


@pytest.mark.gpu
def test_plan_refusals():
    x = torch.zeros(4, 8, device="cuda")
    with pytest.raises(ValueError):
        O.MuonStep([x], [x.t().contiguous()], [x])
    with pytest.raises(TypeError):
        O.MuonStep([x.half()], [x], [x])
    with pytest.raises(TypeError):
        O.MuonStep([torch.zeros(8, 8, device="cuda")[:, :4]], [torch.zeros(8, 4, device="cuda")], [torch.zeros(8, 4, device="cuda")])
    with pytest.raises(ValueError):
        O.MuonStep([x[0]], [x[0]], [x[0]])
    with pytest.raises(ValueError):
        O.MuonStep([x], [x, x], [x])
    with pytest.raises(TypeError):
        O.MuonStep([x], [x], [x], copies=[x])
    with pytest.raises(TulaError):  # twice in the list
        O.MuonStep([x, x], [x.clone(), x.clone()], [x.clone(), x.clone()])
    step = O.MuonStep([x], [x.clone()], [x.clone()])
    with pytest.raises(TypeError):
        step(1e-3, record=torch.zeros(4))
    with pytest.raises(TulaError):
        step(-1.0)
    with pytest.raises(TypeError):
        O.orthogonalize(x, dtype=torch.float32)
    with pytest.raises(TulaError):
        O.orthogonalize(x, steps=-1)
