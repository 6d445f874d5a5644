"""The gradient norm, clipping and AdamW (include/tula_train.h) against their formulas in fp64, and
what they refuse."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2603_18112_gb300 import build as B
from paper_2603_18112_gb300 import optim as O
from paper_2603_18112_gb300 import tula_ags as T

U = 2.0 ** -24                  # fp32's unit roundoff
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
# A norm's sum: chains of 8 squares, two additions, five of a warp, each within U of a sum of
# positive terms; fp64 beyond.  The root halves that; the record and the coefficient round again.
NORM_TOL = (15 / 2 + 2) * U


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    T.lib()


# ---------------------------------------------------------------------------------------------
# Refusals (no GPU)
# ---------------------------------------------------------------------------------------------

def _desc(n=2, numels=(5, 7), grads=None, types=None, params=None, m=None, v=None, copies=None, ctypes_=None):
    keep = []

    def arr(ct, vals):
        if vals is None:
            return None
        a = (ct * len(vals))(*vals)
        keep.append(a)
        return ctypes.cast(a, ctypes.c_void_p)

    P = ctypes.c_void_p
    fake = [0x10000, 0x20000]
    d = O.tula_train_tensors(n, arr(ctypes.c_int64, numels), arr(P, fake if grads is None else grads),
                             arr(ctypes.c_int, types), arr(P, params), arr(P, m), arr(P, v), arr(P, copies),
                             arr(ctypes.c_int, ctypes_))
    return d, keep


def _create(ws=0x40000, size=1 << 20, out=True, **kw):
    d, keep = _desc(**kw)
    h = ctypes.c_void_p(0x1234)
    rc = O._lib().tula_train_plan_create(ctypes.byref(d), ws, size, None, ctypes.byref(h) if out else None)
    if out:
        assert rc != 0 and h.value is None
    return rc


def test_plan_refusals():
    fake = [0x10000, 0x20000]
    assert _create(out=False) == T.TULA_ERR_ARG
    assert _create(n=0) == T.TULA_ERR_ARG
    assert _create(numels=(5, -1)) == T.TULA_ERR_ARG
    assert _create(numels=(1 << 46, 7)) == T.TULA_ERR_ARG              # too many tiles
    assert _create(grads=[0x10000, 0]) == T.TULA_ERR_ARG
    assert _create(grads=[0x10000, 0x20002]) == T.TULA_ERR_ARG        # fp32 off 4 bytes
    assert _create(grads=[0x10000, 0x20001], types=[1, 1]) == T.TULA_ERR_ARG
    assert _create(types=[0, 3]) == T.TULA_ERR_ARG
    assert _create(params=fake) == T.TULA_ERR_ARG                      # no moments
    assert _create(params=fake, m=fake, v=[0x10000, 0]) == T.TULA_ERR_ARG
    assert _create(copies=fake) == T.TULA_ERR_ARG                      # copies of no weights
    assert _create(params=fake, m=fake, v=fake, copies=fake, ctypes_=[1, 0]) == T.TULA_ERR_ARG
    assert _create(ws=0) == T.TULA_ERR_WORKSPACE
    assert _create(ws=0x40010) == T.TULA_ERR_WORKSPACE
    assert _create(size=64) == T.TULA_ERR_WORKSPACE
    L = O._lib()
    assert L.tula_train_plan_destroy(None) == 0
    assert L.tula_grad_norm(None, 1.0, 0.0, 0x1000, None) == T.TULA_ERR_ARG
    assert L.tula_grad_clip(None, 1.0, 0x1000, None) == T.TULA_ERR_ARG
    assert L.tula_adamw_step(None, None, None) == T.TULA_ERR_ARG
    for bad in ([], [3, -1], [1 << 46]):
        with pytest.raises(T.TulaError):
            O.tula_train_workspace_size(bad)
    assert O.tula_train_workspace_size([0]) > 0


def test_binding_refusals():
    with pytest.raises(ValueError):
        O.GradClipper([])
    with pytest.raises(TypeError):
        O.GradClipper([torch.zeros(3)])                                # not on a GPU


def test_header_is_exported():
    import re
    text = re.sub(r"/\*.*?\*/", "", B.TRAIN_HEADER.read_text(), flags=re.S)
    names = set(re.findall(r"\b(tula_\w+)\s*\(", text))
    assert "tula_adamw_step" in names
    for name in names:
        assert hasattr(T.lib(), name), name


# ---------------------------------------------------------------------------------------------
# On the GPU
# ---------------------------------------------------------------------------------------------

SIZES = {
    "one": [1],
    "empty": [0, 0],
    "ragged": [0, 1, 7, 8, 9, 2047, 2048, 2049, 8191, 3, 8193, 0, 20000],
    "many": [17 + 13 * (i % 41) for i in range(700)],
    # beyond 8 * 152 small tiles, so large ones, with groups of them, and over 64 * 64 CTAs
    "large": [3_000_001, 5, 64, 8192 * 40, 16384 * 3 + 1],
    "huge": [60_000_003, 8191],
}


def _flat_views(sizes, dtype, packed, shift, fill):
    """Views into one flat buffer: at 64-element offsets, or back to back, `shift` elements in."""
    offs, at = [], shift
    for n in sizes:
        offs.append(at)
        at += n if packed else (n + 63) // 64 * 64
    flat = fill(at + 1).to(dtype)
    return [flat[o:o + n] for o, n in zip(offs, sizes)]


def _grads(sizes, dtype, layout, seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    packed, shift = {"padded": (False, 0), "packed": (True, 0), "shifted": (True, 3)}[layout]
    return _flat_views(sizes, dtype, packed, shift,
                       lambda n: torch.randn(n, generator=gen, device="cuda") * scale)


def _norm64(grads, scale=1.0):
    return math.sqrt(sum(float((g.double() / scale).square().sum()) for g in grads))


def _f32(x):
    with np.errstate(over="ignore"):
        return float(np.float32(x))


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(SIZES))
@pytest.mark.parametrize("layout", ["padded", "packed", "shifted"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_clip(name, layout, dtype):
    grads = _grads(SIZES[name], dtype, layout, 1)
    before = [g.clone() for g in grads]
    want = _norm64(grads)
    clip = O.GradClipper(grads)
    rec = clip.norm(max_norm=0.5).tolist()
    assert rec[0] == pytest.approx(want, rel=NORM_TOL) and rec[2] == 1.0
    assert all(torch.equal(a, b) for a, b in zip(before, grads))        # read only
    coef = min(1.0, 0.5 / (want + 1e-6))
    assert rec[1] == pytest.approx(coef, rel=2 * NORM_TOL)
    rec2 = clip.clip_(0.5).tolist()
    assert rec2[:3] == rec[:3]
    for a, g in zip(before, grads):
        ref = a.double() * coef
        err = (g.double() - ref).abs()
        tol = ref.abs() * (1.01 * ROUND[dtype] + 2 * NORM_TOL) + TINY[dtype]
        assert bool((err <= tol).all())
    after = [g.clone() for g in grads]
    clip.clip_(2.0 * max(1.0, want))                                     # below the threshold
    assert all(torch.equal(a, g) for a, g in zip(after, grads))
    for a, g in zip(before, grads):
        g.copy_(a)
    # bit for bit, at these alignments
    assert O.GradClipper(grads).norm(max_norm=0.5).tolist() == rec


@pytest.mark.gpu
def test_mixed_types_and_elements_of_their_own_alignment():
    """Tensors of different types and alignments in one list."""
    a = _grads([1000, 3000, 7], torch.float32, "shifted", 2)
    b = _grads([1000, 5001, 9], torch.bfloat16, "shifted", 3)
    c = _grads([12, 4097], torch.float16, "packed", 4)
    grads = a + b + c
    rec = O.GradClipper(grads).norm(grad_scale=4.0, max_norm=1.0).tolist()
    want = _norm64(grads, 4.0)
    assert rec[0] == pytest.approx(want, rel=NORM_TOL)
    assert rec[1] == pytest.approx(1.0 / (want + 1e-6), rel=2 * NORM_TOL)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e-40, 1e-30, 1e-20, 1e15, 1e25, 1e37])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_over_the_whole_range(dtype, scale):
    """Squares that underflow or overflow fp32; also beside ordinary ones and zeros."""
    small = _grads([5000, 33], dtype, "padded", 5, scale)
    rec = O.GradClipper(small).norm().tolist()
    want = _norm64(small)
    # denormal values are exact, their norm rounds to fp32's grid; a norm above its range is
    # finite all the same
    assert rec[0] == pytest.approx(_f32(want), rel=NORM_TOL, abs=2.0 ** -149) and rec[2] == 1.0
    mixed = small + [torch.zeros(10000, dtype=dtype, device="cuda")] + _grads([9000], dtype, "padded", 6)
    rec = O.GradClipper(mixed).norm().tolist()
    assert rec[0] == pytest.approx(_f32(_norm64(mixed)), rel=NORM_TOL) and rec[2] == 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_norm_of_infinities_and_nans(dtype, bad):
    for where in (0, 4321, 19999):
        grads = _grads([100, 20000, 3], dtype, "padded", 7)
        grads[1][where] = bad
        clip = O.GradClipper(grads)
        norm, coef, finite, _ = clip.norm(max_norm=1.0).tolist()
        assert finite == 0.0
        if math.isnan(bad):
            assert math.isnan(norm) and math.isnan(coef)
        else:
            assert norm == math.inf and coef == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_clipping_of_infinities_and_nans(dtype):
    """An infinite norm has coef 0, whatever the threshold, so that finite gradients become zeros and
    infinite ones NaN; a NaN makes them all NaN."""
    for bad, max_norm in ((math.inf, 1.0), (math.inf, math.inf), (-math.inf, 3.0), (math.nan, 1.0), (math.nan, math.inf)):
        for where in (0, 4321, 19999):
            grads = _grads([100, 20000, 3], dtype, "padded", 7)
            grads[1][where] = bad
            norm, coef, finite, _ = O.GradClipper(grads).clip_(max_norm).tolist()
            assert finite == 0.0
            if math.isnan(bad):
                assert math.isnan(norm) and math.isnan(coef)
                assert all(bool(torch.isnan(g).all()) for g in grads)
                continue
            assert norm == math.inf and coef == 0.0
            nans = torch.isnan(grads[1])
            assert bool(nans[where]) and int(nans.sum()) == 1
            assert not grads[0].any() and not grads[2].any() and not grads[1][~nans].any()


def _adam_state(sizes, gdtype, layout, copies, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    packed, shift = {"padded": (False, 0), "packed": (True, 0), "shifted": (True, 3)}[layout]

    def role(dtype, f):
        return _flat_views(sizes, dtype, packed, shift, f)

    def normal(s):
        return lambda n: torch.randn(n, generator=gen, device="cuda") * s

    w, m = role(torch.float32, normal(0.1)), role(torch.float32, normal(0.01))
    v = role(torch.float32, lambda n: torch.rand(n, generator=gen, device="cuda") * 1e-3)
    g = role(gdtype, normal(0.05))
    c = role(copies, normal(1.0)) if copies else None
    return w, g, m, v, c


def _adam64(w, g, m, v, t, mult, lr, b1, b2, eps, wd):
    """(w, m, v) in fp64 and bounds on what fp32 may add to each."""
    w, g, m, v = (x.double() for x in (w, g, m, v))
    d = g * mult
    a, b = b1 * m, (1 - b1) * d
    m2 = a + b
    size_m = a.abs() + b.abs()
    v2 = b2 * v + (1 - b2) * d * d
    c1, c2 = 1 - b1 ** t, 1 - b2 ** t
    den = torch.sqrt(v2 / c2) + eps
    w2 = w * (1 - lr * wd) - lr / c1 * m2 / den
    # m, v: constants, products and the sum, six roundings of parts no larger than size_m and v2;
    # the coefficient's error (2 NORM_TOL, twice in d^2).  w: four of w, a dozen of the quotient.
    tol_m = (6 * U + 2 * NORM_TOL) * size_m + 1e-40
    tol_v = (8 * U + 4 * NORM_TOL) * v2 + 1e-40
    tol_w = 4 * U * w.abs() + (14 * U + 6 * NORM_TOL) * lr / c1 * size_m / den + 1e-40
    return (w2, m2, v2), (tol_w, tol_m, tol_v)


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(SIZES))
@pytest.mark.parametrize("layout,gdtype,copies,max_norm,scale", [
    ("padded", torch.float32, None, 0.0, 1.0),
    ("padded", torch.bfloat16, torch.bfloat16, 0.3, 1.0),
    ("packed", torch.float16, torch.float16, 0.3, 256.0),
    ("packed", torch.bfloat16, torch.bfloat16, 0.0, 1.0),
    ("shifted", torch.float32, torch.bfloat16, 1e9, 1.0),
])
def test_adamw(name, layout, gdtype, copies, max_norm, scale):
    w, g, m, v, c = _adam_state(SIZES[name], gdtype, layout, copies, 11)
    lr, b1, b2, eps, wd = 3e-3, 0.9, 0.98, 1e-8, 0.1
    steps = torch.tensor([4, 1], dtype=torch.int64, device="cuda")
    step = O.AdamWStep(w, g, m, v, copies=c, max_norm=max_norm, steps=steps)
    for t in (5, 6):
        norm = _norm64(g, scale)
        coef = min(1.0, max_norm / (norm + 1e-6)) if max_norm else 1.0
        want = [_adam64(*x, t, coef / scale, lr, b1, b2, eps, wd) for x in zip(w, g, m, v)]
        grads = [x.clone() for x in g]
        step(lr, (b1, b2), eps, wd, grad_scale=scale)
        assert steps.tolist() == [t, 1]
        if max_norm:
            assert step.record[0].item() == pytest.approx(norm, rel=NORM_TOL)
        for i, (ref, tol) in enumerate(want):
            for role, x, r, e in zip("wmv", (w[i], m[i], v[i]), ref, tol):
                assert bool(((x.double() - r).abs() <= e).all()), (t, i, role)
            if c is not None:
                assert torch.equal(c[i], w[i].to(copies))
            assert torch.equal(g[i], grads[i])                           # read only


@pytest.mark.gpu
@pytest.mark.parametrize("offsets", [(0, 1, 0, 0, 0), (1, 2, 3, 4, 5), (0, 0, 0, 0, 1), (4, 0, 4, 4, 4)])
@pytest.mark.parametrize("max_norm", [0.0, 0.5])
@pytest.mark.parametrize("sizes", [[1, 7, 3000], [2_600_000, 5, 20_001]])
def test_adamw_of_buffers_at_offsets_of_their_own(offsets, max_norm, sizes):
    """Weights, gradients, moments and copies that start at different elements of eight: the results are
    those of buffers that lie alike, up to the norm's order of addition."""
    def at(off, xs):
        flat = torch.zeros(sum(sizes) + 8, dtype=xs[0].dtype, device="cuda")
        out, i = [], off
        for x in xs:
            flat[i:i + x.numel()] = x
            out.append(flat[i:i + x.numel()])
            i += x.numel()
        return out

    base = _adam_state(sizes, torch.bfloat16, "padded", torch.bfloat16, 16)
    moved = [at(o, xs) for o, xs in zip(offsets, base)]
    steps = []
    for w, g, m, v, c in (base, moved):
        step = O.AdamWStep(w, g, m, v, copies=c, max_norm=max_norm)
        step(1e-2, (0.9, 0.98), 1e-8, 0.1)
        steps.append(step)
    if max_norm:
        a, b = (s.record.tolist() for s in steps)
        assert a[0] == pytest.approx(b[0], rel=2 * NORM_TOL)
    for i in range(len(sizes)):
        (w, g, m, v, c), (w2, g2, m2, v2, c2) = ([r[i] for r in s] for s in (base, moved))
        if max_norm == 0.0:
            assert torch.equal(w, w2) and torch.equal(m, m2) and torch.equal(v, v2) and torch.equal(c, c2)
        else:
            for x, y in ((w, w2), (m, m2), (v, v2)):
                # coefficients 4 NORM_TOL apart, of which a moment's square takes twice as much
                assert bool(((x - y).abs() <= (8 * NORM_TOL + 8 * U) * (x.abs() + 0.05)).all())
            assert torch.equal(c2, w2.bfloat16())
        assert torch.equal(g, g2)


# exponents (grad_scale, |G| before it) at which the norm, the coefficient or their product with
# 1 / grad_scale leaves fp32's normal range on the way, though what an element is multiplied by does not
ENDS = [(-100, 30), (-99, 30), (-90, 49), (-76, 20), (-60, -20), (-33, 49), (-32, 49), (-31, 49), (0, 49),
        (31, -20), (33, -20), (60, 40), (99, 45), (100, 50)]


@pytest.mark.gpu
@pytest.mark.parametrize("scale2,norm2", ENDS)
@pytest.mark.parametrize("max_norm", [0.0, 2.0 ** -40, 1.0, 2.0 ** 60])
def test_norm_and_adamw_over_the_range_of_grad_scale(scale2, norm2, max_norm):
    w, g, m, v, _ = _adam_state([5000, 33], torch.float32, "padded", None, 17)
    scale = 2.0 ** scale2
    by = 2.0 ** norm2 / _norm64(g)
    for x in g:
        x.mul_(by)
    for x in m + v:
        x.zero_()
    norm = _norm64(g) / scale
    coef = min(1.0, max_norm / (norm + 1e-6)) if max_norm else 1.0
    rec = O.GradClipper(g).norm(grad_scale=scale, max_norm=max_norm).tolist()
    # on fp32's grid, also below its normal range
    assert rec[0] == pytest.approx(_f32(norm), rel=NORM_TOL, abs=2.0 ** -149) and rec[2] == 1.0
    assert rec[1] == pytest.approx(coef, rel=2 * NORM_TOL, abs=2.0 ** -149)
    if not max_norm and norm2 - scale2 > 60:
        return  # squares beyond fp32's range
    lr, b1, b2, eps, wd = 3e-3, 0.9, 0.98, 1e-8, 0.1
    steps = torch.tensor([999, 0], dtype=torch.int64, device="cuda")
    step = O.AdamWStep(w, g, m, v, max_norm=max_norm, steps=steps)
    want = [_adam64(*x, 1000, coef / scale, lr, b1, b2, eps, wd) for x in zip(w, g, m, v)]
    step(lr, (b1, b2), eps, wd, grad_scale=scale)
    for i, (ref, tol) in enumerate(want):
        for role, x, r, e in zip("wmv", (w[i], m[i], v[i]), ref, tol):
            assert bool(((x.double() - r).abs() <= e).all()), (i, role)


@pytest.mark.gpu
def test_adamw_matches_torch_from_the_first_step():
    """Zero moments, steps from 1 on, the defaults of torch.optim.AdamW."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    w = [torch.randn(n, generator=gen, device="cuda", dtype=torch.float64) for n in (1000, 33, 4099)]
    ours = [x.float() for x in w]
    ref = [torch.nn.Parameter(x.float().double()) for x in w]
    grads = [torch.zeros_like(x) for x in ours]
    m, v = [torch.zeros_like(x) for x in ours], [torch.zeros_like(x) for x in ours]
    opt = torch.optim.AdamW(ref, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
    step = O.AdamWStep(ours, grads, m, v)
    for _ in range(20):
        for p, g in zip(ref, grads):
            g.copy_(torch.randn(g.shape, generator=gen, device="cuda"))
            p.grad = g.double()
        opt.step()
        step(1e-3)
    assert step.steps.tolist() == [20, 0]
    for p, x in zip(ref, ours):
        # twenty steps of at most about 1e-3 each, a few roundings of the weight and of each step
        tol = 20 * (4 * U * (p.abs() + 0.02) + 1e-3 * 20 * U * 10)
        assert bool(((x.double() - p).abs() <= tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16, torch.float16])
def test_a_step_that_is_not_finite_is_left_out(bad, gdtype):
    w, g, m, v, c = _adam_state([100, 9000, 5], gdtype, "padded", torch.bfloat16, 12)
    g[1][8999] = bad
    old = [x.clone() for r in (w, m, v, c) for x in r]
    step = O.AdamWStep(w, g, m, v, copies=c, skip_nonfinite=True)
    step(1e-3)
    step(1e-3)
    assert step.steps.tolist() == [0, 2] and step.record[2].item() == 0.0
    assert all(torch.equal(a, b) for a, b in zip(old, [x for r in (w, m, v, c) for x in r]))
    g[1][8999] = 0.25
    step(1e-3)
    assert step.steps.tolist() == [1, 2] and step.record[2].item() == 1.0
    assert not torch.equal(old[0], w[0])


@pytest.mark.gpu
@pytest.mark.parametrize("beta1,beta2,eps,wd", [(0.0, 0.0, 1e-8, 0.0), (0.9, 0.0, 1e-3, 0.5), (0.0, 0.99, 0.0, 0.1)])
def test_adamw_at_the_ends_of_its_hyperparameters(beta1, beta2, eps, wd):
    w, g, m, v, _ = _adam_state([3000, 77], torch.float32, "padded", None, 13)
    step = O.AdamWStep(w, g, m, v)
    want = [_adam64(*x, 1, 1.0, 1e-2, beta1, beta2, eps, wd) for x in zip(w, g, m, v)]
    step(1e-2, (beta1, beta2), eps, wd)
    for i, (ref, tol) in enumerate(want):
        for x, r, e in zip((w[i], m[i], v[i]), ref, tol):
            assert bool(((x.double() - r).abs() <= e).all())


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [0.0, 1e-8, 1.0])
@pytest.mark.parametrize("sizes", [[40_001], [2_600_000, 33]])
def test_adamw_rounds_as_fp32_does(eps, sizes):
    """Zero weights and moments and betas of 0, as of a bias before its first step: v = d^2,
    w = -lr m / (sqrt(v) + eps), a rounding for each operation, bit for bit."""
    _, g, _, _, _ = _adam_state(sizes, torch.float32, "padded", None, 18)
    w, m, v = ([torch.zeros_like(x) for x in g] for _ in range(3))
    O.AdamWStep(w, g, m, v)(3e-3, (0.0, 0.0), eps, 0.0)
    for i, x in enumerate(g):
        d = x.cpu().numpy()
        square = d * d
        with np.errstate(invalid="ignore"):
            quotient = d / (np.sqrt(square) + np.float32(eps))
        assert np.array_equal(m[i].cpu().numpy(), d) and np.array_equal(v[i].cpu().numpy(), square)
        assert np.array_equal(w[i].cpu().numpy(), -(np.float32(3e-3) * quotient), equal_nan=True)


@pytest.mark.gpu
def test_refusals_of_a_plan_in_use():
    w, g, m, v, _ = _adam_state([300], torch.float32, "padded", None, 14)
    clip, step = O.GradClipper(g), O.AdamWStep(w, g, m, v)
    for fn in (lambda: clip.clip_(0.0), lambda: clip.clip_(math.nan), lambda: clip.clip_(-1.0),
               lambda: clip.norm(grad_scale=0.0), lambda: clip.norm(max_norm=-1.0),
               lambda: step(-1.0), lambda: step(math.nan), lambda: step(1e-3, (1.0, 0.9)),
               lambda: step(1e-3, (0.9, -0.1)), lambda: step(1e-3, eps=-1.0), lambda: step(1e-3, grad_scale=0.0)):
        with pytest.raises(T.TulaError) as e:
            fn()
        assert e.value.code == T.TULA_ERR_ARG
    hp = O.tula_adamw_hparams()
    O._lib().tula_adamw_default_hparams(ctypes.byref(hp))
    hp.steps = step.steps.data_ptr()
    assert O._lib().tula_adamw_step(clip._plan.handle, ctypes.byref(hp), None) == T.TULA_ERR_ARG  # no weights
    with pytest.raises(ValueError):
        O.AdamWStep(w, g, m, [torch.zeros(299, device="cuda")])
    with pytest.raises(ValueError):
        O.AdamWStep(w, g, m, v + v)
    with pytest.raises(TypeError):
        O.AdamWStep([w[0].double()], g, m, v)
    with pytest.raises(TypeError):
        O.GradClipper([torch.zeros(4, 4, device="cuda").t()[1:]])
    assert step.steps.tolist() == [0, 0]


@pytest.mark.gpu
def test_graph_and_another_stream():
    """A clip and a step captured together replay as they run, on a stream of their own."""
    def fresh():
        w, g, m, v, c = _adam_state([5000, 100], torch.bfloat16, "padded", torch.bfloat16, 15)
        return w, g, m, v, c, O.AdamWStep(w, g, m, v, copies=c, max_norm=0.5, skip_nonfinite=True)

    a, b = fresh(), fresh()
    for _ in range(3):
        a[-1](1e-3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b[-1](1e-3)
    with torch.cuda.stream(side):
        for _ in range(3):
            graph.replay()
    side.synchronize()
    assert b[-1].steps.tolist() == [3, 0] == a[-1].steps.tolist()
    for r in range(5):
        assert all(torch.equal(x, y) for x, y in zip(a[r], b[r]))


@pytest.mark.gpu
def test_a_plans_memory_waits_for_calls_on_other_streams():
    """A plan that is dropped right after a call on another stream: its workspace does not go to the
    next allocation while that call may be running."""
    g = [torch.full((5000,), 0.5, device="cuda") for _ in range(40)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    clip = O.GradClipper(g)
    at, size = clip._plan.workspace.data_ptr(), clip._plan.workspace.numel()
    at_record = clip.record.data_ptr()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    clip.clip_(1.0, side)
    del clip
    taken = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(32)]
    taken += [torch.empty(4, device="cuda") for _ in range(32)]
    assert not side.query()
    assert all(not at <= t.data_ptr() < at + size and t.data_ptr() != at_record for t in taken)
    torch.cuda.synchronize()
    norm = 0.5 * (40 * 5000) ** 0.5
    for t in g:
        torch.testing.assert_close(t, torch.full_like(t, 0.5 / norm), rtol=1e-5, atol=0)
