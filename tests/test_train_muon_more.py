"""Muon's updates where more can go wrong than elsewhere: matrices of a batch against themselves alone, and what
follows below."""
import pytest
import torch

from paper_2603_18112_gb300 import optim as O
from test_train_muon import SHAPES, _near, _off, _size, _updates, ns64


@pytest.mark.gpu
@pytest.mark.parametrize("n,rows,cols", [s for s in SHAPES if s[0] > 1])
def test_a_matrix_of_a_batch_by_itself(n, rows, cols):
    """The same sums in other blocks, or other loads: a rounding to fp16 may fall on the other side here and there."""
    x = _updates(n, rows, cols, rows + cols + 1)
    got = O.orthogonalize(x, dtype=torch.float16)
    for k in {0, n // 2, n - 1}:
        alone = O.orthogonalize(x[k], dtype=torch.float16).double()
        assert float((got[k].double() - alone).norm()) <= 2.0 ** -9 * float(alone.norm())
    assert O.tula_muon_error() == 0


def test_workspace_of_long_sides():
    """A's sums go by 65536: as many buffers for it, and one for B."""
    for rows, cols in ((65536, 70), (65537, 70), (70, 1 << 20), (200000, 300), (1 << 20, 1)):
        n = min(rows, cols)
        x, a, parts = -(-rows // 128) * -(-cols // 64), -(-n // 128) * -(-n // 64), -(-max(rows, cols) // 65536)
        assert _size([rows], [cols]) == (0, 256 + -(-8 * x // 256) * 256 + (2 * x + (parts + 1) * a) * 16384)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1 << 20, 70), (70, 1 << 20), (1 << 20, 1), (1, 1 << 20), (1 << 17, 1024), (65537, 130), (130, 200000)])
def test_longest_sides(rows, cols):
    """Sums beyond what is taken at a time."""
    x = _updates(1, rows, cols, 6)[0]
    got = O.orthogonalize(x, dtype=torch.float16)
    _near(got, *_off(x, 5), torch.float16)
    assert O.tula_muon_error() == 0


@pytest.mark.gpu
def test_long_sides_among_others():
    """Of several shapes, several matrices each, in a batch and in a plan."""
    x = _updates(3, 150000, 90, 7)
    got = O.orthogonalize(x, dtype=torch.float16)
    for u, o in zip(x, got):
        _near(o, *_off(u, 5), torch.float16)
    assert torch.equal(got, O.orthogonalize(x, dtype=torch.float16))
    shapes = [(150000, 90), (90, 140008), (300, 200), (150000, 90), (65536, 16), (90, 140001)]
    g = [_updates(1, r, c, 8 + i)[0] for i, (r, c) in enumerate(shapes)]
    w, m = [torch.zeros_like(t) for t in g], [torch.zeros_like(t) for t in g]
    record = torch.tensor([1.0, 1.0, 0.0, 0.0], device="cuda")  # left out
    step = O.MuonStep(w, g, m, nesterov=False, scale="aspect")
    step(1.0, 0.0, record=record)
    assert not any(bool(t.any()) for t in (*w, *m))
    step(1.0, 0.0)
    for u, t in zip(g, w):
        s = max(1.0, u.shape[0] / u.shape[1]) ** 0.5
        want, off, most = _off(u, 5)
        d = (t.double() / -s - want).abs()
        assert float(d.norm()) <= off and float(d.max()) <= most
    assert O.tula_muon_error() == 0


# --------------------------------------------------------------------------------------------
# How far off an update is, apart from how it is computed
# --------------------------------------------------------------------------------------------

SPECTRA = {
    "flat": lambda k, n: k * 0 + 1, "falling by e^3": lambda k, n: torch.exp(-3 * k / n), "1/k": lambda k, n: 1 / (k + 1),
    "1/k^2": lambda k, n: 1 / (k + 1) ** 2, "to 1e-4": lambda k, n: 10 ** (-4 * k / n),
    "four of 20": lambda k, n: torch.where(k < 4, 20.0, 1.0), "four of 1000": lambda k, n: torch.where(k < 4, 1000.0, 1.0),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", SPECTRA)
@pytest.mark.parametrize("rows,cols", [(64, 576), (256, 256), (700, 300)])
def test_no_further_off_than_a_matrix_in_bf16(rows, cols, name):
    """However its singular values lie, a matrix's update is less off than a rounding of the matrix itself to bf16
    moves it.  fp16's roundings are a quarter of bf16's; five steps have three each, of which the later ones are
    grown by fewer steps: sqrt(15) / 4, about one, if none is grown, less for the rest; half as much again for
    chance."""
    n = min(rows, cols)
    gen = torch.Generator().manual_seed(rows)
    q, p = (torch.linalg.qr(torch.randn(k, n, generator=gen, dtype=torch.float64))[0] for k in (rows, cols))
    x = (q * SPECTRA[name](torch.arange(n, dtype=torch.float64), n) @ p.t()).float().cuda()
    want = ns64(x)
    moved = float((ns64(x.bfloat16()) - want).norm())
    got = O.orthogonalize(x, dtype=torch.float16)
    off = float((got.double() - want).norm()) - 2.0 ** -11 * float(want.norm())  # (but for the output's own rounding)
    assert off <= 1.5 * moved, (off / moved, off / float(want.norm()))


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [1, 2, 3, 4, 5, 6, 8, 16])
def test_narrow_matrices(cols):
    """A few columns: A and B have a few elements, whose roundings do not average.  Roundings that all fall the worst
    way would be 0.8 to 3.6e-2 (the steps' slope times what there is, and a 2^-11 of A, of B and of X in each);
    1e-2 is what is promised, 4e-3 from 8 columns on."""
    for rows in (100, 874, 3000):
        x = torch.randn(60, rows, cols, generator=torch.Generator().manual_seed(rows)).cuda()
        got = O.orthogonalize(x, dtype=torch.float16)
        for u, o in zip(x, got):
            want = ns64(u)
            assert float((o.double() - want).norm()) <= (1e-2 if cols < 8 else 4e-3) * float(want.norm())
        # and each across, as well
        assert float((O.orthogonalize(x.transpose(1, 2), dtype=torch.float16).transpose(1, 2).double() - got.double()).norm()) <= \
            2e-2 * float(got.double().norm())
