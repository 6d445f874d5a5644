"""Muon's updates where more can go wrong than elsewhere: matrices of a batch against themselves alone, and what
follows below."""
import pytest
import torch

from paper_2603_18112_gb300 import optim as O
from test_train_muon import SHAPES, _near, _off, _size, _updates


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
