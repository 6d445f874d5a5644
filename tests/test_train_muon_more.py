"""Muon's updates where more can go wrong than elsewhere: matrices of a batch against themselves alone, and what
follows below."""
import pytest
import torch

from paper_2603_18112_gb300 import optim as O
from test_train_muon import SHAPES, _updates


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
