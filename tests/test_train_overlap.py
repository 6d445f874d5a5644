"""Buffers of a Muon plan that share memory: refused on the host wherever one of them is written."""
import ctypes

import pytest
import torch

from paper_2603_18112_gb300 import optim as O
from paper_2603_18112_gb300.tula_ags import TulaError

ARG, CUDA = -1, -3
AT = 1 << 20


def _create(matrices):
    """tula_muon_plan_create's answer for matrices of 4 x 8 (w, m, g, gtype, copy), none of them real memory, nor is
    the workspace: what is not refused fails for want of a GPU."""
    w, m, g, t, c = zip(*matrices)
    n = len(matrices)
    arrays = [(ctypes.c_int64 * n)(*[4] * n), (ctypes.c_int64 * n)(*[8] * n), (ctypes.c_void_p * n)(*g), (ctypes.c_int * n)(*t),
              (ctypes.c_void_p * n)(*w), (ctypes.c_void_p * n)(*m), (ctypes.c_void_p * n)(*c), (ctypes.c_int * n)(*[1] * n)]
    d = O.tula_muon_matrices(n, *(ctypes.cast(a, ctypes.c_void_p) for a in arrays))
    plan = ctypes.c_void_p()
    return O._lib().tula_muon_plan_create(ctypes.byref(d), ctypes.c_void_p(1 << 30), 1 << 20, None, ctypes.byref(plan))


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses of no memory: only where no GPU is")
def test_ranges():
    def one(at, **kw):  # 128 bytes of w and of m, 128 of g in fp32, 64 of a copy, back to back
        return list((dict(w=at, m=at + 128, g=at + 256, t=0, c=at + 384) | kw).values())

    a, b = one(AT), one(AT + 448)
    assert _create([a]) == _create([a, b]) == _create([b, a]) == CUDA
    for role in ("w", "m", "c"):  # of the second matrix within each of the first one's buffers, and at their ends
        size = 64 if role == "c" else 128
        for first in (AT, AT + 128, AT + 256, AT + 384):
            length = 64 if first == AT + 384 else 128
            for at in (first - size + 4, first, first + 4, first + length - 4):
                assert _create([a, one(AT + 4096, **{role: at})]) == ARG, (role, first, at)
    assert _create([a, one(AT + 4096, w=AT - 128)]) == CUDA  # next to each other
    # gradients: with written buffers of others or their own momentum, not; with each other and their own end, yes
    for at in (AT, AT + 132, AT + 444):
        assert _create([a, one(AT + 4096, g=at)]) == ARG
    assert _create([one(AT, g=AT + 128)]) == ARG
    assert _create([a, one(AT + 4096, g=AT + 256)]) == _create([a, one(AT + 4096, g=AT + 300, t=1)]) == CUDA
    assert _create([one(AT, g=AT)]) == _create([one(AT, g=AT + 384, t=1)]) == CUDA
    assert _create([one(AT, g=AT + 384)]) == ARG  # fp32, beyond the bf16 copy
    assert _create([one(AT, g=AT + 64)]) == ARG


@pytest.mark.gpu
def test_overlapping_views():
    flat = torch.zeros(200, device="cuda")
    g, m = [torch.ones(4, 8, device="cuda") for _ in range(2)], [torch.zeros(4, 8, device="cuda") for _ in range(2)]
    with pytest.raises(TulaError):
        O.MuonStep([flat[:32].view(4, 8), flat[31:63].view(4, 8)], g, m)
    O.MuonStep([flat[:32].view(4, 8), flat[32:64].view(4, 8)], [g[0], g[0]], m)(1e-3)
    # weights that are their own gradients (of half their squares): as with a copy of them
    w = torch.randn(4, 8, device="cuda")
    w2, g2 = w.clone(), w.clone()
    O.MuonStep([w], [w], [torch.zeros_like(w)])(1e-2)
    O.MuonStep([w2], [g2], [torch.zeros_like(w)])(1e-2)
    assert torch.equal(w, w2)
