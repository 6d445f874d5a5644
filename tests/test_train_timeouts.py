"""Failure detection without a fault: in each operator a bounded wait that runs out is reported once, by that
operator's error word alone, and calls go on."""
import pytest
import torch

from paper_2603_18112_gb300 import fp8, mx, norm
from paper_2603_18112_gb300 import optim as O

WORDS = {"fp8": (fp8.tula_fp8_check_wait_timeout, fp8.tula_fp8_error), "norm": (norm.tula_layer_norm_check_wait_timeout, norm.tula_layer_norm_error),
         "muon": (O.tula_muon_check_wait_timeout, O.tula_muon_error)}


@pytest.mark.gpu
@pytest.mark.parametrize("name", WORDS)
def test_a_wait_that_runs_out_is_reported(name):
    check, _ = WORDS[name]
    x = torch.randn(200, 300, generator=torch.Generator().manual_seed(1)).cuda()

    def results():
        return fp8.linear(x, x), norm.layer_norm(x), O.orthogonalize(x)

    want = results()
    assert all(error() == 0 for _, error in WORDS.values())
    check()
    got = results()
    assert {n: error() for n, (_, error) in WORDS.items()} == {n: int(n == name) for n in WORDS}
    assert mx.tula_mx_error() == 0 and all(error() == 0 for _, error in WORDS.values())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
