"""Forward-mode differentiation: refused, never an output without its tangent.  On the CPU, the library's calls left
out."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2603_18112_gb300 import fp8, mx, norm


def _dual(t):
    return forward_ad.make_dual(t, torch.ones_like(t))


@pytest.fixture
def no_library(monkeypatch):
    for module in (fp8, norm):
        monkeypatch.setattr(module, "_call", lambda *args: None)
        monkeypatch.setattr(module, "_on_gpu", lambda *tensors: 0)


@pytest.mark.parametrize("recorded", [False, True])
def test_layer_norm(no_library, recorded):
    x, w, b = torch.randn(5, 8), torch.ones(8), torch.zeros(8)
    with forward_ad.dual_level():
        for args in ((_dual(x), w, b), (x, _dual(w), b), (x, w, _dual(b)), (_dual(x), None, None), (x, w.clone().requires_grad_(), _dual(b))):
            with torch.set_grad_enabled(recorded), pytest.raises(NotImplementedError):
                norm.layer_norm(*args)
        assert norm.layer_norm(x, w, b).shape == x.shape  # a level alone is no reason
        leaf = x.clone().requires_grad_()
        y = norm.layer_norm(leaf, w, b)
        with pytest.raises(NotImplementedError):
            torch.autograd.grad(y, leaf, _dual(torch.ones_like(y)), retain_graph=True)
        torch.autograd.grad(y, leaf, torch.ones_like(y))
    norm.layer_norm(x, w, b)


@pytest.mark.parametrize("recorded", [False, True])
def test_8_bit_layer(no_library, recorded):
    x, w = torch.randn(3, 5, 8), torch.ones(4, 8)
    with forward_ad.dual_level():
        for args in ((_dual(x), w), (x, _dual(w)), (_dual(x[0]), w), (x, _dual(w.clone().requires_grad_()))):
            with torch.set_grad_enabled(recorded), pytest.raises(NotImplementedError):
                fp8.linear(*args)
        assert fp8.linear(x, w).shape == (3, 5, 4)
        leaf = w.clone().requires_grad_()
        y = fp8.linear(x, leaf)
        with pytest.raises(NotImplementedError):
            torch.autograd.grad(y, leaf, _dual(torch.ones_like(y)), retain_graph=True)
        torch.autograd.grad(y, leaf, torch.ones_like(y))
    fp8.linear(x, w)


def test_gradients_of_the_mxfp4_layer():
    """(Its output goes through torch's function always, which refuses dual tensors.)"""
    dy = torch.ones(5, 4)

    class Context:
        saved_tensors, end, device = (torch.zeros(0, dtype=torch.uint8),), 0, torch.device("cpu")
        sizes, needs_input_grad = (5, 4, 8), (True, True, False)

    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError):
            mx._Linear.backward(Context(), _dual(dy))
        with pytest.raises(TypeError, match="GPU"):  # goes on
            mx._Linear.backward(Context(), dy)
