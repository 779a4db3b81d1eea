"""What the linear operators do with tensors that autograd follows, on the CPU: the refusal comes before anything else."""

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2609_33437_gb300 import linear as L


def _calls(a, b):
    """Every operator, with `a` in each of its places in turn."""
    p = L.Packed8(torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8))
    return {"linear x": lambda: L.linear(a, b), "linear w": lambda: L.linear(b, a), "linear bias": lambda: L.linear(b, b, bias=a),
            "linear residual": lambda: L.linear(b, b, residual=a), "grad_input dy": lambda: L.linear_grad_input(a, b),
            "grad_input w": lambda: L.linear_grad_input(b, a), "grad_weight dy": lambda: L.linear_grad_weight(a, b),
            "grad_weight x": lambda: L.linear_grad_weight(b, a), "grad_weight 8 bits": lambda: L.linear_grad_weight(a, p),
            "pack8": lambda: L.pack8(a), "act_grad8": lambda: L.act_grad8(a, p, "silu")}


NAMES = list(_calls(None, None))


@pytest.mark.parametrize("name", NAMES)
def test_a_gradient_that_would_be_lost_is_refused(name):
    calls = _calls(torch.zeros(4, 8, requires_grad=True), torch.zeros(4, 8))
    with pytest.raises(ValueError, match="no_grad"):
        calls[name]()
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA|must be"):
        calls[name]()  # nobody asks for a gradient: the next thing to object to
    calls = _calls(torch.zeros(4, 8, requires_grad=True).detach(), torch.zeros(4, 8))
    with pytest.raises(ValueError, match="CUDA|must be"):
        calls[name]()


@pytest.mark.parametrize("name", NAMES)
def test_a_tangent_that_would_be_lost_is_refused(name):
    with forward_ad.dual_level(), torch.no_grad():
        calls = _calls(forward_ad.make_dual(torch.zeros(4, 8), torch.ones(4, 8)), torch.zeros(4, 8))
        with pytest.raises(ValueError, match="tangent"):
            calls[name]()


@pytest.mark.parametrize("grad", [True, False])
def test_layers_refuse_tangents(grad):
    for m in (L.Linear8(8, 8, act="silu"), L.Mlp8(8, 16)):
        with forward_ad.dual_level(), torch.set_grad_enabled(grad):
            x = forward_ad.make_dual(torch.zeros(4, 8), torch.ones(4, 8))
            with pytest.raises((ValueError, NotImplementedError), match="tangent|jvp|CUDA" if grad else "tangent"):
                m(x)
