"""The layers' own logic (Linear8, Mlp8) on the CPU: the operators they call are stood in for by torch, so what is tested
is what they save, which gradients they ask for, and what they refuse."""

import pytest
import torch

import _linear_ref as R
from paper_2609_33437_gb300 import linear as L


def _linear(x, w, bias=None, act="none", residual=None, save=False, out=None, stream=None):
    L._no_graph(x, w, bias, residual)
    h = x @ w.T + (bias if bias is not None else 0)
    y = R.act(act, h) + (residual if residual is not None else 0)
    return (y, _pack8(h.detach())) if save else y


def _pack8(x, stream=None):
    L._no_graph(x)
    q, e = R.pack(x.reshape(-1, x.shape[-1]))
    return L.Packed8(q.view(x.shape), e.view(*x.shape[:-1], -1))


def _value(p, dtype):
    return R.unpack(p.q.reshape(-1, p.shape[-1]), p.e.reshape(-1, p.e.shape[-1])).view(p.shape).to(dtype)


def _grad_input(dy, w, act="none", saved=None, out=None, stream=None):
    L._no_graph(dy, w)
    return dy @ w * (R.slope(act, _value(saved, dy.dtype)) if saved is not None else 1)


def _grad_weight(dy, x, act="none", bias=False, out=None, bias_out=None, accumulate=False, stream=None):
    L._no_graph(dy, x if isinstance(x, torch.Tensor) else None)
    v = R.act(act, _value(x, dy.dtype)) if isinstance(x, L.Packed8) else x
    dy = dy.reshape(-1, dy.shape[-1])
    return dy.T @ v.reshape(dy.shape[0], -1), dy.sum(0) if bias else None


def _act_grad8(dy, saved, act, out=None, stream=None):
    L._no_graph(dy)
    return dy * R.slope(act, _value(saved, dy.dtype))


@pytest.fixture(autouse=True)
def _stand_ins(monkeypatch):
    for name, f in (("linear", _linear), ("linear_grad_input", _grad_input), ("linear_grad_weight", _grad_weight),
                    ("pack8", _pack8), ("act_grad8", _act_grad8)):
        monkeypatch.setattr(L, name, f)


def _layers(act):
    torch.manual_seed(0)
    return L.Linear8(40, 40, act=act, dtype=torch.float64), L.Mlp8(40, 64, act=act, dtype=torch.float64)


@pytest.mark.parametrize("act", R.ACTS)
def test_first_derivatives_through_the_stand_ins(act):
    """The stand-ins make the layers torch's own, up to the 8 bits: a sanity check of what follows."""
    for m in _layers(act):
        x = torch.randn(6, 40, dtype=torch.float64, requires_grad=True)
        m(x, residual=x).square().sum().backward()
        assert x.grad.shape == x.shape and all(p.grad.shape == p.shape for p in m.parameters())


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("by", ["backward", "grad of the weight", "grad of the input"])
@pytest.mark.parametrize("power", [1, 2])
def test_a_second_derivative_is_refused(act, by, power):
    """Their backward pass builds no graph. A gradient penalty would otherwise leave out every term that goes through a
    layer, without a word, where another path (here the residual) carries a graph; whether or not the incoming gradient
    depends on anything (power 1: it does not), and by whichever tensor the derivative is taken."""
    for m in _layers(act):
        x = torch.randn(6, 40, dtype=torch.float64, requires_grad=True)
        loss = m(x, residual=x * x).pow(power).sum()
        g, = torch.autograd.grad(loss, x, create_graph=True)
        total = g.square().sum() + loss
        with pytest.raises(RuntimeError, match="first derivatives only"):
            if by == "backward":
                total.backward()
            else:
                torch.autograd.grad(total, next(m.parameters()) if by == "grad of the weight" else x)


def test_a_second_derivative_beside_the_layer_is_right():
    """The residual's gradient is the incoming one, whose own derivatives are first derivatives of the layer: nothing is
    refused there. Whole numbers up to 127 are exact in 8 bits, so the values are torch's."""
    torch.manual_seed(1)
    m = L.Linear8(40, 40, dtype=torch.float64)
    x = torch.randint(-127, 128, (6, 40)).double()
    grads = []
    for f in (lambda r: m(x, residual=r), lambda r: torch.nn.functional.linear(x, m.weight, m.bias) + r):
        r = torch.ones(6, 40, dtype=torch.float64, requires_grad=True)
        g, = torch.autograd.grad(f(r).square().sum(), r, create_graph=True)
        grads.append(torch.autograd.grad(g.square().sum(), (m.weight, m.bias, r)))
    for a, b in zip(*grads):
        assert torch.allclose(a, b, rtol=1e-12, atol=0)


def test_a_first_derivative_with_a_graph_is_the_one_without():
    for m in _layers("gelu"):
        x = torch.randn(6, 40, dtype=torch.float64, requires_grad=True)
        want = [x, *m.parameters()]
        loss = m(x, residual=x).square().sum()
        a = torch.autograd.grad(loss, want, retain_graph=True)
        b = torch.autograd.grad(loss, want, create_graph=True)
        assert all(torch.equal(s, t) for s, t in zip(a, b))
