"""The layers made of the linear operators (Linear8, Mlp8): their outputs and gradients against the same layers in 64
bits by autograd, frozen parts, strided and broadcast gradients, the periodic schedule around them, and what they hold
between the passes.

Tolerance of a gradient: a value saved in 8 bits is off by at most half a step, and a step is at most 2 / 127.5 of its
group's largest magnitude; for a uniform error that is 0.0046 of it in the root mean square, and for normal values,
whose largest of 32 is about 2.1 of their own, 0.0095 of those. An input saved so brings 0.0095 into dW; a
pre-activation brings that times |act''| (up to about 1) over act' (about 0.6 in the mean square) into dh, 0.016. Both, and
a few roundings to bf16 (0.002 each): under 0.03 in the relative 2-norm. Outputs hold no 8-bit value: roundings alone.

That holds where act' is smooth. relu's jumps: a positive pre-activation under half a step reads back as 0 and has the
slope 0. Half a step is at most 2.1 / 127.5 = 0.0165 of a normal group's deviation, whose density there is 0.4: 0.0066 of
the values, out of the half that has slope 1. A relative 2-norm of sqrt(0.0066 / 0.5) = 0.115, and 0.03 as above."""

import importlib.util
import os

import pytest
import torch

import _linear_ref as R
from paper_2609_33437_gb300 import linear as L

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
GRAD, GRAD_RELU = 0.03, 0.145


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


def _rel(got, ref):
    return float((got.double() - ref.double()).norm() / ref.double().norm())


def _leaf(seed, *shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype).requires_grad_(True)


def _wide(t):
    return t.detach().double().requires_grad_(True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("shape", [(300,), (4, 77), (2, 3, 5)])
def test_mlp8_against_autograd_in_64_bits(dtype, act, shape):
    torch.manual_seed(0)
    m = L.Mlp8(96, 256, act=act, device="cuda", dtype=dtype)
    x, r, g = (_leaf(k, *shape, 96, dtype=dtype) for k in (1, 2, 3))
    y = m(x, residual=r)
    y.backward(g.detach())
    xd, rd = _wide(x), _wide(r)
    w1, b1, w2, b2 = (_wide(p) for p in (m.fc1.weight, m.fc1.bias, m.fc2.weight, m.fc2.bias))
    ref = R.act(act, xd @ w1.T + b1) @ w2.T + b2 + rd
    ref.backward(g.detach().double())
    assert _rel(y, ref) < (0.01 if dtype == BF else 1e-5)
    assert torch.equal(r.grad, g.detach())
    for name, got, want in (("x", x, xd), ("w1", m.fc1.weight, w1), ("b1", m.fc1.bias, b1), ("w2", m.fc2.weight, w2),
                            ("b2", m.fc2.bias, b2)):
        assert got.grad.shape == got.shape and got.grad.dtype == dtype
        assert _rel(got.grad, want.grad) < (GRAD_RELU if act == "relu" else GRAD), name


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("bias", [True, False])
def test_linear8_against_autograd_in_64_bits(dtype, act, bias):
    torch.manual_seed(0)
    m = L.Linear8(120, 72, bias=bias, act=act, device="cuda", dtype=dtype)
    x, r, g = _leaf(1, 210, 120, dtype=dtype), _leaf(2, 210, 72, dtype=dtype), _leaf(3, 210, 72, dtype=dtype)
    y = m(x, residual=r)
    y.backward(g.detach())
    xd, rd, w = _wide(x), _wide(r), _wide(m.weight)
    b = _wide(m.bias) if bias else None
    ref = R.act(act, xd @ w.T + (b if bias else 0.0)) + rd
    ref.backward(g.detach().double())
    assert _rel(y, ref) < (0.01 if dtype == BF else 1e-5)
    assert torch.equal(r.grad, g.detach())
    assert _rel(x.grad, xd.grad) < GRAD and _rel(m.weight.grad, w.grad) < GRAD
    if bias:
        assert _rel(m.bias.grad, b.grad) < GRAD


def test_frozen_parts_and_gradients_of_any_stride():
    m = L.Mlp8(64, 128, act="gelu", device="cuda", dtype=BF)
    x = _leaf(1, 50, 64, dtype=BF)
    m(x).sum().backward()  # a gradient that is broadcast from one number
    full = [p.grad.clone() for p in m.parameters()] + [x.grad.clone()]
    # a gradient that arrives transposed is the same gradient
    for p in (*m.parameters(), x):
        p.grad = None
    m(x).T.contiguous().T.mul(1.0).sum().backward()
    for p, ref in zip((*m.parameters(), x), full):
        assert torch.equal(p.grad, ref)
    for frozen in range(4):
        for k, p in enumerate(m.parameters()):
            p.grad = None
            p.requires_grad_(k != frozen)
        y = x.detach()
        m(y).sum().backward()
        for k, p in enumerate(m.parameters()):
            if k == frozen:
                assert p.grad is None
            else:
                assert torch.equal(p.grad, full[k]), (frozen, k)
    # only the first bias learns
    for k, p in enumerate(m.parameters()):
        p.grad = None
        p.requires_grad_(k == 1)
    m(x.detach()).sum().backward()
    assert torch.equal(m.fc1.bias.grad, full[1])
    # nothing learns: nothing is saved, and the result is the same
    with torch.no_grad():
        y = m(x)
    m.requires_grad_(True)
    assert torch.equal(y, m(x).detach())


def test_what_a_layer_holds_between_the_passes():
    """x and the pre-activation, 33 / 32 bytes per element each, and no more of them."""
    rows, width, hidden = 4096, 512, 2048
    m = L.Mlp8(width, hidden, act="gelu", device="cuda", dtype=BF)
    x = torch.randn(rows, width, device="cuda", dtype=BF)
    m(x)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = m(x)
    held = torch.cuda.memory_allocated() - before - y.numel() * 2
    eight = rows * (width + hidden) * 33 // 32
    assert eight <= held <= eight + 16 * 1024
    del y
    p = L.pack8(x)
    assert p.nbytes() == rows * width * 33 // 32


def test_gradients_add_up_over_micro_batches():
    m = L.Linear8(64, 48, act="silu", device="cuda", dtype=F32)
    x = torch.randn(96, 64, device="cuda")
    m(x).square().mean().mul(2).backward()
    whole = [p.grad.clone() for p in m.parameters()]
    for p in m.parameters():
        p.grad = None
    for part in x.chunk(2):
        m(part).square().mean().backward()
    for p, ref in zip(m.parameters(), whole):
        # the same sums in another order: eight roundings of 2^-24 of the magnitudes would be 5e-7
        assert _rel(p.grad, ref) < 1e-5


@pytest.mark.parametrize("dtype", [F32, BF])
def test_example_trains_under_the_periodic_schedule(dtype):
    """The example's network learns its task: simulated-loss steps read theta~ through the operators."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_mlp8.py")
    spec = importlib.util.spec_from_file_location("train_mlp8", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    losses = ex.train(steps=60, width=128, hidden=320, blocks=2, batch=514, dtype=dtype, lr=2e-3)
    assert all(v == v and v < 20 for v in losses)
    first, last = sum(losses[:8]) / 8, sum(losses[-8:]) / 8
    assert last < 0.7 * first, (first, last)
    assert ex.train(steps=8, width=128, hidden=320, blocks=2, batch=514, dtype=dtype, lr=2e-3) == losses[:8]
