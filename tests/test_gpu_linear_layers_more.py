"""The layers (Linear8, Mlp8) on the GPU beside their first derivatives: graphs of gradients, and the inputs that
torch.nn.Linear takes."""

import pytest
import torch

from paper_2609_33437_gb300 import linear as L

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


def _layers(dtype, act="silu"):
    torch.manual_seed(0)
    return (L.Linear8(96, 96, act=act, device="cuda", dtype=dtype), L.Mlp8(96, 160, act=act, device="cuda", dtype=dtype))


def _input(*shape, dtype, grad=True):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype).requires_grad_(grad)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_gradients_with_a_graph(dtype):
    """Asked for with create_graph they are the same gradients, and going through them raises."""
    for m in _layers(dtype):
        x = _input(30, 96, dtype=dtype)
        want = [x, *m.parameters()]
        for power in (1, 2):
            loss = m(x, residual=x * x).float().pow(power).sum()
            a = torch.autograd.grad(loss, want, retain_graph=True)
            b = torch.autograd.grad(loss, want, create_graph=True)
            assert all(torch.equal(s, t) for s, t in zip(a, b))
            with pytest.raises(RuntimeError, match="first derivatives only"):
                (b[0].float().square().sum() + loss).backward()


def test_operators_refuse_what_requires_a_gradient():
    m, _ = _layers(F32)
    x = _input(30, 96, dtype=F32, grad=False)
    with pytest.raises(ValueError, match="no_grad"):
        L.linear(x, m.weight, m.bias)
    with torch.no_grad():
        y = L.linear(x, m.weight, m.bias)
    assert torch.equal(y, L.linear(x, m.weight.detach(), m.bias.detach()))
