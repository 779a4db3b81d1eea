"""The layers (Linear8, Mlp8) on the GPU beside their first derivatives: graphs of gradients, and the inputs that
torch.nn.Linear takes."""

import importlib.util
import os

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


def _same_as_contiguous(m, x, residual=None):
    """Outputs and gradients of inputs of any stride are those of their contiguous copies."""
    res = []
    for f in (lambda t: t, lambda t: t.contiguous()):
        for p in m.parameters():
            p.grad = None
        leaf = x.detach().requires_grad_(True)  # keeps the strides
        y = m(f(leaf), residual=None if residual is None else f(residual))
        y.float().square().sum().backward()
        with torch.no_grad():
            z = m(f(x.detach()), residual=None if residual is None else f(residual))
        res.append([y, z, leaf.grad, *(p.grad for p in m.parameters())])
    assert res[0][0].shape == (*x.shape[:-1], 96)
    for a, b in zip(*res):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_inputs_of_any_stride(dtype):
    for m in _layers(dtype):
        base = _input(12, 10, 96, dtype=dtype, grad=False)
        _same_as_contiguous(m, base.transpose(0, 1))                             # sequence first
        _same_as_contiguous(m, _input(96, 50, dtype=dtype, grad=False).T)        # a transposed view
        _same_as_contiguous(m, _input(20, 192, dtype=dtype, grad=False)[:, ::2])  # every second column
        _same_as_contiguous(m, _input(96, dtype=dtype, grad=False).expand(7, 96))  # one row, broadcast
        _same_as_contiguous(m, base[:, :4], residual=_input(96, 4, 12, dtype=dtype, grad=False).permute(2, 1, 0))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_weights_of_any_stride(dtype):
    """As a parametrisation or a tied, transposed weight leaves them."""
    for m in _layers(dtype):
        other = type(m)(96, 96 if isinstance(m, L.Linear8) else 160, act=m.act, device="cuda", dtype=dtype)
        for p, q in zip(m.parameters(), other.parameters()):
            q.data = p.data.T.contiguous().T if p.dim() == 2 else torch.stack([p.data, p.data], 1)[:, 0]
            assert not q.is_contiguous()
        x = _input(40, 96, dtype=dtype)
        for k in (m, other):
            k(x).float().square().sum().backward()
        for p, q in zip(m.parameters(), other.parameters()):
            assert torch.equal(p.grad, q.grad)


@pytest.mark.parametrize("shape", [(0, 96), (3, 0, 96), (0, 3, 96)])
def test_batches_of_nothing(shape):
    for m in _layers(BF):
        x = _input(*shape, dtype=BF)
        y = m(x, residual=x)
        assert y.shape == shape
        y.sum().backward()
        assert x.grad.shape == shape and all(not p.grad.any() for p in m.parameters())


@pytest.mark.parametrize("grad", [True, False])
def test_autocast(grad):
    """fp32 weights under autocast to bf16 are the bf16 layer's, for inputs of either type; gradients come in the tensors' own
    types; a residual of 32 bits keeps them and the result's type, as beside torch.nn.Linear."""
    for m, low in zip(_layers(F32), _layers(BF)):
        low.load_state_dict({k: v.to(BF) for k, v in m.state_dict().items()})
        plain = torch.nn.Linear(96, 96, device="cuda")
        for dtype in (F32, BF):
            x, y = _input(40, 96, dtype=dtype), _input(40, 96, dtype=BF)
            wide = torch.randn(40, 96, device="cuda")
            with torch.set_grad_enabled(grad):
                want = low(y, residual=y)
                with torch.autocast("cuda", torch.bfloat16):
                    got, bare = m(x, residual=x.to(BF)), m(x)
                    sums = m(x, residual=wide)
                    assert sums.dtype is (plain(x) + wide).dtype is F32
                assert got.dtype is bare.dtype is BF and torch.equal(got, want)
                assert torch.equal(sums, bare + wide)
            if grad:
                for net, z, t in ((m, got, x), (low, want, y)):
                    for p in net.parameters():
                        p.grad = None
                    z.float().square().sum().backward()
                for p, q in zip((x, *m.parameters()), (y, *low.parameters())):
                    assert p.grad.dtype is p.dtype and torch.equal(p.grad.to(BF), q.grad)
        with torch.autocast("cuda", torch.float16), pytest.raises(TypeError):
            m(x)  # a type that the operators do not have
        with torch.autocast("cuda", enabled=False):
            assert m(x.detach().float()).dtype is F32


def test_the_example_does_not_keep_unfinished_results(monkeypatch):
    """A training loop ends with an error, not with losses, where the products' flag is up."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_mlp8.py")
    spec = importlib.util.spec_from_file_location("train_mlp8", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    kw = dict(steps=2, width=64, hidden=96, blocks=1, batch=64)
    assert len(ex.train(**kw)) == 2
    monkeypatch.setattr(ex.L, "poll_errors", lambda stream=None: 1)
    with pytest.raises(RuntimeError, match="unfinished"):
        ex.train(**kw)
