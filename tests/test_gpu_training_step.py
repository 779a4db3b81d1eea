"""A training step made of the operators in a row (norm with the residual, linear layer, norm, loss over a vocabulary, gradients,
AdamW): the same bits eagerly, captured in a graph and replayed, and captured twice on one memory pool; in a padded batch the rows
behind the last sequence change nothing."""

import pytest
import torch

import _loss_ref as R
from paper_2609_33437_gb300 import linear as L
from paper_2609_33437_gb300 import loss as T
from paper_2609_33437_gb300 import norm as N
from paper_2609_33437_gb300 import optim as O

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
K, H, V = 128, 320, 1500


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    yield
    assert L.poll_errors() == 0


def _rand(seed, *shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


class Step:
    """The parameters, what goes in, and one step on them."""

    def __init__(self, dtype, bits, rows):
        shapes = ((K,), (H, K), (H,), (K, H), (K,), (K,), (V, K))
        self.params = [_rand(i, *s, dtype=dtype, scale=0.05) + (1.0 if s == (K,) else 0.0) for i, s in enumerate(shapes)]
        self.moments = O.Moments(self.params, bits=bits)
        self.x, self.r = _rand(20, rows, K, dtype=dtype), _rand(21, rows, K, dtype=dtype)
        g = torch.Generator(device="cuda").manual_seed(22)
        self.t = torch.randint(0, V, (rows,), generator=g, device="cuda")
        self.t[rows // 3:rows // 2] = -100
        self.step = torch.zeros((), dtype=torch.int64, device="cuda")
        self.lr = torch.full((), 1e-3, device="cuda")

    def gradients(self):
        n1, w1, b1, w2, b2, n2, head = self.params
        y1, h, s1 = N.norm(self.x, n1, residual=self.r, kind="rms", save=True)
        a, saved = L.linear(y1, w1, b1, "silu", save=True)
        o = L.linear(a, w2, b2)
        y2, h2, s2 = N.norm(o, n2, residual=h, kind="rms", save=True)
        loss, lse = T.token_loss(y2, head, self.t)
        count = (self.t != -100).sum()
        g = (torch.ones_like(loss) / count).contiguous()
        dy2, dhead = T.token_loss_grad(g, y2, head, self.t, lse)
        do, dn2, _ = N.norm_grad(dy2, h2, s2, n2, kind="rms")  # of o and of h alike
        dw2, db2 = L.linear_grad_weight(do, saved, "silu", bias=True)
        dh = L.linear_grad_input(do, w2, "silu", saved)
        dw1, db1 = L.linear_grad_weight(dh, y1, bias=True)
        _, dn1, _ = N.norm_grad(L.linear_grad_input(dh, w1), h, s1, n1, kind="rms", dh=do)
        return loss, [dn1, dw1, db1, dw2, db2, dn2, dhead]

    def __call__(self):
        loss, grads = self.gradients()
        self.step.add_(1)
        O.adamw(self.params, grads, self.moments, self.step, lr=self.lr, seed=5)
        return loss

    def state(self):
        return [*self.params, *self.moments.buffers().values()]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_captured_step_is_the_eager_one(dtype, bits):
    eager, graphed = Step(dtype, bits, 203), Step(dtype, bits, 203)
    warm = Step(dtype, bits, 203)
    warm()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = graphed()
    second, again = torch.cuda.CUDAGraph(), Step(dtype, bits, 203)
    with torch.cuda.graph(second, pool=graph.pool()):  # another one whose workspaces lie where the first one's do
        again()
    for _ in range(3):
        loss = eager()
        graph.replay()
        second.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, captured)
    for a, b, c in zip(eager.state(), graphed.state(), again.state()):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_behind_the_last_sequence(dtype):
    """A padded batch: rows behind the last one whose targets are ignored, whatever they hold, leave the head's gradient as it is."""
    rows = 150
    s = Step(dtype, 32, rows)
    head, pad = s.params[-1], torch.full((37, K), float("nan"), device="cuda", dtype=dtype)
    y = _rand(30, rows, K, dtype=dtype)
    g = torch.full((rows,), 1.0 / rows, device="cuda")
    _, lse = T.token_loss(y, head, s.t)
    t = torch.cat([s.t, torch.full((37,), -100, device="cuda")])
    loss, lse2 = T.token_loss(torch.cat([y, pad]), head, t)
    dy, dw = T.token_loss_grad(torch.cat([g, pad[:, 0].float()]), torch.cat([y, pad]), head, t, torch.cat([lse, lse2[rows:]]))
    (rx, ex), (rw, ew) = R.gradient(g, y, head, s.t, lse, -100)
    assert bool(((dy[:rows].double() - rx).abs() <= ex).all()) and bool(((dw.double() - rw).abs() <= ew).all())
    assert not bool(dy[rows:].any()) and not bool(loss[rows:].any())
