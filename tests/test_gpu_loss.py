"""The loss over a vocabulary on the GPU (include/smat.h) against its definition in 64 bits: both types, from one row and one
word to several pieces of the vocabulary, odd sizes, strides, addresses off every boundary, rows that are ignored and what they
may hold, targets that are none, infinities, gradients by themselves and added to, streams and graphs, and the differentiable
form. Tolerances: `_loss_ref`."""

import pytest
import torch

import _loss_ref as R
from paper_2609_33437_gb300 import linear as L
from paper_2609_33437_gb300 import loss as T

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
IGNORE = -100


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    yield
    assert L.poll_errors() == 0


def _rand(seed, rows, cols, dtype, scale=1.0, pad=0, off=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (cols + pad) + off + 8,), float("nan"), device="cuda", dtype=dtype)
    t = flat[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.randn(rows, cols, generator=g, device="cuda") * scale)
    return t


def _inputs(seed, m, k, n, dtype, ignored=0.0, **kw):
    x = _rand(seed, m, k, dtype, **kw)
    w = _rand(seed + 1, n, k, dtype, 2.0 / max(k, 1) ** 0.5, **kw)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    t = torch.randint(0, n, (m,), generator=g, device="cuda")
    if m > 1:
        t[0], t[-1] = 0, n - 1
    t = torch.where(torch.rand(m, generator=g, device="cuda") < ignored, IGNORE, t)
    return x, w, t, torch.randn(m, generator=g, device="cuda") / max(m, 1)


def _near(got, ref, tol, what):
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: "
                                 f"{got[bad][0].item()} for {ref[bad][0].item()}, allowed {tol.expand_as(ref)[bad][0].item():.3g}")


def _check(x, w, t, g, **outs):
    loss, lse = T.token_loss(x, w, t, IGNORE)
    _, _, ref_lse, e_lse, ref, e = R.forward(x, w, t, IGNORE)
    _near(lse, ref_lse, e_lse, "lse")
    _near(loss, ref, e, "loss")
    assert not bool(loss[t == IGNORE].any())
    dx, dw = T.token_loss_grad(g, x, w, t, lse, IGNORE, **outs)
    (rx, ex), (rw, ew) = R.gradient(g, x, w, t, lse, IGNORE)
    _near(dx, rx, ex, "dx")
    _near(dw, rw, ew, "dw")
    assert not bool(dx[t == IGNORE].any())
    return loss, lse, dx, dw


# (fp32 products of more than 2^26 terms run on the tensor cores, from 300 rows on)
SIZES = [(1, 64, 500), (1, 8, 1), (2, 1, 3), (3, 130, 33), (17, 96, 256), (24, 512, 1000), (64, 64, 4096), (129, 200, 777),
         (256, 256, 256), (257, 128, 513), (300, 72, 5000), (515, 896, 3001), (1000, 64, 32000), (40, 4096, 2500), (130, 1000, 3001)]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_sizes(m, k, n, dt):
    for i, ignored in enumerate((0.0, 0.4)):
        _check(*_inputs(m + k + n + i, m, k, n, dt, ignored))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("m,n", [(9000, 9000), (700, 150000)])
def test_pieces(m, n, dt):
    """A vocabulary of more than one piece (d: 192 MB): bf16 9000 rows in one, fp32 in two; of 150000 words two and three."""
    _check(*_inputs(m, m, 64, n, dt, 0.2))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("m,k,n", [(5, 33, 70), (130, 101, 600), (300, 66, 1111), (20, 1023, 40000)])
@pytest.mark.parametrize("pad,off", [(0, 0), (1, 0), (8, 3), (7, 1)])
def test_rows_off_every_boundary(m, k, n, pad, off, dt):
    """Odd lengths and strides; results of any stride, and what lies beside them stays as it is."""
    dx, dw = _rand(50, m, k, dt, pad=pad, off=off), _rand(51, n, k, dt, pad=pad, off=off)
    x, w, t, g = _inputs(7, m, k, n, dt, 0.3, pad=pad, off=off)
    got = _check(x, w, t, g, out=dx, weight_out=dw)
    assert got[2] is dx and got[3] is dw
    for v in (dx, dw):
        beside = torch.ones_like(v._base, dtype=torch.bool)
        beside.as_strided(v.shape, v.stride(), v.storage_offset()).fill_(False)
        assert bool(v._base[beside].isnan().all())


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("m,k,n", [(90, 128, 700), (330, 256, 3000)])
def test_ignored_rows_reach_nothing(m, k, n, dt):
    """What rows that are ignored hold, infinities and NaN too, and their gradients; all rows ignored; none."""
    x, w, t, g = _inputs(0, m, k, n, dt, 0.5)
    skip = t == IGNORE
    loss, lse = T.token_loss(x, w, t, IGNORE)
    ref = T.token_loss_grad(g, x, w, t, lse, IGNORE)
    x2, g2, l2 = x.clone(), g.clone(), lse.clone()
    x2[skip], g2[skip], l2[skip] = float("nan"), float("inf"), float("nan")
    x2[skip.nonzero()[0, 0]] = float("inf")
    got = T.token_loss_grad(g2, x2, w, t, l2, IGNORE)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    there = T.token_loss(x2, w, t, IGNORE)[0]
    assert not bool(there[skip].any())
    # (an infinity or NaN anywhere in x has an fp32 product made on other units: other roundings, the same bound)
    *_, value, e = R.forward(x[~skip], w, t[~skip], IGNORE)
    _near(there[~skip], value, e, "loss")
    assert dt is F32 or torch.equal(there[~skip], loss[~skip])
    # the rows that count by themselves: the same numbers
    alone = T.token_loss_grad(g[~skip], x[~skip].contiguous(), w, t[~skip], lse[~skip], IGNORE)
    (rx, ex), (rw, ew) = R.gradient(g[~skip], x[~skip], w, t[~skip], lse[~skip], IGNORE)
    _near(ref[0][~skip], rx, ex, "dx")
    _near(alone[1], rw, ew, "dw")
    none = torch.full_like(t, IGNORE)
    loss, lse = T.token_loss(x2, w, none, IGNORE)
    dx, dw = T.token_loss_grad(g2, x2, w, none, lse, IGNORE)
    assert not bool(loss.any()) and not bool(dx.any()) and not bool(dw.any())
    # another number for them: the old one is then no target
    other = torch.where(skip, 7, t)
    loss, lse = T.token_loss(x, w, other, 7)
    assert bool((loss == 0).sum() >= skip.sum())


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("m,k,n", [(70, 64, 300), (300, 256, 2000)])
def test_targets_that_are_none(m, k, n, dt):
    """A target outside the vocabulary: NaN, and nothing is read or written for it."""
    x, w, t, g = _inputs(0, m, k, n, dt)
    for bad in (n, -1, 1 << 40, -(1 << 62)):
        b = t.clone()
        b[5] = bad
        loss, lse = T.token_loss(x, w, b, IGNORE)
        ok, ref_lse = T.token_loss(x, w, t, IGNORE)
        rest = torch.arange(m, device="cuda") != 5
        assert bool(loss[5].isnan()) and torch.equal(loss[rest], ok[rest]) and torch.equal(lse, ref_lse)
        dx, dw = T.token_loss_grad(g, x, w, b, lse, IGNORE)
        assert bool(dx[5].isnan().all()) and bool(dw.isnan().all()) and not bool(dx[rest].isnan().any())


@pytest.mark.parametrize("dt", [BF, F32])
def test_special_logits(dt):
    """Logits far from one another, of -infinity, and a NaN, which stays in its row."""
    m, k, n = 6, 16, 600
    x, w, t, g = _inputs(0, m, k, n, dt)
    x[0] *= 1000.0
    x[1] = 0.0
    w[7] = 0.0
    w[7, 3] = float("-inf")
    x[:, 3] = x[:, 3].abs() + 0.25  # logit 7 is -infinity, and its gradient's sum is over finite words alone
    t[t == 7] = 8
    loss, lse = T.token_loss(x, w, t, IGNORE)
    _, _, ref_lse, _, ref, _ = R.forward(x, w, t, IGNORE)
    clean = w.clone()
    clean[7] = 0
    keep = torch.arange(n, device="cuda") != 7
    _, _, ref_lse, e_lse, _, _ = R.forward(x, w[keep], torch.zeros_like(t), IGNORE)
    _near(lse, ref_lse, e_lse, "lse")
    t2 = t.clone()
    t2[2] = 7
    assert float(T.token_loss(x, w, t2, IGNORE)[0][2]) == float("inf")
    x[4, 0] = float("nan")
    again, lse2 = T.token_loss(x, w, t, IGNORE)
    rest = torch.arange(m, device="cuda") != 4
    assert bool(again[4].isnan()) and bool(lse2[4].isnan()) and torch.equal(again[rest], loss[rest])


@pytest.mark.parametrize("dt", [BF, F32])
def test_nothing(dt):
    e = torch.empty(0, 32, device="cuda", dtype=dt)
    w = _rand(0, 40, 32, dt)
    t, g = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    loss, lse = T.token_loss(e, w, t)
    assert loss.shape == lse.shape == (0,)
    dx, dw = T.token_loss_grad(g, e, w, t, lse)
    assert dx.shape == (0, 32) and dw.shape == (40, 32) and not bool(dw.any())
    dw.fill_(2.0)
    T.token_loss_grad(g, e, w, t, lse, weight_out=dw, accumulate=True)
    assert bool((dw == 2).all())
    # no columns: every logit is 0
    loss, lse = T.token_loss(torch.empty(5, 0, device="cuda", dtype=dt), torch.empty(1024, 0, device="cuda", dtype=dt),
                             torch.zeros(5, dtype=torch.int64, device="cuda"))
    assert float((lse - torch.log(torch.tensor(1024.0))).abs().max()) < 1e-6 and torch.equal(loss, lse)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("m,k,n", [(20, 1024, 600), (200, 2048, 4000), (33, 515, 500)])
def test_rows_that_are_sure(m, k, n, dt):
    """Where the target has nearly all of the probability its gradient is what is left of two numbers that nearly cancel."""
    x, w, t, g = _inputs(1, m, k, n, dt, 0.1)
    lean = 16.0 / (w[t.clamp(min=0)].float() ** 2).sum(1, keepdim=True)
    x = (0.2 * x.float() + lean * w[t.clamp(min=0)].float()).to(dt)
    p = torch.exp(-_check(x, w, t, g)[0])[t != IGNORE]
    assert float(p.min()) > 0.97 and float(p.max()) < 0.99999


@pytest.mark.parametrize("dt", [BF, F32])
def test_options(dt):
    x, w, t, g = _inputs(3, 140, 160, 3000, dt, 0.2)
    _, lse = T.token_loss(x, w, t)
    dx, dw = T.token_loss_grad(g, x, w, t, lse)
    only = T.token_loss_grad(g, x, w, t, lse, need_w=False)
    assert only[1] is None and torch.equal(only[0], dx)
    only = T.token_loss_grad(g, x, w, t, lse, need_x=False)
    assert only[0] is None and torch.equal(only[1], dw)
    assert T.token_loss_grad(g, x, w, t, lse, need_x=False, need_w=False) == (None, None)
    old = _rand(9, 3000, 160, dt)
    both = old.clone()
    T.token_loss_grad(g, x, w, t, lse, weight_out=both, accumulate=True)
    (_, _), (rw, ew) = R.gradient(g, x, w, t, lse, IGNORE)
    ref = rw + old.double()
    _near(both, ref, ew + R.R.rounding(dt) * 1.01 * ref.abs() + 2 * R.U * old.double().abs(), "added")
    # leading dimensions
    loss3, lse3 = T.token_loss(x.view(7, 20, 160), w, t.view(7, 20))
    assert loss3.shape == (7, 20) and torch.equal(lse3.view(-1), lse)
    dx3, _ = T.token_loss_grad(g.view(7, 20), x.view(7, 20, 160), w, t.view(7, 20), lse3)
    assert torch.equal(dx3.view(140, 160), dx)


@pytest.mark.parametrize("dt", [BF, F32])
def test_same_result_streams_and_graphs(dt):
    x, w, t, g = _inputs(5, 515, 256, 4000, dt, 0.3)

    def both(stream=None):
        loss, lse = T.token_loss(x, w, t, stream=stream)
        return (loss, lse, *T.token_loss_grad(g, x, w, t, lse, stream=stream))

    ref = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(both())
        graphs.append(graph)
    x.mul_(0.5)
    t[::3] = IGNORE  # other rows count at the replay
    for graph in graphs:
        graph.replay()
    ref = both()
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(p, q) for p, q in zip(ref, out))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_differentiable_form(dt, reduction):
    x, w, t, _ = _inputs(11, 60, 48, 900, dt, 0.3)
    x, w = x.clone().requires_grad_(), w.clone().requires_grad_()
    loss = T.cross_entropy(x.view(6, 10, 48), w, t.view(6, 10), reduction=reduction)
    scale = torch.ones((), device="cuda") if reduction != "none" else torch.randn(6, 10, device="cuda")
    (loss * scale).sum().backward()
    xd, wd = x.detach().double(), w.detach().double()
    ref = torch.nn.functional.cross_entropy(xd @ wd.T, t, ignore_index=IGNORE, reduction=reduction)
    _, _, lse, _, _, e = R.forward(x.detach(), w.detach(), t, IGNORE)
    assert bool(((loss.view(-1).double() - ref.view(-1)).abs() <= e.sum() + 70 * R.U * ref.abs().max()).all())
    count = int((t != IGNORE).sum())
    g = (scale.view(-1) if reduction == "none" else torch.full((60,), 1 / count if reduction == "mean" else 1.0, device="cuda"))
    (rx, ex), (rw, ew) = R.gradient(g.float(), x.detach(), w.detach(), t, T.token_loss(x.detach(), w.detach(), t)[1], IGNORE)
    _near(x.grad, rx, ex + 2 * R.U * rx.abs(), "dx")
    _near(w.grad, rw, ew + 2 * R.U * rw.abs(), "dw")
    with torch.no_grad():
        assert torch.equal(T.cross_entropy(x.view(6, 10, 48), w, t.view(6, 10), reduction=reduction), loss)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        d = torch.autograd.grad(T.cross_entropy(x, w, t), x, create_graph=True)[0]
        d.sum().backward()


def test_gradient_against_differences():
    """dx and dw along a direction against differences of the 64-bit loss."""
    x, w, t, _ = _inputs(13, 30, 40, 500, F32, 0.2)
    g = torch.full((30,), 1.0, device="cuda")
    _, lse = T.token_loss(x, w, t)
    dx, dw = T.token_loss_grad(g, x, w, t, lse)
    u, v = _rand(14, 30, 40, F32).double(), _rand(15, 500, 40, F32).double()

    def value(s):
        return float(R.forward(x.double() + s * u, w.double() + s * v, t, IGNORE)[4].sum())

    step = 1e-5
    numeric = (value(step) - value(-step)) / (2 * step)
    exact = float((dx.double() * u).sum() + (dw.double() * v).sum())
    size = float((dx.double() * u).abs().sum() + (dw.double() * v).abs().sum())
    # differences of 64 bits: step^2 and 1e-16 / step of the loss; the gradients: some hundred roundings of their terms
    assert abs(numeric - exact) < 300 * R.U * size + 1e-6


def test_layers_and_autocast():
    """A run of them as a training step has it: norm with the residual, an MLP, norm, loss, gradients, update."""
    from paper_2609_33437_gb300 import norm as N
    from paper_2609_33437_gb300 import optim as O

    torch.manual_seed(0)
    dt = BF
    first, mlp, last = N.Norm(128, "rms", device="cuda", dtype=dt), L.Mlp8(128, 256, device="cuda", dtype=dt), N.Norm(128, "rms", device="cuda", dtype=dt)
    head = torch.nn.Parameter(torch.randn(1000, 128, device="cuda", dtype=dt) * 0.1)
    params = [*first.parameters(), *mlp.parameters(), *last.parameters(), head]
    opt = O.AdamW(params, lr=1e-3, bits=8)
    x, r = _rand(1, 48, 128, dt), _rand(2, 48, 128, dt)
    t = torch.randint(0, 1000, (48,), device="cuda")

    def loss_of(dtype):
        """With torch's own operators, in another type."""
        h = x.to(dtype) + r.to(dtype)
        rms = lambda v, m: v / torch.sqrt((v * v).mean(-1, keepdim=True) + m.eps) * m.weight.to(dtype)  # noqa: E731
        y = torch.nn.functional.gelu(rms(h, first) @ mlp.fc1.weight.to(dtype).T + mlp.fc1.bias.to(dtype))
        h = h + y @ mlp.fc2.weight.to(dtype).T + mlp.fc2.bias.to(dtype)
        return torch.nn.functional.cross_entropy(rms(h, last) @ head.to(dtype).T, t)

    for _ in range(3):
        y, h = first(x, r)
        loss = T.cross_entropy(last(mlp(y, h)), head, t)
        loss.backward()
        # every tensor on the way is rounded to bf16 (2^-8 each) and the activations to 8 bits: ten of those, in parts that add up
        # to no more than the logits' size
        ref = loss_of(torch.float64)
        assert abs(float(loss.detach()) - float(ref.detach())) < 10 * 2.0 ** -8 * 4
        want = torch.autograd.grad(ref, params)
        for p, q in zip(params, want):
            assert float((p.grad.double() - q.double()).norm()) < 0.05 * float(q.double().norm()) + 1e-6
        opt.step()
        opt.zero_grad()
    w32 = torch.randn(300, 64, device="cuda", requires_grad=True)
    x32 = torch.randn(5, 64, device="cuda", requires_grad=True)
    with torch.autocast("cuda", dtype=BF):
        value = T.cross_entropy(x32, w32, t[:5] % 300)
    value.backward()
    assert value.dtype is F32 and w32.grad.dtype is F32 and x32.grad.shape == x32.shape


def _workspaces(m, k, n, dt):
    """Bytes that the loss and its gradient ask for (addresses only have to be aligned)."""
    code, at = 1 if dt is BF else 0, [4096 * i for i in range(1, 8)]
    lib = L.S.load_library()
    fwd = T._TOKEN_LOSS.pack(*at[:5], m, k, n, k, k, IGNORE, code, 0)
    grad = T._TOKEN_LOSS_GRAD.pack(*at, m, k, n, k, k, k, k, IGNORE, code, 0)
    return lib.smat_token_loss_workspace_bytes(fwd), lib.smat_token_loss_grad_workspace_bytes(grad)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("m", [1, 16, 17, 64, 300, 2049, 8192])
@pytest.mark.parametrize("k", [64, 896, 4096])
def test_workspace_is_bounded_in_the_vocabulary(m, k, dt):
    """The gradient's by what the header names, and no larger for four times the words; the loss's grows by its parts alone."""
    n, mib = 151936, 1 << 20
    fwd, grad = _workspaces(m, k, n, dt)
    rows = 2 * m if dt is BF and m <= 128 else m
    d = max(192 * mib, rows * 2048 * (2 if dt is BF else 4))
    x = rows * (k + 32) * 4
    if dt is BF:
        most, part = d + 3 * x + 33 * 256 * (k + 32) * 4, 8 * m * (n // 64 + 400)
    else:
        most, part = 2.5 * d + 1024 * mib + 5 * x, d + 1024 * mib + 2 * x
    slack = 48 * mib  # shares of sums of one tile an SM, flags, numbers of rows, rounding up
    assert 0 < grad <= most + slack and 0 < fwd <= part + slack
    fwd4, grad4 = _workspaces(m, k, 4 * n, dt)
    assert grad4 <= most + slack and fwd4 <= 4 * part + slack
    assert dt is BF or fwd4 <= part + slack


@pytest.mark.parametrize("m,k,n", [(20, 4096, 50000), (300, 2048, 90000), (64, 4100, 45000)])
def test_fp32_pieces_of_a_cut_vocabulary(m, k, n):
    """fp32 on the tensor cores, W in more than one piece for the size of its parts; results added up over them."""
    dx, dw = _check(*_inputs(m + n, m, k, n, F32, 0.3))[2:]
    x, w, t, g = _inputs(m + n, m, k, n, F32, 0.3)
    _, lse = T.token_loss(x, w, t)
    again = T.token_loss_grad(g, x, w, t, lse, need_w=False)[0], T.token_loss_grad(g, x, w, t, lse, need_x=False)[1]
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
