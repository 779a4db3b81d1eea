"""Layer norm and rms norm on the GPU (include/smat.h, "norms") against their definitions in 64 bits: both types and types of
weights, sizes from one column to rows that do not fit in registers, odd sizes, row strides, addresses off every boundary,
special values, streams, graphs, and the layer with its gradients.

Tolerances, u = 2^-24: a sum over a row passes at most `_adds(cols)` roundings of u each on its way (a thread's values in
turn, then five lanes' and five warps' steps); a sum over rows of n terms stays under 8 sqrt(n) u of the magnitudes' sum, see
`_linear_ref.sum_error`; every other operation rounds once, and a result once more to its type."""

import math

import pytest
import torch

import _linear_ref as R
from paper_2609_33437_gb300 import norm as N

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


def _adds(cols):
    return 16 + 12 if cols <= 16384 else -(-cols // 1024) + 12


def _rand(seed, rows, cols, dtype, scale=1.0, shift=0.0, pad=0, off=0):
    """[rows, cols], its rows `pad` elements apart, its address `off` elements off; NaN around it."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (cols + pad) + off + 8,), float("nan"), device="cuda", dtype=dtype)
    t = flat[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.randn(rows, cols, generator=g, device="cuda") * scale + shift)
    return t


def _vec(seed, n, dtype, scale, shift):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, generator=g, device="cuda") * scale + shift).to(dtype)


def _near(got, ref, tol, what):
    got = got.detach().double().cpu()
    off = (got - ref).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: "
                                 f"{got[bad][0].item()} for {ref[bad][0].item()}, allowed {tol.expand_as(ref)[bad][0].item():.3g}")


def _d(t):
    return t.detach().double().cpu()


def _forward(x, w, b, r, kind, eps):
    """h, y, stats and how far y and the statistics may be off."""
    h = _d(x)
    if r is not None:
        h = _d((x.float() + r.float()).to(x.dtype))
    n, adds = h.shape[1], _adds(h.shape[1])
    layer = kind == "layer"
    mu = h.mean(1, keepdim=True) if layer else torch.zeros(h.shape[0], 1, dtype=torch.float64)
    e_mu = (adds + 2) * U * h.abs().mean(1, keepdim=True) if layer else 0 * mu
    d = h - mu
    v = (d * d).mean(1, keepdim=True)
    s = 1 / torch.sqrt(v + eps)
    e_v = (adds + 4) * U * v + 2 * e_mu * d.abs().mean(1, keepdim=True) + e_mu ** 2
    rel_s = 0.5 * e_v / (v + eps) * 1.01 + 4 * U
    xh = d * s
    e_xh = s * (e_mu + U * d.abs()) * 1.01 + xh.abs() * (rel_s + 2 * U)
    wd = _d(w) if w is not None else torch.ones(n, dtype=torch.float64)
    bd = _d(b) if b is not None else torch.zeros(n, dtype=torch.float64)
    y = xh * wd + bd
    tol = wd.abs() * e_xh * 1.01 + U * y.abs() + R.rounding(x.dtype) * 1.01 * (y.abs() + wd.abs() * e_xh) + 1e-38
    stats = torch.cat([mu, s], 1).T if layer else s.T
    e_stats = torch.cat([e_mu + U * mu.abs() + 1e-38, s * rel_s], 1).T if layer else (s * rel_s).T
    return h, y, tol, stats, e_stats


def _check_forward(x, w, b, r, kind, eps=1e-5):
    got = N.norm(x, w, b, residual=r, kind=kind, eps=eps, save=True)
    h, y, tol, stats, e_stats = _forward(x, w, b, r, kind, eps)
    if r is not None:
        assert torch.equal(_d(got[1]), h)
    _near(got[-1], stats, e_stats, "stats")
    _near(got[0], y, tol, "y")
    return got


def _check_grad(dy, h, stats, w, bias, kind, dh, **outs):
    dx, dw, db = N.norm_grad(dy, h, stats, w, bias=bias, kind=kind, dh=dh, **outs)
    hd, dyd, sd = _d(h), _d(dy), _d(stats)
    rows, n = hd.shape
    adds, layer = _adds(n), kind == "layer"
    inv = sd[-1][:, None]
    xh = (hd - sd[0][:, None] if layer else hd) * inv
    wd = _d(w) if w is not None else torch.ones(n, dtype=torch.float64)
    a = dyd * wd
    by, off = (a * xh).mean(1, keepdim=True), a.mean(1, keepdim=True) if layer else torch.zeros(rows, 1, dtype=torch.float64)
    e_by = (adds + 6) * U * (a * xh).abs().mean(1, keepdim=True)
    e_off = (adds + 3) * U * a.abs().mean(1, keepdim=True) if layer else 0.0
    dx_ref = (a - off - xh * by) * inv
    e = inv * (e_off + xh.abs() * e_by + 6 * U * (a.abs() + off.abs() + (xh * by).abs()))
    if dh is not None:
        dx_ref = dx_ref + _d(dh)
        e = e + U * dx_ref.abs()
    _near(dx, dx_ref, e * 1.01 + R.rounding(dy.dtype) * 1.01 * (dx_ref.abs() + e) + 1e-38, "dx")
    by_rows = (8 * math.sqrt(rows) + 8) * U
    ref = (dyd * xh).sum(0)
    tol = by_rows * (dyd * xh).abs().sum(0)
    _near(dw, ref, tol + R.rounding(dw.dtype) * 1.01 * (ref.abs() + tol) + 1e-38, "dw")
    assert (db is not None) == bias
    if bias:
        ref = dyd.sum(0)
        tol = by_rows * dyd.abs().sum(0)
        _near(db, ref, tol + R.rounding(db.dtype) * 1.01 * (ref.abs() + tol) + 1e-38, "db")


SIZES = [(1, 1), (1, 4096), (3, 7), (5, 33), (64, 128), (257, 1024), (2, 2048), (3, 2050), (17, 896), (300, 100), (7, 8200),
         (2, 11008), (3, 16384), (2, 16386), (5, 20001), (1300, 64), (641, 255),
         (1300, 1023), (700, 2047), (650, 4095), (330, 8191), (20, 16383), (4000, 13), (2500, 770)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("types", [(BF, BF), (BF, F32), (F32, F32)], ids=["bf16", "bf16_f32", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(rows, cols, types, kind):
    dt, wt = types
    seed = rows * 31 + cols
    x = _rand(seed, rows, cols, dt, 2.0, 0.5)
    r = _rand(seed + 1, rows, cols, dt)
    w, b = _vec(seed + 2, cols, wt, 0.2, 1.0), _vec(seed + 3, cols, wt, 0.1, 0.0) if kind == "layer" else None
    _check_forward(x, w, b, None, kind)
    _, h, stats = _check_forward(x, w, b, r, kind)
    dy, dh = _rand(seed + 4, rows, cols, dt, 0.1), _rand(seed + 5, rows, cols, dt, 0.1)
    _check_grad(dy, h, stats, w, b is not None, kind, None)
    _check_grad(dy, h, stats, w, True, kind, dh)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("pad,off", [(8, 0), (2, 2), (1, 0), (0, 1), (3, 3), (4, 4)])
@pytest.mark.parametrize("rows,cols", [(9, 64), (33, 1032), (6, 4100)])
def test_strides_and_addresses(rows, cols, pad, off, dt):
    """Rows apart and off every boundary; what lies between the rows stays as it is."""
    x, r, dy, dh = (_rand(i, rows, cols, dt, pad=pad, off=off) for i in range(4))
    w, b = _vec(5, cols + 4, dt, 0.2, 1.0)[off:off + cols], _vec(6, cols + 4, dt, 0.1, 0.0)[off:off + cols]
    y, h, dx = (_rand(i, rows, cols, dt, pad=pad, off=off) for i in range(7, 10))
    got = N.norm(x, w, b, residual=r, save=True, out=y, sum_out=h)
    assert got[0] is y and got[1] is h
    href, yref, tol, _, _ = _forward(x, w, b, r, "layer", 1e-5)
    assert torch.equal(_d(h), href)
    _near(y, yref, tol, "y")
    _check_grad(dy, h, got[-1], w, True, "layer", dh, out=dx)
    for t in (y, h, dx):
        base = t._base if t._base is not None else t
        whole = torch.ones_like(base, dtype=torch.bool)
        whole.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(False)
        assert bool(base[whole].isnan().all()) and not bool(t.isnan().any())


def test_in_place_and_leading_dimensions():
    x, r = _rand(0, 24, 72, BF).reshape(2, 3, 4, 72), _rand(1, 24, 72, BF).reshape(2, 3, 4, 72)
    y, h = N.norm(x, residual=r, kind="rms")
    assert y.shape == h.shape == x.shape
    r2 = r.clone()
    y2, h2 = N.norm(x, residual=r2, kind="rms", sum_out=r2)
    assert h2 is r2 and torch.equal(h, h2) and torch.equal(y, y2)
    _, stats = N.norm(h, kind="rms", save=True)
    dy, dh = _rand(2, 24, 72, BF).reshape(2, 3, 4, 72), _rand(3, 24, 72, BF).reshape(2, 3, 4, 72)
    dx = N.norm_grad(dy, h, stats, kind="rms", dh=dh)[0]
    assert torch.equal(N.norm_grad(dy, h, stats, kind="rms", dh=dh, out=dh)[0], dx) and torch.equal(dh, dx)
    one = _rand(4, 1, 50, F32)[0]
    assert N.norm(one).shape == (50,)
    # (rows of 50 lie off 16 bytes in turn, and their sums' order goes by that: the same row in a batch is as near, not the same bits)
    _check_forward(one.expand(5, 50).contiguous(), None, None, None, "layer")


@pytest.mark.parametrize("wt", [BF, F32])
def test_options(wt):
    """Each gradient by itself, gradients added to, no weights, and what is not asked for."""
    x, dy = _rand(0, 530, 96, BF), _rand(1, 530, 96, BF)
    w = _vec(2, 96, wt, 0.2, 1.0)
    _, stats = N.norm(x, w, save=True)
    dx, dw, db = N.norm_grad(dy, x, stats, w, bias=True)
    assert torch.equal(N.norm_grad(dy, x, stats, w, need_w=False)[0], dx)
    only = N.norm_grad(dy, x, stats, w, need_x=False)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dw)
    only = N.norm_grad(dy, x, stats, w, bias=True, need_x=False, need_w=False)
    assert only[0] is None and only[1] is None and torch.equal(only[2], db)
    assert N.norm_grad(dy, x, stats, w, need_x=False, need_w=False) == (None, None, None)
    w0, b0 = _vec(3, 96, wt, 1.0, 0.0), _vec(4, 96, wt, 1.0, 0.0)
    w1, b1 = w0.clone(), b0.clone()
    N.norm_grad(dy, x, stats, w, bias=True, weight_out=w1, bias_out=b1, accumulate=True)
    full = N.norm_grad(dy, x, stats, w.float(), bias=True)
    for got, old, add in ((w1, w0, full[1]), (b1, b0, full[2])):
        ref = _d(old) + _d(add)
        _near(got, ref, R.rounding(wt) * 1.01 * ref.abs() + 2 * U * (_d(old).abs() + _d(add).abs()), "added")
    _check_forward(x, None, None, None, "layer")
    _check_grad(dy, x, stats, None, True, "layer", None)


@pytest.mark.parametrize("dt", [BF, F32])
def test_nothing_and_constant_rows(dt):
    x = torch.empty(0, 40, device="cuda", dtype=dt)
    y, stats = N.norm(x, save=True)
    assert y.shape == (0, 40) and stats.shape == (2, 0)
    dw, db = torch.ones(40, device="cuda", dtype=dt), torch.ones(40, device="cuda", dtype=dt)
    N.norm_grad(x, x, stats, bias=True, weight_out=dw, bias_out=db)
    assert not bool(dw.any()) and not bool(db.any())
    dw.fill_(3.0)
    N.norm_grad(x, x, stats, weight_out=dw, accumulate=True)
    assert bool((dw == 3.0).all())
    # a row of one value: nothing is left of it, whatever its size; of zeros nothing divides by 0
    c = torch.full((3, 128), 1024.0, device="cuda", dtype=dt)
    assert not bool(N.norm(c).any()) and not bool(N.norm(torch.zeros_like(c), kind="rms").any())
    assert bool(N.norm(c, eps=0.0).isnan().all()) and bool(torch.isfinite(N.norm(c, kind="rms", eps=0.0)).all())


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("cols", [64, 4096, 20000])
def test_special_values_stay_in_their_rows(kind, cols):
    x = _rand(0, 6, cols, F32)
    ref = N.norm(x, kind=kind)
    x[1, 3], x[4, 5] = float("nan"), float("inf")
    y = N.norm(x, kind=kind)
    keep = torch.tensor([0, 2, 3, 5], device="cuda")
    assert torch.equal(y[keep], ref[keep])
    assert bool(y[1].isnan().all()) and bool(y[4, 5].isnan())


def test_large_mean():
    """A row whose mean is far above its spread: the squares are of what is left of the mean."""
    x = _rand(0, 4, 4096, F32, scale=0.01, shift=100.0)
    _check_forward(x, None, None, None, "layer", eps=1e-12)


def test_same_result_streams_and_graphs():
    x, r, dy = (_rand(i, 1031, 1024, BF) for i in range(3))
    w, b = _vec(5, 1024, BF, 0.2, 1.0), _vec(6, 1024, BF, 0.1, 0.0)

    def both(stream=None):
        y, h, stats = N.norm(x, w, b, residual=r, save=True, stream=stream)
        return (y, h, stats, *N.norm_grad(dy, h, stats, w, bias=True, dh=x, stream=stream))

    ref = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    graphs, outs = [], []
    for _ in range(2):  # two captured graphs, each with its own workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(both())
        graphs.append(g)
    for t in (x, r, dy):
        t.mul_(0.5)
    for g in graphs:
        g.replay()
    ref = both()
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(p, q) for p, q in zip(ref, out))


def test_offsets_past_32_bits():
    rows, ld = 3, (1 << 30) + 8
    flat = torch.empty(2 * ld + 64, device="cuda", dtype=BF)
    x = flat.as_strided((rows, 64), (ld, 1))
    x.copy_(_rand(0, rows, 64, BF))
    _check_forward(x, None, None, None, "layer")


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dt", [BF, F32])
def test_layer_matches_autograd(kind, dt):
    """The layer's gradients against torch's own in 64 bits, through two uses of the residual stream."""
    rows, cols = 37, 192
    layer = N.Norm(cols, kind=kind, device="cuda", dtype=dt)
    with torch.no_grad():
        layer.weight.copy_(_vec(1, cols, dt, 0.2, 1.0))
        if layer.bias is not None:
            layer.bias.copy_(_vec(2, cols, dt, 0.1, 0.0))
    x, r = _rand(3, rows, cols, dt).clone().requires_grad_(), _rand(4, rows, cols, dt).clone().requires_grad_()
    dy, dh = _rand(5, rows, cols, dt), _rand(6, rows, cols, dt)
    y, h = layer(x, r)
    torch.autograd.backward((y, h), (dy, dh))
    xd, rd = _d(x).requires_grad_(), _d(r).requires_grad_()
    wd = _d(layer.weight).requires_grad_()
    bd = _d(layer.bias).requires_grad_() if layer.bias is not None else None
    hd = xd + rd
    hd = hd + (_d(h) - hd.detach())  # as it was rounded
    off = hd - hd.mean(1, keepdim=True) if kind == "layer" else hd
    yd = off / torch.sqrt((off * off).mean(1, keepdim=True) + 1e-5) * wd
    if bd is not None:
        yd = yd + bd
    torch.autograd.backward((yd, hd), (_d(dy), _d(dh)))
    # an output's rounding beside its size, and the chain's roundings beside the largest
    for got, ref in ((x.grad, xd.grad), (r.grad, rd.grad), (layer.weight.grad, wd.grad),
                     *(((layer.bias.grad, bd.grad),) if bd is not None else ())):
        _near(got, ref, R.rounding(dt) * 1.01 * ref.abs() + 200 * U * ref.abs().max(), "gradient")
    assert torch.equal(x.grad, r.grad)
    with torch.no_grad():
        y2, h2 = layer(x, r)
        assert torch.equal(y, y2) and torch.equal(h, h2)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        g = torch.autograd.grad(layer(x).sum(), x, create_graph=True)[0]
        g.sum().backward()


def test_layer_uses_one_output_only():
    layer = N.Norm(64, device="cuda")
    x, r = _rand(0, 5, 64, F32).clone().requires_grad_(), _rand(1, 5, 64, F32).clone().requires_grad_()
    layer(x, r)[1].sum().backward()
    assert bool((x.grad == 1).all()) and bool((r.grad == 1).all()) and not bool(layer.weight.grad.any())
    x.grad = r.grad = None
    layer(x, r.detach())[0].sum().backward()
    assert x.grad is not None
    layer(x.t().contiguous().t()[:, :64]).sum().backward()
    layer.weight.requires_grad_(False)
    layer.bias.requires_grad_(False)
    layer.weight.grad = None
    layer(x)[0].sum().backward()
    assert layer.weight.grad is None


def test_gradient_against_differences():
    """dx against differences of the 64-bit definition along a direction, in fp32."""
    x, w = _rand(0, 4, 40, F32), _vec(1, 40, F32, 0.2, 1.0)
    dy, u = _rand(2, 4, 40, F32), _d(_rand(3, 4, 40, F32))
    _, stats = N.norm(x, w, save=True)
    dx = _d(N.norm_grad(dy, x, stats, w)[0])

    def value(t):
        off = t - t.mean(1, keepdim=True)
        return float((off / torch.sqrt((off * off).mean(1, keepdim=True) + 1e-5) * _d(w) * _d(dy)).sum())

    step = 1e-5
    numeric = (value(_d(x) + step * u) - value(_d(x) - step * u)) / (2 * step)
    exact = float((dx * u).sum())
    # 64-bit differences are good to about step^2; dx is good to 100 roundings of its terms
    assert abs(numeric - exact) < 1e-7 * float((dx * u).abs().sum()) * 100 + 1e-6
