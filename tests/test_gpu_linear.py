"""The linear layers' operators on the GPU (include/smat.h, "linear layers") against their definitions in 64 bits:
every type, activation and option over sizes from nothing to several tiles, odd sizes, row strides, addresses off
every boundary, other streams, special values, offsets past 32 bits, and the same result every time.

Tolerances: an output is off by its one rounding, by the sums' error (`_linear_ref.sum_error`) times the largest
slope of an activation (1.13), and by an activation's own error, 4e-6 of |h| (a 2-ulp exponential of an argument
rounded to 2^-24, up to |h| = 20, beyond which it no longer shows; erfc's 4 ulp)."""

import pytest
import torch

import _linear_ref as R
from paper_2609_33437_gb300 import linear as L
from paper_2609_33437_gb300 import smat as S

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


def _rand(seed, *shape, scale=1.0, dtype=BF, pad=0, shift=0):
    """A matrix of this shape; its rows `pad` elements apart from one another, its address `shift` elements off."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols = shape
    flat = torch.empty(rows * (cols + pad) + shift + 8, device="cuda", dtype=dtype).fill_(float("nan"))
    t = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.randn(rows, cols, generator=g, device="cuda") * scale)
    return t


def _vec(seed, n, dtype, scale=0.1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, generator=g, device="cuda") * scale).to(dtype)


def _near(got, ref, tol, what):
    got, ref = got.detach().double().cpu(), ref.double()
    off = (got - ref).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} off, first at "
                                 f"{bad.nonzero()[0].tolist()}: {got[bad][0].item()} for {ref[bad][0].item()}, "
                                 f"largest excess {float((off - tol)[bad].max()):.3g}")


def _d(t):
    return t.detach().double().cpu()


def _linear_ref(x, w, b, act, r):
    """(y, h, error of h)"""
    dx, dw = _d(x), _d(w)
    h = dx @ dw.T
    mag = dx.abs() @ dw.abs().T
    if b is not None:
        h = h + _d(b)
        mag = mag + _d(b).abs()
    err = R.sum_error(mag, x.dtype, x.shape[-1])
    y = R.act(act, h)
    if r is not None:
        y = y + _d(r)
    return y, h, err


def _check_linear(x, w, b, act, r, y, saved=None):
    ref, h, err = _linear_ref(x, w, b, act, r)
    tol = R.rounding(x.dtype) * ref.abs() * 1.01 + 1.13 * err + 4e-6 * h.abs() + 1e-30
    if r is not None:
        tol = tol + 2.0 ** -23 * (_d(r).abs() + h.abs())
    _near(y, ref, tol, "y")
    if saved is not None:
        _check_saved(saved, h, err)


def _check_saved(saved, h, err):
    """Values within half a step of h, steps as small as they may be."""
    val = R.unpack(saved.q, saved.e)
    e = saved.e.cpu().to(torch.int64)
    step = torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e - 127)
    wide = step.repeat_interleave(32, -1)[:, :h.shape[1]]
    _near(val, h, 0.5 * wide * (1 + 1e-12) + err, "saved")
    assert int(saved.q.cpu().to(torch.int32).abs().max()) <= 127
    groups = e.shape[1]
    pad = torch.zeros(h.shape[0], groups * 32, dtype=torch.float64)
    pad[:, :h.shape[1]] = h.abs() + err
    top = pad.view(h.shape[0], groups, 32).amax(-1)
    assert bool(((e == 1) | (top >= 127.5 * step / 2 * (1 - 1e-12))).all()), "a step larger than needed"


# sizes: (rows, k, n)
SIZES = [(1, 1, 1), (1, 64, 128), (1, 4096, 257), (2, 40, 33), (5, 896, 130), (17, 8, 4096), (33, 129, 65), (64, 576, 320),
         (77, 588, 200), (100, 1000, 1000), (128, 128, 128), (129, 64, 256), (257, 1024, 96), (300, 72, 520),
         (513, 200, 264), (1000, 520, 384), (128, 4160, 256)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_linear_sizes(dtype, rows, k, n):
    act = R.ACTS[(rows + k + n) % 6]
    x, w = _rand(1, rows, k, dtype=dtype), _rand(2, n, k, scale=k ** -0.5, dtype=dtype)
    b, r = _vec(3, n, dtype), _rand(4, rows, n, dtype=dtype)
    _check_linear(x, w, None, "none", None, L.linear(x, w))
    y, saved = L.linear(x, w, b, act, r, save=True)
    _check_linear(x, w, b, act, r, y, saved)
    assert torch.equal(y, L.linear(x, w, b, act, r)), "y differs with and without saving"


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("rows", [3, 200])
def test_linear_activations(dtype, act, rows):
    x, w = _rand(1, rows, 96, scale=3.0, dtype=dtype), _rand(2, 160, 96, scale=0.3, dtype=dtype)
    b = _vec(3, 160, dtype, 2.0)
    y, saved = L.linear(x, w, b, act, save=True)
    _check_linear(x, w, b, act, None, y, saved)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (3, 5), (16, 8), (4, 4)])
@pytest.mark.parametrize("rows", [4, 150])
def test_strides_and_addresses(dtype, pad, shift, rows):
    """Rows apart by any stride, starting at any element; nothing outside the outputs is written."""
    k, n = 136, 144
    kw = dict(dtype=dtype, pad=pad, shift=shift)
    x, w, r = _rand(1, rows, k, **kw), _rand(2, n, k, scale=0.1, **kw), _rand(4, rows, n, **kw)
    b = _vec(3, n, dtype)
    out = _rand(5, rows, n, **kw)
    whole = out._base if out._base is not None else out
    before = whole.clone()
    y = L.linear(x, w, b, "silu", r, out=out)
    assert y.data_ptr() == out.data_ptr()
    _check_linear(x, w, b, "silu", r, out)
    hole = torch.ones_like(whole, dtype=torch.bool)
    hole[shift:shift + rows * (n + pad)].view(rows, n + pad)[:, :n] = False
    assert torch.equal(whole[hole].nan_to_num(7.0), before[hole].nan_to_num(7.0)), "written outside the output"
    dy = _rand(6, rows, n, scale=1e-2, **kw)
    _check_grad_input(dy, w, "none", None, L.linear_grad_input(dy, w, out=_rand(7, rows, k, **kw)))
    dw, db = L.linear_grad_weight(dy, x, bias=True, out=_rand(8, n, k, **kw))
    _check_grad_weight(dy, _d(x), dw, db)
    p = L.pack8(x)
    q, e = R.pack(_d(x))
    assert torch.equal(p.q.cpu(), q) and torch.equal(p.e.cpu(), e)
    qq = torch.empty(rows * (k + pad) + shift, dtype=torch.int8, device="cuda")[shift:].view(rows, k + pad)[:, :k]
    qq.copy_(p.q)
    s = L.Packed8(qq, p.e)
    assert torch.equal(L.unpack8(s, dtype=dtype).double().cpu(), R.unpack(q, e))
    _check_grad_input(dy, w, "gelu", s, L.linear_grad_input(dy, w, "gelu", s))
    dw, _ = L.linear_grad_weight(dy, s)
    _check_grad_weight(dy, R.unpack(q, e), dw, None)


def _check_grad_input(dy, w, act, saved, dx):
    a, b = _d(dy), _d(w)
    ref, mag = a @ b, a.abs() @ b.abs()
    err = R.sum_error(mag, dy.dtype, dy.shape[-1])
    if act != "none":
        h = R.unpack(saved.q, saved.e)
        f = R.slope(act, h)
        # the slope's own error: 4e-6 of 1 + |h|, as for the activation
        err = err * f.abs() + ref.abs() * 4e-6 * (1 + h.abs())
        ref = ref * f
    _near(dx, ref, R.rounding(dy.dtype) * ref.abs() * 1.01 + err + 1e-30, "dx")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_grad_input_sizes(dtype, rows, k, n):
    dy, w = _rand(1, rows, n, scale=1e-2, dtype=dtype), _rand(2, n, k, scale=n ** -0.5, dtype=dtype)
    _check_grad_input(dy, w, "none", None, L.linear_grad_input(dy, w))
    act = R.ACTS[1 + (rows + k + n) % 5]
    saved = L.pack8(_rand(3, rows, k, scale=2.0, dtype=dtype))
    _check_grad_input(dy, w, act, saved, L.linear_grad_input(dy, w, act, saved))


def _check_grad_weight(dy, x, dw, db, old=None, old_b=None):
    """x: float64, as the product takes it"""
    a = _d(dy)
    rows = a.shape[0]
    ref, mag = a.T @ x, a.abs().T @ x.abs()
    err = R.sum_error(mag, dy.dtype, rows)
    if old is not None:
        ref = ref + old
        err = err + 2.0 ** -23 * old.abs()
    _near(dw, ref, R.rounding(dy.dtype) * ref.abs() * 1.01 + err + 1e-30, "dw")
    if db is not None:
        ref, mag = a.sum(0), a.abs().sum(0)
        if old_b is not None:
            ref, mag = ref + old_b, mag + old_b.abs()
        tol = R.rounding(dy.dtype) * ref.abs() * 1.01 + R.sum_error(mag, F32, rows) + 1e-30
        _near(db, ref, tol, "db")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_grad_weight_sizes(dtype, rows, k, n):
    dy, x = _rand(1, rows, n, scale=1e-2, dtype=dtype), _rand(2, rows, k, scale=2.0, dtype=dtype)
    dw, db = L.linear_grad_weight(dy, x, bias=True)
    _check_grad_weight(dy, _d(x), dw, db)
    dw, db = L.linear_grad_weight(dy, x)
    assert db is None
    # from 8 bits, through an activation, added to what was there
    p = L.pack8(x)
    act = R.ACTS[(rows + k + n) % 6]
    xs = L.unpack8(p, act, dtype)
    v = R.unpack(p.q, p.e)
    ref = R.act(act, v)
    _near(xs, ref, R.rounding(dtype) * ref.abs() * 1.01 + 4e-6 * v.abs() + 1e-30, "x through its activation")
    old, old_b = _rand(4, n, k, scale=0.05, dtype=dtype), _vec(5, n, dtype)
    out, bout = old.clone(), old_b.clone()
    dw, db = L.linear_grad_weight(dy, p, act, bias=True, out=out, bias_out=bout, accumulate=True)
    assert dw.data_ptr() == out.data_ptr() and db.data_ptr() == bout.data_ptr()
    # x^ as the product takes it may differ from unpack8's by the activation's own error, which a rounding to bf16
    # can turn into one unit in its last place
    a, slack = _d(dy).abs(), (2.0 ** -7 if dtype == BF else 2.0 ** -23) * _d(xs).abs() + 4e-6 * v.abs()
    if act in ("none", "relu"):
        slack = torch.zeros_like(slack)
    _check_near_weight(dy, _d(xs), dw, _d(old), a.T @ slack)
    ref = _d(dy).sum(0) + _d(old_b)
    tol = R.rounding(dtype) * ref.abs() * 1.01 + R.sum_error(a.sum(0) + _d(old_b).abs(), F32, rows) + 1e-30
    _near(db, ref, tol, "db")


def _check_near_weight(dy, x, dw, old, slack):
    a = _d(dy)
    ref = a.T @ x + old
    err = R.sum_error(a.abs().T @ x.abs(), dy.dtype, a.shape[0]) + 2.0 ** -23 * old.abs() + slack
    _near(dw, ref, R.rounding(dy.dtype) * ref.abs() * 1.01 + err + 1e-30, "dw")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_empty_sizes(dtype):
    def z(*s):
        return torch.zeros(*s, dtype=dtype, device="cuda")

    b = _vec(1, 24, dtype)
    assert L.linear(z(0, 16), z(24, 16), b).shape == (0, 24)
    assert L.linear(z(5, 16), z(0, 16)).shape == (5, 0)
    y, s = L.linear(z(5, 0), z(24, 0), b, "relu", save=True)
    assert torch.equal(y, torch.relu(b).expand(5, 24))
    q, e = R.pack(_d(b).expand(5, 24))
    assert torch.equal(s.q.cpu(), q) and torch.equal(s.e.cpu(), e)
    assert torch.equal(L.linear_grad_input(z(5, 0), z(0, 16)), z(5, 16))
    assert L.linear_grad_input(z(0, 24), z(24, 16)).shape == (0, 16)
    for x in (z(0, 16), L.pack8(z(0, 16))):
        out, bout = _rand(2, 24, 16, dtype=dtype), _vec(3, 24, dtype)
        a, c = out.clone(), bout.clone()
        L.linear_grad_weight(z(0, 24), x, bias=True, out=out, bias_out=bout, accumulate=True)
        assert torch.equal(out, a) and torch.equal(bout, c)
        dw, db = L.linear_grad_weight(z(0, 24), x, bias=True)
        assert not dw.any() and not db.any()
    dw, db = L.linear_grad_weight(b.expand(7, 24).contiguous(), z(7, 0), bias=True)
    assert dw.shape == (24, 0)
    _near(db, 7 * _d(b), R.rounding(dtype) * 7 * _d(b).abs() * 1.01 + 8 * 2.0 ** -24 * 7 * _d(b).abs(), "db")
    assert L.unpack8(L.pack8(z(0, 40)), "silu", dtype).shape == (0, 40)
    assert L.pack8(z(3, 0)).e.shape == (3, 0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (2, 32), (7, 33), (64, 48), (257, 1024), (5, 8191), (700, 96)])
def test_pack_exact(dtype, rows, cols):
    """Every bit of q and e, over magnitudes from below the smallest step to the largest numbers."""
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    power = torch.randint(-140, 128, (rows, (cols + 31) // 32), generator=g, device="cuda").float()
    x = torch.ldexp(x.clamp(-0.999, 0.999), power.repeat_interleave(32, 1)[:, :cols]).to(dtype)
    x[torch.rand(rows, cols, generator=g, device="cuda") < 0.05] = 0.0
    p = L.pack8(x)
    q, e = R.pack(_d(x))
    assert torch.equal(p.e.cpu(), e)
    assert torch.equal(p.q.cpu(), q)
    for dt in (BF, F32):
        assert torch.equal(L.unpack8(p, dtype=dt).double().cpu(), R.unpack(q, e)), dt


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pack_thresholds(dtype):
    """Largest values around 127.5 steps, where the step doubles, and ties to even."""
    tops = torch.tensor([127.0, 127.5, 128.0, 126.5, 64.0, 63.5, 127.49, 127.51, 254.0, 255.0, 1.0])
    x = torch.zeros(len(tops), 32)
    x[:, 5] = -tops
    x[:, 6:16] = torch.tensor([0.5, 1.5, 2.5, -0.5, -1.5, 3.5, 63.5, 62.5, -62.5, 0.25])
    x = x.to(dtype).cuda()
    p = L.pack8(x)
    q, e = R.pack(_d(x))
    assert torch.equal(p.e.cpu(), e) and torch.equal(p.q.cpu(), q)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pack_infinities_and_nan(dtype):
    x = _rand(1, 6, 100, dtype=dtype).clone()
    x[1, 3], x[2, 40], x[3, 70], x[3, 71], x[4, 99] = float("inf"), float("nan"), -float("inf"), float("nan"), -float("inf")
    p = L.pack8(x)
    back = L.unpack8(p, dtype=dtype)
    q, e = R.pack(_d(x).nan_to_num(0, 0, 0))
    ref = R.unpack(q, e)
    for r, grp in ((1, 0), (2, 1), (3, 2), (4, 3)):
        assert int(p.e[r, grp]) == 255
        ref[r, 32 * grp:32 * grp + 32] = float("nan")
    ref[1, 3], ref[3, 70], ref[4, 99] = float("inf"), -float("inf"), -float("inf")
    got = back.double().cpu()
    assert torch.equal(got.nan_to_num(1e30, 2e30, 3e30), ref.nan_to_num(1e30, 2e30, 3e30))
    # through the products: poisoned rows and columns, and no others
    w = _rand(2, 40, 100, scale=0.1, dtype=dtype)
    y, s = L.linear(x, w, save=True)
    bad = ~torch.isfinite(y).all(1)
    assert bad.tolist() == [False, True, True, True, True, False]
    assert torch.isfinite(y[~bad]).all() and (s.e[bad] == 255).all() and (s.e[~bad] < 255).all()
    dw, _ = L.linear_grad_weight(_rand(3, 6, 40, dtype=dtype), p)
    cols = torch.isfinite(dw).all(0)
    assert torch.equal(cols.cpu(), torch.isfinite(ref).all(0))


@pytest.mark.parametrize("rows,k,n", [(40, 200, 300), (300, 520, 392), (1030, 4160, 136)])
def test_f32_infinities_and_nan_as_in_the_definition(rows, k, n):
    """Infinities and NaN in fp32 operands, and products that overflow: finite, infinite (of the same sign) and NaN
    where the definition's sums are, at sizes for the fp32 units and for the tensor cores."""
    x, w, dy = _rand(1, rows, k, dtype=F32), _rand(2, n, k, dtype=F32), _rand(3, rows, n, dtype=F32)
    x[5, 7], x[9, 3], x[9, 4], x[11, 0] = float("inf"), float("inf"), -float("inf"), float("nan")
    w[:, 7] = w[:, 7].abs() + 0.5  # no infinity meets a 0
    w[:, 3:5] = w[:, 3:5].abs() + 0.5
    w[20, 9], dy[7, 20], dy[8, 20] = -float("inf"), 3.0, 1.0

    def same(got, ref):
        got, ref = got.double().cpu(), ref.double()
        assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isposinf(), ref.isposinf())
        assert torch.equal(got.isneginf(), ref.isneginf())
        fine = torch.isfinite(ref)
        size = ref[fine].abs().max()
        assert bool(((got - ref)[fine].abs() <= 1e-4 * size).all())

    same(L.linear(x, w), _d(x) @ _d(w).T)
    same(L.linear_grad_input(dy, w), _d(dy) @ _d(w))
    same(L.linear_grad_weight(dy, x)[0], _d(dy).T @ _d(x))
    big = torch.zeros(rows, k, device="cuda")
    big[:, ::8] = 3e38
    pos = w.nan_to_num(1.0, 1.0, 1.0).abs() + 1.0
    y = L.linear(big, pos)
    assert bool(y.isposinf().all())  # at least 3e38 (1 + ... ) more than twice
    assert bool(torch.isfinite(L.linear(big * 1e-5, pos)).all())
    assert L.poll_errors() == 0


@pytest.mark.parametrize("rows,k,n", [(600, 896, 1000), (2100, 333, 515), (65, 5000, 2049)])
def test_f32_small_and_large_values(rows, k, n):
    """fp32 accuracy whatever the scale: each value in bits that one bf16 does not hold, rows scaled by powers of two."""
    g = torch.Generator(device="cuda").manual_seed(5)
    scale = torch.ldexp(torch.ones(rows, 1, device="cuda"), torch.randint(-60, 60, (rows, 1), generator=g, device="cuda"))
    x = _rand(1, rows, k, dtype=F32) * scale
    w, dy = _rand(2, n, k, dtype=F32), _rand(3, rows, n, dtype=F32)
    _check_linear(x, w, None, "none", None, L.linear(x, w))
    _check_grad_input(dy * scale, w, "none", None, L.linear_grad_input(dy * scale, w))
    _check_grad_weight(dy, _d(x / scale), L.linear_grad_weight(dy, x / scale)[0], None)
    assert L.poll_errors() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", R.ACTS)
def test_slopes_by_formula_and_by_differences(dtype, act):
    """act_grad8 with dy = 1: act' at the saved values, by its formula and by central differences of the activation
    (error h^2 / 6 of a third derivative below 8, and 1e-16 / h of rounding; away from relu's corner)."""
    x = torch.linspace(-12.0, 12.0, 33 * 64, device="cuda").view(33, 64)
    p = L.pack8(x.to(dtype))
    one = torch.ones(33, 64, dtype=dtype, device="cuda")
    got = L.act_grad8(one, p, act)
    h = R.unpack(p.q, p.e)
    ref = R.slope(act, h)
    tol = R.rounding(dtype) * ref.abs() * 1.01 + 4e-6 * (1 + h.abs())
    _near(got, ref, tol, "slope")
    d = 1e-5
    diff = (R.act(act, h + d) - R.act(act, h - d)) / (2 * d)
    away = h.abs() > 2 * d
    _near(got.cpu()[away], diff[away], (tol + 8 * d * d / 6 + 1e-9)[away], "slope by differences")
    val = L.unpack8(p, act, dtype)
    ref = R.act(act, h)
    _near(val, ref, R.rounding(dtype) * ref.abs() * 1.01 + 4e-6 * h.abs() + 1e-30, "value")


def test_slopes_at_huge_values_are_their_limits():
    x = torch.tensor([[1e30, -1e30, 3e38, -3e38] + [0.0] * 28, [float("inf")] * 32, [float("nan")] * 32], device="cuda")
    p = L.pack8(x)
    for act in R.ACTS[1:]:
        s = L.act_grad8(torch.ones_like(x), p, act).cpu()
        assert s[0, :4].tolist()[2:] == [1.0, 0.0], act
        assert (s[1] == 1.0).all() and s[2].isnan().all(), act


@pytest.mark.parametrize("dtype", [BF, F32])
def test_gradients_by_differences(dtype):
    """d/dt of sum(dy * layer) along random directions of x and W, in 64 bits by central differences of the forward
    pass's definition, against the operators' gradients at h^ = h (h chosen to be exact in 8 bits)."""
    rows, k, n = 40, 64, 48
    h0 = torch.randint(-127, 128, (rows, k), generator=torch.Generator().manual_seed(1)).double() / 64
    h0[:, ::32] = 127 / 64  # every group's step is 1 / 64
    saved = L.pack8(h0.to(F32).cuda())
    assert torch.equal(R.unpack(saved.q, saved.e), h0)
    w, dy = _rand(2, n, k, dtype=dtype), _rand(3, rows, n, dtype=dtype)
    g = torch.Generator().manual_seed(4)
    for act in R.ACTS[2:]:
        dx = L.linear_grad_input(dy, w, act, saved)
        dw, db = L.linear_grad_weight(dy, saved, act, bias=True)

        def f(h, ww, b):
            return float(((R.act(act, h) @ ww.T + b) * _d(dy)).sum())

        dh, dww, dbb = torch.randn(rows, k, generator=g).double(), torch.randn(n, k, generator=g).double(), \
            torch.randn(n, generator=g).double()
        t, zero = 1e-4, torch.zeros(n, dtype=torch.float64)
        for got, step, size in (((_d(dx) * dh).sum(), (dh, 0 * dww, zero), (_d(dx).abs() * dh.abs()).sum()),
                                ((_d(dw) * dww).sum(), (0 * dh, dww, zero), (_d(dw).abs() * dww.abs()).sum()),
                                ((_d(db) * dbb).sum(), (0 * dh, 0 * dww, dbb), (_d(db).abs() * dbb.abs()).sum())):
            num = (f(h0 + t * step[0], _d(w) + t * step[1], t * step[2])
                   - f(h0 - t * step[0], _d(w) - t * step[1], -t * step[2])) / (2 * t)
            # one rounding of each gradient value (three for dW: its input's too), t^2 of the third derivative
            tol = (4 * R.rounding(dtype) + 1e-5 + t * t * 8) * float(size)
            assert abs(float(got) - num) <= tol, (act, float(got), num, tol)


def test_leading_dimensions_views_and_vectors():
    x = _rand(1, 6 * 7, 64).view(6, 7, 64)
    w, b = _rand(2, 96, 64, scale=0.1), _vec(3, 96, BF)
    y, s = L.linear(x, w, b, "gelu", save=True)
    assert y.shape == (6, 7, 96) and s.shape == (6, 7, 96) and s.e.shape == (6, 7, 3)
    flat = L.linear(x.reshape(42, 64), w, b, "gelu")
    assert torch.equal(y.reshape(42, 96), flat)
    assert torch.equal(L.linear(x[2, 3], w, b, "gelu"), flat[17])
    # slices of one joint projection, in place of one another's neighbours
    joint = torch.zeros(42, 3 * 96, dtype=BF, device="cuda")
    for i in range(3):
        L.linear(x.reshape(42, 64), w, b, "gelu", out=joint[:, 96 * i:96 * i + 96])
    assert torch.equal(joint, flat.repeat(1, 3))
    # out is the residual
    r = _rand(5, 42, 96)
    ref = L.linear(x.reshape(42, 64), w, b, "gelu", r)
    z = r.clone()
    L.linear(x.reshape(42, 64), w, b, "gelu", z, out=z)
    assert torch.equal(z, ref)
    wide = _rand(6, 6 * 7, 200).view(6, 7, 200)[:, :, 8:72]
    assert torch.equal(L.linear(wide, w), L.linear(wide.contiguous(), w))


@pytest.mark.parametrize("rows,k,n", [(1, 2048, 512), (40, 512, 640), (600, 1024, 512), (2000, 256, 256)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_same_result_every_time(dtype, rows, k, n):
    x, w, dy = _rand(1, rows, k, dtype=dtype), _rand(2, n, k, dtype=dtype), _rand(3, rows, n, dtype=dtype)
    p = L.pack8(x)

    def once():
        y, s = L.linear(x, w, save=True)
        return (y, s.q, s.e, L.linear_grad_input(dy, w, "silu", p), *L.linear_grad_weight(dy, p, "silu", bias=True))

    first = once()
    for _ in range(5):
        for a, b in zip(first, once()):
            assert torch.equal(a, b)


def test_rows_do_not_depend_on_one_another():
    """A row's result does not depend on what the other rows hold (bitwise, for one number of rows)."""
    x, w = _rand(1, 300, 256), _rand(2, 512, 256, scale=0.1)
    y = L.linear(x, w, act="silu")
    z = x.clone()
    z[::2] = float("nan")
    z[1::4] = 1e30
    assert torch.equal(L.linear(z, w, act="silu")[3::4], y[3::4])


def test_other_stream():
    s = torch.cuda.Stream()
    x, w, dy = _rand(1, 700, 512), _rand(2, 640, 512, scale=0.1), _rand(3, 700, 640)
    ref = [L.linear(x, w, act="silu", save=True), L.linear_grad_input(dy, w), L.linear_grad_weight(dy, x, bias=True)]
    p_ref = L.pack8(x)
    torch.cuda.synchronize()
    for _ in range(3):
        s.wait_stream(torch.cuda.current_stream())
        y, h = L.linear(x, w, act="silu", save=True, stream=s)
        dx = L.linear_grad_input(dy, w, stream=s)
        p = L.pack8(x, stream=s)
        dw, db = L.linear_grad_weight(dy, p, bias=True, stream=s)
        v = L.unpack8(h, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(y, ref[0][0]) and torch.equal(h.q, ref[0][1].q) and torch.equal(h.e, ref[0][1].e)
        assert torch.equal(dx, ref[1]) and torch.equal(db, ref[2][1]) and torch.equal(p.q, p_ref.q)
        assert torch.equal(v, L.unpack8(ref[0][1])) and torch.equal(dw, L.linear_grad_weight(dy, p_ref)[0])


def test_under_graph_capture():
    x, w, r = _rand(1, 300, 512), _rand(2, 640, 512, scale=0.1), _rand(3, 300, 640)
    y, dw = torch.empty(300, 640, dtype=BF, device="cuda"), torch.empty(640, 512, dtype=BF, device="cuda")
    L.linear(x, w, residual=r, out=y)
    L.linear_grad_weight(r, L.pack8(x), out=dw)
    ref = (y.clone(), dw.clone())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.linear(x, w, residual=r, out=y)
        L.linear_grad_weight(r, L.pack8(x), out=dw)
    y.zero_(), dw.zero_()
    g.replay()
    assert torch.equal(y, ref[0]) and torch.equal(dw, ref[1])
    x2 = _rand(9, 300, 512)
    x.copy_(x2)
    g.replay()
    assert torch.equal(y, L.linear(x2, w, residual=r))


def test_offsets_past_32_bits():
    """Outputs and inputs of more than 2^32 bytes and 2^31 elements: the last rows."""
    rows, n, k = 70001, 32768, 16
    x, w = _rand(1, rows, k), _rand(2, n, k)
    y, s = L.linear(x, w, act="relu", save=True)
    for a in (0, rows // 2, rows - 3):
        one, os = L.linear(x[a:a + 3].contiguous(), w, act="relu", save=True)
        _check_linear(x[a:a + 3], w, None, "relu", None, y[a:a + 3], L.Packed8(s.q[a:a + 3], s.e[a:a + 3]))
    p = L.pack8(y)
    q, e = R.pack(_d(y[-3:]))
    assert torch.equal(p.q[-3:].cpu(), q) and torch.equal(p.e[-3:].cpu(), e)
    v = L.unpack8(p)
    assert torch.equal(_d(v[-3:]), R.unpack(q, e))
    del v
    dx = L.linear_grad_input(y, w)
    _check_grad_input(y[-3:], w, "none", None, dx[-3:])
    # a weight gradient over all rows, of which only the last two are not zero
    y[:-2] = 0
    dw, db = L.linear_grad_weight(y, x, bias=True)
    a, b = _d(y[-2:]), _d(x[-2:])
    ref, mag = a.T @ b, a.abs().T @ b.abs()
    _near(dw, ref, R.rounding(BF) * ref.abs() * 1.01 + R.sum_error(mag, BF, 2) + 1e-30, "dw")
    _near(db, a.sum(0), R.rounding(BF) * a.sum(0).abs() * 1.01 + 2.0 ** -22 * a.abs().sum(0) + 1e-30, "db")


def _refused(f, *args, **kw):
    with pytest.raises((ValueError, TypeError, S.SmatError)):
        f(*args, **kw)


def test_refusals_leave_outputs_alone():
    x, w, b = _rand(1, 8, 64), _rand(2, 32, 64), _vec(3, 32, BF)
    dy = _rand(4, 8, 32)
    out = torch.full((8, 32), 5.0, dtype=BF, device="cuda")
    _refused(L.linear, x, w.float(), out=out)
    _refused(L.linear, x, w[:, :32], out=out)
    _refused(L.linear, x, w.T, out=out)
    _refused(L.linear, x, w, b.float(), out=out)
    _refused(L.linear, x, w, b[:31], out=out)
    _refused(L.linear, x, w, act="swish", out=out)
    _refused(L.linear, x, w, residual=dy[:4], out=out)
    _refused(L.linear, x, w, residual=dy[:1].expand(8, 32), out=out)
    _refused(L.linear, x.cpu(), w, out=out)
    _refused(L.linear, x, w.cpu(), out=out)
    _refused(L.linear, x.half(), w.half())
    _refused(L.linear, x.T, w, out=out)
    _refused(L.linear, x, w, out=out[:, :16])
    _refused(L.linear, x, w, out=out.float())
    _refused(L.linear, x[:, :32], w[:, :32], out=x[:, 16:48])
    _refused(L.linear, x[:, :32], _rand(5, 32, 32), out=x[:, 16:48])
    _refused(L.linear, dy, _rand(5, 32, 32), residual=out, out=dy)
    _refused(L.linear_grad_input, dy, w, "silu")
    _refused(L.linear_grad_input, dy, w, "none", L.pack8(x))
    _refused(L.linear_grad_input, dy, w, "silu", L.pack8(dy))
    _refused(L.linear_grad_weight, dy, x, "silu")
    _refused(L.linear_grad_weight, dy, x[:4])
    _refused(L.linear_grad_weight, dy, x, accumulate=True)
    _refused(L.linear_grad_weight, dy, x, bias_out=b)
    _refused(L.linear_grad_weight, dy, L.pack8(x[:4]))
    _refused(L.unpack8, L.pack8(x), "tanh")
    _refused(L.unpack8, L.pack8(x), dtype=torch.float16)
    _refused(L.Packed8, torch.zeros(4, 40, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8))
    _refused(L.Packed8, torch.zeros(4, 40), torch.zeros(4, 2, dtype=torch.uint8))
    torch.cuda.synchronize()
    assert (out == 5.0).all()
    y = L.linear(x, w, b, out=out)  # and the next call works
    _check_linear(x, w, b, "none", None, y)


@pytest.mark.parametrize("rows,k,n", [(64, 1024, 1024), (65, 1024, 1024), (129, 515, 1031)])
def test_f32_products_around_the_size_from_which_operands_are_cut(rows, k, n):
    x, w, dy = _rand(1, rows, k, dtype=F32), _rand(2, n, k, dtype=F32), _rand(3, rows, n, dtype=F32)
    _check_linear(x, w, None, "none", None, L.linear(x, w))
    _check_grad_input(dy, w, "none", None, L.linear_grad_input(dy, w))
    _check_grad_weight(dy, _d(x), L.linear_grad_weight(dy, x)[0], None)
    assert L.poll_errors() == 0


def test_f32_infinities_and_nan_just_above_that_size():
    test_f32_infinities_and_nan_as_in_the_definition(330, 536, 392)
