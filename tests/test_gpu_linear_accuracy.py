"""How near the linear operators come to their definitions in 64 bits, with bounds that follow the arithmetic and not the
size of the sum, on the GPU: fp32 products, and the activations of both types.

fp32 products of large matrices are six of the nine products of three bf16 parts (smat_linear_f32.cu). With parts rounded to
nearest |mid| <= 2^-8 and |lo| <= 2^-17 of a value's power of two, so what is left out, mid lo + lo mid + lo lo, is at most
2^-24 (1 + 2^-9) of a product. An addition in tensor memory may cut off one unit in the last place, 2^-23 of the partial
sum; the parts' products come small ones first, so that only the last ones, of hi and hi, are added to sums of full size:
those before are below 2^-6 of it."""

import math

import pytest
import torch

import _linear_ref as R
from paper_2609_33437_gb300 import linear as L

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24  # half a unit in the last place, relative
DROPPED = U * (1 + 2.0 ** -9)


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


def _d(t):
    return t.double().cpu()


def _products(a, b):
    """forward, input's and weight's gradient, each as [i, l] times [j, l]: (name, result, A, B) of one pair."""
    return (("linear", L.linear(a, b), a, b),
            ("grad_input", L.linear_grad_input(a, b.T.contiguous()), a, b),
            ("grad_weight", L.linear_grad_weight(a.T.contiguous(), b.T.contiguous())[0], a, b))


def _single(values_a, values_b, length, at):
    """[i, length] and [j, length] whose only column that is not 0 is `at`: every result is one product."""
    a = torch.zeros(len(values_a), length, device="cuda")
    b = torch.zeros(len(values_b), length, device="cuda")
    a[:, at], b[:, at] = values_a.cuda(), values_b.cuda()
    return a, b


@pytest.mark.parametrize("length,at", [(600, 7), (1030, 1029), (5000, 2500)])
def test_f32_single_products(length, at):
    """One product per result, on the tensor cores (more than 2^26 products): what is left out, and one addition's cut."""
    g = torch.Generator().manual_seed(length)
    i, j = 400, 520
    va = (1 + torch.rand(i, generator=g)) * torch.ldexp(torch.ones(i), torch.randint(-30, 30, (i,), generator=g))
    vb = (1 + torch.rand(j, generator=g)) * torch.where(torch.rand(j, generator=g) < 0.5, -1.0, 1.0)
    va[:50] = 1.0078124  # just under a bf16 number: cut off instead of rounded, its parts are 1.0, 0.0078, 3e-5
    vb[:60] = 1.0078124
    a, b = _single(va, vb, length, at)
    ref = va.double()[:, None] * vb.double()[None, :]
    for name, got, _, _ in _products(a, b):
        off = ((_d(got) - ref) / ref).abs().max()
        assert off <= DROPPED + 2 * U * (1 + 2.0 ** -4), (name, float(off) / U)
    assert L.poll_errors() == 0


@pytest.mark.parametrize("value", [1.0078124, 1.5, 1.9960937])
def test_f32_sums_of_one_sign(value):
    """Sums whose terms are all alike, so that no error averages out. A slice of 64 adds four times 16 products of hi and hi
    (each addition cuts off up to 2^-23 of the sum so far: 1/4, 2/4, 3/4 and all of it) after 20 additions below 2^-6; the
    slices are added with one rounding each, of partial sums 1/S, 2/S, ..., and up to 8 shares."""
    i, j, length = 300, 300, 1024
    a = torch.full((i, length), value, device="cuda")
    b = torch.full((j, length), value, device="cuda")
    ref = float(length) * float(a[0, 0].double()) ** 2
    slices = length // 64
    bound = DROPPED + 2 * U * (2.5 + 20 * 2.0 ** -6) + U * ((slices + 1) / 2 + 8)
    for name, got, _, _ in _products(a, b):
        off = float(((_d(got) - ref) / ref).abs().max())
        assert off <= bound, (name, off / U, bound / U)
    assert L.poll_errors() == 0


def test_f32_products_next_to_the_largest_number():
    """Parts that are rounded up do not make infinities of products under the largest number."""
    most = torch.finfo(F32).max
    for va, vb in ((2.0 ** 64 * (1 - 2.0 ** -10), 2.0 ** 64), (2.0 ** 64 * (1 - 2.0 ** -10), 2.0 ** 64 * (1 - 2.0 ** -10)),
                   (most, 1.0), (most, -0.75), (-2.0 ** 127 * 1.9970703, 1.0), (1.0000001, most * 0.9999)):
        a, b = _single(torch.full((400,), va), torch.full((520,), vb), 600, 3)
        ref = float(a[0, 3].double() * b[0, 3].double())
        for name, got, _, _ in _products(a, b):
            assert bool(((_d(got) - ref).abs() <= (DROPPED + 2 * U * (1 + 2.0 ** -4)) * abs(ref)).all()), (name, va, vb)
    assert L.poll_errors() == 0


@pytest.mark.parametrize("rows,k,n", [(300, 520, 520), (1100, 300, 260)])
@pytest.mark.parametrize("power", [-88, -100, -118])
def test_f32_operands_that_are_small_all_over(rows, k, n, power):
    """An operand below the size at which three bf16 parts hold its bits, times one that makes up for it: fp32's bound for a
    sum, 8 sqrt(terms) + 4 roundings of the magnitudes' sum. (Values below 2^-126 have fewer bits themselves: inputs are
    normal numbers, of one sign and at least 2^power, and results are.)"""
    g = torch.Generator(device="cuda").manual_seed(power + 200)
    small = torch.ldexp(1 + torch.rand(rows, k, generator=g, device="cuda"), torch.tensor(float(power), device="cuda"))
    large = torch.ldexp(torch.randn(n, k, generator=g, device="cuda"), torch.tensor(40.0, device="cuda"))
    for a, b in ((small, large), (large, small)):
        ref, mag = _d(a) @ _d(b).T, _d(a).abs() @ _d(b).abs().T
        for name, got, _, _ in _products(a, b):
            worst = float(((_d(got) - ref).abs() / mag).max()) / U
            assert worst <= 8 * k ** 0.5 + 4, (name, worst)
    assert L.poll_errors() == 0


def test_f32_operands_of_nothing_and_of_mixed_sizes():
    """Zeros all over are 0, not small; one value of 2^-86 keeps the parts in use, and what is below them then is off by
    2^-134 of its factor at most (and the sum's roundings)."""
    zero, one = torch.zeros(300, 520, device="cuda"), torch.ones(520, 520, device="cuda")
    for name, got, _, _ in _products(zero, one):
        assert not got.any(), name
    g = torch.Generator(device="cuda").manual_seed(1)
    a = torch.ldexp(torch.randn(300, 520, generator=g, device="cuda"), torch.tensor(-116.0, device="cuda"))
    a[7, 9] = 2.0 ** -86
    b = torch.ldexp(torch.randn(520, 520, generator=g, device="cuda"), torch.tensor(40.0, device="cuda"))
    ref, mag = _d(a) @ _d(b).T, _d(a).abs() @ _d(b).abs().T
    tol = (8 * 520 ** 0.5 + 4) * U * mag + 2.0 ** -134 * _d(b).abs().sum(1)
    for name, got, _, _ in _products(a, b):
        assert bool(((_d(got) - ref).abs() <= tol).all()), name
    assert L.poll_errors() == 0


@pytest.mark.parametrize("power", [-90, -112, -120])
def test_f32_single_products_of_small_values(power):
    """As test_f32_single_products, one operand small all over: the result's bits are there all the same."""
    g = torch.Generator().manual_seed(3)
    va = torch.ldexp(1 + torch.rand(400, generator=g), torch.tensor(float(power)))
    vb = torch.ldexp(1 + torch.rand(520, generator=g), torch.tensor(40.0))
    for x, y in ((va, vb), (vb, va)):
        a, b = _single(x, y, 600, 599)
        ref = x.double()[:, None] * y.double()[None, :]
        for name, got, _, _ in _products(a, b):
            off = ((_d(got) - ref) / ref).abs().max()
            assert off <= DROPPED + 2 * U * (1 + 2.0 ** -4), (name, float(off) / U)


# Activations and slopes, relative to themselves: nothing hides behind an absolute tolerance where they are small.
# Errors in units of 2^-24, by the steps taken. fp32: expf 2 ulp (4), 1 + e (1), reciprocal 1 ulp (2), e r (1), h s (1): 9; the
# argument's own relative error, times its size: 0 for silu, 1.702 h 1.5, the tanh form's 6. GELU: polynomial with its roundings
# (5), reciprocal (2), ex2 (4) of h^2 log2(e) / 2 (a square, a constant, a product: 1.5 h^2), two products (2), 1 - s (1),
# h Phi (1): 15 + 1.5 h^2.
# bf16: ex2 2 ulp (4), 1 + e (1), reciprocal 2, product 1: 8; the exponent's relative error, times its size: its constant (1)
# and its product (1), the tanh form's four more; then the rounding to bf16.
EXPF, ARGUMENT_FULL, ARGUMENT_FAST = 9, {"silu": 0, "quick_gelu": 1.5, "gelu_tanh": 6}, {"silu": 2, "quick_gelu": 3, "gelu_tanh": 7}
GAIN = 2.0 * math.sqrt(2.0 / math.pi)


def _argument(act, h):
    return {"silu": h, "quick_gelu": 1.702 * h, "gelu_tanh": GAIN * (h + 0.044715 * h ** 3)}[act]


def _published_cdf(h):
    """Abramowitz and Stegun's 7.1.26 for Phi(-|h|), what bf16 calls' GELU goes by, in 64 bits."""
    t = 1 / (1 + 0.3275911 * h.abs() / math.sqrt(2.0))
    p = t * (0.254829592 + t * (-0.284496736 + t * (1.421413741 + t * (-1.453152027 + t * 1.061405429))))
    return 0.5 * p * torch.exp(-0.5 * h * h)


def _saved_range(low, high, dtype):
    """Values in 8 bits from low to high, and what they stand for (in groups of 32 neighbours, steps small near 0)."""
    x = torch.cat([torch.linspace(low, high, 4096), torch.linspace(low / 64, high / 64, 4096)]).view(-1, 64)
    p = L.pack8(x.to(dtype).cuda())
    return p, R.unpack(p.q, p.e)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "quick_gelu", "silu"])
def test_activations_keep_their_digits(act, dtype):
    low = {"gelu": -12.5, "gelu_tanh": -7.0, "quick_gelu": -48.0, "silu": -80.0}[act]  # down to about 2^-116
    p, h = _saved_range(low, 30.0, dtype)
    got, ref = _d(L.unpack8(p, act, dtype)), R.act(act, h)
    if act == "gelu":
        if dtype == F32:
            tol = (15 + 1.5 * h * h) * U * ref.abs()
        else:  # its published form's error; then 1 - s, polynomial (20) and exponent (its argument twice rounded)
            tail = (_published_cdf(h) - 0.5 * torch.special.erfc(h.abs() / math.sqrt(2.0))).abs() * h.abs()
            tol = tail + (24 + 3 * 0.5 * h * h) * U * ref.abs()
    else:
        x = _argument(act, h).abs()
        tol = (EXPF + x * (ARGUMENT_FULL if dtype == F32 else ARGUMENT_FAST)[act]) * U * ref.abs()
    if dtype == BF:
        tol = tol * 1.01 + R.rounding(BF) * ref.abs()
    bad = (got - ref).abs() > tol
    assert not bool(bad.any()), (h[bad][0].item(), got[bad][0].item(), ref[bad][0].item(), int(bad.sum()))
    # a product's epilogue applies the same function: times the unit matrix, in few rows and in many
    x, y = L.unpack8(p, dtype=dtype).view(16, 512), L.unpack8(p, act, dtype).view(16, 512)
    eye = torch.eye(512, device="cuda", dtype=dtype)
    for rows in (1, 2, 16, 40, 640):
        reps = -(-rows // 16)
        assert torch.equal(L.linear(x.repeat(reps, 1)[:rows], eye, act=act), y.repeat(reps, 1)[:rows]), rows


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "quick_gelu", "silu"])
def test_f32_slopes_keep_their_digits(act):
    """s + c h s (1 - s) (Phi + h phi): relative to the two terms' magnitudes, since they may cancel. The second term has the
    first's exponential, one more factor s (1 + 2 + 2) and its own products (3)."""
    low = {"gelu": -12.5, "gelu_tanh": -7.0, "quick_gelu": -48.0, "silu": -80.0}[act]
    p, h = _saved_range(low, 30.0, F32)
    got = _d(L.act_grad8(torch.ones(p.shape, device="cuda"), p, act))
    if act == "gelu":
        first, second = 0.5 * torch.special.erfc(-h / math.sqrt(2.0)), h * torch.exp(-0.5 * h * h) / math.sqrt(2 * math.pi)
        tol = (15 + 1.5 * h * h) * U * first + (4 + 4 + 1.5 * h * h) * U * second.abs()
    else:
        x = _argument(act, h)
        s = torch.sigmoid(x)
        by = {"silu": h, "quick_gelu": 1.702 * h, "gelu_tanh": GAIN * h * (1 + 3 * 0.044715 * h * h)}[act]
        first, second = s, by * s * torch.sigmoid(-x)
        tol = (EXPF + x.abs() * ARGUMENT_FULL[act]) * U * (first + second.abs()) + 12 * U * second.abs()
    ref = first + second
    tol = tol + U * ref.abs()
    bad = (got - ref).abs() > tol
    assert not bool(bad.any()), (h[bad][0].item(), got[bad][0].item(), ref[bad][0].item(), int(bad.sum()))
