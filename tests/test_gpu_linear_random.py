"""The linear operators over random sizes, row strides and offsets, options and types, against their definitions in 64 bits:
operands lie in buffers of NaN, results in wider buffers of which nothing else may change. Bounds as in test_gpu_linear."""

import math
import random

import pytest
import torch

import _linear_ref as R
import test_gpu_linear as T
from paper_2609_33437_gb300 import linear as L

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


class Draw:
    def __init__(self, seed):
        self.r, self.seed = random.Random(seed), 1000 * seed

    def size(self, most):
        """Spread over its logarithm; odd ones, and multiples of 8 to 128."""
        v, step = round(math.exp(self.r.uniform(0, math.log(most)))), self.r.choice((1, 1, 1, 8, 32, 64, 128))
        return max(1, min(most, (v + step // 2) // step * step or v))

    def place(self):
        return dict(pad=self.r.choice((0, 0, 1, 3, 8, 16, 40)), shift=self.r.choice((0, 0, 1, 2, 4, 8)))

    def matrix(self, rows, cols, dtype, scale=1.0):
        self.seed += 1
        return T._rand(self.seed, rows, cols, scale=scale, dtype=dtype, **self.place())

    def result(self, rows, cols, dtype):
        """A place for a result, and a check that nothing around it has changed."""
        at = self.place()
        ld, shift = cols + at["pad"], at["shift"]
        flat = torch.full((rows * ld + shift + 8,), 7.0, device="cuda").to(dtype)
        out = flat[shift:shift + rows * ld].view(rows, ld)[:, :cols]

        def untouched():
            keep = flat.clone()
            keep[shift:shift + rows * ld].view(rows, ld)[:, :cols] = 7.0
            return bool((keep == 7.0).all())

        return out, untouched

    def packed(self, x):
        """x in 8 bits, exact against the definition; half the time in buffers of other strides and offsets."""
        p = L.pack8(x)
        q, e = R.pack(T._d(x))
        assert torch.equal(p.q.cpu(), q) and torch.equal(p.e.cpu(), e)
        if self.r.random() < 0.5:
            return p
        (rows, cols), groups = p.shape, p.e.shape[1]
        pad, shift = self.r.choice((0, 1, 8, 16)), self.r.choice((0, 1, 8, 16))
        q = torch.zeros(rows * (cols + pad) + shift, dtype=torch.int8, device="cuda")[shift:].view(rows, cols + pad)[:, :cols]
        e = torch.zeros(rows, groups + 3, dtype=torch.uint8, device="cuda")[:, 1:1 + groups]
        return L.Packed8(q.copy_(p.q), e.copy_(p.e))


def _linear(d, dtype, rows, k, n, act):
    x, w = d.matrix(rows, k, dtype), d.matrix(n, k, dtype, k ** -0.5)
    b = T._vec(d.seed, n + 1, dtype)[d.r.randrange(2):][:n] if d.r.random() < 0.5 else None
    residual, save = d.matrix(rows, n, dtype) if d.r.random() < 0.5 else None, d.r.random() < 0.5
    out, untouched = d.result(rows, n, dtype)
    got = L.linear(x, w, b, act, residual, save=save, out=out)
    T._check_linear(x, w, b, act, residual, *(got if save else (got, None)))
    assert untouched()


def _grad_input(d, dtype, rows, k, n, act):
    dy, w = d.matrix(rows, n, dtype, 1e-2), d.matrix(n, k, dtype, n ** -0.5)
    saved = d.packed(d.matrix(rows, k, dtype, 2.0)) if act != "none" else None
    out, untouched = d.result(rows, k, dtype)
    T._check_grad_input(dy, w, act, saved, L.linear_grad_input(dy, w, act, saved, out=out))
    assert untouched()


def _grad_weight(d, dtype, rows, k, n, act):
    dy, x = d.matrix(rows, n, dtype, 1e-2), d.matrix(rows, k, dtype, 2.0)
    bias, add = d.r.random() < 0.6, d.r.random() < 0.4
    out, untouched = d.result(n, k, dtype)
    old = torch.zeros(n, k, dtype=torch.float64)
    if add:
        out.copy_(d.matrix(n, k, dtype, 0.05))
        old = T._d(out)
    if d.r.random() < 0.6:
        p = d.packed(x)
        dw, db = L.linear_grad_weight(dy, p, act, bias=bias, out=out, accumulate=add)
        # x^ may differ from unpack8's by the activation's own error, which a rounding can turn into a last place
        xs, v = T._d(L.unpack8(p, act, dtype)), R.unpack(p.q, p.e)
        slack = (2.0 ** -7 if dtype == BF else 2.0 ** -23) * xs.abs() + 4e-6 * v.abs()
        T._check_near_weight(dy, xs, dw, old, T._d(dy).abs().T @ (slack if act not in ("none", "relu") else 0 * slack))
    else:
        dw, db = L.linear_grad_weight(dy, x, bias=bias, out=out, accumulate=add)
        T._check_grad_weight(dy, T._d(x), dw, None, old=old)
    if bias:
        a = T._d(dy)
        T._near(db, a.sum(0), R.rounding(dtype) * a.sum(0).abs() * 1.01 + R.sum_error(a.abs().sum(0), F32, rows) + 1e-30, "db")
    assert untouched()


def _elementwise(d, dtype, rows, k, n, act):
    p, other = d.packed(d.matrix(rows, k, dtype, 2.0)), d.r.choice((BF, F32))
    h, dy = R.unpack(p.q, p.e), d.matrix(rows, k, other)
    for got, ref, error in ((lambda out: L.unpack8(p, act, other, out=out), R.act(act, h), h.abs()),
                            (lambda out: L.act_grad8(dy, p, act, out=out), T._d(dy) * R.slope(act, h),
                             (1 + h.abs()) * T._d(dy).abs())):
        out, untouched = d.result(rows, k, other)
        T._near(got(out), ref, R.rounding(other) * ref.abs() * 1.01 + 4e-6 * error + 1e-30, act)
        assert untouched()


@pytest.mark.parametrize("seed", range(24))
def test_random_calls(seed):
    d = Draw(seed)
    for _ in range(25):
        op = d.r.choice((_linear, _grad_input, _grad_weight, _elementwise))
        dtype, act = d.r.choice((BF, BF, F32)), d.r.choice(R.ACTS)
        rows, k, n = d.size(1500), d.size(1500), d.size(1500)
        if rows * k * n <= 2e8:
            try:
                op(d, dtype, rows, k, n, act)
            except AssertionError as e:
                raise AssertionError(f"{op.__name__} {dtype} rows {rows} k {k} n {n} {act}: {e}") from e
    assert L.poll_errors() == 0
