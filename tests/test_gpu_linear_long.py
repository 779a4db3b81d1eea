"""The longest sums that the linear operators accept, and tiles in several rounds with everything that an epilogue reads."""

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


def test_the_longest_sum_is_finished():
    """2^31 - 2^16 rows, the most there may be: a share of the sum takes longer than the two seconds that a wait inside the
    product has for one slice. All rows are 0 but a few in every share, whose products are whole numbers: the sums are exact."""
    rows, n, k = (1 << 31) - (1 << 16), 8, 8
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    dy, x = torch.zeros(rows, n, dtype=BF, device="cuda"), torch.zeros(rows, k, dtype=BF, device="cuda")
    at = torch.tensor([0, 1, rows // 5, rows // 2 - 1, rows // 2, rows // 4 * 3 + 7, rows - 65, rows - 1], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    dy[at] = torch.randint(-8, 9, (len(at), n), generator=g, device="cuda").to(BF)
    x[at] = torch.randint(-8, 9, (len(at), k), generator=g, device="cuda").to(BF)
    dw, _ = L.linear_grad_weight(dy, x)
    assert L.poll_errors() == 0
    ref = dy[at].double().T @ x[at].double()
    assert torch.equal(dw.double(), ref.to(BF).double())


# 17 x 17 tiles of 256 x 256 and more of the smaller ones, where 76 pairs or 152 single CTAs work at once: every warp's space
# for what comes in and goes out is used in turn. Widths off 16 bytes take the warps' own copies.
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("wide", [4104, 4101])
def test_tiles_in_several_rounds(dtype, wide):
    rows, short, act = 4200, 72, "silu"
    x, w = T._rand(1, rows, short, dtype=dtype), T._rand(2, wide, short, scale=short ** -0.5, dtype=dtype)
    b, r = T._vec(3, wide, dtype), T._rand(4, rows, wide, dtype=dtype)
    y, saved = L.linear(x, w, b, act, r, save=True)
    T._check_linear(x, w, b, act, r, y, saved)
    out = r.clone()
    assert torch.equal(L.linear(x, w, b, act, out, out=out), y)  # added to in place
    # back through an activation
    dy, w = T._rand(5, rows, short, scale=1e-2, dtype=dtype), T._rand(6, short, wide, scale=short ** -0.5, dtype=dtype)
    T._check_grad_input(dy, w, "gelu", saved, L.linear_grad_input(dy, w, "gelu", saved))
    # an older gradient added to
    dy, x = T._rand(7, short, rows, scale=1e-2, dtype=dtype), T._rand(8, short, wide, dtype=dtype)
    old = T._rand(9, rows, wide, scale=0.05, dtype=dtype)
    dw, _ = L.linear_grad_weight(dy, x, out=old.clone(), accumulate=True)
    T._check_grad_weight(dy, T._d(x), dw, None, old=T._d(old))
    assert L.poll_errors() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("rows,cols,pad,shift", [(37, 333, 0, 0), (3, 33, 1, 3), (5, 31, 0, 1), (130, 1100, 8, 4), (7, 4097, 3, 0),
                                                 (64, 96, 0, 0)])
def test_slopes_over_rows_off_every_boundary(dtype, act, rows, cols, pad, shift):
    """act_grad8 with a gradient and a result whose rows start anywhere: dy * act'(h^), one rounding and the slope's own
    error (4e-6 of 1 + |h|), and nothing written outside."""
    kw = dict(dtype=dtype, pad=pad, shift=shift)
    dy, saved = T._rand(1, rows, cols, **kw), L.pack8(T._rand(2, rows, cols, scale=2.0, dtype=dtype))
    h = R.unpack(saved.q, saved.e)
    ref = T._d(dy) * R.slope(act, h)
    tol = R.rounding(dtype) * ref.abs() * 1.01 + 4e-6 * (1 + h.abs()) * T._d(dy).abs() + 1e-30
    flat = torch.full((rows * (cols + pad) + shift + 8,), 7.0, dtype=dtype, device="cuda")
    out = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    got = L.act_grad8(dy, saved, act, out=out)
    T._near(got, ref, tol, "dh")
    T._near(L.act_grad8(dy, saved, act), ref, tol, "dh in memory of its own")
    out.fill_(7.0)
    assert bool((flat == 7.0).all())
