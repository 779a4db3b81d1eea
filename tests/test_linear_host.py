"""CPU-only checks of the linear layers' part of the C ABI and of its binding: what is refused on the host, before
anything reaches a GPU. Pointers here are numbers; none is read."""

import pytest
import torch

import _linear_ref as R
from paper_2609_33437_gb300 import linear as L
from paper_2609_33437_gb300 import smat as S

INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE, CUDA = 1, 2, 3, 4, 6
BASE = 0x10000000


@pytest.fixture(scope="module")
def lib():
    return S.load_library()


def _linear(**kw):
    v = dict(x=BASE, w=2 * BASE, bias=0, residual=0, y=3 * BASE, q=0, e=0, rows=8, k=64, n=32, ldx=64, ldw=64, ldr=32,
             ldy=32, ldq=32, lde=1, dtype=1, act=0)
    v.update(kw)
    return L._LINEAR.pack(*v.values())


def _grad_input(**kw):
    v = dict(dy=BASE, w=2 * BASE, q=0, e=0, dx=3 * BASE, rows=8, k=64, n=32, lddy=32, ldw=64, ldq=64, lde=2, lddx=64,
             dtype=1, act=0)
    v.update(kw)
    return L._GRAD_INPUT.pack(*v.values())


def _grad_weight(**kw):
    v = dict(dy=BASE, x=2 * BASE, q=0, e=0, dw=3 * BASE, db=0, rows=8, k=64, n=32, lddy=32, ldx=64, ldq=64, lde=2,
             lddw=64, dtype=1, act=0, accumulate=0, reserved=0)
    v.update(kw)
    return L._GRAD_WEIGHT.pack(*v.values())


@pytest.mark.parametrize("bad,code", [
    (dict(rows=-1), INVALID), (dict(k=-1), INVALID), (dict(n=1 << 31), INVALID), (dict(rows=1 << 31), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(act=6), UNSUPPORTED), (dict(act=-1), UNSUPPORTED), (dict(x=0), INVALID),
    (dict(w=0), INVALID), (dict(y=0), INVALID), (dict(ldx=63), INVALID), (dict(ldw=0), INVALID), (dict(ldy=31), INVALID),
    (dict(x=BASE + 1), ALIGNMENT), (dict(y=BASE * 3 + 1), ALIGNMENT), (dict(bias=BASE * 5 + 1), ALIGNMENT),
    (dict(dtype=0, w=BASE * 2 + 2), ALIGNMENT), (dict(q=4 * BASE), INVALID), (dict(e=4 * BASE), INVALID),
    (dict(q=4 * BASE, e=5 * BASE, ldq=31), INVALID), (dict(y=BASE), INVALID), (dict(y=2 * BASE + 64), INVALID),
    (dict(residual=3 * BASE + 2), INVALID), (dict(residual=3 * BASE, ldr=33), INVALID),
    (dict(q=3 * BASE + 8, e=5 * BASE), INVALID), (dict(q=4 * BASE, e=4 * BASE + 16), INVALID),
])
def test_linear_refuses(lib, bad, code):
    assert lib.smat_linear(_linear(**bad), None, 0, None) == code
    assert lib.smat_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(act=5), INVALID), (dict(q=4 * BASE, e=5 * BASE), INVALID), (dict(act=5, q=4 * BASE), INVALID),
    (dict(act=9), UNSUPPORTED), (dict(lddx=63), INVALID), (dict(dx=2 * BASE), INVALID), (dict(dy=0), INVALID),
    (dict(act=1, q=4 * BASE, e=5 * BASE, lde=1), INVALID), (dict(act=1, q=3 * BASE, e=5 * BASE), INVALID),
])
def test_grad_input_refuses(lib, bad, code):
    assert lib.smat_grad_input(_grad_input(**bad), None, 0, None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(x=0), INVALID), (dict(q=4 * BASE, e=5 * BASE), INVALID), (dict(q=4 * BASE), INVALID), (dict(act=5), INVALID),
    (dict(accumulate=4), UNSUPPORTED), (dict(reserved=1), UNSUPPORTED), (dict(dw=BASE), INVALID),
    (dict(db=3 * BASE + 64), INVALID), (dict(db=6 * BASE + 1), ALIGNMENT), (dict(lddw=32), INVALID),
])
def test_grad_weight_refuses(lib, bad, code):
    assert lib.smat_grad_weight(_grad_weight(**bad), None, 0, None) == code


def test_null_args_and_elementwise_refusals(lib):
    assert lib.smat_linear(None, None, 0, None) == INVALID
    assert lib.smat_grad_input(None, None, 0, None) == INVALID
    assert lib.smat_grad_weight(None, None, 0, None) == INVALID
    for f in ("linear", "grad_input", "grad_weight"):
        assert getattr(lib, f"smat_{f}_workspace_bytes")(None) == 0
    x, q, e, o = BASE, 2 * BASE, 3 * BASE, 4 * BASE
    assert lib.smat_pack8(x, 64, q, 64, 0, 2, 8, 64, 1, None) == INVALID
    assert lib.smat_pack8(x, 64, q, 64, e, 1, 8, 64, 1, None) == INVALID
    assert lib.smat_pack8(x, 64, x, 64, e, 2, 8, 64, 1, None) == INVALID
    assert lib.smat_pack8(x, 64, q, 64, e, 2, 8, 64, 3, None) == UNSUPPORTED
    assert lib.smat_unpack8(q, 64, e, 2, q, 64, 8, 64, 1, 0, None) == INVALID
    assert lib.smat_unpack8(q, 64, e, 2, o, 64, 8, 64, 1, 7, None) == UNSUPPORTED
    assert lib.smat_act_grad8(0, 64, q, 64, e, 2, o, 64, 8, 64, 1, 1, None) == INVALID
    assert lib.smat_act_grad8(o, 64, q, 64, e, 2, o, 64, 8, 64, 1, 1, None) == INVALID


def test_slices_of_one_buffer_are_no_overlap(lib):
    """Columns 0..31 and 32..63 of rows 64 apart lie between one another and share nothing: what is refused next is
    the address itself, which is no GPU memory (or there is no GPU to ask)."""
    st = lib.smat_linear(_linear(x=BASE, ldx=128, y=BASE + 128, ldy=128), None, 0, None)
    assert st in (INVALID, CUDA)
    assert "overlaps" not in lib.smat_last_error().decode()
    assert lib.smat_linear(_linear(x=BASE, ldx=128, y=BASE + 126, ldy=128), None, 0, None) == INVALID
    assert "overlaps" in lib.smat_last_error().decode()


def test_structures_match_the_header():
    """The C structures' sizes: pointers and 64-bit sizes of 8 bytes, then 32-bit words, no padding."""
    assert L._LINEAR.size == 8 * (7 + 9) + 4 * 2
    assert L._GRAD_INPUT.size == 8 * (5 + 8) + 4 * 2
    assert L._GRAD_WEIGHT.size == 8 * (6 + 8) + 4 * 4


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    for f in (lambda: L.linear(x, w), lambda: L.linear_grad_input(x, w), lambda: L.linear_grad_weight(x, x),
              lambda: L.pack8(x), lambda: L.act_grad8(x, None, "relu")):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(ValueError):
        L.linear(x, w, act="swish")
    with pytest.raises(ValueError):
        L.Mlp8(8, 16, act="swish")


def test_rows_of_strided_tensors():
    """Leading dimensions taken as rows of one stride, on shapes and strides alone."""
    class Fake:
        is_cuda = True

        def __init__(self, t):
            self.shape, self.stride, self.dim = t.shape, t.stride, t.dim

    t = torch.zeros(5, 6, 40)
    assert L._rows("t", Fake(t)) == (30, 40, 40)
    assert L._rows("t", Fake(t[:, :, 8:24])) == (30, 16, 40)
    assert L._rows("t", Fake(t[:, 2])) == (5, 40, 240)
    assert L._rows("t", Fake(t[:, :1])) == (5, 40, 240)
    assert L._rows("t", Fake(t[:, ::2])) == (15, 40, 80)
    assert L._rows("t", Fake(t[0, 0])) == (1, 40, 40)
    assert L._rows("t", Fake(t[:1])) == (6, 40, 40)
    assert L._rows("t", Fake(torch.zeros(0, 3, 8)))[:2] == (0, 8)
    for bad in (t[:, :4], t.transpose(0, 1), t[:, :, ::2], torch.zeros(1, 8).expand(4, 8), torch.zeros(())):
        with pytest.raises(ValueError):
            L._rows("t", Fake(bad))


def test_reference_pack_against_a_search():
    """The tests' own packing: no smaller power of two keeps every |q| within 127, and values are within half a
    step."""
    x = torch.randn(7, 75, generator=torch.Generator().manual_seed(3)).double() * 10.0 ** torch.arange(-3, 4)[:, None]
    q, e = R.pack(x)
    v = R.unpack(q, e)
    step = torch.ldexp(torch.ones(7, 3, dtype=torch.float64), e.to(torch.int64) - 127).repeat_interleave(32, 1)[:, :75]
    assert bool(((v - x).abs() <= step / 2).all())
    assert bool((q.to(torch.int32).abs() <= 127).all())
    top = torch.zeros(7, 96, dtype=torch.float64)
    top[:, :75] = (x / step * 2).abs()
    assert bool((top.view(7, 3, 32).amax(-1).round() > 127).all())
