"""CPU-only checks of the norms' part of the C ABI and of its binding: what is refused on the host, before anything reaches a
GPU. Pointers here are numbers; none is read."""

import pytest
import torch

from paper_2609_33437_gb300 import norm as N
from paper_2609_33437_gb300 import smat as S

INVALID, UNSUPPORTED, ALIGNMENT = 1, 2, 3
BASE = 0x10000000


@pytest.fixture(scope="module")
def lib():
    return S.load_library()


def _norm(**kw):
    v = dict(x=BASE, r=0, w=2 * BASE, b=0, h=0, y=3 * BASE, stats=0, rows=8, cols=64, ldx=64, ldr=64, ldh=64, ldy=64, dtype=1,
             wdtype=1, kind=0, eps=1e-5)
    v.update(kw)
    return N._NORM.pack(*v.values())


def _grad(**kw):
    v = dict(dy=BASE, h=2 * BASE, stats=3 * BASE, w=4 * BASE, dh=0, dx=5 * BASE, dw=6 * BASE, db=0, rows=8, cols=64, lddy=64,
             ldh=64, lddh=64, lddx=64, dtype=1, wdtype=1, kind=0, accumulate=0)
    v.update(kw)
    return N._NORM_GRAD.pack(*v.values())


@pytest.mark.parametrize("bad,code", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(cols=1 << 31), INVALID), (dict(rows=1 << 31), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(dtype=0, wdtype=1), UNSUPPORTED), (dict(kind=2), UNSUPPORTED), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(x=0), INVALID), (dict(y=0), INVALID), (dict(r=4 * BASE), INVALID),
    (dict(h=4 * BASE), INVALID), (dict(ldx=63), INVALID), (dict(ldy=1), INVALID), (dict(x=BASE + 1), ALIGNMENT),
    (dict(stats=5 * BASE + 2), ALIGNMENT), (dict(wdtype=0, w=2 * BASE + 2), ALIGNMENT), (dict(y=BASE), INVALID),
    (dict(y=2 * BASE), INVALID), (dict(stats=3 * BASE + 8), INVALID), (dict(r=4 * BASE, h=3 * BASE), INVALID),
    (dict(r=4 * BASE, h=4 * BASE, ldh=65), INVALID), (dict(r=4 * BASE, h=BASE), INVALID),
])
def test_norm_refuses(lib, bad, code):
    assert lib.smat_norm(_norm(**bad), None) == code
    assert lib.smat_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(dtype=3), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED),
    (dict(accumulate=2), UNSUPPORTED), (dict(dy=0), INVALID), (dict(h=0), INVALID), (dict(stats=0), INVALID),
    (dict(dx=BASE), INVALID), (dict(dx=2 * BASE + 2), INVALID), (dict(dw=4 * BASE + 4), INVALID), (dict(db=6 * BASE + 64), INVALID),
    (dict(dh=5 * BASE, lddh=72), INVALID), (dict(lddx=1), INVALID), (dict(stats=3 * BASE + 1), ALIGNMENT),
])
def test_norm_grad_refuses(lib, bad, code):
    assert lib.smat_norm_grad(_grad(**bad), None, 0, None) == code


def test_nothing(lib):
    assert lib.smat_norm(None, None) == INVALID and lib.smat_norm_grad(None, None, 0, None) == INVALID
    assert lib.smat_norm_grad_workspace_bytes(None) == 0
    assert lib.smat_norm_grad_workspace_bytes(_grad(rows=-4)) == 0


def test_binding_refuses():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="CUDA"):
        N.norm(x)
    with pytest.raises(ValueError, match="kind"):
        N.norm(x, kind="batch")
    with pytest.raises(ValueError, match="residual"):
        N.norm(x, sum_out=x)
    with pytest.raises(ValueError, match="graph"):
        N.norm(x.clone().requires_grad_())
    with pytest.raises(ValueError, match="accumulate"):
        N.norm_grad(x, x, x, accumulate=True)
    with pytest.raises(ValueError, match="not asked for"):
        N.norm_grad(x, x, x, need_w=False, weight_out=x)
    with pytest.raises(ValueError, match="kind"):
        N.Norm(8, kind="group")
    assert N.Norm(8, kind="rms").bias is None and N.Norm(8).bias is not None


def test_binding_checks_the_weights():
    meta = torch.device("cpu")
    with pytest.raises(ValueError, match="w: must be"):
        N._weights(8, torch.float32, meta, torch.zeros(8, dtype=torch.bfloat16), None)
    with pytest.raises(ValueError, match="b: must be"):
        N._weights(8, torch.bfloat16, meta, torch.zeros(8), torch.zeros(8, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="w: must be"):
        N._weights(8, torch.float32, meta, torch.zeros(9), None)


def test_a_gradient_that_would_be_lost_names_the_layers():
    x = torch.zeros(2, 4, requires_grad=True)
    for call in (lambda: N.norm(x), lambda: N.norm_grad(x, x, x)):
        with pytest.raises(ValueError, match="norm.Norm, loss.cross_entropy"):
            call()
