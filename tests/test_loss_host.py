"""CPU-only checks of the loss over a vocabulary: what its part of the C ABI and its binding refuse before anything reaches a
GPU. Pointers here are numbers; none is read."""

import pytest
import torch

from paper_2609_33437_gb300 import loss as T
from paper_2609_33437_gb300 import smat as S

INVALID, UNSUPPORTED, ALIGNMENT = 1, 2, 3
BASE = 0x10000000


@pytest.fixture(scope="module")
def lib():
    return S.load_library()


def _loss(**kw):
    v = dict(x=BASE, w=2 * BASE, t=3 * BASE, loss=4 * BASE, lse=5 * BASE, rows=8, k=64, n=500, ldx=64, ldw=64, ignore=-100, dtype=1,
             reserved=0)
    v.update(kw)
    return T._TOKEN_LOSS.pack(*v.values())


def _grad(**kw):
    v = dict(g=BASE, x=2 * BASE, w=3 * BASE, t=4 * BASE, lse=5 * BASE, dx=6 * BASE, dw=7 * BASE, rows=8, k=64, n=500, ldx=64, ldw=64,
             lddx=64, lddw=64, ignore=-100, dtype=1, accumulate=0)
    v.update(kw)
    return T._TOKEN_LOSS_GRAD.pack(*v.values())


@pytest.mark.parametrize("bad,code", [
    (dict(rows=-1), INVALID), (dict(k=-1), INVALID), (dict(n=0), INVALID), (dict(n=1 << 31), INVALID), (dict(rows=1 << 31), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(reserved=1), UNSUPPORTED), (dict(x=0), INVALID), (dict(w=0), INVALID), (dict(t=0), INVALID),
    (dict(loss=0), INVALID), (dict(lse=0), INVALID), (dict(ldx=63), INVALID), (dict(ldw=1), INVALID), (dict(x=BASE + 1), ALIGNMENT),
    (dict(t=3 * BASE + 4), ALIGNMENT), (dict(lse=5 * BASE + 2), ALIGNMENT), (dict(loss=5 * BASE), INVALID), (dict(lse=BASE), INVALID),
    (dict(loss=3 * BASE + 8), INVALID),
])
def test_loss_refuses(lib, bad, code):
    assert lib.smat_token_loss(_loss(**bad), None, 0, None) == code
    assert lib.smat_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(rows=-1), INVALID), (dict(n=0), INVALID), (dict(dtype=-1), UNSUPPORTED), (dict(accumulate=2), UNSUPPORTED),
    (dict(g=0), INVALID), (dict(x=0), INVALID), (dict(w=0), INVALID), (dict(t=0), INVALID), (dict(lse=0), INVALID),
    (dict(dx=2 * BASE), INVALID), (dict(dw=3 * BASE + 2), INVALID), (dict(dw=6 * BASE), INVALID), (dict(lddx=63), INVALID),
    (dict(lddw=0), INVALID), (dict(g=BASE + 2), ALIGNMENT), (dict(dw=7 * BASE + 1), ALIGNMENT),
])
def test_grad_refuses(lib, bad, code):
    assert lib.smat_token_loss_grad(_grad(**bad), None, 0, None) == code


def test_nothing(lib):
    assert lib.smat_token_loss(None, None, 0, None) == INVALID and lib.smat_token_loss_grad(None, None, 0, None) == INVALID
    for f, pack in (("smat_token_loss", _loss), ("smat_token_loss_grad", _grad)):
        size = getattr(lib, f + "_workspace_bytes")
        assert size(None) == 0 and size(pack(rows=-1)) == 0 and size(pack(rows=0)) == 0 and size(pack(dtype=7)) == 0


def test_binding_refuses():
    x, w, t = torch.zeros(4, 8), torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        T.token_loss(x, w, t)
    with pytest.raises(ValueError, match="graph"):
        T.token_loss(x.clone().requires_grad_(), w, t)
    with pytest.raises(ValueError, match="targets"):
        T._targets(t.int(), (4,), t.device)
    with pytest.raises(ValueError, match="targets"):
        T._targets(t, (5,), t.device)
    with pytest.raises(ValueError, match="g: must be"):
        T._row_values("g", torch.zeros(4, 2)[:, 0], (4,), t.device)
    with pytest.raises(ValueError, match="accumulate"):
        T.token_loss_grad(x[:, 0], x, w, t, x[:, 0], accumulate=True)
    with pytest.raises(ValueError, match="not asked for"):
        T.token_loss_grad(x[:, 0], x, w, t, x[:, 0], out=x, need_x=False)
    with pytest.raises(ValueError, match="reduction"):
        T.cross_entropy(x, w, t, reduction="max")
