"""Results whose rows start on 16 bytes and end anywhere, in a wider buffer: what lies beside them stays as it was."""

import pytest
import torch

import _linear_ref as R
import test_gpu_linear as T
from paper_2609_33437_gb300 import linear as L
from paper_2609_33437_gb300 import smat as S

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


def _inside(rows, cols, dtype, beside):
    """A [rows, cols] matrix whose rows are `beside` and up to 7 more elements apart, on 16 bytes; and the buffer."""
    ld = (cols + 15) // 16 * 16 + beside
    flat = torch.full((rows, ld), 7.0, device="cuda").to(dtype)
    return flat[:, :cols], flat


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("wide", [5, 7, 31, 33, 117, 250, 1063])
@pytest.mark.parametrize("rows", [3, 100, 300])
def test_nothing_is_written_beside_a_result(dtype, wide, rows):
    short = 72
    x, w = T._rand(1, rows, short, dtype=dtype), T._rand(2, wide, short, scale=0.1, dtype=dtype)
    res, whole_res = _inside(rows, wide, dtype, 16)
    res.copy_(T._rand(3, rows, wide, dtype=dtype))
    for residual in (None, res):
        out, whole = _inside(rows, wide, dtype, 0)
        T._check_linear(x, w, None, "silu", residual, L.linear(x, w, act="silu", residual=residual, out=out))
        assert bool((whole[:, wide:] == 7.0).all())
    # in place of the residual, in a buffer of three results side by side
    part = (wide + 15) // 16 * 16
    joint = torch.full((rows, 3 * part), 7.0, device="cuda").to(dtype)
    joint[:, part:part + wide] = res
    L.linear(x, w, act="silu", residual=joint[:, part:part + wide], out=joint[:, part:part + wide])
    assert torch.equal(joint[:, part:part + wide], out)
    joint[:, part:part + wide] = 7.0
    assert bool((joint == 7.0).all())

    dy, w2 = T._rand(4, rows, short, scale=1e-2, dtype=dtype), T._rand(5, short, wide, scale=0.1, dtype=dtype)
    saved = L.pack8(T._rand(6, rows, wide, scale=2.0, dtype=dtype))
    ld = (wide + 15) // 16 * 16
    q = torch.zeros(rows, ld, dtype=torch.int8, device="cuda")[:, :wide]
    q.copy_(saved.q)
    for act, h in (("none", None), ("gelu", saved), ("gelu", L.Packed8(q, saved.e))):
        out, whole = _inside(rows, wide, dtype, 16)
        T._check_grad_input(dy, w2, act, h, L.linear_grad_input(dy, w2, act, h, out=out))
        assert bool((whole[:, wide:] == 7.0).all())

    for m in (2, 40):  # rows of the sum
        dy, x = T._rand(7, m, rows, scale=1e-2, dtype=dtype), T._rand(8, m, wide, dtype=dtype)
        old = T._rand(9, rows, wide, scale=0.05, dtype=dtype)
        for acc in (False, True):
            out, whole = _inside(rows, wide, dtype, 0)
            out.copy_(old)
            dw, _ = L.linear_grad_weight(dy, x, out=out, accumulate=acc)
            T._check_grad_weight(dy, T._d(x), dw, None, old=T._d(old) if acc else None)
            assert bool((whole[:, wide:] == 7.0).all())
    assert bool((whole_res[:, wide:] == 7.0).all()) and L.poll_errors() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("wide", [5, 24, 40, 117, 264])
@pytest.mark.parametrize("rows", [3, 100, 300])
def test_nothing_is_written_beside_saved_bits(dtype, wide, rows):
    """q and e of a forward pass and of pack8 in rows of a wider buffer, through the C ABI."""
    k, ld, groups = 72, (wide + 15) // 16 * 16, -(-wide // 32)
    x, w = T._rand(1, rows, k, dtype=dtype), T._rand(2, wide, k, scale=0.1, dtype=dtype)
    ref, saved = L.linear(x, w, act="gelu", save=True)
    q = torch.full((rows, ld + 16), 77, dtype=torch.int8, device="cuda")
    e = torch.full((rows, groups + 3), 77, dtype=torch.uint8, device="cuda")
    y, whole = _inside(rows, wide, dtype, 16)
    lib, code = S.load_library(), S.dtype_code(dtype)
    args = L._LINEAR.pack(x.data_ptr(), w.data_ptr(), 0, 0, y.data_ptr(), q.data_ptr(), e.data_ptr(), rows, k, wide, k, k, wide,
                          whole.shape[1], q.shape[1], e.shape[1], code, L.ACTS["gelu"])
    size = lib.smat_linear_workspace_bytes(args)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    S.check("smat_linear", lib.smat_linear(args, ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream))

    def there(p):
        assert torch.equal(q[:, :wide], p.q) and torch.equal(e[:, :groups], p.e)
        assert bool((q[:, wide:] == 77).all()) and bool((e[:, groups:] == 77).all())

    assert torch.equal(y, ref) and bool((whole[:, wide:] == 7.0).all())
    there(saved)
    q.fill_(77), e.fill_(77)
    S.check("smat_pack8", lib.smat_pack8(y.data_ptr(), whole.shape[1], q.data_ptr(), q.shape[1], e.data_ptr(), e.shape[1], rows,
                                         wide, code, torch.cuda.current_stream().cuda_stream))
    there(L.pack8(ref))
