"""The longest sums that the linear operators accept, and tiles in several rounds with everything that an epilogue reads."""

import pytest
import torch

import _linear_ref as R
from paper_2609_33437_gb300 import linear as L

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


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
