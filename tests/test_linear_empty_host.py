"""Activations in 8 bits of no rows, whose memory has no address, on the host side of the C ABI."""

import pytest

from paper_2609_33437_gb300 import linear as L
from paper_2609_33437_gb300 import smat as S

INVALID, CUDA, BASE = 1, 6, 0x10000000


@pytest.fixture(scope="module")
def lib():
    return S.load_library()


def test_gradients_of_no_rows_through_an_activation(lib):
    def grad_input(rows, k, q, e, act):
        return lib.smat_grad_input(L._GRAD_INPUT.pack(BASE, 2 * BASE, q, e, 3 * BASE, rows, k, 32, 32, 64, 64, 2, 64, 1, act),
                                   None, 0, None)

    assert grad_input(0, 64, 0, 0, 5) == 0  # nothing to do
    assert grad_input(0, 64, 4 * BASE, 5 * BASE, 5) == 0
    assert grad_input(0, 64, 4 * BASE, 5 * BASE, 0) == INVALID
    assert grad_input(8, 64, 0, 0, 5) == INVALID and grad_input(8, 64, 4 * BASE, 0, 5) == INVALID

    def grad_weight(rows, k, x, act):
        return lib.smat_grad_weight(L._GRAD_WEIGHT.pack(BASE, x, 0, 0, 3 * BASE, 0, rows, k, 32, 32, 64, 64, 2, 64, 1, act, 0, 0),
                                    None, 0, None)

    # no column either, so that nothing is written to what is only a number here; what may come next is the lack of a GPU
    assert grad_weight(0, 0, 0, 5) in (0, CUDA)
    assert grad_weight(0, 64, 2 * BASE, 5) == INVALID and "activation" in lib.smat_last_error().decode()
    assert grad_weight(8, 64, 0, 5) == INVALID
