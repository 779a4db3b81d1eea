"""What the binding takes as rows of one stride, on shapes and strides alone: tensors of nothing, of any dimensions."""

import pytest
import torch

from paper_2609_33437_gb300 import linear as L


class Fake:
    is_cuda = True

    def __init__(self, t):
        self.shape, self.stride, self.dim = t.shape, t.stride, t.dim


@pytest.mark.parametrize("shape", [(0, 8), (0, 3, 8), (3, 0, 8), (2, 3, 0, 8), (2, 0, 3, 8), (0, 0, 8)])
def test_no_rows(shape):
    for t in (torch.zeros(shape), torch.zeros(*shape[:-1], 16)[..., 4:12], torch.zeros(*shape[:-2], shape[-2] + 2, 8)[..., :shape[-2], :]):
        assert L._rows("t", Fake(t)) == (0, 8, 8)
    # as the gradient of a sum arrives: one number for all, of which there are none
    assert L._rows("t", Fake(torch.zeros(()).expand(shape))) == (0, 8, 8)


@pytest.mark.parametrize("shape,rows", [((5, 0), 5), ((2, 3, 0), 6), ((0, 0), 0)])
def test_no_columns(shape, rows):
    assert L._rows("t", Fake(torch.zeros(shape)))[:2] == (rows, 0)
