"""Norms of rows that start and end on 16 bytes, more of them than the GPU takes at once: every CTA goes on to further rows, with
the next row's loads under way and the weights' sums carried along. Against the definitions in 64 bits, with the tolerances of
`test_gpu_norm`; a thread adds up to 32 values of a row here, so a sum over it passes 32 + 12 roundings."""

import pytest
import torch

import test_gpu_norm as T
from paper_2609_33437_gb300 import norm as N

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _cuda(monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    monkeypatch.setattr(T, "_adds", lambda cols: 32 + 12)


# a warp per row and 32 values a thread forward: 512 < columns <= 1024; the others by the threads that a row takes
SIZES = [(4112, 1024), (1500, 1024), (2600, 768), (1500, 512), (6000, 64), (1400, 2048), (700, 4096), (400, 8192), (400, 11008),
         (200, 16384)]


@pytest.mark.parametrize("dt,wt,kind", [(BF, BF, "rms"), (BF, F32, "layer"), (F32, F32, "layer"), (F32, F32, "rms")])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_many_rows(rows, cols, dt, wt, kind):
    seed = rows * 37 + cols
    x, r = T._rand(seed, rows, cols, dt, 2.0, 0.5), T._rand(seed + 1, rows, cols, dt)
    w, b = T._vec(seed + 2, cols, wt, 0.2, 1.0), T._vec(seed + 3, cols, wt, 0.1, 0.0) if kind == "layer" else None
    T._check_forward(x, w, b, None, kind)
    _, h, stats = T._check_forward(x, w, b, r, kind)
    dy, dh = T._rand(seed + 4, rows, cols, dt, 0.1), T._rand(seed + 5, rows, cols, dt, 0.1)
    T._check_grad(dy, h, stats, w, b is not None, kind, None)
    T._check_grad(dy, h, stats, w, True, kind, dh)


def test_rows_of_padded_batches():
    """A row's result and gradient in a batch that takes another number of CTAs: as near the definition, whatever stands beside it."""
    x, dy, w = T._rand(0, 4112, 1024, BF), T._rand(1, 4112, 1024, BF), T._vec(2, 1024, BF, 0.2, 1.0)
    for rows in (4112, 600, 5, 1):
        _, stats = N.norm(x[:rows], w, kind="rms", save=True)
        T._check_forward(x[:rows], w, None, None, "rms")
        T._check_grad(dy[:rows], x[:rows], stats, w, False, "rms", None)
