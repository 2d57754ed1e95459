"""Root-mean-square norm over very long rows, whose sums a thread makes of thousands of terms.

Bounds.  U = 2^-24.  Squares and products are exact in the 64 bits in which they are summed, so the inverse root is rounded to U/2 and its own steps leave
as much: 2 U in all, and a result in fp32 4 U.  The gradient: h rstd and dy weight carry 3 U, so do the terms of the mean, 8 U in all of their
magnitudes, and the last differences and products 4 U more.
"""
import numpy as np
import pytest

import oracle.lm as olm

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("D", [16392, 30001, 1 << 18, (1 << 20) + 5])
@pytest.mark.parametrize("value", [0.3, 1.7, 3.3])
def test_rows_of_one_value(value, D):
    import torch
    import paper_2407_09453_amd as bsp
    X = torch.full((2, D), value, device="cuda")
    X[1, ::3] = -0.77
    Y, H, rstd = bsp.rms_norm(X)
    dY = torch.full((2, D), 1.1, device="cuda")
    dY[0, ::5] = 0.7
    dX, _ = bsp.rms_norm_grad(dY, H, rstd)
    x, dy, y, q, dx = (t.double().cpu().numpy() for t in (X, dY, Y, rstd, dX))
    wy, wq = olm.rms_norm(x)
    wx, _ = olm.rms_norm_grad(dy, x)
    assert (np.abs(q - wq) <= 2 * U * wq).all(), (q / wq - 1) / U
    assert (np.abs(y - wy) <= 4 * U * np.abs(wy)).all()
    n = np.abs(wy)
    spread = wq[:, None] * (np.abs(dy) + n * (np.abs(dy) * n).mean(1, keepdims=True))
    assert (np.abs(dx - wx) <= 12 * U * spread).all(), (np.abs(dx - wx) / spread).max() / U
