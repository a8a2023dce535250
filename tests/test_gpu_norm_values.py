"""Values that are not finite in the norm's backward pass: the gradients that they reach are what the formula gives, and no others."""
import numpy as np
import pytest
import torch

import act8_ref as R
from test_gpu_rmsnorm import DTYPES, Grad, U, half

pytestmark = pytest.mark.gpu


# whole pieces, rows on any boundary, tensors on boundaries of their own, rows beyond the registers; more rows than teams
@pytest.mark.parametrize("rows, cols, strides", [(9, 256, (0, 0, 0, 0)), (9, 257, (0, 0, 0, 0)), (9, 100, (101, 0, 102, 103)), (7, 17000, (0, 0, 0, 0)), (3000, 640, (0, 0, 0, 0)), (3000, 643, (0, 0, 0, 0))])
@pytest.mark.parametrize("dtype", DTYPES)
def test_backward_values(rows, cols, strides, dtype):
    g = Grad(rows, cols, dtype, strides=strides)
    nan, inf = float("nan"), float("inf")
    g.dy[0, 3], g.s[1, cols - 1], g.ds[2, 5], g.ds[3, 6], g.dy[4, cols // 2], g.rstd[5], g.dy[6, 7] = nan, nan, nan, -inf, inf, nan, -inf
    g.run()
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        dx, dw, size, wsize = R.norm_grad(*(R.f64(t[:, :cols]) for t in (g.dy, g.ds, g.s)), R.f64(g.w), R.f64(g.rstd))
        for got, want, tol in ((R.f64(g.dx[:, :cols]), dx, half(dtype) * np.abs(dx) + 80 * U * size), (R.f64(g.dw[:cols]), dw, (100 + rows / 100) * U * wsize)):
            for kind in (np.isnan, np.isposinf, np.isneginf):
                assert np.array_equal(kind(got), kind(want)), kind
            fine = np.isfinite(want)
            assert np.all(np.abs(got - want)[fine] <= tol[fine])
    assert np.isfinite(dx[7:]).all() and not np.isfinite(dx[:7]).all(1).any()
