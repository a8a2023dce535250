"""The weight's gradient of the norm over very many rows.

Terms of one sign, alike in every row, so that roundings do not cancel: a chain of n additions is then off by up to n u, u = 2^-24.  Bounds, in u of the sum: two roundings of a term; chains of
64; how the chains are added up (64 u for the 63 chains of a team here, 2 u where what is rounded off is kept); 37 for the blocks' sums, five in a thread and 32 threads: 168 u and 106 u."""
import numpy as np
import pytest
import torch

import act8_ref as R
from paper_1908_05460_b200 import binding as B
from test_gpu_rmsnorm import Grad

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def weight_gradient(rows, cols, dtype, y_stride=0):
    """dweight, and what it is in 64 bits, for rows that are all the same."""
    g = torch.Generator().manual_seed(cols)
    dy, s = ((0.5 + torch.rand(cols, generator=g)).to(dtype) for _ in range(2))
    buf = torch.zeros(rows, y_stride or cols, dtype=dtype, device="cuda")
    buf[:, :cols] = dy.cuda()
    rstd = torch.full((rows,), 1.1, device="cuda")
    dx, dw, w = torch.empty(rows, cols, dtype=dtype, device="cuda"), torch.empty(cols, device="cuda"), torch.ones(cols, dtype=dtype, device="cuda")
    d = B.make_rows_desc(rows, cols, dtype, y_stride=y_stride)
    B.gaconv_rmsnorm_backward(buf, None, s.cuda().repeat(rows, 1), w, rstd, dx, dw, d, B.rmsnorm_workspace(d))
    return R.f64(dw), rows * R.f64(dy) * R.f64(s) * R.f64(rstd[:1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_on_different_boundaries(dtype):
    """dy's rows lie four elements apart, the sum's three: a thread a channel, 16384 rows each."""
    got, want = weight_gradient(1 << 20, 3, dtype, 4)
    assert np.all(np.abs(got - want) <= 106 * U * want)


def test_rows_that_a_team_takes_in_turn():
    """A row takes a block of 288 threads, and a block 4000 rows."""
    got, want = weight_gradient(4000 * 148, 2052, torch.float32)
    assert np.all(np.abs(got - want) <= 168 * U * want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_an_infinite_rstd_stays_in_its_row(dtype):
    """A row whose squares underflow has, without eps, an infinite rstd, and the weight's gradient is infinite; a team that then has no row left adds nothing to it."""
    rows, cols = 148 * 64 + 1, 8          # (teams of 8 threads, 64 a block, a block an SM: one row is left for the second round)
    s = torch.ones(rows, cols, dtype=dtype, device="cuda")
    s[1:64] = 1e-25
    w, y, rstd = torch.ones(cols, dtype=dtype, device="cuda"), torch.empty_like(s), torch.empty(rows, device="cuda")
    d = B.make_rows_desc(rows, cols, dtype, eps=0.0)
    B.gaconv_rmsnorm_forward(s, None, w, None, y, None, None, rstd, d)
    assert torch.isinf(rstd[1:64]).all() and (rstd[64:] == 1).all()
    dy, dx, dw = torch.ones_like(s), torch.empty_like(s), torch.empty(cols, device="cuda")
    B.gaconv_rmsnorm_backward(dy, None, s, w, rstd, dx, dw, d, B.rmsnorm_workspace(d))
    assert (dw == float("inf")).all()
    assert torch.isfinite(dx[0]).all() and torch.isfinite(dx[64:]).all()


@pytest.mark.parametrize("cols", [8200, 8203])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_rows_beyond_the_registers(cols, dtype):
    """Ranges of forty rows, and one that is shorter."""
    g = Grad(2533, cols, dtype)
    g.run()
    g.check()
