"""The root-mean-square norm and its backward pass against 64-bit references.

Tolerances.  u = 2^-24, half the relative spacing of fp32.  A row's mean square is a chain of at most 40 products and 30 additions of subtotals, all of one
sign, so its relative error is below 70 u and that of 1/sqrt(.) below 35 u + 3 u; an output takes three more roundings: 80 u, and half a step of its
type.  A gradient's mean is summed in the same way, off by at most 70 u of the sum of magnitudes; a weight's gradient is a chain over the rows of one thread, the teams of a
block and the blocks: below 100 + rows / 100 additions for the sizes here, on grids of at least 100 teams."""
import numpy as np
import pytest
import torch

import act8_ref as R
from paper_1908_05460_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = [torch.bfloat16, torch.float32]
SIZES = [(1, 1), (3, 5), (2, 8), (1, 16), (7, 40), (64, 256), (5, 257), (300, 264), (33, 1000), (9, 1024), (4, 1333), (17, 2048), (3, 4096), (700, 72), (2, 8200), (3, 16384), (2, 16392), (1, 20001), (5000, 96), (1500, 4096)]


def half(dtype):
    return torch.finfo(dtype).eps / 2 if dtype is torch.bfloat16 else 0.0


def draw(rows, cols, seed, dtype, scale=1.0, stride=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((rows, stride or cols), 7.0, dtype=dtype, device="cuda")
    buf[:, :cols] = (scale * torch.randn(rows, cols, generator=g, device="cuda")).to(dtype)
    return buf


class Norm:
    def __init__(self, rows, cols, dtype, fmt=B.ACT_E4M3, eps=1e-6, seed=0, strides=(0, 0, 0, 0), residual=True):
        self.rows, self.cols, self.dtype, self.eps, self.fmt = rows, cols, dtype, eps, fmt
        xs, rs, ss, ys = strides
        self.x = draw(rows, cols, seed + 1, dtype, 1.0, xs)
        self.res = draw(rows, cols, seed + 2, dtype, 2.0, rs) if residual else None
        self.w = draw(1, cols, seed + 3, dtype, 0.5)[0] + 1
        self.sum = torch.full((rows, ss or cols), 9.0, dtype=dtype, device="cuda") if residual else None
        self.y = torch.full((rows, ys or cols), 9.0, dtype=dtype, device="cuda")
        self.rstd = torch.full((rows + 8,), -1.0, device="cuda")
        self.desc = B.make_rows_desc(rows, cols, dtype, fmt=fmt, eps=eps, x_stride=xs, r_stride=rs, s_stride=ss, y_stride=ys)
        nc, ns = B.gaconv_act_sizes(self.desc)
        self.codes, self.scales = (torch.full((n + 32,), 0xA5, dtype=torch.uint8, device="cuda") for n in (nc, ns))
        self.nc, self.ns = nc, ns

    def forward(self):
        B.gaconv_rmsnorm_forward(self.x, self.res, self.w, self.sum, self.y, self.codes, self.scales, self.rstd, self.desc)

    def check_forward(self):
        torch.cuda.synchronize()
        c = self.cols
        x = R.f64(self.x[:, :c])
        if self.res is not None:
            t = x + R.f64(self.res[:, :c])
            s = R.f64(self.sum[:, :c])
            assert np.all(np.abs(s - t) <= (torch.finfo(self.dtype).eps / 2 + U) * np.abs(t))
            assert (self.sum[:, c:] == 9).all()
        else:
            s = x
        y, rstd = R.norm(s, R.f64(self.w), self.eps)
        assert np.all(np.abs(R.f64(self.rstd[: self.rows]) - rstd) <= 40 * U * rstd) and (self.rstd[self.rows:] == -1).all()
        mine = R.f64(self.y[:, :c])
        assert np.all(np.abs(mine - y) <= (half(self.dtype) + 80 * U) * np.abs(y))
        assert (self.y[:, c:] == 9).all()
        codes, scales, _ = R.pack(mine, self.fmt)
        assert np.array_equal(self.codes[: self.nc].cpu().numpy().reshape(codes.shape), codes)
        assert np.array_equal(self.scales[: self.ns].cpu().numpy().reshape(scales.shape), scales)
        assert (self.codes[self.nc:] == 0xA5).all() and (self.scales[self.ns:] == 0xA5).all()


class Grad:
    def __init__(self, rows, cols, dtype, seed=0, strides=(0, 0, 0, 0), dsum=True, eps=1e-6):
        self.rows, self.cols, self.dtype = rows, cols, dtype
        xs, _, ss, ys = strides
        self.dy = draw(rows, cols, seed + 1, dtype, 0.01, ys)
        self.ds = draw(rows, cols, seed + 2, dtype, 0.01, ss) if dsum else None
        self.s = draw(rows, cols, seed + 3, dtype, 2.0, ss)
        self.w = draw(1, cols, seed + 4, dtype, 0.5)[0] + 1
        self.rstd = torch.rsqrt(self.s[:, :cols].double().square().mean(1) + eps).float()
        self.dx = torch.full((rows, xs or cols), 9.0, dtype=dtype, device="cuda")
        self.dw = torch.full((cols + 8,), 9.0, device="cuda")
        self.desc = B.make_rows_desc(rows, cols, dtype, eps=eps, x_stride=xs, s_stride=ss, y_stride=ys)
        self.ws = B.rmsnorm_workspace(self.desc)

    def run(self, dx=None, dw=True):
        B.gaconv_rmsnorm_backward(self.dy, self.ds, self.s, self.w, self.rstd, self.dx if dx is None else dx, self.dw if dw else None, self.desc, self.ws if dw else None)

    def check(self, ds=None, dx=None, dw=True):
        torch.cuda.synchronize()
        c = self.cols
        ds = ds if ds is not None else R.f64(self.ds[:, :c]) if self.ds is not None else np.zeros((self.rows, c))
        want, wdw, size, wsize = R.norm_grad(R.f64(self.dy[:, :c]), ds, R.f64(self.s[:, :c]), R.f64(self.w), R.f64(self.rstd))
        got = R.f64((self.dx if dx is None else dx)[:, :c])
        assert np.all(np.abs(got - want) <= half(self.dtype) * np.abs(want) + 80 * U * size)
        if dx is None:
            assert (self.dx[:, c:] == 9).all()
        if dw:
            assert np.all(np.abs(R.f64(self.dw[:c]) - wdw) <= (100 + self.rows / 100) * U * wsize)
            assert (self.dw[c:] == 9).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, cols", SIZES)
def test_forward(rows, cols, dtype):
    n = Norm(rows, cols, dtype, fmt=rows % 2)
    n.forward()
    n.check_forward()


# many rows of more than 128 threads, whole pieces and not, more rows than teams
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, cols", [(2500, 2600), (2500, 2603), (700, 1333), (480, 1400), (1400, 1999)])
def test_forward_of_wide_rows(rows, cols, dtype):
    n = Norm(rows, cols, dtype, fmt=rows % 2)
    n.forward()
    n.check_forward()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("strides", [(104, 112, 128, 120), (101, 100, 102, 103), (112, 0, 0, 101)])
def test_forward_strides(strides, dtype):
    n = Norm(37, 100, dtype, strides=strides)
    n.forward()
    n.check_forward()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [96, 1000, 17000])
def test_forward_optional_parts(cols, dtype):
    n = Norm(21, cols, dtype, residual=False, fmt=B.ACT_INT8)
    n.forward()
    n.check_forward()
    want = n.y.clone(), n.codes.clone(), n.rstd.clone()
    n.y.fill_(9)
    B.gaconv_rmsnorm_forward(n.x, None, n.w, None, n.y, None, None, None, n.desc)          # the output alone
    assert torch.equal(n.y, want[0])
    n.codes.fill_(0xA5)
    B.gaconv_rmsnorm_forward(n.x, None, n.w, None, None, n.codes, n.scales, None, n.desc)  # its 8-bit form alone
    assert torch.equal(n.codes, want[1])
    copy = torch.zeros_like(n.x)
    B.gaconv_rmsnorm_forward(n.x, None, n.w, copy, n.y, None, None, n.rstd, n.desc)        # a sum without a residual is x
    assert torch.equal(copy, n.x) and torch.equal(n.rstd, want[2])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [96, 1001, 17000])
def test_forward_in_place(cols, dtype):
    """The sum in the residual's buffer, and in x's."""
    for which in ("res", "x"):
        n = Norm(50, cols, dtype)
        n.forward()
        want = n.sum.clone(), n.y.clone(), n.codes.clone()
        n.sum = getattr(n, which)
        n.y.fill_(9); n.codes.fill_(0xA5)
        n.forward()
        assert torch.equal(n.sum, want[0]) and torch.equal(n.y, want[1]) and torch.equal(n.codes, want[2])


@pytest.mark.parametrize("dtype", DTYPES)
def test_forward_values(dtype):
    """Rows of zeros (only eps is left; none: not finite, as the formula has it), large and tiny rows, and rows that are not finite stay to themselves."""
    n = Norm(8, 200, dtype, residual=False)
    n.x[0] = 0
    n.x[1] *= 1e15
    n.x[2] *= 1e-15
    n.forward()
    n.check_forward()
    assert (n.y[0] == 0).all()
    n.x[3, 7] = float("nan")
    n.x[4, 9] = float("inf")
    n.forward()
    torch.cuda.synchronize()
    y = R.f64(n.y)
    assert np.isnan(y[3]).all() and np.isnan(y[4, 9]) and np.isfinite(y[[0, 1, 2, 5, 6, 7]]).all()
    assert (n.scales[: n.ns].view(8, -1)[3] == 255).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, cols", SIZES)
def test_backward(rows, cols, dtype):
    g = Grad(rows, cols, dtype, dsum=rows % 3 != 0)
    g.run()
    g.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("strides", [(104, 0, 128, 120), (101, 0, 102, 103), (112, 0, 0, 101)])
def test_backward_strides(strides, dtype):
    g = Grad(137, 100, dtype, strides=strides)
    g.run()
    g.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [96, 1001, 17000])
def test_backward_in_place_and_alone(cols, dtype):
    g = Grad(50, cols, dtype)
    g.run(dw=False)                                      # dx alone, without a workspace
    g.check(dw=False)
    want, ds = g.dx.clone(), R.f64(g.ds)
    g.run(dx=g.ds)                                       # into the incoming gradient's buffer
    assert torch.equal(g.ds, want)
    g.check(ds=ds, dx=g.ds)


def test_no_rows():
    g = Grad(0, 40, torch.float32)
    g.run()
    torch.cuda.synchronize()
    assert (g.dw[:40] == 0).all() and (g.dw[40:] == 9).all()


def test_gradients_are_differences():
    """dx and dweight against central differences of the norm itself in 64 bits."""
    g = Grad(3, 24, torch.float32, dsum=False, eps=1e-3)
    g.run()
    torch.cuda.synchronize()
    s, w, dy = R.f64(g.s), R.f64(g.w), R.f64(g.dy)
    loss = lambda s, w: (R.norm(s, w, 1e-3)[0] * dy).sum()  # noqa: E731
    h = 1e-6         # truncation ~h^2, cancellation ~2^-52 |loss| / h: both below 1e-8
    for i in range(3):
        for j in range(24):
            e = np.zeros_like(s)
            e[i, j] = h
            assert abs((loss(s + e, w) - loss(s - e, w)) / (2 * h) - float(g.dx[i, j])) < 1e-7
    for j in range(24):
        e = np.zeros_like(w)
        e[j] = h
        assert abs((loss(s, w + e) - loss(s, w - e)) / (2 * h) - float(g.dw[j])) < 1e-6


@pytest.mark.parametrize("dtype", DTYPES)
def test_same_bits_again_and_in_a_graph(dtype):
    n, g = Norm(333, 1000, dtype), Grad(333, 1000, dtype)
    n.forward(); g.run()
    first = [t.clone() for t in (n.sum, n.y, n.codes, n.scales, n.rstd, g.dx, g.dw)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n.forward(); g.run()
    for t in (n.sum, n.y, n.rstd, g.dx, g.dw):
        t[..., : n.cols].fill_(5)
    graph.replay()
    n.rstd[n.rows:] = -1
    for a, b in zip((n.sum, n.y, n.codes, n.scales, n.rstd, g.dx, g.dw), first):
        assert torch.equal(a, b)


def test_rows_beyond_32_bits():
    rows, cols = 1 << 19, 8256
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-1] = 2.0
    x[rows // 2 + 3] = -4.0
    y, rstd = torch.full_like(x, 9.0), torch.empty(rows, device="cuda")
    d = B.make_rows_desc(rows, cols, torch.bfloat16, eps=0.25)
    w = torch.full((cols,), 1.5, dtype=torch.bfloat16, device="cuda")
    B.gaconv_rmsnorm_forward(x, None, w, None, y, None, None, rstd, d)
    assert rows * cols > 1 << 32
    for row, v in ((-1, 2.0), (rows // 2 + 3, -4.0), (0, 0.0)):
        want = 1.5 * v / (v * v + 0.25) ** 0.5
        assert abs(float(y[row, 8000]) - want) <= 2.0 ** -8 * abs(want) + 1e-6 and abs(float(rstd[row]) - (v * v + 0.25) ** -0.5) < 1e-6
    assert int((y != 0).any(1).sum()) == 2
