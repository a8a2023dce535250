"""Activations in 8 bits and the filter gradients taken from them, against 64-bit references.

Codes, scales and values read back have to be equal bit for bit.  Filter gradients: the products of an 8-bit value with a bf16 gradient are exact, and
what is added up is off by at most 2^-23 of the running sum for each addition of a chain (the tensor core truncates); chains are at most 64
products of matrix instructions, 16 products within one, and then the partial sums, so CHAIN = 128 covers them: 128 * 2^-23 = 1.6e-5
of the sum of magnitudes.  fp32 gradients: 2^-23 more for what their planes leave out."""
import numpy as np
import pytest
import torch

import act8_ref as R
from oracle import oracle
from helpers import norm_err, oshape
from paper_1908_05460_b200 import binding as B
from paper_1908_05460_b200.layers import ConvLayer

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
FORMATS = [B.ACT_E4M3, B.ACT_INT8]
TOL = 129 * 2.0 ** -23


def rows_of(rows, cols, dtype, seed, kind="tokens"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64)
    if kind == "relu":
        x = x.relu()
    elif kind == "wide":                                 # magnitudes over the whole range of the type
        x = x * torch.exp2(torch.randint(-140, 127, (rows, cols), generator=g).double())
    elif kind == "edges":                                # around largest codes, ties and powers of two
        pick = torch.tensor([0.0, -0.0, 448, -448, 449, 450, 127, 127.5, 126.5, 1, 0.5, 1.5, 2.5, 3 * 2.0 ** -10, 2.0 ** -10, 2.0 ** -9, 464, 63.75])
        x = pick[torch.randint(0, len(pick), (rows, cols), generator=g)].double()
    elif kind == "special":
        x = x.clone()
        x[torch.rand(rows, cols, generator=g) < 0.02] = float("inf")
        x[torch.rand(rows, cols, generator=g) < 0.02] = float("nan")
        x[torch.rand(rows, cols, generator=g) < 0.02] = -float("inf")
        x[torch.rand(rows, cols, generator=g) < 0.02] = 3.3895e38
        x[:, : cols // 2] = torch.where(torch.rand(rows, cols // 2, generator=g) < 0.5, 3.38e38, 1.0).double()
    return x.to(dtype)


class Packed:
    def __init__(self, x, fmt, stride=None):
        """x: plain rows on the CPU; packed on the GPU, from a tensor whose rows lie `stride` apart."""
        rows, cols = x.shape
        self.buf = torch.full((rows, stride or cols), 77.0, dtype=x.dtype, device="cuda")
        self.buf[:, :cols] = x.cuda()
        self.desc = B.make_rows_desc(rows, cols, x.dtype, fmt=fmt, x_stride=stride or 0)
        nc, ns = B.gaconv_act_sizes(self.desc)
        self.codes, self.scales = (torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda") for n in (nc, ns))      # (64 bytes behind: left alone)
        B.gaconv_act_pack(self.buf, self.codes, self.scales, self.desc)
        torch.cuda.synchronize()
        assert (self.codes[nc:] == 0xA5).all() and (self.scales[ns:] == 0xA5).all()
        self.codes, self.scales = self.codes[:nc], self.scales[:ns]
        self.c, self.s = self.codes.cpu().numpy().reshape(rows, -1), self.scales.cpu().numpy().reshape(rows, -1)


def check_round_trip(x, fmt, stride=None):
    rows, cols = x.shape
    p = Packed(x, fmt, stride)
    codes, scales, value = R.pack(R.f64(x), fmt)
    assert np.array_equal(p.s, scales)
    assert np.array_equal(p.c, codes)
    out = torch.full_like(p.buf, 55.0)
    B.gaconv_act_unpack(p.codes, p.scales, out, p.desc)
    torch.cuda.synchronize()
    assert np.array_equal(R.f64(out[:, :cols]), value, equal_nan=True)
    assert (out[:, cols:] == 55).all()
    if fmt == B.ACT_E4M3:          # half a step of the format is 2^-4 of a normal code, and half the smallest step is 2^-10 of the scale
        fine = np.isfinite(value) & (np.abs(R.f64(x)) < 2.9e38)
        step = np.repeat(2.0 ** (scales.astype(float) - 127), 32, 1)[:, :cols]
        assert np.all(np.abs(value - R.f64(x))[fine] <= np.maximum(2.0 ** -4 * np.abs(R.f64(x)), 2.0 ** -10 * step)[fine])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, cols", [(1, 1), (3, 7), (1, 16), (5, 31), (64, 32), (33, 33), (2, 48), (17, 100), (9, 256), (100, 64), (7, 1000), (300, 1333), (2, 5000), (1, 40000), (4099, 96)])
def test_round_trip(rows, cols, dtype, fmt):
    check_round_trip(rows_of(rows, cols, dtype, 10 * rows + cols), fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["relu", "wide", "edges", "special"])
def test_round_trip_values(kind, dtype, fmt):
    check_round_trip(rows_of(40, 330, dtype, 5, kind), fmt)
    check_round_trip(torch.zeros(3, 40, dtype=dtype), fmt)
    check_round_trip(torch.full((2, 70), 1e-45 if dtype is torch.float32 else 9.2e-41, dtype=dtype), fmt)      # smallest subnormals


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("stride", [104, 112, 101, 128])
def test_round_trip_strides(stride, dtype, fmt):
    check_round_trip(rows_of(37, 100, dtype, 3), fmt, stride)


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_code_reads_back(fmt):
    codes = torch.arange(256, dtype=torch.uint8)
    if fmt == B.ACT_E4M3:
        codes = codes[(codes & 127) != 127]              # (stand for no number)
    codes = torch.nn.functional.pad(codes, (0, 256 - len(codes)))
    for byte in (10, 60, 127, 200, 246 if fmt == B.ACT_E4M3 else 248):
        scales = torch.full((8,), byte, dtype=torch.uint8)
        for dtype in DTYPES:
            out = torch.zeros(1, 256, dtype=dtype, device="cuda")
            B.gaconv_act_unpack(codes.cuda(), scales.cuda(), out, B.make_rows_desc(1, 256, dtype, fmt=fmt))
            want = R.values(codes.numpy()[None], scales.numpy()[None], 256, fmt)
            if fmt == B.ACT_INT8 and byte == 248:
                want = np.where(want == -128 * 2.0 ** 121, -np.inf, want)        # (a code that is never written)
            assert np.array_equal(R.f64(out), want)


def test_round_trip_beyond_32_bits():
    """More than 2^32 bytes of codes: the last rows are where they belong."""
    rows, cols = 1 << 20, 4160
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.arange(cols, device="cuda") % 97 + 1
    x[rows // 2 + 1] = 3.0
    d = B.make_rows_desc(rows, cols, torch.bfloat16, fmt=B.ACT_INT8)
    nc, ns = B.gaconv_act_sizes(d)
    assert nc > 1 << 32
    codes, scales = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")
    B.gaconv_act_pack(x, codes, scales, d)
    y = torch.full_like(x, 9.0)
    B.gaconv_act_unpack(codes, scales, y, d)
    assert torch.equal(x, y)                             # (whole numbers up to 97 are exact)


# ---------------------------------------------------------------- filter gradients
class Case:
    def __init__(self, layer, dtype, fmt, seed=1, dy_layout=B.DY_NPQK, dw_layout=B.DW_KCRS, alpha=1.0, methods=(B.METHOD_EXACT,), kind="tokens", topk=1, sm_budget=0):
        self.layer, self.dw_layout, self.fmt = layer, dw_layout, fmt
        x = rows_of(layer.n * layer.h * layer.w, layer.c, dtype, seed, kind)
        self.packed = Packed(x, fmt)
        g = torch.Generator().manual_seed(seed + 1)
        dy = torch.randn(layer.n, layer.k, layer.p, layer.q, generator=g, dtype=torch.float64).mul(0.01).to(dtype)
        self.x64 = R.values(self.packed.c, self.packed.s, layer.c, fmt).reshape(layer.n, layer.h, layer.w, layer.c).transpose(0, 3, 1, 2).copy()
        self.dy64 = R.f64(dy)
        self.dy = (dy if dy_layout == B.DY_NKPQ else dy.permute(0, 2, 3, 1)).contiguous().cuda()
        self.shape = {B.DW_KRSC: (layer.k, layer.r, layer.s, layer.c), B.DW_KCRS: (layer.k, layer.c, layer.r, layer.s), B.DW_RSCK: (layer.r, layer.s, layer.c, layer.k)}[dw_layout]
        self.desc = B.make_desc(layer, dtype, dy_layout=dy_layout, dw_layout=dw_layout, alpha=alpha, topk=topk, sm_budget=sm_budget)
        self.ws = B.attach_packed_workspace(self.desc, methods=methods)
        self.guard = torch.full((int(np.prod(self.shape)) + 64,), float("nan"), device="cuda")
        self.dw = self.guard[:-64]

    def run(self, method=B.METHOD_EXACT, seed=0, stream=None):
        B.gaconv_dw_from_packed(method, self.packed.codes, self.packed.scales, self.fmt, self.dy, self.dw, self.desc, seed, stream)

    def result(self):
        torch.cuda.synchronize()
        assert torch.isnan(self.guard[-64:]).all(), "written behind dW"
        assert B.gaconv_poll_async_status(self.desc) == B.OK
        d = R.f64(self.dw).reshape(self.shape)
        return {B.DW_KRSC: (0, 3, 1, 2), B.DW_KCRS: (0, 1, 2, 3), B.DW_RSCK: (3, 2, 0, 1)}[self.dw_layout], d

    def reference(self):
        """dW and the sums of the magnitudes of its products."""
        l = self.layer
        if l.r == l.s == l.h == l.w == 1:
            x, dy = self.x64[:, :, 0, 0], self.dy64[:, :, 0, 0]
            return (dy.T @ x)[:, :, None, None], (np.abs(dy).T @ np.abs(x))[:, :, None, None]
        return oracle.dw_exact(self.x64, self.dy64, oshape(l))

    def check(self):
        self.run()
        order, d = self.result()
        want, size = self.reference()
        err = norm_err(d.transpose(order), self.desc.alpha * want, abs(self.desc.alpha) * size)
        assert err <= TOL, err


def linear(m, c, k):
    return ConvLayer("linear", m, c, 1, 1, k, 1, 1)


# tokens, channels, outputs: one of each, less than a tile, ragged, more than a tile, long reductions, no multiple of eight
LINEAR = [(1, 1, 1), (1, 300, 70), (2, 8, 8), (3, 16, 24), (31, 40, 48), (64, 128, 128), (65, 129, 136), (100, 33, 17), (257, 255, 264), (500, 1000, 333),
          (1, 4096, 8), (5000, 24, 8), (4099, 160, 72), (300, 520, 1048), (20000, 16, 16), (1029, 272, 264)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, c, k", LINEAR)
def test_linear(m, c, k, dtype, fmt):
    Case(linear(m, c, k), dtype, fmt).check()


# more tiles than CTA pairs (whole tiles and split ones), splits of few and of many rows, a tile and a bit
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, c, k", [(1500, 2050, 2600), (700, 2304, 2048), (2500, 1000, 1333), (300, 257, 2000), (9000, 256, 257), (129, 1100, 1030), (40000, 64, 72), (3000, 520, 128)])
def test_linear_of_many_tiles(m, c, k, dtype):
    Case(linear(m, c, k), dtype, B.ACT_INT8 if m % 2 else B.ACT_E4M3).check()


# fp32 gradients in rows of 16 bytes, which are split into bf16 planes inside the kernel: tiles of 64 and of 128 channels, pairs; a last tile of four outputs;
# few rows, rows that end inside a stage, an odd number of stages a split; and rows of dY that do not start on 16 bytes beside them
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m, c, k", [(20000, 64, 64), (200, 700, 700), (1000, 1000, 1000), (4097, 300, 516), (2048, 128, 1000), (33, 1400, 1300), (65, 2100, 1156), (2111, 515, 2052),
                                     (30001, 256, 260), (4097, 300, 518), (33, 1400, 1301)])
def test_linear_fp32_gradients(m, c, k, fmt):
    Case(linear(m, c, k), torch.float32, fmt).check()


@pytest.mark.parametrize("m, c, k", [(1000, 200, 400), (4097, 300, 516), (30001, 256, 260), (4097, 300, 518)])
def test_fp32_gradients_of_every_magnitude(m, c, k):
    """Outputs whose gradients lie far apart; an Inf and a NaN stay in the output that they belong to, and zeros are zeros."""
    case = Case(linear(m, c, k), torch.float32, B.ACT_E4M3)
    dy = case.dy.reshape(m, k)
    dy[:, 0] *= 1e-28
    dy[:, 1] *= 1e30
    dy[:, 2] = 0.0
    dy[m - 1, 4] = float("inf")
    dy[m // 2, k - 1] = float("nan")
    case.dy64 = R.f64(dy).reshape(m, k, 1, 1)
    case.run()
    d = case.result()[1][:, :, 0, 0]
    assert not np.isfinite(d[4]).any() and not np.isfinite(d[k - 1]).any()
    assert (d[2] == 0).all()
    case.dy64 = np.nan_to_num(case.dy64, nan=0.0, posinf=0.0)
    want, size = case.reference()
    rest = [i for i in range(k) if i not in (4, k - 1)]
    assert norm_err(d[rest], want[rest, :, 0, 0], size[rest, :, 0, 0]) <= TOL


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_transposed_result_of_many_tiles(dtype):
    Case(linear(700, 1300, 1100), dtype, B.ACT_E4M3, dw_layout=B.DW_RSCK, alpha=0.5).check()


@pytest.mark.parametrize("dw_layout", [B.DW_KRSC, B.DW_KCRS, B.DW_RSCK])
@pytest.mark.parametrize("dy_layout", [B.DY_NKPQ, B.DY_NPQK])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layer", [ConvLayer("1x1", 6, 72, 9, 11, 40, 1, 1), ConvLayer("1x1", 3, 50, 7, 7, 35, 1, 1), ConvLayer("1x1", 300, 264, 4, 4, 520, 1, 1)], ids=lambda l: "%d_%d" % (l.c, l.k))
def test_pointwise_layouts(layer, dtype, dy_layout, dw_layout):
    """Pixels of feature maps as rows, and every order of gradient and result."""
    Case(layer, dtype, B.ACT_E4M3, dy_layout=dy_layout, dw_layout=dw_layout, alpha=1 / 128).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layer", [ConvLayer("3x3", 4, 16, 16, 16, 24, 3, 3, 1, 1), ConvLayer("3x3s2", 5, 40, 9, 9, 32, 3, 3, 2, 1), ConvLayer("5x5", 3, 17, 8, 8, 13, 5, 5, 1, 2),
                                   ConvLayer("1x1s2", 9, 64, 8, 8, 128, 1, 1, 2, 0), ConvLayer("1x1p", 2, 24, 5, 5, 16, 1, 1, 1, 1), ConvLayer("3x3", 16, 128, 8, 8, 128, 3, 3, 1, 1)], ids=lambda l: l.name + "_%d" % l.c)
def test_convolutions(layer, dtype, fmt):
    Case(layer, dtype, fmt, kind="relu").check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_wide_range_of_magnitudes(dtype):
    """Scales and codes far apart: 2^-100 to 2^100 in X."""
    c = Case(linear(300, 200, 136), dtype, B.ACT_E4M3)
    g = torch.Generator().manual_seed(9)
    x = torch.randn(300, 200, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-100, 100, (300, 1), generator=g).double())
    c.packed = Packed(x.to(dtype), B.ACT_E4M3)
    c.x64 = R.values(c.packed.c, c.packed.s, 200, B.ACT_E4M3).reshape(300, 200, 1, 1)
    c.check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_approximated_methods(dtype):
    layer = ConvLayer("l", 12, 32, 8, 8, 48, 3, 3, 1, 1)
    methods = (B.METHOD_EXACT, B.METHOD_ZERO, B.METHOD_RANDOM, B.METHOD_TOP1, B.METHOD_TOPK)
    c = Case(layer, dtype, B.ACT_INT8, methods=methods, topk=3, kind="relu", dw_layout=B.DW_KCRS)
    for method, want in ((B.METHOD_TOP1, oracle.dw_top1(c.x64, c.dy64, oshape(layer))), (B.METHOD_TOPK, oracle.dw_topk(c.x64, c.dy64, oshape(layer), 3))):
        c.run(method)
        # (one sum of 64 gradients and 12 images for an element; bf16: a map's sum may be rounded to bf16 on its way to the tensor cores)
        assert norm_err(c.result()[1], want[0], want[1]) <= (2.0 ** -8 if dtype is torch.bfloat16 else TOL)
    c.run(B.METHOD_ZERO)
    assert (c.result()[1] == 0).all()
    c.run(B.METHOD_RANDOM, seed=5)
    plain = torch.empty_like(c.dw)
    B.gaconv_dw_approx(B.METHOD_RANDOM, None, None, plain, c.desc, 5)
    assert torch.equal(c.dw, plain)


def test_rows_that_are_not_finite():
    """A group with a NaN or Inf is NaN throughout, and so is every element of dW that it is summed into; the others are untouched."""
    m, c, k = 200, 96, 64
    x = rows_of(m, c, torch.bfloat16, 3)
    x[17, 40] = float("inf")
    x[150, 41] = float("nan")
    case = Case(linear(m, c, k), torch.bfloat16, B.ACT_E4M3)
    case.packed = Packed(x, B.ACT_E4M3)
    case.x64 = R.values(case.packed.c, case.packed.s, c, B.ACT_E4M3).reshape(m, c, 1, 1)
    case.run()
    d = case.result()[1][:, :, 0, 0]
    assert np.isnan(d[:, 32:64]).all()
    case.x64 = np.nan_to_num(case.x64)
    want, size = case.reference()
    rest = np.r_[0:32, 64:96]
    assert norm_err(d[:, rest], want[:, rest, 0, 0], size[:, rest, 0, 0]) <= TOL


def test_same_bits_again_and_in_a_graph():
    """Run twice, on another stream, and captured and replayed on new inputs in the same buffers."""
    for layer, dtype in ((linear(1029, 272, 264), torch.bfloat16), (linear(4099, 160, 72), torch.float32), (linear(700, 100, 51), torch.bfloat16)):
        c = Case(layer, dtype, B.ACT_E4M3)
        c.run()
        first = c.result()[1]
        c.dw.fill_(float("nan"))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        c.run(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert np.array_equal(c.result()[1], first)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run()
        c.dw.fill_(float("nan"))
        graph.replay()
        assert np.array_equal(c.result()[1], first)
        other = Case(layer, dtype, B.ACT_E4M3, seed=8)
        c.packed.codes.copy_(other.packed.codes); c.packed.scales.copy_(other.packed.scales); c.dy.copy_(other.dy)
        graph.replay()
        other.run()
        assert np.array_equal(c.result()[1], other.result()[1])


def test_two_at_once():
    """Calls on two streams with a workspace each."""
    cases = [Case(linear(3000 + 7 * i, 260, 200), torch.bfloat16, B.ACT_INT8, seed=i) for i in range(4)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip(cases, streams):
            c.run(stream=s)
    torch.cuda.synchronize()
    for c in cases:
        got = c.result()[1]
        c.check()
        assert np.array_equal(got, c.result()[1])


def test_fewer_sms():
    for dtype in DTYPES:
        Case(linear(2000, 300, 136), dtype, B.ACT_E4M3, sm_budget=20).check()
