"""Filter gradients from inputs in 8 bits by each instance of the tensor-core kernel, and by the routes that a descriptor asks for by name.

Which kernel a call takes is read from a graph that it is captured into.  Tolerances as in test_gpu_packed.py."""
import ctypes
import re
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest
import torch

import act8_ref as R
from helpers import norm_err
from paper_1908_05460_b200 import binding as B
from paper_1908_05460_b200.graph_names import kernel_names
from paper_1908_05460_b200.layers import ConvLayer
from test_gpu_packed import DTYPES, FORMATS, TOL, Case, Packed, linear, rows_of

pytestmark = pytest.mark.gpu

# tokens, channels (the last group of 32 is not whole), outputs -> the kernel's instance: CTAs of a tile, planes of dY, channels of a CTA, planes made inside
INSTANCES = [(torch.bfloat16, (300, 200, 136), "1, 1, 64, 0"), (torch.bfloat16, (2100, 330, 1030), "1, 1, 128, 0"), (torch.bfloat16, (700, 2311, 2048), "1, 1, 128, 0"),
             (torch.bfloat16, (700, 2300, 2048), "2, 1, 128, 0"),
             (torch.float32, (300, 200, 136), "1, 3, 64, 1"), (torch.float32, (4000, 130, 250), "1, 3, 64, 0"), (torch.float32, (1000, 1001, 1000), "1, 3, 128, 1"),
             (torch.float32, (2100, 330, 1030), "1, 3, 128, 0"), (torch.float32, (1500, 1100, 1500), "2, 3, 128, 1"), (torch.float32, (2500, 1000, 1333), "2, 3, 128, 0")]


def instance(names):
    """Of packed_dw_kernel, if it is among them."""
    for name in names:
        m = re.search(r"packed_dw_kernelILi(\d)ELi(\d)ELi(\d+)ELb(\d)E", name)
        if m:
            return ", ".join(m.groups())


def tensor_case(dtype, sizes, fmt, want, x=None):
    """A linear layer whose gradient is asked of the tensor cores (few products go to the FP32 pipes otherwise); x: other rows than normal ones."""
    c = Case(linear(*sizes), dtype, fmt)
    c.desc.algo = B.ALGO_TENSOR
    c.ws = B.attach_packed_workspace(c.desc)
    if x is not None:
        c.packed = Packed(x.to(dtype), fmt)
        c.x64 = R.values(c.packed.c, c.packed.s, sizes[1], fmt).reshape(sizes[0], sizes[1], 1, 1)
    assert instance(kernel_names(c.run)) == want
    return c


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype, sizes, want", INSTANCES)
def test_scales_far_apart(dtype, sizes, want, fmt):
    """A scale of its own, from 2^-100 to 2^100 times a few, for every group of every row: bytes beyond 134 take E4M3's second factor."""
    m, c, _ = sizes
    g = torch.Generator().manual_seed(3)
    scale = torch.exp2(torch.randint(-100, 100, (m, R.groups(c)), generator=g).double()).repeat_interleave(32, 1)[:, :c]
    case = tensor_case(dtype, sizes, fmt, want, torch.randn(m, c, generator=g, dtype=torch.float64) * scale)
    assert (case.packed.s > 134).any() and (case.packed.s < 100).any()
    case.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype, sizes, want", INSTANCES)
def test_groups_that_are_not_finite(dtype, sizes, want, fmt):
    """A group with an Inf or NaN, the first, one in the middle and the last, which is not whole: its channels of dW are NaN, the others are untouched."""
    m, c, _ = sizes
    last = R.groups(c) - 1
    x = rows_of(m, c, dtype, 4)
    x[0, 5], x[m // 2, 32 * (last // 2) + 31], x[m - 1, c - 1] = float("nan"), float("inf"), -float("inf")
    case = tensor_case(dtype, sizes, fmt, want, x)
    assert int((case.packed.s == 255).sum()) == 3
    case.run()
    d = case.result()[1][:, :, 0, 0]
    bad = np.isin(np.arange(c) // 32, (0, last // 2, last))
    assert np.isnan(d[:, bad]).all()
    case.x64 = np.nan_to_num(case.x64)
    ref, size = case.reference()
    assert norm_err(d[:, ~bad], ref[:, ~bad, 0, 0], size[:, ~bad, 0, 0]) <= TOL


@pytest.mark.parametrize("math", [B.MATH_DEFAULT, B.MATH_TF32])
@pytest.mark.parametrize("algo", [B.ALGO_AUTO, B.ALGO_DIRECT, B.ALGO_TENSOR])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layer", [linear(500, 64, 72), ConvLayer("3x3", 4, 16, 16, 16, 24, 3, 3, 1, 1), ConvLayer("3x3", 8, 64, 8, 8, 64, 3, 3, 1, 1)], ids=lambda l: "%s_%d" % (l.name, l.c))
def test_routes_by_name(layer, dtype, algo, math):
    """What the plain call refuses is refused; what it takes gives the plain call's bits on the values that are kept, unless the kernel for linear layers takes it."""
    lib, fmt = B.load(), B.ACT_INT8
    case = Case(layer, dtype, fmt)
    d = case.desc
    d.algo, d.math, d.workspace, d.workspace_bytes = algo, math, None, 0
    x = torch.empty(layer.n * layer.h * layer.w, layer.c, dtype=dtype, device="cuda")
    B.gaconv_act_unpack(case.packed.codes, case.packed.scales, x, B.make_rows_desc(x.shape[0], layer.c, dtype, fmt=fmt))
    room = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
    d.workspace, d.workspace_bytes = room.data_ptr(), room.numel()
    plain = torch.empty_like(case.dw)
    want = lib.gaconv_dw_exact(x.data_ptr(), case.dy.data_ptr(), plain.data_ptr(), ctypes.byref(d), B._stream(None))
    got = lib.gaconv_dw_from_packed(B.METHOD_EXACT, case.packed.codes.data_ptr(), case.packed.scales.data_ptr(), fmt, case.dy.data_ptr(), case.dw.data_ptr(), ctypes.byref(d), 0, B._stream(None))
    fused = layer.r == 1 and algo != B.ALGO_DIRECT and math == B.MATH_DEFAULT
    if got != want:
        assert fused and got == B.OK          # (a linear layer that the plain tensor-core kernels do not take)
    if got != B.OK:
        return
    names = kernel_names(case.run)
    assert any("act_unpack" in n for n in names) != fused
    if fused:
        case.check()
        assert algo != B.ALGO_TENSOR or instance(names) is not None
    else:
        torch.cuda.synchronize()
        assert torch.equal(case.dw, plain)


def test_threads():
    """Four host threads, a stream each, calls of many sizes in turn: the plans and kernels are shared."""
    sizes = [(m, c, k) for m in (300, 2100) for c in (64, 130, 330) for k in (72, 250)]
    cases = [[Case(linear(*s), torch.bfloat16, B.ACT_E4M3) for s in sizes] for _ in range(4)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]

    def work(i):
        order = np.random.default_rng(i).permutation(len(sizes) * 5)
        for j in order:
            cases[i][j % len(sizes)].run(stream=streams[i])
    with ThreadPoolExecutor(4) as pool:
        list(pool.map(work, range(4)))
    torch.cuda.synchronize()
    for row in zip(*cases):
        first = row[0].result()[1]
        assert all(np.array_equal(first, c.result()[1]) for c in row[1:])
        row[0].check()
