"""Layers that keep their inputs in 8 bits, as a training program uses them, against 64-bit references of the values that are kept.

Tolerances.  A filter gradient from kept values is exact up to its fp32 sum (129 * 2^-23 of the sum of magnitudes) and its rounding to the weight's type, half
a step: 2^-8 (bf16).  What reaches a layer as dy went through torch's kernels and is taken from there (a hook), so that only this library's arithmetic is compared."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

import act8_ref as R
from oracle import oracle
from paper_1908_05460_b200 import binding as B
from paper_1908_05460_b200.autograd import GAConv2d, GALinear, GARMSNorm, linear_filter_gradient
from paper_1908_05460_b200.packed import FORMATS, PackedActivation

pytestmark = pytest.mark.gpu
TOL = 129 * 2.0 ** -23
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DTYPES = [torch.bfloat16, torch.float32]


def kept(x, fmt):
    """What is kept of x [rows, cols], float64."""
    return R.pack(R.f64(x), FORMATS[fmt])[2]


def check_linear_gradient(grad, x64, dy64):
    want, size = dy64.T @ x64, np.abs(dy64).T @ np.abs(x64)
    assert np.all(np.abs(R.f64(grad) - want) <= HALF[grad.dtype] * np.abs(want) + TOL * size)


@pytest.mark.parametrize("fmt", sorted(FORMATS))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape, features", [((7, 5, 24), 40), ((300, 33), 17), ((1, 64), 8), ((2, 3, 130), 129), ((2000, 72), 264)])
def test_linear(shape, features, dtype, fmt):
    torch.manual_seed(1)
    x = torch.randn(shape, device="cuda").to(dtype).requires_grad_()
    layer = GALinear(shape[-1], features, checkpoint=fmt, dtype=dtype)
    y = layer(x)
    assert torch.equal(y, F.linear(x, layer.weight, layer.bias))
    dy = (0.01 * torch.randn(y.shape, device="cuda")).to(dtype)
    y.backward(dy)
    rows, grad = x.detach().reshape(-1, shape[-1]), dy.reshape(-1, features)
    check_linear_gradient(layer.weight.grad, kept(rows, fmt), R.f64(grad))
    assert torch.equal(x.grad, dy.matmul(layer.weight)) and torch.equal(layer.bias.grad, grad.sum(0))


def test_linear_inputs_of_all_kinds():
    """Rows apart from one another, a transposed input, a view off the 16-byte boundary, no tokens, and a frozen weight."""
    torch.manual_seed(2)
    layer = GALinear(48, 32, bias=False)
    wide = torch.randn(60, 100, device="cuda").bfloat16()
    for x in (wide[:, :48], wide[:, 4:52], wide.t()[:48].t(), wide[:48, :60].t(), wide[0, :48]):
        layer.weight.grad = None
        y = layer(x)
        dy = torch.randn_like(y)
        y.backward(dy)
        check_linear_gradient(layer.weight.grad, kept(x.reshape(-1, 48), "e4m3"), R.f64(dy.reshape(-1, 32)))
    layer.weight.grad = None
    layer(wide[:0, :48]).sum().backward()
    assert (layer.weight.grad == 0).all()
    layer.weight.requires_grad_(False)
    before = B.gaconv_launch_count()
    x = wide[:, :48].clone().requires_grad_()
    layer(x).sum().backward()
    assert B.gaconv_launch_count() == before and x.grad is not None          # nothing was kept
    strided = layer.weight.requires_grad_()
    y = layer(wide[:, :48].contiguous())
    y.backward(torch.randn(60, 64, device="cuda").bfloat16()[:, ::2])        # a gradient whose channels are apart
    assert strided.grad is not None


def test_linear_refuses():
    with pytest.raises(ValueError):
        GALinear(8, 8, checkpoint=None)
    with pytest.raises(ValueError):
        GALinear(8, 8, checkpoint="fp4")
    with pytest.raises(ValueError):
        GALinear(8, 8, dtype=torch.float16)
    layer = GALinear(16, 8)
    x = torch.zeros(4, 16, device="cuda", dtype=torch.bfloat16)
    for bad in (x.float(), x[:, :8]):
        with pytest.raises(ValueError):
            layer(bad)
    with pytest.raises(ValueError):
        layer(x, PackedActivation.pack(x[:2]))
    with pytest.raises(TypeError):
        PackedActivation.pack(x.half())
    with pytest.raises(ValueError):
        linear_filter_gradient(PackedActivation.pack(x), x[:2])
    with pytest.raises(ValueError):
        GARMSNorm(16)(x[:, :8])
    with pytest.raises(ValueError):
        GARMSNorm(16)(x, x[:2])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layer_args, hw", [((16, 24, 3, 1, 1), 12), ((40, 32, 3, 2, 1), 9), ((17, 13, 5, 1, 2), 8), ((64, 128, 1, 1, 0), 8)])
@pytest.mark.parametrize("fmt", sorted(FORMATS))
def test_convolution(fmt, layer_args, hw, dtype):
    torch.manual_seed(3)
    c, k, r, stride, pad = layer_args
    layer = GAConv2d(c, k, r, stride, pad, dtype=dtype, checkpoint=fmt)
    x = torch.randn(6, c, hw, hw, device="cuda").relu().to(dtype).requires_grad_()
    y = layer(x)
    dy = (0.01 * torch.randn(y.shape, device="cuda")).to(dtype)
    y.backward(dy)
    x64 = kept(x.detach().permute(0, 2, 3, 1).reshape(-1, c), fmt).reshape(6, hw, hw, c).transpose(0, 3, 1, 2)
    want, size = oracle.dw_exact(x64, R.f64(dy), oracle.Shape(6, c, hw, hw, k, r, r, stride, stride, pad, pad))
    assert np.all(np.abs(R.f64(layer.weight.grad) - want) <= HALF[dtype] * np.abs(want) + TOL * size)
    plain = GAConv2d(c, k, r, stride, pad, dtype=dtype)
    plain.weight.data.copy_(layer.weight.data)
    x2 = x.detach().clone().requires_grad_()
    plain(x2).backward(dy)
    # the same call of torch's with the same values: its algorithm may differ by the alignment of a placeholder, so one rounding of the sums is allowed
    assert torch.allclose(x2.grad.float(), x.grad.float(), rtol=2 * HALF[dtype], atol=1e-5)


def test_convolution_with_a_schedule():
    """Every method of a schedule from kept values."""
    torch.manual_seed(4)
    x = torch.randn(8, 16, 8, 8, device="cuda").relu()
    x64 = kept(x.permute(0, 2, 3, 1).reshape(-1, 16), "int8").reshape(8, 8, 8, 16).transpose(0, 3, 1, 2)
    shape = oracle.Shape(8, 16, 8, 8, 24, 3, 3, 1, 1, 1, 1)
    for method in (B.METHOD_ZERO, B.METHOD_RANDOM, B.METHOD_TOP1):
        sched = B.Schedule(2, B.SCHED_ALL_LAYERS_EVERY_4TH_BATCH, method, 0.0, 9)
        layer = GAConv2d(16, 24, 3, 1, 1, schedule=sched, layer_index=1, checkpoint="int8")
        for step in (0, 3):
            layer.step = step
            layer.weight.grad = None
            y = layer(x)
            dy = torch.randn_like(y) * 0.01
            y.backward(dy)
            got = R.f64(layer.weight.grad)
            if step == 0:
                want, size = oracle.dw_exact(x64, R.f64(dy), shape)
            elif method == B.METHOD_TOP1:
                want, size = oracle.dw_top1(x64, R.f64(dy), shape)
            else:
                plain = torch.empty(24, 16, 3, 3, device="cuda")
                d = B.make_desc(__import__("paper_1908_05460_b200.layers", fromlist=["ConvLayer"]).ConvLayer("l", 8, 16, 8, 8, 24, 3, 3, 1, 1), torch.float32, dw_layout=B.DW_KCRS)
                sched.run_layer(1, step, None, None, plain, d)
                assert np.array_equal(got, R.f64(plain))
                continue
            assert np.all(np.abs(got - want) <= TOL * size)
    with pytest.raises(ValueError):
        GAConv2d(4, 4, 3, checkpoint="e5m2")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [40, 64, 333])
def test_norm(cols, dtype):
    torch.manual_seed(5)
    u = 2.0 ** -24
    norm = GARMSNorm(cols, checkpoint="int8", dtype=dtype)
    norm.weight.data += 0.1 * torch.randn(cols, device="cuda").to(dtype)
    x = torch.randn(4, 7, cols, device="cuda").to(dtype).requires_grad_()
    res = torch.randn(4, 7, cols, device="cuda").to(dtype).requires_grad_()
    y, s, packed = norm(x, res)
    assert torch.equal(s, x + res)
    s64, w64 = R.f64(s).reshape(-1, cols), R.f64(norm.weight)
    y64, rstd = R.norm(s64, w64, 1e-6)
    assert np.all(np.abs(R.f64(y).reshape(-1, cols) - y64) <= ((HALF[dtype] if dtype is torch.bfloat16 else 0) + 80 * u) * np.abs(y64))
    codes, scales, _ = R.pack(R.f64(y).reshape(-1, cols), 1)
    assert np.array_equal(packed.codes.cpu().numpy().reshape(codes.shape), codes) and np.array_equal(packed.scales.cpu().numpy().reshape(scales.shape), scales)
    dy, ds = torch.randn_like(y), torch.randn_like(s)
    torch.autograd.backward((y, s), (dy, ds))
    dx, dw, size, wsize = R.norm_grad(R.f64(dy).reshape(-1, cols), R.f64(ds).reshape(-1, cols), s64, w64, rstd)
    half = HALF[dtype] if dtype is torch.bfloat16 else 0
    assert np.all(np.abs(R.f64(x.grad).reshape(-1, cols) - dx) <= half * np.abs(dx) + 120 * u * size)        # (rstd is the library's own: 40 u more)
    assert torch.equal(x.grad, res.grad)
    assert np.all(np.abs(R.f64(norm.weight.grad) - dw) <= half * np.abs(dw) + 240 * u * wsize)
    # the parts on their own: without a residual, and with only the sum used behind it
    x.grad = None
    out = norm(x)
    assert out.sum is None
    out.y.backward(dy)
    assert x.grad is not None
    x.grad = None
    norm(x, res).sum.backward(ds)
    assert torch.equal(x.grad, ds)


@pytest.mark.parametrize("dtype", DTYPES)
def test_block_of_layers(dtype):
    """A norm, two projections of its output that share what it kept, a gate, a projection back and the residual: a run of the calls as a model makes them."""
    torch.manual_seed(6)
    tokens, d, hidden = 130, 96, 200
    norm = GARMSNorm(d, checkpoint="e4m3", dtype=dtype)
    gate, up = (GALinear(d, hidden, bias=False, dtype=dtype) for _ in range(2))
    down = GALinear(hidden, d, bias=False, checkpoint="int8", dtype=dtype)
    x = torch.randn(tokens, d, device="cuda").to(dtype).requires_grad_()
    res = torch.randn(tokens, d, device="cuda").to(dtype).requires_grad_()
    grads = {}

    def watch(name, t):
        t.register_hook(lambda g: grads.__setitem__(name, g.clone()))
        return t

    def step():
        y, s, packed = norm(x, res)
        g, u = watch("gate", gate(y, packed)), watch("up", up(y, packed))
        h = F.silu(g) * u
        out = watch("down", down(h))
        return y, h, out + s

    y, h, out = step()
    out.square().mean().backward()
    for name, layer, inp, fmt in (("gate", gate, y, "e4m3"), ("up", up, y, "e4m3"), ("down", down, h, "int8")):
        check_linear_gradient(layer.weight.grad, kept(inp.detach(), fmt), R.f64(grads[name]))
    assert all(p.grad is not None and torch.isfinite(p.grad).all() for p in (x, res, norm.weight))


def test_training_step_in_a_graph():
    """Forward and backward captured and replayed on another input give what the calls give."""
    torch.manual_seed(7)
    norm, lin = GARMSNorm(72, checkpoint="e4m3"), GALinear(72, 40)
    params = [norm.weight, lin.weight, lin.bias]
    x = torch.randn(50, 72, device="cuda").bfloat16()
    res = torch.randn(50, 72, device="cuda").bfloat16()
    target = torch.randn(50, 40, device="cuda").bfloat16()

    def grads():
        y, s, packed = norm(x, res)
        loss = (lin(y, packed) - target).float().square().sum() + s.float().square().sum()
        return torch.autograd.grad(loss, params)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            grads()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = grads()
    for seed in (8, 9):
        torch.manual_seed(seed)
        x.copy_(torch.randn(50, 72, device="cuda")); res.copy_(torch.randn(50, 72, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [g.clone() for g in captured]
        want = grads()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_memory_that_is_kept():
    """A layer holds one byte and a thirty-second an element of its input, not the input."""
    layer = GALinear(1024, 64, bias=False)
    x = torch.randn(4096, 1024, device="cuda").bfloat16()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = layer(x)
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated() - before - y.numel() * 2
    assert 4096 * 1024 <= held <= 4096 * 1024 * 1.1
    del x
    loss = y.sum()
    del y
    loss.backward()
    assert torch.isfinite(layer.weight.grad).all()
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - before < 4096 * 1024          # freed with the backward pass, though the loss lives on
