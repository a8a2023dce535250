"""The layers as parts of larger programs on the GPU: gradients that arrive as parts of others, evaluation, status of calls whose scratch is gone."""
import numpy as np
import pytest
import torch

import act8_ref as R
from oracle import oracle
from paper_1908_05460_b200 import binding as B
from paper_1908_05460_b200.autograd import GAConv2d, GALinear, GARMSNorm, check_async_status
from paper_1908_05460_b200.graph_names import kernel_names
from paper_1908_05460_b200.packed import FORMATS

pytestmark = pytest.mark.gpu
TOL = 129 * 2.0 ** -23          # of the sum of magnitudes: chains of at most 128 additions, each off by 2^-23 of the running sum, and the planes of fp32 operands
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("order", [torch.contiguous_format, torch.channels_last])
@pytest.mark.parametrize("checkpoint", [None, "e4m3"])
def test_outputs_joined_by_cat(checkpoint, order, dtype):
    """The second branch's gradient starts 3 * 13 * 49 elements into the joint one, off the 16-byte boundary."""
    torch.manual_seed(11)
    layers = [GAConv2d(5, 13, 3, 1, 1, dtype=dtype, checkpoint=checkpoint) for _ in range(2)]
    x = torch.randn(6, 5, 7, 7, device="cuda").to(dtype).contiguous(memory_format=torch.channels_last)
    parts = [x[:3], x[3:]]
    dy = (0.01 * torch.randn(6, 13, 7, 7, device="cuda")).to(dtype).contiguous(memory_format=order)
    assert dy[3:].data_ptr() % 16 != 0
    torch.cat([layer(part) for layer, part in zip(layers, parts)]).backward(dy)
    for layer, part, grad in zip(layers, parts, (dy[:3], dy[3:])):
        x64 = R.f64(part)
        if checkpoint is not None:
            x64 = R.pack(R.f64(part.permute(0, 2, 3, 1).reshape(-1, 5)), FORMATS[checkpoint])[2].reshape(3, 7, 7, 5).transpose(0, 3, 1, 2)
        want, size = oracle.dw_exact(x64, R.f64(grad), oracle.Shape(3, 5, 7, 7, 13, 3, 3, 1, 1, 1, 1))
        assert np.all(np.abs(R.f64(layer.weight.grad) - want) <= HALF[dtype] * np.abs(want) + TOL * size)


def test_evaluation_launches_nothing():
    """GALinear and GAConv2d without gradients: torch's forward and no kernel of this library; the norm alone, without codes."""
    torch.manual_seed(12)
    linear, conv, norm = GALinear(72, 40), GAConv2d(8, 16, 3, 1, 1, checkpoint="e4m3"), GARMSNorm(72, checkpoint="int8")
    x, maps = torch.randn(9, 72, device="cuda").bfloat16(), torch.randn(2, 8, 6, 6, device="cuda")
    y, z, n = linear(x), conv(maps), norm(x).y
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            before = B.gaconv_launch_count()
            assert torch.equal(linear(x), y) and torch.equal(conv(maps), z)
            assert B.gaconv_launch_count() == before
            out = norm(x, keep=False)
            assert out.packed is None and torch.equal(out.y, n) and B.gaconv_launch_count() == before + 1


def test_status_outlives_the_workspace(monkeypatch):
    """A status word that is raised in a call's workspace (from the host: no wait is made to run out) is reported after the workspace went back and was used again, once."""
    torch.manual_seed(13)
    layer, conv = GALinear(72, 40), GAConv2d(8, 16, 3, 1, 1, checkpoint="e4m3")
    x, maps = torch.randn(9, 72, device="cuda").bfloat16(), torch.randn(2, 8, 6, 6, device="cuda")
    check_async_status(layer, conv)
    attach, run = B.attach_packed_workspace, B.gaconv_dw_from_packed
    held = []

    def attach_and_hold(*a, **k):
        held.append(attach(*a, **k))
        return held[-1]

    def run_and_give_up(*a):
        run(*a)
        held.pop()[:4].copy_(torch.tensor([1, 0, 0, 0], dtype=torch.uint8))
    for module, inp in ((layer, x), (conv, maps)):
        with monkeypatch.context() as m:
            m.setattr(B, "attach_packed_workspace", attach_and_hold)
            m.setattr(B, "gaconv_dw_from_packed", run_and_give_up)
            module(inp).sum().backward()
        for _ in range(3):          # later calls, in the same memory
            module(inp).sum().backward()
        with pytest.raises(B.GaconvError) as e:
            check_async_status(module)
        assert e.value.status == B.ERR_TIMEOUT
        check_async_status(module)
        check_async_status()


def test_status_of_a_captured_step():
    """The collection is part of a captured backward pass; a word that the graph's call does not raise stays down."""
    torch.manual_seed(14)
    layer = GALinear(64, 48)
    x = torch.randn(40, 64, device="cuda").bfloat16()
    step = lambda: torch.autograd.grad(layer(x).float().square().sum(), [layer.weight])[0]  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = step().clone()
    torch.cuda.current_stream().wait_stream(side)
    assert sum("collect_status" in name for name in kernel_names(step)) == 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    graph.replay()
    check_async_status(layer)
    assert torch.equal(got, want)
