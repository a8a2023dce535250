"""What the layers that keep their inputs in 8 bits hand to the library, and what they refuse: no GPU needed, the library's calls are replaced by recorders."""
import contextlib
import ctypes
import random
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

from paper_1908_05460_b200 import binding as B
from paper_1908_05460_b200 import build as build_mod
from paper_1908_05460_b200.autograd import GAConv2d, GALinear, GARMSNorm, check_async_status
from paper_1908_05460_b200.layers import ConvLayer
from paper_1908_05460_b200.packed import PackedActivation

ENQUEUE = ["gaconv_act_pack", "gaconv_act_unpack", "gaconv_dw_from_packed", "gaconv_dw_exact", "gaconv_rmsnorm_forward", "gaconv_rmsnorm_backward", "gaconv_workspace_init"]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()
    B.load()


@pytest.fixture
def calls(monkeypatch):
    """The calls that would have been made, in order: (name, arguments).  "cpu" and "meta" stand for two devices."""
    made = []
    for name in ENQUEUE:
        monkeypatch.setattr(B, name, lambda *a, name=name, **k: made.append((name, a)))
    monkeypatch.setattr(B, "gaconv_collect_async_status", lambda *a, **k: None, raising=False)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    return made


def linear_desc(rows=4, c=16, k=8):
    return B.make_desc(ConvLayer("linear", rows, c, 1, 1, k, 1, 1), torch.bfloat16, dy_layout=B.DY_NPQK)


def test_tensors_on_several_devices_are_refused(calls):
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    for norm in (GARMSNorm(16, device="cpu"), GARMSNorm(16, checkpoint="int8", device="cpu")):
        norm(x, x)
        assert calls.pop()[0] == "gaconv_rmsnorm_forward"
        with pytest.raises(ValueError, match="several devices"):
            norm(x, x.to("meta"))
        with pytest.raises(ValueError, match="several devices"):
            norm(x.to("meta"))
    here, there = PackedActivation(4, 16, x.dtype, "e4m3", "cpu"), PackedActivation(4, 16, x.dtype, "e4m3", "meta")
    layer = GALinear(16, 8, device="cpu")
    layer(x, here)
    with pytest.raises(ValueError, match="several devices"):
        layer(x, there)
    dy, dw = torch.zeros(4, 8, dtype=x.dtype), torch.zeros(8, 16)
    for packed, dy, dw in ((there, dy, dw), (here, dy.to("meta"), dw), (here, dy, dw.to("meta"))):
        with pytest.raises(ValueError, match="several devices"):
            packed.filter_gradient(dy, dw, linear_desc())
    assert not calls


def test_gradients_with_gaps_or_repeats_are_refused(calls):
    """An expanded gradient ends before the kernel does; what lies between the rows of a view is not the gradient's."""
    packed = PackedActivation(4, 16, torch.bfloat16, "e4m3", "cpu")
    one, dw = torch.zeros(1, 8, dtype=torch.bfloat16), torch.zeros(8, 16)
    for dy in (one.expand(4, 8), one[:, :1].expand(4, 8), torch.zeros(4, 10, dtype=one.dtype)[:, :8], torch.zeros(8, 8, dtype=one.dtype)[::2],
               torch.zeros(64, dtype=one.dtype).as_strided((4, 8), (7, 1)), torch.zeros(64, dtype=one.dtype).as_strided((4, 8), (3, 3))):
        with pytest.raises(ValueError, match="gaps"):
            packed.filter_gradient(dy, dw, linear_desc())
    for dw in (torch.zeros(8, 32)[:, :16], torch.zeros(1, 16).expand(8, 16)):
        with pytest.raises(ValueError, match="gaps"):
            packed.filter_gradient(torch.zeros(4, 8, dtype=one.dtype), dw, linear_desc())
    assert not calls
    for dy, dw in ((torch.zeros(4, 8, dtype=one.dtype), torch.zeros(8, 16)), (torch.zeros(8, 4, dtype=one.dtype).t(), torch.zeros(8, 16, 1, 1)),
                   (torch.zeros(4, 8, 1, 1, dtype=one.dtype).contiguous(memory_format=torch.channels_last), torch.zeros(8, 16))):
        packed.filter_gradient(dy, dw, linear_desc())
        assert calls.pop()[0] == "gaconv_dw_from_packed"


def test_norm_weights_that_are_not_dense(calls):
    """A weight that is every other element of a longer one, or one element for all channels, is read as its values, not as the memory behind its first."""
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    norm = GARMSNorm(16, device="cpu")
    for weight in (torch.arange(32.0).bfloat16()[::2], torch.ones(1).bfloat16().expand(16), torch.arange(40.0).bfloat16()[3:19]):
        norm.weight = torch.nn.Parameter(weight)
        norm(x)
        given = calls.pop()[1][2]
        assert given.is_contiguous() and given.data_ptr() % 16 == 0 and torch.equal(given, weight)


@pytest.mark.parametrize("rows, cols", [(1, (1 << 32) + 8), (1, 1 << 31), ((1 << 64) + 4, 8), (1, 8 - (1 << 32))])
def test_rows_that_the_descriptor_has_no_room_for(rows, cols):
    """They were another, smaller problem: 8 channels of 2^32 + 8."""
    with pytest.raises(B.GaconvError) as e:
        B.make_rows_desc(rows, cols, torch.bfloat16)
    assert e.value.status == B.ERR_UNSUPPORTED


@pytest.mark.filterwarnings("ignore:Initializing zero-element")
@pytest.mark.parametrize("shape, features", [((3, 0), 5), ((2, 3, 0), 5), ((0,), 5), ((3, 5), 0), ((2, 3, 5), 0), ((5,), 0), ((0, 5), 4), ((2, 0, 5), 4), ((3, 0), 0)])
def test_linear_layers_without_tokens_or_features(shape, features, calls):
    """Nothing is kept, and the gradients are torch's."""
    layer, plain = GALinear(shape[-1], features, dtype=torch.float32, device="cpu"), torch.nn.Linear(shape[-1], features)
    x, z = torch.zeros(shape, requires_grad=True), torch.zeros(shape, requires_grad=True)
    layer(x).sum().backward()
    plain(z).sum().backward()
    for got, want in ((x.grad, z.grad), (layer.weight.grad, plain.weight.grad), (layer.bias.grad, plain.bias.grad)):
        assert got.shape == want.shape and torch.equal(got, want)
    assert not calls


@pytest.mark.parametrize("checkpoint", [None, "e4m3"])
@pytest.mark.parametrize("order", [torch.contiguous_format, torch.channels_last])
def test_convolution_gradients_off_the_boundary(checkpoint, order, calls):
    """The gradients of two outputs that torch.cat has joined are parts of one tensor, the second one's from an odd element on; an input may be such a part, too."""
    layer = GAConv2d(4, 13, 3, 1, 1, dtype=torch.bfloat16, device="cpu", checkpoint=checkpoint)
    whole = torch.zeros(6 * 13 * 49, dtype=torch.bfloat16)
    dy = (whole.view(6, 13, 7, 7) if order is torch.contiguous_format else whole.view(6, 7, 7, 13).permute(0, 3, 1, 2))[3:]
    dy.copy_(torch.randn(dy.shape))
    x = torch.zeros(6 * 4 * 49 + 5, dtype=torch.bfloat16)[5:].view(6, 7, 7, 4).permute(0, 3, 1, 2)[3:]
    assert dy.data_ptr() % 16 != 0 and x.data_ptr() % 16 != 0 and dy.is_contiguous(memory_format=order)
    if checkpoint is None:
        layer.filter_gradient(x, dy)
        (_, _), (name, (given_x, given, _, desc)) = calls
        assert name == "gaconv_dw_exact" and given_x.data_ptr() % 16 == 0 and given_x.is_contiguous(memory_format=torch.channels_last)
    else:
        layer.packed_filter_gradient(PackedActivation(3 * 49, 4, x.dtype, checkpoint, "cpu"), x.shape, dy)
        name, (_, _, _, _, given, _, desc, _) = calls[-1]
        assert name == "gaconv_dw_from_packed"
    assert given.data_ptr() % 16 == 0 and given.is_contiguous(memory_format=order) and torch.equal(given, dy)
    assert desc.dy_layout == (B.DY_NPQK if order is torch.channels_last else B.DY_NKPQ)


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_evaluation_keeps_nothing(mode, calls):
    """Where no gradients are recorded nothing is packed, though the weights require them; the norm's 8-bit form can be left out."""
    linear, conv = GALinear(16, 8, device="cpu"), GAConv2d(4, 8, 3, 1, 1, device="cpu", checkpoint="int8")
    norm = GARMSNorm(16, device="cpu", checkpoint="int8")
    x, maps = torch.randn(3, 16).bfloat16(), torch.randn(2, 4, 5, 5)
    with mode():
        y, z = linear(x), conv(maps)
        assert not calls
        assert torch.equal(y, torch.nn.functional.linear(x, linear.weight, linear.bias)) and torch.equal(z, torch.nn.functional.conv2d(maps, conv.weight, None, 1, 1))
        assert linear(x, PackedActivation(3, 16, x.dtype, "e4m3", "cpu")).shape == (3, 8)
        out = norm(x, keep=False)
        assert out.packed is None and out.y.shape == x.shape
        name, given = calls.pop()
        assert name == "gaconv_rmsnorm_forward" and given[5] is None and given[6] is None
        assert norm(x).packed is not None
    calls.clear()
    linear(x), conv(maps)
    assert [name for name, _ in calls] == ["gaconv_act_pack"] * 2


def test_offsets_beyond_64_bits_are_refused():
    """Rows times their distance, in bytes, is a number of the kernels' address arithmetic."""
    for stride, rows, fine in ((1 << 40, 1 << 20, True), (1 << 40, (1 << 20) + 1, False), (1 << 40, (1 << 31) - 1, False), (1 << 29, (1 << 31) - 1, True), ((1 << 29) + 2, (1 << 31) - 1, False)):
        for name in ("x_stride", "r_stride", "s_stride", "y_stride"):
            desc = B.make_rows_desc(rows, 8, torch.float32, **{name: stride})
            if fine:
                assert B.gaconv_act_sizes(desc) == (rows * 16, rows)
            else:
                with pytest.raises(B.GaconvError) as e:
                    B.gaconv_act_sizes(desc)
                assert e.value.status == B.ERR_UNSUPPORTED


def test_a_descriptor_keeps_its_own_workspace(calls, monkeypatch):
    """filter_gradient brings a workspace for the call; afterwards the descriptor has the caller's again, or none, also where the library refuses."""
    packed, dy, dw = PackedActivation(4, 16, torch.bfloat16, "e4m3", "cpu"), torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8, 16)
    seen = []
    for refuse in (False, True):
        def call(*a):
            seen.append(a[6].workspace)
            if refuse:
                raise B.GaconvError(B.ERR_BAD_DESC, "gaconv_dw_from_packed")
        monkeypatch.setattr(B, "gaconv_dw_from_packed", call)
        for own in ((None, 0), (4096, 512)):
            desc = linear_desc()
            desc.workspace, desc.workspace_bytes = own
            with pytest.raises(B.GaconvError) if refuse else contextlib.nullcontext():
                packed.filter_gradient(dy, dw, desc)
            assert (desc.workspace, desc.workspace_bytes) == own and seen.pop() not in (None, 4096)


def test_a_kernel_that_gave_up_is_reported(calls, monkeypatch):
    """The workspace of a layer's call is given back at once; its status is collected before, and check_async_status raises for it once."""
    raised = [B.OK]
    workspaces = []
    monkeypatch.setattr(B, "gaconv_workspace_init", lambda ws, n, **k: workspaces.append(ws) or ws[:256].zero_())

    def kernel(*a):
        calls.append(("gaconv_dw_from_packed", a))
        workspaces[-1][0] = 1          # what a kernel does that gives up

    def collect(desc, stream=None):
        ws = workspaces.pop()
        assert desc.workspace == ws.data_ptr() and calls[-1][0] == "gaconv_dw_from_packed"
        if int(ws[:4].view(torch.int32)) != 0:
            raised[0] = B.ERR_TIMEOUT

    def poll(stream=None):
        status, raised[0] = raised[0], B.OK
        return status
    monkeypatch.setattr(B, "gaconv_dw_from_packed", kernel)
    monkeypatch.setattr(B, "gaconv_collect_async_status", collect)
    monkeypatch.setattr(B, "gaconv_poll_collected_status", poll)
    layer = GALinear(16, 8, device="cpu")
    check_async_status()
    layer(torch.randn(3, 16).bfloat16()).sum().backward()
    with pytest.raises(B.GaconvError) as e:
        check_async_status()
    assert e.value.status == B.ERR_TIMEOUT
    check_async_status()
    # a convolution without a checkpoint keeps its workspaces, which are asked one by one, all of them before anything is raised
    conv = GAConv2d(4, 8, 3, 1, 1, device="cpu")
    words = {}
    for hw in (5, 6):
        conv(torch.randn(2, 4, hw, hw)).sum().backward()
    descs = [desc for desc, _ in conv._desc_cache.values()]
    assert len(descs) == 2
    words = {id(d): B.ERR_TIMEOUT for d in descs}
    monkeypatch.setattr(B, "gaconv_poll_async_status", lambda desc, stream=None: words.pop(id(desc), B.OK))
    with pytest.raises(B.GaconvError):
        check_async_status(torch.nn.Sequential(conv))
    check_async_status(conv)


def test_status_calls_check_their_arguments():
    lib, desc = B.load(), linear_desc()
    ref = ctypes.byref(desc)
    assert lib.gaconv_collect_async_status(None, None) == B.ERR_NULL_POINTER and lib.gaconv_collect_async_status(ref, None) == B.ERR_NULL_POINTER
    desc.workspace, desc.workspace_bytes = 4096 + 8, 1 << 20
    assert lib.gaconv_collect_async_status(ref, None) == B.ERR_MISALIGNED
    desc.workspace, desc.workspace_bytes = 4096, 255
    assert lib.gaconv_collect_async_status(ref, None) == B.ERR_WORKSPACE_TOO_SMALL


def test_plans_asked_for_by_several_threads():
    """More sizes than the table of plans has room for, in other orders, by eight threads at once: each gets what one thread alone gets."""
    sizes = [(m, c, k) for m in (1, 7, 100, 513, 4099, 20000) for c in (8, 33, 130, 512, 1000) for k in range(40, 1240, 80)]

    def workspace(size):
        return B.gaconv_packed_workspace_size(linear_desc(*size), B.METHOD_EXACT)
    want = {size: workspace(size) for size in sizes}

    def work(seed):
        order = sizes * 3
        random.Random(seed).shuffle(order)
        return all(workspace(size) == want[size] for size in order)
    with ThreadPoolExecutor(8) as pool:
        assert all(pool.map(work, range(8)))


def test_descriptors_of_another_type_are_refused(calls):
    """The kernels read dy as what the descriptor says: bf16 gradients under an fp32 descriptor are half as long as what is read."""
    for dtype, other in ((torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)):
        packed, dy, dw = PackedActivation(4, 16, dtype, "e4m3", "cpu"), torch.zeros(4, 8, dtype=dtype), torch.zeros(8, 16)
        desc = {t: B.make_desc(ConvLayer("linear", 4, 16, 1, 1, 8, 1, 1), t, dy_layout=B.DY_NPQK) for t in (dtype, other)}
        with pytest.raises(ValueError, match="descriptor"):
            packed.filter_gradient(dy, dw, desc[other])
        assert not calls
        packed.filter_gradient(dy, dw, desc[dtype])
        assert calls.pop()[0] == "gaconv_dw_from_packed"
        calls.clear()


def test_a_layer_moved_to_another_device_takes_a_workspace_there(calls):
    layer = GAConv2d(4, 8, 3, 1, 1, device="cpu")
    x = torch.zeros(2, 4, 5, 5)
    here, there = layer._desc(x), layer._desc(x.to("meta"))
    assert here is layer._desc(x) and here is not there
    assert [ws.device.type for _, ws in layer._desc_cache.values()] == ["cpu", "meta"]


def test_convolutions_off_the_current_device(calls, monkeypatch):
    """The library's calls go to the current device, so that the tensors' one is made current around them; tensors of several are refused."""
    current, at = [], []

    @contextlib.contextmanager
    def device(d):
        current.append(d)
        yield
        current.pop()
    monkeypatch.setattr(torch.cuda, "device", device)
    for name in ("gaconv_dw_exact", "gaconv_workspace_init"):
        monkeypatch.setattr(B, name, lambda *a, name=name, **k: at.append((name, list(current))))
    layer = GAConv2d(4, 8, 3, 1, 1, device="cpu")
    x, dy = torch.zeros(2, 4, 5, 5), torch.zeros(2, 8, 5, 5)
    layer.filter_gradient(x, dy)
    assert [name for name, _ in at] == ["gaconv_workspace_init", "gaconv_dw_exact"] and all(devices == [x.device] for _, devices in at)
    for bad in ((x.to("meta"), dy), (x, dy.to("meta"))):
        with pytest.raises(ValueError, match="several devices"):
            layer.filter_gradient(*bad)
    assert len(at) == 2


def test_gradients_of_another_layer_are_refused(calls):
    """A gradient that is smaller than the activations' shape says was read past its end."""
    layer = GAConv2d(4, 8, 3, 2, 1, device="cpu")
    x, dy = torch.zeros(2, 4, 7, 6), torch.zeros(2, 8, 4, 3)
    layer.filter_gradient(x, dy)
    assert calls.pop()[0] == "gaconv_dw_exact"
    calls.clear()
    for bad in ((x, dy[:1]), (x, dy[:, :7]), (x, dy[:, :, :3]), (x, dy[0]), (x[:, :3], dy), (x[0], dy), (torch.zeros(3, 4, 7, 6), dy), (torch.zeros(2, 4, 9, 6), dy)):
        with pytest.raises(ValueError):
            layer.filter_gradient(*bad)
    assert not calls
