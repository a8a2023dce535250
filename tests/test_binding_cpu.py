"""What the binding makes of its arguments and of the process around it: no GPU needed."""
import os

import numpy as np
import pytest
import torch

from paper_1908_05460_b200 import binding as B
from paper_1908_05460_b200 import build as build_mod
from paper_1908_05460_b200.autograd import GAConv2d
from paper_1908_05460_b200.layers import config1_layer


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()
    B.load()


def test_pointers_are_tensors_addresses_or_none():
    t = torch.zeros(4)
    assert B._ptr(t) == t.data_ptr() and B._ptr(4096) == 4096 and B._ptr(None) is None
    desc = B.make_rows_desc(1, 16, torch.bfloat16)
    for wrong in (b"\0" * 32, "text", np.zeros(16), bytearray(16), 1.5):
        with pytest.raises(AttributeError):
            B._ptr(wrong)
        with pytest.raises(AttributeError):
            B.gaconv_act_pack(wrong, t, t, desc, 0)


def test_a_forked_process_hears_it_from_torch(monkeypatch):
    """A process forked after CUDA has started cannot use it, and torch.cuda.current_device() says so; the short way to the stream does not ask."""
    ways = []
    monkeypatch.setattr(B, "_cuda_runs", True)
    monkeypatch.setattr(B, "_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda device: ways.append("short") or 7)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: ways.append("torch") or 0)
    assert B._stream(None) == 7 and ways == ["short"]
    read, write = os.pipe()
    pid = os.fork()
    if pid == 0:
        try:
            del ways[:]
            B._stream(None)
            os.write(write, ways[0].encode())
        finally:
            os._exit(0)
    os.close(write)
    with os.fdopen(read, "rb") as f:
        assert f.read() == b"torch"
    os.waitpid(pid, 0)
    assert B._cuda_runs          # the parent's own is left alone


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int8, torch.float8_e4m3fn])
def test_layers_of_other_types_are_refused(dtype):
    """They were fp32 to the library, which reads four bytes an element."""
    with pytest.raises(TypeError):
        B.make_desc(config1_layer(), dtype)
    with pytest.raises(TypeError):
        GAConv2d(4, 8, 3, device="cpu").filter_gradient(torch.zeros(2, 4, 5, 5).to(dtype), torch.zeros(2, 8, 3, 3).to(dtype))
