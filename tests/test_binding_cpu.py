"""What the binding makes of its arguments and of the process around it: no GPU needed."""
import numpy as np
import pytest
import torch

from paper_1908_05460_b200 import binding as B
from paper_1908_05460_b200 import build as build_mod


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
