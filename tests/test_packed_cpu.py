"""Refusals and sizes of the calls on rows of activations, and the reference that the GPU tests use: no GPU needed."""
import ctypes

import numpy as np
import pytest
import torch

import act8_ref as R
from paper_1908_05460_b200 import binding as B
from paper_1908_05460_b200 import build as build_mod
from paper_1908_05460_b200.layers import ConvLayer

P = 4096        # an aligned address that is never read


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()
    B.load()


def test_sizes():
    for rows, cols in ((0, 5), (1, 1), (7, 31), (3, 32), (2, 33), (5, 1000), (1 << 20, 8192)):
        assert B.gaconv_act_sizes(B.make_rows_desc(rows, cols, torch.bfloat16)) == (rows * R.pitch(cols), rows * R.groups(cols))
    d = B.make_rows_desc(0, 5, torch.float32)
    assert B.gaconv_rmsnorm_workspace_size(d) > 0


@pytest.mark.parametrize("field, value, status", [
    ("struct_size", 8, B.ERR_BAD_DESC), ("cols", 0, B.ERR_BAD_DESC), ("cols", -3, B.ERR_BAD_DESC), ("rows", -1, B.ERR_BAD_DESC),
    ("dtype", 2, B.ERR_BAD_DESC), ("dtype", -1, B.ERR_BAD_DESC), ("format", 2, B.ERR_BAD_DESC), ("eps", -1.0, B.ERR_BAD_DESC),
    ("eps", float("nan"), B.ERR_BAD_DESC), ("x_stride", 63, B.ERR_BAD_DESC), ("r_stride", -64, B.ERR_BAD_DESC), ("s_stride", 1, B.ERR_BAD_DESC),
    ("y_stride", 63, B.ERR_BAD_DESC), ("rows", 1 << 31, B.ERR_UNSUPPORTED), ("cols", (1 << 28) + 1, B.ERR_UNSUPPORTED), ("x_stride", 1 << 50, B.ERR_UNSUPPORTED)])
def test_bad_rows_descriptors(field, value, status):
    lib, d = B.load(), B.make_rows_desc(4, 64, torch.bfloat16)
    setattr(d, field, value)
    r, n = ctypes.byref(d), ctypes.c_size_t(0)
    assert lib.gaconv_act_sizes(r, ctypes.byref(n), ctypes.byref(n)) == status
    assert lib.gaconv_act_pack(P, P, P, r, None) == status
    assert lib.gaconv_act_unpack(P, P, P, r, None) == status
    assert lib.gaconv_rmsnorm_forward(P, P, P, P, P, P, P, P, r, None) == status
    assert lib.gaconv_rmsnorm_backward(P, P, P, P, P, P, P, r, P, 1 << 30, None) == status
    assert lib.gaconv_rmsnorm_workspace_size(r, ctypes.byref(n)) == status


def test_bad_types():
    for dtype in (torch.float16, torch.int8, torch.float64):
        with pytest.raises(TypeError):
            B.make_rows_desc(4, 64, dtype)


def test_bad_pointers():
    lib = B.load()
    d = B.make_rows_desc(4, 64, torch.bfloat16)
    r = ctypes.byref(d)
    assert lib.gaconv_act_pack(P, P, P, None, None) == B.ERR_NULL_POINTER
    for call in (lib.gaconv_act_pack, lib.gaconv_act_unpack):
        for i in range(3):
            a = [P, P, P]
            a[i] = None
            assert call(*a, r, None) == B.ERR_NULL_POINTER
            a[i] = P + 8
            assert call(*a, r, None) == B.ERR_MISALIGNED
    ok = dict(x=P, residual=P, weight=P, sum=P, y=P, codes=P, scales=P, rstd=P)

    def forward(**change):
        return lib.gaconv_rmsnorm_forward(*dict(ok, **change).values(), r, None)
    for change in (dict(x=None), dict(weight=None), dict(sum=None), dict(codes=None), dict(scales=None), dict(y=None, codes=None, scales=None)):
        assert forward(**change) == B.ERR_NULL_POINTER, change
    for name in ok:
        assert forward(**{name: P + 4}) == B.ERR_MISALIGNED, name
    good = dict(dy=P, dsum=P, sum=P, weight=P, rstd=P, dx=P, dweight=P)

    def backward(ws=P, size=1 << 30, **change):
        return lib.gaconv_rmsnorm_backward(*dict(good, **change).values(), r, ws, size, None)
    for name in ("dy", "sum", "weight", "rstd", "dx"):
        assert backward(**{name: None}) == B.ERR_NULL_POINTER, name
    assert backward(ws=None) == B.ERR_NULL_POINTER
    assert backward(ws=P + 8) == B.ERR_MISALIGNED
    assert backward(size=16) == B.ERR_WORKSPACE_TOO_SMALL
    for name in good:
        assert backward(**{name: P + 8}) == B.ERR_MISALIGNED, name


def test_no_rows_is_no_work():
    """Nothing is read, written or enqueued, whatever the pointers."""
    lib, d = B.load(), B.make_rows_desc(0, 64, torch.float32)
    r, before = ctypes.byref(d), B.gaconv_launch_count()
    assert lib.gaconv_act_pack(None, None, None, r, None) == B.OK
    assert lib.gaconv_act_unpack(None, None, None, r, None) == B.OK
    assert lib.gaconv_rmsnorm_forward(None, None, None, None, None, None, None, None, r, None) == B.OK
    assert lib.gaconv_rmsnorm_backward(None, None, None, None, None, None, None, r, None, 0, None) == B.OK
    assert B.gaconv_launch_count() == before


def test_filter_gradient_refusals():
    lib = B.load()
    layer = ConvLayer("l", 64, 40, 1, 1, 48, 1, 1)
    d = B.make_desc(layer, torch.bfloat16, dy_layout=B.DY_NPQK)
    r, n = ctypes.byref(d), ctypes.c_size_t(0)

    def run(method=B.METHOD_EXACT, codes=P, scales=P, fmt=B.ACT_E4M3, dy=P, dw=P):
        return lib.gaconv_dw_from_packed(method, codes, scales, fmt, dy, dw, r, 0, None)
    assert lib.gaconv_packed_workspace_size(r, B.METHOD_EXACT, None) == B.ERR_NULL_POINTER
    assert lib.gaconv_packed_workspace_size(r, 9, ctypes.byref(n)) == B.ERR_BAD_DESC
    assert lib.gaconv_dw_from_packed(B.METHOD_EXACT, P, P, 0, P, P, None, 0, None) == B.ERR_NULL_POINTER
    assert run() == B.ERR_NULL_POINTER                                   # no workspace
    d.workspace, d.workspace_bytes = P, 64
    assert run() == B.ERR_WORKSPACE_TOO_SMALL
    need = B.gaconv_packed_workspace_size(d, B.METHOD_EXACT)
    d.workspace_bytes = need - 1
    assert run() == B.ERR_WORKSPACE_TOO_SMALL
    d.workspace_bytes = need
    assert run(fmt=2) == B.ERR_BAD_DESC and run(fmt=-1) == B.ERR_BAD_DESC and run(method=7) == B.ERR_BAD_DESC
    for name in ("codes", "scales", "dy", "dw"):
        assert run(**{name: None}) == B.ERR_NULL_POINTER, name
        assert run(**{name: P + 4}) == B.ERR_MISALIGNED, name
    assert run(method=B.METHOD_ZERO, codes=None, scales=None, dy=None, dw=None) == B.ERR_NULL_POINTER
    d.workspace = P + 8
    assert run() == B.ERR_MISALIGNED
    d.x_layout = B.X_NCHW
    assert run() == B.ERR_UNSUPPORTED and lib.gaconv_packed_workspace_size(r, B.METHOD_EXACT, ctypes.byref(n)) == B.ERR_UNSUPPORTED
    d.x_layout, d.k = B.X_NHWC, 0
    assert run() == B.ERR_BAD_DESC


def test_reference_values_of_every_code():
    """The reference's two directions agree on every code, and its E4M3 table is torch's."""
    every = np.arange(256, dtype=np.uint8)[None]
    one = np.full((1, 8), 127, np.uint8)
    theirs = torch.from_numpy(every.copy()).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    mine = R.values(every, one, 256, 0)
    number = ~np.isnan(theirs)
    assert np.array_equal(mine[number], theirs[number]) and number.sum() == 254
    assert np.array_equal(R.e4m3_byte(mine[number]), every[number])
    assert np.array_equal(R.values(every, one, 256, 1)[0], np.r_[0:128, -128:0])


def test_reference_rounding():
    x = np.zeros((1, 32))
    x[0, :8] = [448, 1.0625, 1.1875, -1.0625, 17, 19, 2.0 ** -10, 3 * 2.0 ** -10]       # scale 1: ties go to the even neighbour
    _, s, v = R.pack(x, 0)
    assert s[0, 0] == 127 and list(v[0, :8]) == [448, 1.0, 1.25, -1.0, 16, 20, 0, 2.0 ** -8]
    x[0, 0] = np.nextafter(448, 1000)                                                    # one step beyond: the next scale
    assert R.pack(x, 0)[1][0, 0] == 128
    x[:] = 0
    x[0, :4] = [127, 0.5, 1.5, -2.5]
    _, s, v = R.pack(x, 1)
    assert s[0, 0] == 127 and list(v[0, :4]) == [127, 0, 2, -2]
