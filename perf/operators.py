"""Activations kept in 8 bits for the backward pass: what is measured of the operators that make, restore and use them.

  pack     gaconv_act_pack            a layer's input X -> one byte an element and a power-of-two scale for every 32 neighbouring channels
  unpack   gaconv_act_unpack          and back
  dw       gaconv_dw_from_packed      filter gradient of a layer whose X was kept in that form; a linear layer is a 1x1 filter on rows of tokens
  fwd      gaconv_rmsnorm_forward     root-mean-square norm behind the addition of the residual, with its output also in 8 bits
  bwd      gaconv_rmsnorm_backward    its backward pass

A case names the operator (`op`), the type of the tensors (`dtype`), the 8-bit format (`fmt`) and the sizes.  Rows are tokens, or pixels of
channels-last feature maps.  Activations are normal values whose channels differ in size, a few by much, as inputs of linear layers do, or ReLU
outputs (convolutions); gradients are small normal values.  Where `own` is false the operators are computed in plain torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32                                             # neighbouring channels that share a scale
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
TOP = {"e4m3": 448.0, "int8": 127.0}                   # largest code
E_MIN, E_MAX = -117, {"e4m3": 119, "int8": 121}        # exponents of the scales: codes times scales are finite, normal bf16 numbers
EPS = 1e-6


# ---------------------------------------------------------------- cases
def listed():
    return [
        # the input of one of ResNet-20's last layers at batch 128, kept when its forward pass has run: launch latency counts
        dict(name="pack_8192x64", op="pack", dtype="bf16", fmt="e4m3", rows=8192, cols=64),
        # the input of a wide linear layer, a long batch of tokens
        dict(name="pack_16384x4096", op="pack", dtype="bf16", fmt="e4m3", rows=16384, cols=4096),
        # an activation restored for code that wants it whole, ragged in both directions
        dict(name="unpack_5003x1000_f32", op="unpack", dtype="f32", fmt="int8", rows=5003, cols=1000),
        # a linear layer on a short batch of tokens: latency
        dict(name="dw_512_512_512", op="dw", dtype="bf16", fmt="e4m3", n=512, hw=1, c=512, k=512, r=1, stride=1),
        # a projection of a large model on a long batch of tokens: the tensor cores' rate
        dict(name="dw_16384_4096_4096", op="dw", dtype="bf16", fmt="e4m3", n=16384, hw=1, c=4096, k=4096, r=1, stride=1),
        # tokens, inputs and outputs (a vocabulary's remainder) that no tile divides
        dict(name="dw_4099_1000_1333", op="dw", dtype="bf16", fmt="int8", n=4099, hw=1, c=1000, k=1333, r=1, stride=1),
        # the same for fp32 training
        dict(name="dw_4096_512_512_f32", op="dw", dtype="f32", fmt="e4m3", n=4096, hw=1, c=512, k=512, r=1, stride=1),
        # VGG-19's 256->256 layers at batch 128, from a checkpoint of their ReLU inputs
        dict(name="dw_conv_256_8x8", op="dw", dtype="bf16", fmt="int8", n=128, hw=8, c=256, k=256, r=3, stride=1),
        # the norm in front of a wide linear layer on a long batch of tokens, forward and backward: memory bandwidth
        dict(name="fwd_16384x4096", op="fwd", dtype="bf16", fmt="e4m3", rows=16384, cols=4096),
        dict(name="bwd_16384x4096", op="bwd", dtype="bf16", fmt="e4m3", rows=16384, cols=4096),
        # a few tokens: launch latency
        dict(name="fwd_64x1024", op="fwd", dtype="bf16", fmt="e4m3", rows=64, cols=1024),
        # fp32, ragged in both directions
        dict(name="bwd_5003x1000_f32", op="bwd", dtype="f32", fmt="e4m3", rows=5003, cols=1000),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("pack", "unpack", "dw", "dw", "dw", "fwd", "bwd"))
    c = dict(op=op, dtype=rng.choice(("bf16", "bf16", "f32")), fmt="e4m3" if op in ("fwd", "bwd") else rng.choice(("e4m3", "int8")))
    if op != "dw":
        c.update(rows=_log(rng, 1, 16384), cols=_log(rng, 8, 4096))
    elif rng.random() < 0.7:        # tokens
        c.update(n=_log(rng, 1, 16384), hw=1, c=_log(rng, 8, 4096), k=_log(rng, 8, 4096), r=1, stride=1)
    else:                           # feature maps, sizes around those of the networks of layers.py
        hw, r = rng.randint(4, 32), rng.choice((1, 3, 3, 5))
        most = max(1, min(128, 131072 // (hw * hw)))
        c.update(n=_log(rng, 1, most), hw=hw, c=_log(rng, 8, 256), k=_log(rng, 8, 256), r=r, stride=rng.choice((1, 1, 2)))
    return c


def _out(case):
    """Side of the layer's output map ("same" padding)."""
    pad = case["r"] // 2
    return (case["hw"] + 2 * pad - case["r"]) // case["stride"] + 1


def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "dw":
        px, out = case["n"] * case["hw"] ** 2, case["n"] * _out(case) ** 2
        taps = case["k"] * case["c"] * case["r"] ** 2
        return {"bytes": px * (case["c"] + -(-case["c"] // GROUP)) + out * case["k"] * b + 4 * taps, "flops": 2 * out * taps}
    n, rows, cols = case["rows"] * case["cols"], case["rows"], case["cols"]
    kept = n + rows * -(-cols // GROUP)
    if case["op"] in ("pack", "unpack"):
        return {"bytes": n * b + kept, "flops": n}
    if case["op"] == "fwd":         # x, residual -> their sum, the output, and the output in 8 bits
        return {"bytes": 4 * n * b + kept + 4 * rows + cols * b, "flops": 6 * n}
    return {"bytes": 4 * n * b + 4 * rows + cols * (b + 4), "flops": 12 * n}       # dy, the sum and its gradient -> dx


# ---------------------------------------------------------------- plain forms
def _pow2(e):
    """2^e in fp32, exactly, for whole e in [-126, 127] (a power function may be an ulp off)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x, fmt):
    """x [rows, cols] -> codes as values (e4m3: float8, int8: int8) [rows, pitch], scales (float8 powers of two) [rows, groups]."""
    rows, cols = x.shape
    groups, pitch = -(-cols // GROUP), -(-cols // 16) * 16
    v = torch.nn.functional.pad(x.float(), (0, groups * GROUP - cols)).view(rows, groups, GROUP)
    a = v.abs().amax(2)
    m, p = torch.frexp(a)
    top, bits = (0.875, 9) if fmt == "e4m3" else (127 / 128, 7)        # the largest code is top * 2^bits
    e = torch.where(m <= top, p - bits, p - bits + 1)
    e = torch.where(a == 0, E_MIN, e).clamp(E_MIN, E_MAX[fmt])
    fine = torch.isfinite(a)
    half = (-e).div(2, rounding_mode="floor")                          # 2^-e in two factors: each is a normal number
    q = v * _pow2(half)[..., None] * _pow2(-e - half)[..., None]
    q = torch.where(fine[..., None], q, 0.0).clamp(-TOP[fmt], TOP[fmt]).view(rows, -1)
    q = torch.nn.functional.pad(q, (0, max(0, pitch - q.shape[1])))[:, :pitch]
    q = q.to(torch.float8_e4m3fn) if fmt == "e4m3" else q.round().to(torch.int8)
    s = torch.where(fine, e + 127, 255).to(torch.uint8).view(torch.float8_e8m0fnu)
    return q.contiguous(), s.contiguous()


def _restore(codes, scales, cols):
    """The values that codes and scales stand for, fp32 [rows, cols]."""
    s = scales.float().repeat_interleave(GROUP, 1)[:, :cols]
    return codes[:, :cols].float() * s


def _windows(x, case):
    """x [n, hw, hw, c] -> [n*out*out, c*r*r], the window under each output pixel."""
    pad, st, r = case["r"] // 2, case["stride"], case["r"]
    if r == 1 and st == 1:
        return x.reshape(-1, case["c"])
    x = torch.nn.functional.pad(x, (0, 0, pad, pad, pad, pad))
    return x.unfold(1, r, st).unfold(2, r, st).reshape(-1, case["c"] * r * r)


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _tokens(rows, cols, g):
    """Rows of activations: channels of different sizes, about one in a hundred large."""
    size = torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda"))
    size = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 16 * size, size)
    return torch.randn(rows, cols, generator=g, device="cuda") * size


def prepare(case, seed):
    g, dt, op, fmt = _gen(seed), DTYPES[case["dtype"]], case["op"], case["fmt"]
    state = {"case": case}
    if op == "dw":
        n, hw, c, k = case["n"], case["hw"], case["c"], case["k"]
        x = _tokens(n, c, g) if hw == 1 else torch.randn(n * hw * hw, c, generator=g, device="cuda").relu_()
        q, s = _quantise(x.to(dt), fmt)
        state["codes"], state["scales"] = q, s
        state["dy"] = (0.01 * torch.randn(n * _out(case) ** 2, k, generator=g, device="cuda")).to(dt)
        state["dw"] = torch.zeros(k, c, case["r"], case["r"], device="cuda")          # the weight's gradient buffer
        return state
    rows, cols = case["rows"], case["cols"]
    x = _tokens(rows, cols, g).to(dt)
    groups, pitch = -(-cols // GROUP), -(-cols // 16) * 16
    if op == "unpack":
        state["codes"], state["scales"] = _quantise(x, fmt)
        state["x"] = torch.zeros_like(x)
        return state
    if op in ("pack", "fwd"):
        state["codes"] = torch.zeros(rows, pitch, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn if fmt == "e4m3" else torch.int8)
        state["scales"] = torch.zeros(rows, groups, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    state["x"] = x
    if op == "pack":
        return state
    state["w"] = (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(dt)
    other = torch.randn(rows, cols, generator=g, device="cuda")
    if op == "fwd":
        state["res"] = (2 * other).to(dt)
        state["sum"], state["y"] = torch.zeros_like(x), torch.zeros_like(x)
        state["rstd"] = torch.zeros(rows, device="cuda")
    else:       # x is the sum that the forward pass has kept
        state["rstd"] = torch.rsqrt(x.float().square().mean(1) + EPS)
        state["dy"] = (0.01 * other).to(dt)
        state["dsum"] = (0.01 * torch.randn(rows, cols, generator=g, device="cuda")).to(dt)
        state["dx"], state["dweight"] = torch.zeros_like(x), torch.zeros(cols, device="cuda")
    return state


# ---------------------------------------------------------------- the framework's operators
_plans = {}        # descriptors and workspaces by the sizes of a layer, as a training program holds them


def _plan(case):
    key = tuple(sorted((k, v) for k, v in case.items() if k != "name"))
    if key not in _plans:
        from paper_1908_05460_b200 import binding as B
        from paper_1908_05460_b200.layers import ConvLayer
        dt, fmt = DTYPES[case["dtype"]], B.ACT_E4M3 if case["fmt"] == "e4m3" else B.ACT_INT8
        if case["op"] == "dw":
            layer = ConvLayer("layer", case["n"], case["c"], case["hw"], case["hw"], case["k"], case["r"], case["r"], case["stride"], case["r"] // 2)
            d = B.make_desc(layer, dt, x_layout=B.X_NHWC, dw_layout=B.DW_KCRS, dy_layout=B.DY_NPQK)
            ws = B.attach_packed_workspace(d, methods=(B.METHOD_EXACT,))
        else:
            d = B.make_rows_desc(case["rows"], case["cols"], dt, fmt=fmt, eps=EPS)
            ws = B.rmsnorm_workspace(d) if case["op"] == "bwd" else None
        while len(_plans) > 40:
            _plans.pop(next(iter(_plans)))
        _plans[key] = (B, d, fmt, ws)
    return _plans[key]


def _run_own(state):
    B, d, fmt, ws = _plan(state["case"])
    op = state["case"]["op"]
    if op == "pack":
        B.gaconv_act_pack(state["x"], state["codes"], state["scales"], d)
        return state["codes"], state["scales"]
    if op == "unpack":
        B.gaconv_act_unpack(state["codes"], state["scales"], state["x"], d)
        return state["x"]
    if op == "dw":
        B.gaconv_dw_from_packed(B.METHOD_EXACT, state["codes"], state["scales"], fmt, state["dy"], state["dw"], d)
        return state["dw"]
    if op == "fwd":
        B.gaconv_rmsnorm_forward(state["x"], state["res"], state["w"], state["sum"], state["y"], state["codes"], state["scales"], state["rstd"], d)
        return state["sum"], state["y"], state["codes"], state["scales"], state["rstd"]
    B.gaconv_rmsnorm_backward(state["dy"], state["dsum"], state["x"], state["w"], state["rstd"], state["dx"], state["dweight"], d, ws)
    return state["dx"], state["dweight"]


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    op, dt, fmt = case["op"], DTYPES[case["dtype"]], case["fmt"]
    if op == "pack":
        return _quantise(state["x"], fmt)
    if op == "unpack":
        return _restore(state["codes"], state["scales"], case["cols"]).to(dt)
    if op == "dw":
        x = _restore(state["codes"], state["scales"], case["c"]).view(case["n"], case["hw"], case["hw"], case["c"])
        dw = state["dy"].float().t() @ _windows(x, case)
        return dw.view(case["k"], case["c"], case["r"], case["r"])
    if op == "fwd":
        s = (state["x"].float() + state["res"].float()).to(dt)
        v = s.float()
        rstd = torch.rsqrt(v.square().mean(1) + EPS)
        y = (v * rstd[:, None] * state["w"].float()).to(dt)
        return (s, y) + _quantise(y, fmt) + (rstd,)
    dy, v, rstd = state["dy"].float(), state["x"].float(), state["rstd"][:, None]
    xh, gr = v * rstd, dy * state["w"].float()
    dx = state["dsum"].float() + rstd * (gr - xh * (gr * xh).mean(1, keepdim=True))
    return dx.to(dt), (dy * xh).sum(0)


# ---------------------------------------------------------------- the same from the definitions, in 64 bits
def _two64(e):
    """2^e in fp64, exactly, for whole e."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _decode64(codes, scales, fmt, cols):
    """Values of codes and scales, taken apart bit by bit."""
    b = codes.view(torch.uint8)[:, :cols].to(torch.int32)
    if fmt == "int8":
        v = (b - 256 * (b > 127)).double()
    else:
        ex, man = (b >> 3) & 15, (b & 7).double()
        v = torch.where(ex == 0, man * 2.0 ** -9, _two64(ex - 7) * (1 + man / 8)) * (1 - 2 * (b >> 7)).double()
    at = torch.arange(cols, device=codes.device) // GROUP
    return v * _two64(scales.view(torch.uint8).to(torch.int32) - 127)[:, at]


def _codes64(x, fmt):
    """Codes and scales, as values, of x [rows, cols]."""
    x = x.double()
    rows, cols = x.shape
    groups, pitch = -(-cols // GROUP), -(-cols // 16) * 16
    a = torch.zeros(rows, groups * GROUP, dtype=torch.float64, device=x.device)
    a[:, :cols] = x.abs()
    a = a.view(rows, groups, GROUP).amax(2)
    e = torch.full_like(a, float(E_MIN))
    # the least exponent whose largest code reaches the group's largest value: a guess by the logarithm, put right by comparison
    guess = torch.floor(torch.log2(torch.clamp(a, min=1e-300) / TOP[fmt]))
    for up in (2.0, 1.0, 0.0, -1.0):
        e = torch.where(TOP[fmt] * _two64(guess + up) >= a, guess + up, e)
    e = e.clamp(E_MIN, E_MAX[fmt])
    q = (x / _two64(e)[:, torch.arange(cols, device=x.device) // GROUP]).clamp(-TOP[fmt], TOP[fmt])
    if fmt == "e4m3":
        step = _two64(torch.frexp(q.abs().clamp(min=2.0 ** -6))[1] - 4)
        q = torch.round(q / step) * step
    else:
        q = torch.round(q)
    full = torch.zeros(rows, pitch, dtype=torch.float64, device=x.device)
    full[:, :cols] = q
    return full, _two64(e)


def exact(case, seed):
    state = prepare(case, seed)
    op, fmt, dt = case["op"], case["fmt"], DTYPES[case["dtype"]]
    if op == "pack":
        return _codes64(state["x"], fmt)
    if op == "unpack":
        return _decode64(state["codes"], state["scales"], fmt, case["cols"])
    if op == "dw":
        n, hw, c, k, r, st = (case[i] for i in ("n", "hw", "c", "k", "r", "stride"))
        pad, out = r // 2, _out(case)
        x = torch.zeros(n, hw + 2 * pad, hw + 2 * pad, c, dtype=torch.float64, device="cuda")
        x[:, pad:pad + hw, pad:pad + hw] = _decode64(state["codes"], state["scales"], fmt, c).view(n, hw, hw, c)
        dy = state["dy"].double()
        dw = torch.empty(k, c, r, r, dtype=torch.float64, device="cuda")
        for i in range(r):
            for j in range(r):
                at = x[:, i:i + (out - 1) * st + 1:st, j:j + (out - 1) * st + 1:st].reshape(-1, c)
                dw[:, :, i, j] = torch.einsum("mk,mc->kc", dy, at)
        return dw
    w = state["w"].double()
    if op == "fwd":
        s = (state["x"].double() + state["res"].double()).to(dt).double()
        rstd = 1 / torch.sqrt((s * s).sum(1) / case["cols"] + EPS)
        y = s * rstd[:, None] * w
        return (s, y) + _codes64(y.to(dt), fmt) + (rstd,)
    dy, s, rstd = state["dy"].double(), state["x"].double(), state["rstd"].double()[:, None]
    # from the quotient rule: d(s_i rstd)/ds_j = rstd (delta_ij - s_i s_j rstd^2 / cols)
    g = dy * w
    along = torch.einsum("rc,rc->r", g, s)[:, None]
    return state["dsum"].double() + rstd * g - rstd ** 3 * s * along / case["cols"], torch.einsum("rc,rc->c", dy, s * rstd)
