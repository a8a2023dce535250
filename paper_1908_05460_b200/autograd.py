"""Training-step integration: a convolution whose filter gradient comes from this library.

Forward and the input gradient stay with the framework (torch / cuDNN); only the filter gradient --
the operation the paper approximates, "roughly a third" of a layer's time (Section 2) -- is computed
by gaconv, exactly or by the method the approximation schedule picks for this layer at this training
step (Sections 2.5 and 3).  Weights and inputs are bf16 or fp32 CUDA tensors; the layer keeps its
activations in channels-last memory (the NHWC layout of the paper's kernel, Section 2.4), so the
library reads torch's buffers in place and writes the gradient straight in torch's [K,C,R,S] layout.

With `checkpoint` a layer keeps its input for the backward pass in 8 bits (packed.py) instead of its own type, and takes the filter
gradient from that.  GALinear is the linear layer among them, and GARMSNorm the norm in front of one, which hands its output over
in both forms.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch
import torch.nn.functional as F
from torch.autograd.function import once_differentiable

from . import binding as B
from .layers import ConvLayer
from .packed import DTYPES, PackedActivation, as_rows, check_devices, check_format, row_stride


def _on_boundary(t, memory_format):
    """t, of that format, where it starts on 16 bytes, or a copy that does."""
    return t if t.data_ptr() % 16 == 0 else t.clone(memory_format=memory_format)


class _Conv2dFilterGrad(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, module):
        ctx.module = module
        ctx.packed, ctx.shape = None, x.shape
        if module.checkpoint is None:
            ctx.save_for_backward(weight, x)
        elif ctx.needs_input_grad[1]:
            kept, ctx.packed = PackedActivation.pack(x.permute(0, 2, 3, 1), module.checkpoint).saved()
            ctx.save_for_backward(weight, *kept)
        else:
            ctx.save_for_backward(weight)
        return F.conv2d(x, weight, None, module.stride, module.padding)

    @staticmethod
    def backward(ctx, dy):
        weight, *kept = ctx.saved_tensors
        m = ctx.module
        x = kept[0] if len(kept) == 1 else None              # (one tensor: the input; two: its codes and scales; none: not needed)
        dx = None
        if ctx.needs_input_grad[0]:
            if x is None:        # (the gradient of the input does not read it; its shape and memory order count)
                x = torch.empty(ctx.shape, dtype=dy.dtype, device=dy.device, memory_format=torch.channels_last)
            # with the layer's own input, which is channels-last: torch.nn.grad.conv2d_input hands the framework a placeholder
            # without a memory format, upon which it turns gradient and result (128->128 on 16x16 maps, N = 128: 57 -> 23 us)
            st, pad = m.stride, m.padding
            dx = torch.ops.aten.convolution_backward(dy, x, weight, None, (st, st) if isinstance(st, int) else st,
                                                     (pad, pad) if isinstance(pad, int) else pad, (1, 1), False, (0, 0), 1,
                                                     (True, False, False))[0]
        dw = None
        if ctx.needs_input_grad[1]:
            dw = m.filter_gradient(x, dy) if ctx.packed is None else m.packed_filter_gradient(PackedActivation.restored(kept, ctx.packed), ctx.shape, dy)
        return dx, dw, None


class GAConv2d(torch.nn.Module):
    """3x3 / 5x5 / ... convolution (no bias, dilation 1, one group) with the library's filter gradient.

    `schedule` (binding.Schedule) and `layer_index` say which method this layer uses at `step`; advance
    `step` once per batch (`module.step += 1`, or share one counter object across layers).  Without a
    schedule the gradient is always exact.

    `checkpoint`: "e4m3" or "int8" to keep the input for the backward pass in 8 bits (a scale for every 32 channels of a pixel); every
    method's gradient is then that of the kept values."""

    def __init__(self, in_channels, out_channels, kernel_size, stride=1, padding=0, schedule=None, layer_index=0,
                 dtype=torch.float32, device="cuda", checkpoint=None):
        super().__init__()
        self.checkpoint = check_format(checkpoint)
        self.stride, self.padding, self.kernel_size = stride, padding, kernel_size
        self.weight = torch.nn.Parameter(torch.empty(out_channels, in_channels, kernel_size, kernel_size, dtype=dtype, device=device))
        torch.nn.init.kaiming_normal_(self.weight)
        self.schedule, self.layer_index, self.step = schedule, layer_index, 0
        self._desc_cache = {}

    def forward(self, x):
        # (inside a Function needs_input_grad is true of a weight with requires_grad, whether or not gradients are recorded)
        if not torch.is_grad_enabled():
            return F.conv2d(x.contiguous(memory_format=torch.channels_last), self.weight, None, self.stride, self.padding)
        return _Conv2dFilterGrad.apply(x.contiguous(memory_format=torch.channels_last), self.weight, self)

    def _desc(self, x, dy_layout=B.DY_NKPQ):
        key = (x.shape, x.dtype, x.device, dy_layout)
        found = self._desc_cache.get(key)
        if found is None:
            n, c, h, w = x.shape
            k = self.weight.shape[0]
            layer = ConvLayer("gaconv2d", n, c, h, w, k, self.kernel_size, self.kernel_size, self.stride, self.padding)
            d = B.make_desc(layer, x.dtype, x_layout=B.X_NHWC, dw_layout=B.DW_KCRS, alpha=1.0, dy_layout=dy_layout)
            with torch.cuda.device(x.device):
                found = self._desc_cache[key] = (d, B.attach_workspace(d, methods=(B.METHOD_EXACT, B.METHOD_TOP1), device=x.device))
        return found[0]

    @staticmethod
    def _dy_in_place(dy):
        """dy as the library takes it, and its layout: the gradient of a channels-last forward arrives channels-last and is taken as it is ([N,P,Q,K] memory).
        A part of a larger gradient (torch.cat's, of a batch) may start anywhere, and is copied unless that is a 16-byte boundary."""
        if dy.dim() == 4 and dy.shape[1] > 1 and not dy.is_contiguous() and dy.is_contiguous(memory_format=torch.channels_last):
            return _on_boundary(dy, torch.channels_last), B.DY_NPQK
        return _on_boundary(dy.contiguous(), torch.contiguous_format), B.DY_NKPQ                           # [N,K,P,Q]

    def packed_filter_gradient(self, packed, shape, dy):
        """filter_gradient for activations of `shape` that were kept in 8 bits."""
        n, c, h, w = shape
        dy, dy_layout = self._dy_in_place(dy if dy.dtype == packed.dtype else dy.to(packed.dtype))
        layer = ConvLayer("gaconv2d", n, c, h, w, self.weight.shape[0], self.kernel_size, self.kernel_size, self.stride, self.padding)
        d = B.make_desc(layer, packed.dtype, x_layout=B.X_NHWC, dw_layout=B.DW_KCRS, dy_layout=dy_layout)
        dw = torch.empty(self.weight.shape, dtype=torch.float32, device=dy.device)
        method = B.METHOD_EXACT if self.schedule is None else self.schedule.method(self.layer_index, self.step)
        if method in (B.METHOD_ZERO, B.METHOD_RANDOM):              # (the schedule seeds the random method)
            with torch.cuda.device(dy.device):
                self.schedule.run_layer(self.layer_index, self.step, None, None, dw, d)
        else:
            packed.filter_gradient(dy, dw, d, method)
        return dw.to(self.weight.dtype)

    def filter_gradient(self, x, dy):
        """dW [K,C,R,S] (the weight's dtype) of this layer for activations x and output gradient dy."""
        B.load()
        check_devices(activations=x, gradient=dy, weight=self.weight)
        k, c, r, _ = self.weight.shape
        out = [(size + 2 * self.padding - r) // self.stride + 1 for size in x.shape[2:]]
        if x.dim() != 4 or x.shape[1] != c or dy.shape != (x.shape[0], k, *out):          # (the kernels go by x's shape alone)
            raise ValueError("activations %s and a gradient %s of a layer of %s" % (tuple(x.shape), tuple(dy.shape), tuple(self.weight.shape)))
        x = _on_boundary(x.contiguous(memory_format=torch.channels_last), torch.channels_last)        # NHWC memory under an NCHW-shaped tensor
        if dy.dtype != x.dtype:
            dy = dy.to(x.dtype)
        dy, dy_layout = self._dy_in_place(dy)
        dw = torch.empty(self.weight.shape, dtype=torch.float32, device=x.device)
        d = self._desc(x, dy_layout)
        with torch.cuda.device(x.device):
            if self.schedule is None:
                B.gaconv_dw_exact(x, dy, dw, d)
            else:
                self.schedule.run_layer(self.layer_index, self.step, x, dy, dw, d)
        return dw.to(self.weight.dtype)


class _LinearFilterGrad(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, packed, fmt):
        kept, ctx.packed = (), None
        if ctx.needs_input_grad[1] and x.numel() > 0 and weight.numel() > 0:
            kept, ctx.packed = (PackedActivation.pack(x, fmt) if packed is None else packed).saved()
        ctx.save_for_backward(weight, *kept)
        return F.linear(x, weight, bias)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        weight, *kept = ctx.saved_tensors
        dx = dw = db = None
        if ctx.needs_input_grad[0]:
            dx = dy.matmul(weight)
        if ctx.needs_input_grad[2]:
            db = dy.flatten(0, -2).sum(0) if dy.dim() > 1 else dy.clone()
        if ctx.needs_input_grad[1]:
            dw = torch.zeros_like(weight) if ctx.packed is None else linear_filter_gradient(PackedActivation.restored(kept, ctx.packed), dy).to(weight.dtype)
        return dx, dw, db, None, None


def linear_filter_gradient(packed: PackedActivation, dy: torch.Tensor) -> torch.Tensor:
    """Filter gradient [out, in] (fp32) of a linear layer whose input was kept in 8 bits, for the output gradient dy [..., out]."""
    rows = as_rows(dy if dy.dtype == packed.dtype else dy.to(packed.dtype)).contiguous()
    layer = ConvLayer("linear", packed.rows, packed.cols, 1, 1, rows.shape[1], 1, 1)
    dw = torch.empty(rows.shape[1], packed.cols, dtype=torch.float32, device=dy.device)
    packed.filter_gradient(rows, dw, B.make_desc(layer, packed.dtype, dy_layout=B.DY_NPQK))
    return dw


class GALinear(torch.nn.Module):
    """Linear layer that keeps its input for the backward pass in 8 bits ("e4m3" or "int8") and takes its filter gradient, a 1x1 convolution's on rows of
    tokens, from that.  Forward and the input gradient stay with the framework, as in GAConv2d.  `packed`: the input as it was already kept (GARMSNorm, or a
    second layer on the same input); otherwise the layer packs it."""

    def __init__(self, in_features, out_features, bias=True, checkpoint="e4m3", dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        if check_format(checkpoint) is None or dtype not in DTYPES:
            raise ValueError("GALinear keeps bf16 or fp32 inputs in 8 bits (checkpoint: e4m3 or int8)")
        self.checkpoint = checkpoint
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, dtype=dtype, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(out_features, dtype=dtype, device=device)) if bias else None
        torch.nn.init.kaiming_normal_(self.weight)

    def forward(self, x, packed: Optional[PackedActivation] = None):
        if x.dtype != self.weight.dtype or x.shape[-1] != self.weight.shape[1]:
            raise ValueError("input %s %s for a layer of %s %s" % (tuple(x.shape), x.dtype, tuple(self.weight.shape), self.weight.dtype))
        check_devices(input=x, weight=self.weight, kept=None if packed is None else packed.codes)
        if packed is not None and (packed.rows * packed.cols != x.numel() or packed.cols != x.shape[-1] or packed.dtype != x.dtype):
            raise ValueError("the kept input has %d x %d values of %s, the input %s" % (packed.rows, packed.cols, packed.dtype, tuple(x.shape)))
        if not torch.is_grad_enabled():          # (as in GAConv2d)
            return F.linear(x, self.weight, self.bias)
        return _LinearFilterGrad.apply(x, self.weight, self.bias, packed, self.checkpoint)


def check_async_status(*modules: torch.nn.Module):
    """Raises GaconvError if a kernel of a filter gradient gave up on a bounded wait since the last look, so that the gradient is not to be used.

    Waits for the current stream of each device, so it belongs where a program reads its loss.  Looked at are the gradients from inputs that were kept in 8 bits, of
    whatever layer, on the devices that `modules` have parameters on (none given: the current one), and those of the GAConv2d layers in `modules`."""
    failed = []
    devices = {p.device for module in modules for p in module.parameters() if p.is_cuda}
    for device in sorted(devices, key=str) if modules else [None]:
        with torch.cuda.device(device):
            failed.append(B.gaconv_poll_collected_status())
    for layer in (m for module in modules for m in module.modules() if isinstance(m, GAConv2d)):
        for desc, workspace in layer._desc_cache.values():
            with torch.cuda.device(workspace.device):
                failed.append(B.gaconv_poll_async_status(desc))
    for status in failed:          # (every word has been looked at and cleared)
        B._check(status, "check_async_status")


class NormOutput(NamedTuple):
    y: torch.Tensor
    sum: Optional[torch.Tensor]                 # x + residual, the next residual; None without one
    packed: Optional[PackedActivation]          # y in 8 bits; None without `checkpoint` or `keep`


class _RMSNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps, packed):
        rows = as_rows(x)
        res = None if residual is None else as_rows(residual)
        n, cols = rows.shape
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        s = None if res is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        rstd = torch.empty(n, dtype=torch.float32, device=x.device)
        w = weight if weight.is_contiguous() and weight.data_ptr() % 16 == 0 else weight.clone(memory_format=torch.contiguous_format)
        with torch.cuda.device(x.device):
            d = B.make_rows_desc(n, cols, x.dtype, fmt=packed.format if packed else B.ACT_E4M3, eps=eps, x_stride=row_stride(rows),
                                 r_stride=0 if res is None else row_stride(res))
            B.gaconv_rmsnorm_forward(rows, res, w, s, y, packed.codes if packed else None, packed.scales if packed else None, rstd, d)
        ctx.save_for_backward(rows if s is None else s, w, rstd)
        ctx.set_materialize_grads(False)
        return y if s is None else (y, s)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, ds=None):
        s, w, rstd = ctx.saved_tensors
        if dy is None:          # only the sum was used
            return ds, ds if ctx.needs_input_grad[1] else None, None, None, None
        cols = w.shape[0]
        grad = as_rows(dy.to(s.dtype))
        rows = s.reshape(-1, cols) if s.dim() != 2 else s
        dsum = None if ds is None else as_rows(ds.to(s.dtype))
        s_stride = row_stride(rows)
        if dsum is not None and row_stride(dsum) != s_stride:          # (the sum's gradient lies as the sum does, which is dense where there is one)
            dsum = dsum.contiguous()
        dx = torch.empty(dy.shape, dtype=s.dtype, device=dy.device)
        dw = torch.empty(cols, dtype=torch.float32, device=dy.device) if ctx.needs_input_grad[2] else None
        with torch.cuda.device(dy.device):
            d = B.make_rows_desc(grad.shape[0], cols, s.dtype, s_stride=s_stride, y_stride=row_stride(grad))
            B.gaconv_rmsnorm_backward(grad, dsum, rows, w, rstd, dx, dw, d, None if dw is None else B.rmsnorm_workspace(d, dy.device))
        return dx, dx if ctx.needs_input_grad[1] else None, None if dw is None else dw.to(w.dtype), None, None


class GARMSNorm(torch.nn.Module):
    """Root-mean-square norm of the last dimension, of x + residual where one is given; with `checkpoint` its output comes in 8 bits as well, for the linear layers
    behind it.  Returns NormOutput(y, sum, packed).  `keep=False` in a call: without the 8-bit form, for evaluation, where no layer reads it."""

    def __init__(self, features, eps=1e-6, checkpoint=None, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        if dtype not in DTYPES:
            raise ValueError("GARMSNorm is for bf16 and fp32")
        self.eps, self.checkpoint = eps, check_format(checkpoint)
        self.weight = torch.nn.Parameter(torch.ones(features, dtype=dtype, device=device))

    def forward(self, x, residual=None, keep=True) -> NormOutput:
        if x.dtype != self.weight.dtype or x.shape[-1] != self.weight.shape[0] or (residual is not None and (residual.shape != x.shape or residual.dtype != x.dtype)):
            raise ValueError("input %s %s for a norm of %s %s, and a residual alike" % (tuple(x.shape), x.dtype, tuple(self.weight.shape), self.weight.dtype))
        check_devices(input=x, residual=residual, weight=self.weight)
        packed = None
        if self.checkpoint is not None and keep:
            packed = PackedActivation(x.numel() // x.shape[-1], x.shape[-1], x.dtype, self.checkpoint, x.device)
        out = _RMSNorm.apply(x, residual, self.weight, self.eps, packed)
        return NormOutput(out, None, packed) if residual is None else NormOutput(out[0], out[1], packed)
