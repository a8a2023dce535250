"""Activations kept in 8 bits between the forward and the backward pass: owner of the codes and scales that the library's calls write.

Rows are tokens, or the pixels of a channels-last activation; the memory comes from torch's allocator on the current stream, as every
workspace here does, so that calls on several streams and captured graphs keep apart."""
from __future__ import annotations

import torch

from . import binding as B

FORMATS = {"e4m3": B.ACT_E4M3, "int8": B.ACT_INT8}
DTYPES = (torch.bfloat16, torch.float32)


def check_format(name):
    if name is not None and name not in FORMATS:
        raise ValueError("checkpoint: %r is none of %s" % (name, ", ".join(sorted(FORMATS))))
    return name


def check_devices(**tensors):
    """A kernel is given addresses alone, and one of another device's memory, or the host's, faults there."""
    at = {name: t.device for name, t in tensors.items() if t is not None}
    if len(set(at.values())) > 1:
        raise ValueError("tensors on several devices: " + ", ".join("%s on %s" % i for i in at.items()))


def is_dense(t: torch.Tensor) -> bool:
    """Whether t's elements fill the memory from its first to its last one, each once, in whatever order."""
    step = 1
    for stride, size in sorted((stride, size) for size, stride in zip(t.shape, t.stride()) if size != 1):
        if stride != step:
            return t.numel() == 0
        step *= size
    return True


def as_rows(x: torch.Tensor) -> torch.Tensor:
    """x [..., cols] as rows that the library can read: neighbouring channels, on a 16-byte boundary."""
    if x.dtype not in DTYPES:
        raise TypeError("activations are bf16 or fp32, not %s" % x.dtype)
    rows = x.reshape(-1, x.shape[-1])
    if rows.shape[1] > 1 and rows.stride(1) != 1 or rows.shape[0] > 1 and rows.stride(0) < rows.shape[1]:
        rows = rows.contiguous()
    return rows if rows.data_ptr() % 16 == 0 else rows.clone(memory_format=torch.contiguous_format)


def row_stride(rows: torch.Tensor) -> int:
    return rows.stride(0) if rows.shape[0] > 1 else 0


class PackedActivation:
    """`rows` x `cols` values of `dtype` in 8 bits: codes and scales as gaconv_act_pack writes them."""

    def __init__(self, rows: int, cols: int, dtype: torch.dtype, fmt: str, device):
        self.rows, self.cols, self.dtype, self.fmt = rows, cols, dtype, check_format(fmt)
        codes, scales = B.gaconv_act_sizes(self.desc())
        self.codes = torch.empty(codes, dtype=torch.uint8, device=device)
        self.scales = torch.empty(scales, dtype=torch.uint8, device=device)

    @property
    def format(self) -> int:
        return FORMATS[self.fmt]

    def desc(self, x_stride: int = 0) -> B.RowsDesc:
        return B.make_rows_desc(self.rows, self.cols, self.dtype, fmt=FORMATS[self.fmt], x_stride=x_stride)

    def saved(self):
        """What autograd keeps of it, and what is needed to put it together again."""
        return (self.codes, self.scales), (self.rows, self.cols, self.dtype, self.fmt)

    @classmethod
    def restored(cls, tensors, what) -> "PackedActivation":
        p = cls.__new__(cls)
        (p.codes, p.scales), (p.rows, p.cols, p.dtype, p.fmt) = tensors, what
        return p

    @classmethod
    def pack(cls, x: torch.Tensor, fmt: str = "e4m3") -> "PackedActivation":
        """x [..., cols], bf16 or fp32."""
        rows = as_rows(x)
        with torch.cuda.device(x.device):
            p = cls(rows.shape[0], rows.shape[1], x.dtype, fmt, x.device)
            B.gaconv_act_pack(rows, p.codes, p.scales, p.desc(row_stride(rows)))
        return p

    def unpack(self) -> torch.Tensor:
        """The values that are kept, [rows, cols]."""
        x = torch.empty(self.rows, self.cols, dtype=self.dtype, device=self.codes.device)
        with torch.cuda.device(x.device):
            B.gaconv_act_unpack(self.codes, self.scales, x, self.desc())
        return x

    def filter_gradient(self, dy, dw, desc: B.ConvDesc, method: int = B.METHOD_EXACT, seed: int = 0):
        """gaconv_dw_from_packed in a workspace of this call's own; desc says what layer the rows belong to."""
        check_devices(kept=self.codes, dy=dy, dw=dw)
        if desc.in_dtype != B.make_rows_desc(0, 1, self.dtype).dtype:
            raise ValueError("the descriptor's gradients are not of %s, as the kept values are" % self.dtype)
        if desc.n * desc.h * desc.w != self.rows or desc.c != self.cols:
            raise ValueError("%d x %d values are kept, the layer has %d x %d" % (self.rows, self.cols, desc.n * desc.h * desc.w, desc.c))
        p = (desc.h + 2 * desc.pad_h - desc.r) // desc.stride_h + 1
        q = (desc.w + 2 * desc.pad_w - desc.s) // desc.stride_w + 1
        if dy.numel() != desc.n * desc.k * p * q or dw.numel() != desc.k * desc.c * desc.r * desc.s or dy.dtype != self.dtype or dw.dtype != torch.float32:
            raise ValueError("dy %s %s or dw %s %s is not the layer's" % (tuple(dy.shape), dy.dtype, tuple(dw.shape), dw.dtype))
        if not is_dense(dy) or not is_dense(dw):          # (the kernels go by desc's layouts alone: past the end of an expanded tensor, over what lies between the rows of a view)
            raise ValueError("dy %s with strides %s or dw %s with strides %s has gaps or repeated elements" % (tuple(dy.shape), dy.stride(), tuple(dw.shape), dw.stride()))
        own = desc.workspace, desc.workspace_bytes
        with torch.cuda.device(self.codes.device):
            try:
                workspace = B.attach_packed_workspace(desc, methods=(method,), device=self.codes.device)
                B.gaconv_dw_from_packed(method, self.codes, self.scales, self.format, dy, dw, desc, seed)
                B.gaconv_collect_async_status(desc)          # (whether a kernel gave up is asked when the workspace is gone: autograd.check_async_status)
            finally:          # (a descriptor that went on pointing at this call's workspace would have later calls write to memory that is others' by then)
                desc.workspace, desc.workspace_bytes = own
        del workspace          # (back to the allocator, which hands it out again in the order of this stream)
