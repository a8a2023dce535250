"""64-bit reference of the 8-bit form of activations and of the norm, for tests (numpy, on the CPU; shares no code with the library)."""
from __future__ import annotations

import numpy as np
import torch

GROUP = 32
TOP = {0: 448.0, 1: 127.0}              # binding.ACT_E4M3, ACT_INT8
E_MIN, E_MAX = -117, {0: 119, 1: 121}


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().to(torch.float64).numpy()


def pitch(cols: int) -> int:
    return -(-cols // 16) * 16


def groups(cols: int) -> int:
    return -(-cols // GROUP)


def e4m3_byte(q: np.ndarray) -> np.ndarray:
    """Whole codes of numbers that E4M3 represents."""
    sign = np.signbit(q).astype(np.int64) << 7
    a = np.abs(q)
    m, p = np.frexp(a)                                   # a = m 2^p, m in [0.5, 1)
    normal = a >= 2.0 ** -6
    exp = np.where(normal, p - 1 + 7, 0)
    frac = np.where(normal, (2 * m - 1) * 8, a * 2.0 ** 9)
    assert np.all(frac == np.round(frac)) and np.all(a <= 448)
    return (sign | (exp.astype(np.int64) << 3) | frac.astype(np.int64)).astype(np.uint8)


def pack(x: np.ndarray, fmt: int):
    """x [rows, cols] (float64) -> codes uint8 [rows, pitch], scale bytes uint8 [rows, groups], values float64 [rows, cols]."""
    rows, cols = x.shape
    G, top = groups(cols), TOP[fmt]
    full = np.zeros((rows, G * GROUP))
    full[:, :cols] = x
    g = full.reshape(rows, G, GROUP)
    fine = np.isfinite(g).all(2)
    a = np.where(fine, np.abs(np.where(np.isfinite(g), g, 0)).max(2), 0.0)
    e = np.full(a.shape, E_MIN, dtype=np.int64)
    for k in range(E_MAX[fmt], E_MIN - 1, -1):           # the least exponent that reaches, by trying all
        e = np.where(a <= top * 2.0 ** k, k, e)
    e = np.where(a > top * 2.0 ** E_MAX[fmt], E_MAX[fmt], e)
    q = np.where(fine[..., None], np.where(np.isfinite(g), g, 0) / (2.0 ** e)[..., None], 0.0)
    q = np.clip(q, -top, top)
    if fmt == 0:
        _, p = np.frexp(np.maximum(np.abs(q), 2.0 ** -6))
        step = 2.0 ** (p - 4)
        q = np.rint(q / step) * step                     # (rint: ties to even)
        codes = e4m3_byte(q)
    else:
        q = np.rint(q)
        codes = q.astype(np.int64).astype(np.int8).view(np.uint8)
    value = q * (2.0 ** e)[..., None]
    value = np.where(fine[..., None], value, np.nan).reshape(rows, -1)[:, :cols]
    codes = codes.reshape(rows, -1)
    codes = np.pad(codes, ((0, 0), (0, max(0, pitch(cols) - codes.shape[1]))))[:, :pitch(cols)]
    return codes, np.where(fine, e + 127, 255).astype(np.uint8), value


def values(codes: np.ndarray, scales: np.ndarray, cols: int, fmt: int) -> np.ndarray:
    """What codes and scale bytes stand for."""
    if fmt == 0:
        b = codes.astype(np.int64)
        exp, frac = (b >> 3) & 15, b & 7
        v = np.where(exp == 0, frac * 2.0 ** -9, (8 + frac) * 2.0 ** (exp - 10.0)) * np.where(b >> 7, -1.0, 1.0)
    else:
        v = codes.view(np.int8).astype(np.float64)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v[:, :cols] * np.repeat(s, GROUP, 1)[:, :cols]


def norm(s: np.ndarray, w: np.ndarray, eps: float):
    rstd = 1 / np.sqrt((s * s).mean(1) + eps)
    return s * rstd[:, None] * w, rstd


def norm_grad(dy, ds, s, w, rstd):
    """dx, dweight, and for each the sum of magnitudes that its rounding errors are relative to."""
    h, g = s * rstd[:, None], dy * w
    m = (g * h).mean(1, keepdims=True)
    dx = ds + rstd[:, None] * (g - h * m)
    size = np.abs(ds) + rstd[:, None] * (np.abs(g) + np.abs(h) * np.abs(g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), size, np.abs(dy * h).sum(0)
