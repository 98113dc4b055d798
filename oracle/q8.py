"""Training in 8 bits, restated in plain NumPy: the q8 format, the RMS norm with an 8-bit output, the product of 8-bit
matrices, and their gradients.  64-bit arithmetic; what an operator rounds by definition is rounded where it says so."""
from __future__ import annotations

import math

import numpy as np

MIN_EXP, MAX_EXP = -126, 121


def round_bf16(x) -> np.ndarray:
    """float64 / float32 -> nearest bfloat16 (half to even), as float64.  Finite values and NaN."""
    x = np.asarray(x, dtype=np.float64)
    out = np.array(x, copy=True)
    fine = np.isfinite(x) & (x != 0.0)
    _, e = np.frexp(x[fine])
    unit = np.ldexp(1.0, np.maximum(e, -125) - 8)  # eight significant bits; below 2^-126 the spacing stays
    out[fine] = np.rint(x[fine] / unit) * unit
    out[np.abs(out) >= 2.0 ** 128] *= math.inf
    return out


def scale_of(amax: float) -> float:
    """The smallest power of two, between 2^-126 and 2^121, whose 127 steps reach amax; 0 for 0, NaN if not finite."""
    if amax == 0.0:
        return 0.0
    if not math.isfinite(amax):
        return math.nan
    e = MIN_EXP
    while e < MAX_EXP and 127.0 * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


def pack(x):
    """(codes int8, scales float64) of the rows of x."""
    x = np.asarray(x, dtype=np.float64)
    codes, scales = np.zeros(x.shape, np.int8), np.zeros(x.shape[0])
    for r, row in enumerate(x):
        scales[r] = scale_of(float(np.max(np.abs(row))) if np.all(np.isfinite(row)) else math.inf)
        if scales[r] > 0.0:
            codes[r] = np.clip(np.rint(row / scales[r]), -127, 127).astype(np.int8)
    return codes, scales


def unpack(codes, scales) -> np.ndarray:
    return codes.astype(np.float64) * np.asarray(scales, dtype=np.float64)[:, None]


def rms_norm(h, weight, eps):
    """(rstd, y) of rows h."""
    h = np.asarray(h, dtype=np.float64)
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=1) + eps)
    return rstd, h * rstd[:, None] * np.asarray(weight, dtype=np.float64)


def rms_norm_backward(dy, h, rstd, weight, dh=None):
    """(dx, dweight) for given rows h and reciprocal norms rstd."""
    dy, h, rstd = (np.asarray(v, dtype=np.float64) for v in (dy, h, rstd))
    n, g = h * rstd[:, None], dy * np.asarray(weight, dtype=np.float64)
    dx = rstd[:, None] * (g - n * np.mean(g * n, axis=1, keepdims=True))
    return (dx if dh is None else dx + np.asarray(dh, dtype=np.float64)), np.sum(dy * n, axis=0)


def matmul(a, a_scales, b, b_scales) -> np.ndarray:
    s = a.astype(np.int64) @ b.astype(np.int64).T
    return s * np.asarray(a_scales, np.float64)[:, None] * np.asarray(b_scales, np.float64)


def matmul_grad_input(dy, b, b_scales) -> np.ndarray:
    return np.asarray(dy, np.float64) @ round_bf16(unpack(b, b_scales))


def matmul_grad_weight(dy, a, a_scales) -> np.ndarray:
    return np.asarray(dy, np.float64).T @ round_bf16(unpack(a, a_scales))
