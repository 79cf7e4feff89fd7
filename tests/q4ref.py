"""The 4-bit cache's format in numpy, float64, from its definition: the reference
of the tests of the ``*_q4`` entry points."""
from __future__ import annotations

import numpy as np

MAG = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """Rows [..., d] (any float type, taken as they are) as codes [..., d / 2]
    and scale bytes [..., d / 32]."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    with np.errstate(all="ignore"):
        a = np.abs(b)
        top = a.max(-1)
        fine = np.isfinite(b).all(-1)
        e = np.full(top.shape, -125)
        for k in range(-125, 125):  # the smallest e with top <= 7 * 2^e
            e = np.where(top > 7 * 2.0 ** k, k + 1, e)
        a = a / 2.0 ** e[..., None]
        # nearest of MAG, ties to the even code
        code = np.zeros(a.shape, dtype=np.uint8)
        for c in range(1, 8):
            border = (MAG[c] + MAG[c - 1]) / 2
            code += ((a > border) if c % 2 else (a >= border)).astype(np.uint8)
        code += 8 * (b < 0).astype(np.uint8)
    code = np.where(fine[..., None], code, 0).astype(np.uint8).reshape(x.shape)
    scale = np.where(fine, e + 127, 255).astype(np.uint8)
    return code[..., ::2] | (code[..., 1::2] << 4), scale


def values(codes, scales):
    """What codes and scales stand for (float64)."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    x = MAG[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return x * np.repeat(s, 32, axis=-1)


def span_means(x, off, anchor=None):
    """Quantised spans of x [L][H][T][d] (float64 of the stored rows): codes and scales."""
    out = np.empty(x.shape[:2] + (len(off) - 1, x.shape[-1]))
    for j in range(len(off) - 1):
        n = off[j + 1] - off[j]
        s = x[:, :, off[j]: off[j + 1]].sum(2)
        out[:, :, j] = (s if anchor is None else s + n * anchor[:, :, j]) / n
    return quantise(out)
