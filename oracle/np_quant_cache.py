"""NumPy restatement of the quantised paged cache: the codes by fp32 operations rounded one by one (bit for bit what the format
says), the values that codes stand for in 64 bits.
"""
from __future__ import annotations

import numpy as np


def bf16(x):
    """fp32 values rounded to bf16 (nearest, ties to even; NaN stays), as fp32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = ((u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r)


def rotate32(x, cos, sin):
    """Heads [..][D] fp32, half split, two products and a sum, each rounded to fp32."""
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    f = np.float32
    return np.concatenate([f(a * cos) - f(b * sin), f(b * cos) + f(a * sin)], axis=-1)


def quantise(v, bits):
    """(codes, scale, zero) of heads v [..][D] fp32: codes as whole numbers, one scale (and zero point) per head."""
    v = np.asarray(v, dtype=np.float32)
    with np.errstate(all="ignore"):
        if bits == 8:
            s = bf16(np.abs(v).max(axis=-1) / np.float32(127.0))
        else:
            lo, hi = np.minimum(v.min(axis=-1), np.float32(0)), np.maximum(v.max(axis=-1), np.float32(0))
            s = bf16((hi - lo) / np.float32(15.0))
        strange = ~np.isfinite(v).all(axis=-1) | ~np.isfinite(s)
        none = ~strange & (s < np.float32(2.0 ** -126))
        s = np.where(strange | none, np.float32(1.0), s)
        skip = (strange | none)[..., None]
        q = np.where(skip, np.float32(0), np.rint(v / s[..., None]))
        z = np.zeros_like(s)
        if bits == 8:
            q = np.clip(q, -128, 127)
        else:
            z = np.where(strange | none, np.float32(0), np.clip(np.rint(-lo / s), 0, 15))
            q = np.where(skip, np.float32(0), np.clip(q + z[..., None], 0, 15))
    return q.astype(np.int64), np.where(strange, np.float32(np.nan), s), z


def values(codes, scale, zero, bits):
    """What codes stand for, in 64 bits."""
    c = codes.astype(np.float64)
    if bits == 4:
        c = c - zero.astype(np.float64)[..., None]
    with np.errstate(invalid="ignore"):
        return c * scale.astype(np.float64)[..., None]


def unpack(words):
    """4-bit codes [..][D] of words [..][D / 8] (code d: word d / 8, bits 4 (d % 8))."""
    w = words.astype(np.int64) & 0xFFFFFFFF
    return ((w[..., None] >> (4 * np.arange(8))) & 15).reshape(*w.shape[:-1], -1)
