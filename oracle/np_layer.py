"""NumPy restatement, in 64 bits, of the operators between the linears of a decoder layer: residual RMS norm, rotary
embedding with append to a paged cache, attention of new tokens over the cache, low-rank adapters of many requests.

Inputs are float64 arrays (bf16 values widened exactly); nothing is rounded.
"""
from __future__ import annotations

import numpy as np


def rmsnorm(x, weight, eps, residual=None):
    """(v, h): the normalised rows and the sum they were taken of."""
    h = x if residual is None else x + residual
    return h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps) * weight, h


def a8_scale(v):
    """Per-row scale of the int8 output: max |v| / 127, 1 for a row of zeros."""
    s = np.abs(v).max(axis=1) / 127.0
    return np.where(s == 0, 1.0, s)


def positions(cu_q, kv_len):
    """(request, position) of every packed row."""
    seq, pos = [], []
    for b, kv in enumerate(kv_len):
        n = int(cu_q[b + 1]) - int(cu_q[b])
        seq += [b] * n
        pos += [int(kv) - n + i for i in range(n)]
    return seq, pos


def rope_rotate(x, pos, theta):
    """x [heads][D] at one position, half split."""
    half = x.shape[1] // 2
    angle = pos * theta ** (-np.arange(half) / half)
    c, s = np.cos(angle), np.sin(angle)
    a, b = x[:, :half], x[:, half:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=1)


def gather_cache(cache, table_row, n):
    """The first n cached tokens of a request: [n][Hk][D] from [pages][Hk][page][D]."""
    page = cache.shape[2]
    return np.stack([cache[table_row[j // page], :, j % page] for j in range(n)]) if n else np.zeros((0,) + cache.shape[1::2])


def attn(q, k, v, first_pos, scale):
    """One request: q [n][H][D] at positions first_pos + i over k, v [kv][Hk][D].  Returns (out, spread, score error scale):
    spread = sum_j w_j |v_j| and the largest sum_d |q_d k_d| |scale| of a row, for tolerances."""
    n, H, D = q.shape
    Hk = k.shape[1]
    out, spread, absdot = np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((n, H))
    for h in range(H):
        kh, vh = k[:, h * Hk // H], v[:, h * Hk // H]
        for i in range(n):
            end = first_pos + i + 1
            if end <= 0:
                continue
            s = kh[:end] @ q[i, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ vh[:end]
            spread[i, h] = w @ np.abs(vh[:end])
            absdot[i, h] = (np.abs(kh[:end]) @ np.abs(q[i, h])).max() * abs(scale)
    return out, spread, absdot


def lora_batch(x, a, b, cu_q, adapter, scales):
    """(side, absolute side): what the adapters add to the rows, and the same of absolute values."""
    M, N = x.shape[0], b.shape[1]
    side, absside = np.zeros((M, N)), np.zeros((M, N))
    for i, ad in enumerate(adapter):
        if 0 <= ad < a.shape[0]:
            lo, hi = int(cu_q[i]), int(cu_q[i + 1])
            side[lo:hi] = scales[ad] * (x[lo:hi] @ a[ad].T) @ b[ad].T
            absside[lo:hi] = abs(scales[ad]) * (np.abs(x[lo:hi]) @ np.abs(a[ad]).T) @ np.abs(b[ad]).T
    return side, absside
