"""The choice of a token from one row of logits, restated on the host in 64 bits (sums by math.fsum)."""
from __future__ import annotations

import math

import numpy as np


def distribution(x, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """(indices that stay, ascending; their weights).  Empty where no logit is above -inf."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, dtype=np.float64))
    if not (x > -np.inf).any():
        return np.zeros(0, dtype=np.int64), np.zeros(0)
    if (x == np.inf).any():
        x = np.where(x == np.inf, 0.0, -np.inf)
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    if not temperature > 0:
        return order[:1], np.ones(1)
    w = np.exp((x[order] - x[order[0]]) / temperature)
    live = w >= 2.0 ** -43
    order, w = order[live], w[live]
    if top_k > 0:
        order, w = order[:top_k], w[:top_k]
    if top_p < 1:
        goal, before = top_p * math.fsum(w), np.concatenate([[0.0], np.cumsum(w)[:-1]])
        n = max(1, int((before < goal).sum()))
        order, w = order[:n], w[:n]
    stay = (w >= min_p) if min_p <= 1 else np.zeros(len(w), dtype=bool)
    stay[0] = True
    order, w = order[stay], w[stay]
    by_index = np.argsort(order)
    return order[by_index], w[by_index]


def pick(x, u, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """(token, how far u times the total is from the nearest running sum, relative to the total): within rounding of one, the
    token on its other side would be as right."""
    index, w = distribution(x, temperature, top_k, top_p, min_p)
    if not len(index):
        return -1, 1.0
    run = np.cumsum(w)
    want = (u if u >= 0 else 0.0) * run[-1]
    at = min(int((run <= want).sum()), len(index) - 1)
    return int(index[at]), float(np.abs(run - want).min() / run[-1]) if len(index) > 1 else 1.0
