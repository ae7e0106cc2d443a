"""Sampling by temperature, top-k, top-p and min-p in 64 bits on the CPU: a row
sorted, its cumulative weights, its inverse CDF."""
from __future__ import annotations

import numpy as np


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row.  Returns (token, probs, kept ids, margin): margin is the least
    distance of a sum from a border that it was compared with, as a share of the
    total weight, infinite where no sum decides anything."""
    x = np.asarray(logits, np.float64).copy()
    x[np.isnan(x)] = -np.inf
    V = x.size
    probs = np.zeros(V)
    if not (x > -np.inf).any():
        return -1, probs, np.zeros(0, np.int64), np.inf
    order = np.lexsort((np.arange(V), -x))
    order = order[x[order] > -np.inf]
    s = x[order]
    one = not temperature > 0 or not top_p > 0 or not min_p <= 1
    margin = np.inf
    if one:
        n, w = 1, np.ones(1)
    else:
        n = min(top_k, s.size) if top_k > 0 else s.size
        with np.errstate(invalid="ignore", over="ignore", under="ignore"):
            w = np.where(s == s[0], 1.0, np.exp((s - s[0]) / np.float64(temperature)))[:n]
        w[np.isnan(w)] = 0.0
        if top_p < 1:
            total = np.cumsum(w)
            mark = np.float64(top_p) * total[-1]
            m = int(np.searchsorted(total, mark)) + 1
            near = np.abs(total - mark).min() / total[-1]
            margin = min(margin, near)
            n = min(n, m)
        n = min(n, max(1, int((w >= np.float64(min_p)).sum())))
        w = w[:n]
    ids = np.sort(order[:n])
    q = np.zeros(V)
    q[order[:n]] = w
    total = np.cumsum(q[ids])
    probs = q / total[-1]
    mark = np.float64(u) * total[-1]
    token = int(ids[min(np.searchsorted(total, mark, side="right"), n - 1)])
    if n > 1 and mark > 0:                 # a mark of zero is met by the first weight, whatever the sums' rounding
        margin = min(margin, np.abs(total[:-1] - mark).min() / total[-1])
    return token, probs, ids, margin
