"""Sampling from scores by its definition in float64 numpy, one row at a time. Test infrastructure; shares no
code with the GPU path."""
import numpy as np


def kept_entries(s, T, k, p, q):
    """(entries that stay, in order; their w; how near any decision is to its edge)."""
    s = np.asarray(s, np.float64)
    order = np.argsort(-s, kind="stable")
    order = order[(s > -np.inf)[order]]                # masked entries (also NaN) are out
    if len(order) == 0:
        return order, np.zeros(0), np.inf
    v = s[order]
    with np.errstate(invalid="ignore"):
        w = np.where(v == v[0], 1.0, np.exp((v - v[0]) / T))
    margin = np.inf
    if k > 0:
        order, w = order[:k], w[:k]
    if p < 1:
        before = np.cumsum(w) - w
        stay = before < p * w.sum()
        stay[0] = True
        if len(w) > 1:
            margin = min(margin, np.abs(before[1:] / w.sum() - p).min())
        order, w = order[stay], w[stay]
    stay = w >= min(q, 1.0)
    if q > 0:
        edge = np.abs(w[w < 1] / q - 1)
        margin = min(margin, edge.min() if len(edge) else np.inf)
    return order[stay], w[stay], margin


def sample(s, noise, T=1.0, k=0, p=1.0, q=0.0):
    """(index, log probability, how near any decision is to its edge, how near the second draw is to the best)."""
    s = np.asarray(s, np.float64)
    if not (s > -np.inf).any():
        return -1, -np.inf, np.inf, np.inf
    if not T > 0:
        return int(np.nanargmax(np.where(s > -np.inf, s, -np.inf))), 0.0, np.inf, np.inf
    at, w, margin = kept_entries(s, T, k, p, q)
    key = w / np.asarray(noise, np.float64)[at]
    best = np.lexsort((at, -key))                      # larger key, then lower index
    tie = np.inf
    if len(key) > 1 and key[best[0]] != key[best[1]]:
        tie = key[best[0]] / key[best[1]] - 1 if key[best[1]] > 0 else np.inf
    i = best[0]
    return int(at[i]), float(np.log(w[i] / w.sum())), margin, tie
