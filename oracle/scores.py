"""Log probabilities and distillation by their definitions in float64 numpy, one row at a time. Test infrastructure;
shares no code with the GPU path."""
import numpy as np


FAR = 2.0 ** 128 - 2.0 ** 103                         # rounds to infinity in 32 bits


def live(s):
    """The scores of a row in 64 bits with masked entries at -inf; rows with +inf keep only those, as 0."""
    s = np.asarray(s, np.float64)
    s = np.where(np.isnan(s), -np.inf, s)
    if (s == np.inf).any():
        s = np.where(s == np.inf, 0.0, -np.inf)
    return s


def log_p(s, T=1.0):
    """Log probabilities of a row's entries, -inf for masked ones and for those that lie further below the largest
    than 32 bits can say (lowest - largest = -6.8e38), whatever T."""
    v = live(s)
    out = np.full(v.shape, -np.inf)
    on = v > -np.inf
    if not on.any():
        return out
    if not T > 0:
        out[np.argmax(v)] = 0.0
        return out
    on &= v - v.max() > -FAR
    d = (v[on] - v.max()) / T
    out[on] = d - np.log(np.exp(d).sum())
    return out


def entropy(lp):
    on = lp > -np.inf
    return float(-(np.exp(lp[on]) * lp[on]).sum())


def best(s, k):
    """The k largest scores' places, larger first, then by index; -1 past those that are not masked."""
    v = live(s)
    order = np.argsort(-v, kind="stable")[:k]
    order = np.where(v[order] > -np.inf, order, -1)
    return np.concatenate([order, np.full(k - len(order), -1)]).astype(np.int64)


def log_p_gradient(s, target, a, b, T=1.0):
    """Gradient of a log p[target] + b entropy."""
    v, n = live(s), len(s)
    lp = log_p(s, T)
    if target >= n:
        return np.full(n, np.nan)
    g = np.zeros(n)
    on = v > -np.inf
    if not T > 0 or not on.any():
        return g
    p, h = np.exp(lp), entropy(lp)
    g = -b * p * (np.where(p > 0, lp, 0.0) + h)
    if target >= 0:
        g -= a * p
        if on[target]:
            g[target] += a
    return g / T
