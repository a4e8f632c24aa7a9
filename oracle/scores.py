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


def distill(s, index, l, T=1.0, tail=True, with_gradient=True):
    """(loss, its gradient, the sum of the magnitudes of the loss's terms) of a row's scores against a teacher's list."""
    v, n = live(s), len(s)
    index, l = np.asarray(index, np.int64), np.asarray(l, np.float64)
    on = index >= 0
    if (index >= n).any() or np.isnan(l[on]).any() or not T > 0:
        return np.nan, np.full(n, np.nan), np.nan
    index, l = index[on], l[on]
    lp = log_p(s, T)
    p = np.exp(lp)
    rest = np.ones(n, bool)
    rest[index] = False
    rest &= v > -np.inf
    t_rest = 0.0
    if tail:
        t = np.exp(l)
        if rest.any():
            t_rest = max(0.0, 1.0 - t.sum())
    else:
        e = np.exp(l - l.max()) if len(l) and l.max() > -np.inf else np.zeros(len(l))
        t = e / e.sum() if e.sum() > 0 else e
    some = t > 0
    with np.errstate(divide="ignore"):
        terms = t[some] * (np.log(t[some]) - lp[index[some]])
        if t_rest > 0:
            m = lp[rest].max()
            lr = m + np.log(np.exp(lp[rest] - m).sum()) if m > -np.inf else -np.inf
            terms = np.append(terms, t_rest * (np.log(t_rest) - lr))
    g = (t.sum() + t_rest) * p
    np.add.at(g, index, -t)
    if t_rest > 0 and lr > -np.inf:
        e = np.exp(lp[rest] - m)  # lr = m + log(sum) has nothing left of the logarithm where m is -1e38
        g[rest] -= t_rest * e / e.sum()
    g[~(v > -np.inf)] = 0.0
    return terms.sum(), g / T, np.abs(terms).sum()
