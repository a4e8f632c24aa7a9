"""Sampling from scores against its definition in float64 (oracle.sampling). Indices have to be equal, except
that a decision of the definition (the end of the top-p prefix, a min-p edge, the two best draws) that is within
1e-5 relative of its edge may fall either way: w is a 32-bit exponential of a 32-bit quotient, good to (|x| + 4) 2^-23 relative, under 4e-6 for the
x = (s - s_max) / T > -30 that matter here, and sums of w are exact to 2^-44 an entry. The log of a probability is
then within 4e-6 + 2^-23 |log p|."""
import numpy as np
import pytest
import torch

from oracle import sampling as OS
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu

EDGE = 1e-5


def inputs(rows, n, seed, dtype=torch.float32, spread=2.0):
    g = np.random.default_rng(seed)
    s = torch.from_numpy((spread * g.standard_normal((rows, n))).astype(np.float32)).cuda().to(dtype)
    e = torch.from_numpy(np.maximum(g.standard_exponential((rows, n)), 1e-20).astype(np.float32)).cuda()
    return s, e


def check(s, e, T=1.0, k=0, p=1.0, q=0.0):
    index, logp = emr.sample(s, e, T, k, p, q)
    again = emr.sample(s, e, T, k, p, q)
    assert torch.equal(index, again[0]) and torch.equal(logp, again[1])
    index, logp, sn, en = index.cpu().numpy(), logp.double().cpu().numpy(), s.double().cpu().numpy(), e.double().cpu().numpy()
    at = lambda v, r: float(v[r]) if isinstance(v, torch.Tensor) else float(np.float32(v))
    ties = 0
    for r in range(len(sn)):
        t, kk, pp, qq = at(T, r), int(at(k, r)), at(p, r), at(q, r)
        want = [OS.sample(sn[r], en[r], t, kk, pp, qq)]
        if want[0][2] < EDGE:                         # a decision near its edge may fall either way
            want += [OS.sample(sn[r], en[r], t, kk, pp * (1 + x) if pp < 1 else pp, qq * (1 + y)) for x in (-EDGE, EDGE)
                     for y in (-EDGE, EDGE)]
        lps = [w[1] for w in want if w[0] == index[r]]
        if not lps:
            assert min(w[3] for w in want) < EDGE, (r, index[r], want)   # the two best draws are that close
            ties += 1
        elif np.isinf(lps[0]):
            assert logp[r] == lps[0]
        else:
            tol = 4e-6 + 2.0 ** -23 * abs(lps[0])
            assert min(lps) - tol <= logp[r] <= max(lps) + tol, (r, logp[r], lps)
    assert ties <= max(1, 0.01 * len(sn))


# slices of one block and of clusters of 2, 4 and 8; in shared memory and beyond it; odd lengths
SHAPES = [(1, 1), (3, 2), (5, 31), (7, 1364), (200, 1000), (40, 5460), (1, 4097), (70, 8193), (20, 20001), (2, 87380),
          (160, 30011), (9, 349524), (2, 600001)]


@pytest.mark.parametrize("rows,n", SHAPES)
@pytest.mark.parametrize("T,k,p,q", [(1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.02), (1.3, 0, 0.9, 0.0), (1.0, 3, 1.0, 0.0),
                                     (0.5, 5000, 0.8, 0.0), (1.0, 0, 0.0, 0.0), (2.0, 0, 1.0, 0.3), (0.0, 7, 0.5, 0.1)])
def test_sample(rows, n, T, k, p, q):
    s, e = inputs(rows, n, 1)
    check(s, e, T, k, p, q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n", [(30, 5461), (6, 87380), (3, 700001)])
def test_sample_types(dtype, rows, n):
    s, e = inputs(rows, n, 2, dtype)
    check(s, e, 0.8, 40, 0.95)
    check(s, e, 0.8, 0, 1.0)
    check(s, e, 0.8, 3000, 1.0)


def test_top_p_keeps_the_prefix():
    """Kept sets themselves: noise so small at one entry that it is drawn whenever it stays."""
    n = 4001
    s, e = inputs(1, n, 3)
    sn = s.double().cpu().numpy()[0]
    for p in (0.1, 0.5, 0.9, 0.99):
        at, w, margin = OS.kept_entries(sn, 1.0, 0, p, 0.0)
        for place, stays in ((0, True), (len(at) - 2, True), (len(at) + 1, False), (n - 1, False)):
            entry = int(np.argsort(-sn, kind="stable")[place])
            noise = torch.ones_like(e)
            noise[0, entry] = 1e-30
            index, _ = emr.sample(s, noise, top_p=p)
            assert (int(index) == entry) == stays


def test_equal_scores_are_taken_by_index():
    n = 20000
    s = torch.zeros(1, n, device="cuda")
    s[0, 100:15000] = 1.0
    for k in (1, 2, 513, 14899, 14900, 14901, 19999):
        for entry in (i for i in (100, 100 + k - 1, 100 + k, 14999, 0, n - 1) if i < n):
            noise = torch.ones(1, n, device="cuda")
            noise[0, entry] = 1e-30
            index, logp = emr.sample(s, noise, top_k=k)
            kept = 100 <= entry < 100 + min(k, 14900) or (k > 14900 and entry < k - 14900)
            assert (int(index) == entry) == (kept or entry == 100), (k, entry)
            mass = min(k, 14900) + max(0, k - 14900) * np.exp(-1)
            if kept:
                w = 1.0 if 100 <= entry < 15000 else np.exp(-1)
                assert abs(float(logp) - np.log(w / mass)) < 1e-6
    # the same by mass: a prefix of 10,000 of the equal ones
    p = 9999.5 / (14900 + 5100 * np.exp(-1))
    for entry, stays in ((100, True), (10099, True), (10100, False), (0, False)):
        noise = torch.ones(1, n, device="cuda")
        noise[0, entry] = 1e-30
        index, _ = emr.sample(s, noise, top_p=float(p))
        assert (int(index) == entry) == stays


@pytest.mark.parametrize("n", [50, 6000, 90000])
def test_few_distinct_scores(n):
    g = np.random.default_rng(4)
    s = torch.from_numpy(g.integers(-3, 4, (12, n)).astype(np.float32)).cuda()
    e = torch.from_numpy(g.standard_exponential((12, n)).astype(np.float32)).cuda()
    check(s, e, 1.0, n // 3, 1.0)
    check(s, e, 0.9, n // 2, 1.0, 0.01)
    check(s, e, 1.0, 0, 0.7)


def test_masked_rows_and_infinities():
    n = 3000
    s, e = inputs(8, n, 5)
    s[0] = float("-inf")                              # nothing left
    s[1] = float("nan")
    s[2, :-1] = float("-inf")                         # one entry left, the last
    s[3, 7] = float("nan")
    s[4, 5] = s[4, 2999] = float("inf")               # only these two
    s[5, ::2] = float("-inf")
    s[6] = -3.4028234e38                              # a mask of the type's lowest value everywhere
    s[7, 1:] = -3.4028234e38
    for kw in (dict(), dict(k=5), dict(k=2900), dict(p=0.9), dict(k=2000, p=0.5, q=0.1), dict(T=0.0)):
        check(s, e, **kw)
    index, logp = emr.sample(s, e, top_p=0.5)
    assert index[:3].tolist() == [-1, -1, n - 1] and logp[:3].tolist() == [-np.inf, -np.inf, 0.0]
    assert int(index[4]) in (5, 2999) and abs(float(emr.sample(s, e)[1][4]) - np.log(0.5)) < 1e-6
    assert int(index[7]) == 0
    h = s.half()                                      # overflows to -inf there
    assert emr.sample(h, e)[0][6] == -1


def test_parameters_for_each_row_and_strides():
    rows, n = 64, 2500
    s, e = inputs(rows, 2 * n, 6)
    g = np.random.default_rng(7)
    T = torch.from_numpy(g.choice([0.0, 0.5, 1.0, 2.0], rows).astype(np.float32)).cuda()
    k = torch.from_numpy(g.choice([0, 1, 10, 2000, 2500, 9999, -1], rows).astype(np.int32)).cuda()
    p = torch.from_numpy(g.choice([0.3, 0.9, 1.0, 1.5], rows).astype(np.float32)).cuda()
    q = torch.from_numpy(g.choice([0.0, 0.05, 1.0, 2.0], rows).astype(np.float32)).cuda()
    check(s[:, 3:n + 3], e[:, 1:n + 1], T, k, p, q)
    check(s[:, ::2], e[:, ::2], T, k, p, q)
    check(s[:1, :n].expand(rows, n), e[:, :n], T, k, p, q)
    one, _ = emr.sample(s[0], e[0])
    assert one.shape == (1,)


def test_draws_follow_the_probabilities():
    """20,000 draws from one row of 6 kept entries: each frequency within 5 standard deviations."""
    rows = 20000
    s = torch.tensor([1.0, 0.5, 3.0, -2.0, 2.0, 2.5, 0.0, 1.5], device="cuda").expand(rows, 8)
    g = torch.Generator(device="cuda").manual_seed(8)
    e = torch.empty(rows, 8, device="cuda").exponential_(generator=g).clamp_min_(1e-30)
    index, logp = emr.sample(s, e, temperature=1.5, top_k=6)
    at, w, _ = OS.kept_entries(s[0].double().cpu().numpy(), 1.5, 6, 1.0, 0.0)
    prob = w / w.sum()
    got = np.bincount(index.cpu().numpy(), minlength=8)
    assert got.sum() == got[at].sum() == rows
    assert np.all(np.abs(got[at] - rows * prob) <= 5 * np.sqrt(rows * prob * (1 - prob)))
    assert np.allclose(logp.cpu().numpy(), np.log(prob)[[list(at).index(i) for i in index.cpu().numpy()]], atol=1e-6)


def test_refusals():
    s, e = inputs(4, 10, 9)
    for call in (lambda: emr.sample(s, e[:, :9]), lambda: emr.sample(s, e.half()), lambda: emr.sample(s.double(), e),
                 lambda: emr.sample(s.cpu(), e.cpu()), lambda: emr.sample(s[None], e[None]),
                 lambda: emr.sample(s, e, top_k=torch.zeros(4, device="cuda")),
                 lambda: emr.sample(s, e, temperature=torch.ones(3, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    L = emr.lib()
    import ctypes as C
    ok = [s.data_ptr(), 0, 4, 10, 10, e.data_ptr(), 10, None, 1.0, None, 0, None, 1.0, None, 0.0, e.data_ptr(), None, None]
    for i, v, want in ((0, None, emr.EMR_ERR_ARG), (1, 3, emr.EMR_ERR_ARG), (2, 0, emr.EMR_ERR_ARG), (3, 0, emr.EMR_ERR_ARG),
                       (3, 2 ** 31, emr.EMR_ERR_RANGE), (4, -1, emr.EMR_ERR_ARG), (5, None, emr.EMR_ERR_ARG),
                       (5, e.data_ptr() + 2, emr.EMR_ERR_ARG), (6, -1, emr.EMR_ERR_ARG), (15, None, emr.EMR_ERR_ARG),
                       (2, 2 ** 27 + 1, emr.EMR_ERR_RANGE)):
        args = list(ok)
        args[i] = v
        assert L.emr_sample(*args) == want, (i, v)
    assert emr.sample(s[:0], e[:0])[0].shape == (0,)
