"""Log probabilities, entropies, best answers and their gradient against their definitions in float64 (oracle.scores).

Tolerances, in units u = 2^-24. (s - s_max) / T is off by 2u of itself, its multiple of log2 e in units of log2 by 3u, and w =
2^x by |x| ln 2 times that and the 2^-22 of the special function unit: (3 |d| + 4) u relative, where d = (s - s_max) / T. The entries that
count have |d| < 25, most of the mass |d| < 6; sums of at most 16 terms are added with their rounding kept, so Z is good to
80 u relative at most, log Z to that and u |log Z|, and log p to 80 u + 3u |d| + u |log p| < 100 u + 4 u |log p|, as
|d| <= |log p|: 6e-6 + 2.4e-7 |log p|. The entropy is log Z - (sum w d) / Z with the same relative errors of w and d in
both: 80 u (1 + H) + 3 u max |d w| ... < 1e-5 (1 + H). A gradient's element is p times (a + b (log p + H)): p good to
120 u relative with |log p| < 30, the bracket to 2e-5 (|a| + |b| (1 + H + |log p|)) of its terms, and rounded to its type."""
import numpy as np
import pytest
import torch

from oracle import scores as OS
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}


def inputs(rows, n, seed, dtype=torch.float32, spread=2.0, masked=True):
    g = np.random.default_rng(seed)
    s = (spread * g.standard_normal((rows, n))).astype(np.float32)
    if masked and n > 3:
        s[g.random((rows, n)) < 0.1] = -np.inf
        s[g.random((rows, n)) < 0.05] = np.nan
    t = torch.from_numpy(g.integers(0, n, rows).astype(np.int32)).cuda()
    return torch.from_numpy(s).cuda().to(dtype), t


def at(v, r):
    return float(v[r]) if isinstance(v, torch.Tensor) else float(np.float32(v))


def check(s, t, T=1.0, top=0, rows=None):
    out = emr.log_probs(s, t, T, top)
    again = emr.log_probs(s, t, T, top)
    for x, y in zip((out.logp, out.entropy, out.top_index, out.top_logp), (again.logp, again.entropy, again.top_index, again.top_logp)):
        assert x is None and y is None or torch.equal(x.view(torch.int32), y.view(torch.int32))
    sn, tn = s.double().cpu().numpy(), t.cpu().numpy()
    logp, h = out.logp.double().cpu().numpy(), out.entropy.double().cpu().numpy()
    if top:
        index, best = out.top_index.cpu().numpy(), out.top_logp.double().cpu().numpy()
    near = lambda x, y: x == y or abs(x - y) <= 6e-6 + 2.4e-7 * abs(y)
    for r in range(len(sn)) if rows is None else rows:
        lp = OS.log_p(sn[r], at(T, r))
        want = np.nan if tn[r] >= len(lp) else 0.0 if tn[r] < 0 else lp[tn[r]]
        assert near(logp[r], want) or (np.isnan(want) and np.isnan(logp[r])), (r, logp[r], want)
        want = OS.entropy(lp)
        assert abs(h[r] - want) <= 1e-5 * (1 + want), (r, h[r], want)
        if top:
            order = OS.best(sn[r], top)
            assert np.array_equal(index[r], order), r
            assert all(near(x, lp[i] if i >= 0 else -np.inf) for x, i in zip(best[r], order)), r


def check_gradient(s, t, a, b, T=1.0, out_dtype=None, rows=None):
    ds, logp, h = emr.log_probs_grad(s, t, a, b, T, out_dtype)
    again = emr.log_probs_grad(s, t, a, b, T, out_dtype)
    plain = emr.log_probs(s, t, T)
    assert ds.dtype == (out_dtype or s.dtype) and ds.shape == s.shape
    for x, y in ((ds, again[0]), (logp, plain.logp), (h, plain.entropy)):
        assert torch.equal(torch.nan_to_num(x, 7.0), torch.nan_to_num(y, 7.0))
    sn, tn = s.double().cpu().numpy(), t.cpu().numpy()
    for r in range(len(sn)) if rows is None else rows:
        da, db, heat = at(a, r), at(b, r) if b is not None else 0.0, at(T, r)
        want, got = OS.log_p_gradient(sn[r], int(tn[r]), da, db, heat), ds[r].double().cpu().numpy()
        assert np.array_equal(np.isnan(want), np.isnan(got))
        lp = OS.log_p(sn[r], heat)
        on = lp > -np.inf
        size = np.zeros(len(want))
        size[on] = np.exp(lp[on]) * (abs(da) + abs(db) * (1 + OS.entropy(lp) + np.abs(lp[on])))
        if 0 <= tn[r] < len(want):
            size[tn[r]] += abs(da)
        tol = (4e-5 * size) / (heat if heat > 0 else 1.0) + HALF[ds.dtype] * np.abs(want) + LEAST[ds.dtype]
        ok = np.isnan(want) | (np.abs(got - want) <= tol)
        assert ok.all(), (r, np.argmin(ok), got[~ok][:3], want[~ok][:3])


# a warp's rows (many and short), a block's, a cluster's; odd lengths
SHAPES = [(1, 1), (3, 2), (5, 31), (7, 1364), (1300, 33), (2000, 340), (1220, 2047), (40, 5460), (1, 4097), (70, 8193),
          (20, 20001), (2, 87380), (200, 30011), (9, 349524), (2, 600001)]


def some(rows):
    return range(rows) if rows <= 300 else list(range(0, rows, 97)) + [rows - 1]


@pytest.mark.parametrize("rows,n", SHAPES)
@pytest.mark.parametrize("T,top", [(1.0, 0), (0.7, 5), (1.3, 32), (2.0, 100), (1.0, 256), (0.0, 3)])
def test_log_probs(rows, n, T, top):
    s, t = inputs(rows, n, 1)
    check(s, t, T, top, some(rows))


@pytest.mark.parametrize("dtype", TYPES[1:])
@pytest.mark.parametrize("rows,n", [(1300, 333), (30, 5461), (6, 87380), (3, 700001)])
def test_types(dtype, rows, n):
    s, t = inputs(rows, n, 2, dtype)
    check(s, t, 0.8, 20, some(rows))


@pytest.mark.parametrize("rows,n", SHAPES)
@pytest.mark.parametrize("T,entropy", [(1.0, False), (0.6, True)])
def test_gradient(rows, n, T, entropy):
    s, t = inputs(rows, n, 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    a = torch.randn(rows, device="cuda", generator=g)
    check_gradient(s, t, a, torch.randn(rows, device="cuda", generator=g) if entropy else None, T, rows=some(rows))


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(1250, 341), (9, 5461), (3, 87381)])
def test_gradient_types(dtype, out, rows, n):
    s, t = inputs(rows, n, 5, dtype)
    check_gradient(s, t, 1.5, -0.25, 0.9, out, some(rows))


def test_equal_scores_are_ordered_by_index():
    """More equal scores than the list of candidates holds: the k-th entry is looked for by bytes."""
    for rows, n in ((2, 1000), (1300, 300), (3, 20000), (2, 400000)):
        s = torch.zeros(rows, n, device="cuda")
        s[0, n // 3:] = 1.0
        s[1, ::2] = -1.0
        s[-1, n - 1] = 2.0
        t = torch.zeros(rows, dtype=torch.int32, device="cuda")
        for top in (1, 31, 256):
            check(s, t, 1.0, top, [0, 1, rows - 1])
            check(s.bfloat16(), t, 1.0, top, [0, 1, rows - 1])


def test_the_best_lie_together():
    """Rows in order, up and down: the largest entries belong to few threads."""
    for n in (2000, 50000, 349524):
        s = torch.arange(n, device="cuda", dtype=torch.float32).mul_(20.0 / n).expand(3, n).clone()
        s[1] = s[1].flip(0)
        s[2, 100:400] = 50.0
        t = torch.tensor([n - 1, 0, 5], dtype=torch.int32, device="cuda")
        for top in (7, 256):
            check(s, t, 1.0, top)
            check(s.half(), t, 1.0, top)


@pytest.mark.parametrize("n", [50, 6000, 90000])
def test_few_distinct_scores(n):
    g = np.random.default_rng(6)
    s = torch.from_numpy(g.integers(-3, 4, (12, n)).astype(np.float32)).cuda()
    t = torch.from_numpy(g.integers(0, n, 12).astype(np.int32)).cuda()
    check(s, t, 0.9, 200)
    check_gradient(s, t, 1.0, 0.5, 0.9)


@pytest.mark.parametrize("rows,n", [(12, 3000), (12, 100001), (1300, 300)])
def test_masked_rows_and_infinities(rows, n):
    s, t = inputs(rows, n, 7)
    s[0] = float("-inf")                              # nothing left
    s[1] = float("nan")
    s[2, :-1] = float("-inf")                         # one entry left, the last
    t[2] = n - 1
    s[3, 7] = float("nan")
    t[3] = 7                                          # a masked answer
    s[4, 5] = s[4, n - 1] = float("inf")              # only these two
    t[4] = 5
    s[5, 6] = float("inf")
    t[5] = 9
    s[6] = -3.4028234e38                              # a mask of the type's lowest value everywhere
    s[7, 1:] = -3.4028234e38
    s[7, 0] = 3.4028234e38
    t[7] = 0
    t[8], t[9], t[10] = -1, n, 2 ** 31 - 1
    s[11] = 80.0 + s[11]
    for T, top in ((1.0, 0), (0.7, 9), (0.0, 4), (float("nan"), 2), (float("inf"), 3)):
        check(s, t, T, top, range(12))
        check_gradient(s, t, 1.0, 0.25, T, rows=range(12))
    r = emr.log_probs(s, t, top=3)
    assert r.logp[0] == r.logp[1] == -np.inf and r.entropy[:3].tolist() == [0, 0, 0] and r.logp[2] == 0
    assert r.top_index[0].tolist() == [-1, -1, -1] and r.top_index[4].tolist() == [5, n - 1, -1]
    h = s.half()                                      # overflows to -inf, and +inf, there
    check(h, t, 1.0, 5, range(12))
    check_gradient(h, t, 1.0, 0.25, rows=range(12))


def test_parameters_for_each_row_and_strides():
    rows, n = 64, 2500
    s, t = inputs(rows, 2 * n, 8)
    g = np.random.default_rng(9)
    f = lambda v: torch.from_numpy(g.choice(v, rows).astype(np.float32)).cuda()
    T, a, b = f([0.0, 0.5, 1.0, 2.0, -1.0]), f([0.0, 1.0, -2.0]), f([0.0, 0.5])
    t = t % n
    for v in (s[:, 3:n + 3], s[:, ::2], s[:1, :n].expand(rows, n)):
        check(v, t, T, 12)
        check_gradient(v, t, a, b, T)
    one = emr.log_probs(s[0], t[:1], top=2)
    assert one.logp.shape == one.entropy.shape == (1,) and one.top_index.shape == (1, 2)
    assert emr.log_probs_grad(s[0], t[:1], 1.0)[0].shape == (2 * n,)
    none = emr.log_probs(s, top=1)
    assert none.logp is None and emr.log_probs(s).top_index is None


def test_gradient_against_differences():
    """The kernel's own values, central differences in T = 1 units of 1/8: the third derivative of log p and H is below 1, so
    they are off by at most 1/8^2 / 6 of a step; 0.02 with the values' 1e-5 / (1/4)."""
    s, t = inputs(3, 40, 10, masked=False)
    ds, _, _ = emr.log_probs_grad(s, t, 1.0, 0.5)
    for i in range(40):
        v = []
        for e in (0.125, -0.125):
            x = s.clone()
            x[:, i] += e
            r = emr.log_probs(x, t)
            v.append(r.logp + 0.5 * r.entropy)
        assert torch.allclose((v[0] - v[1]) / 0.25, ds[:, i], atol=0.02)


def test_values_agree_with_draws():
    """log_probs of drawn answers is what the draw itself says (no filters): both within 4e-6 + 2^-23 |log p| and ours."""
    s, _ = inputs(200, 5460, 11, masked=False)
    e = torch.empty_like(s).exponential_().clamp_min_(1e-30)
    for T in (0.0, 0.7, 1.0):
        index, logp = emr.sample(s, e, temperature=T)
        assert torch.allclose(emr.log_probs(s, index, T).logp, logp, atol=1.2e-5)
        index, logp = emr.sample(s, e, temperature=T, top_k=1)
        assert torch.equal(emr.log_probs(s, index, T, top=1).top_index[:, 0], index)


def test_refusals():
    s, t = inputs(4, 10, 12)
    f = torch.ones(4, device="cuda")
    for call in (lambda: emr.log_probs(s.double(), t), lambda: emr.log_probs(s.cpu(), t.cpu()), lambda: emr.log_probs(s[None], t),
                 lambda: emr.log_probs(s, t.long()), lambda: emr.log_probs(s, t[:3]), lambda: emr.log_probs(s, t.cpu()),
                 lambda: emr.log_probs(s, [1, 2, 3, 4]), lambda: emr.log_probs(s, t, top=257), lambda: emr.log_probs(s, t, top=-1),
                 lambda: emr.log_probs(s, t, f[:3]), lambda: emr.log_probs(s[:, :0], t), lambda: emr.log_probs_grad(s, None, 1.0),
                 lambda: emr.log_probs_grad(s, t, f.double()), lambda: emr.log_probs_grad(s, t, 1.0, f[:2]),
                 lambda: emr.log_probs_grad(s, t, 1.0, out_dtype=torch.float64)):
        with pytest.raises(ValueError):
            call()
    empty = emr.log_probs(s[:0], t[:0], top=2)
    assert empty.logp.shape == (0,) and empty.top_index.shape == (0, 2)
    assert emr.log_probs_grad(s[:0], t[:0], 1.0)[0].shape == (0, 10)
