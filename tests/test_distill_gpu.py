"""Distillation and its gradient against their definition in float64 (oracle.scores).

Tolerances, in units u = 2^-24. A student's log p is good to 100 u + 4 u |log p| (as log_probs), t = exp(l) to 4 u relative for
expf and (with tail 0) 100 u for the sum and its log: a term t (log t - log p) is off by at most 110 u t + 4 u t |log p| + 104
u |term|, the sum of k <= 256 terms by trees of at most 9 additions by 9 u of their magnitudes, together 2e-5 of the sum of t (1 + |log p|) and
of |terms|, of which sum t <= 1. What the teacher leaves over, t_r = 1 - sum t, is off by 110 u absolutely, its term by that times (1 +
|log t_r - log p_r|), where a difference of up to 5 is met: 4e-5. Together 4e-5 (1 + the sum of |terms|). A gradient's
element has p to 120 u relative and t to 104 u, and what is left of p_r sum t - t_r p_l to 240 u of each: 2e-5 (M p_i + t_i + e_i / z_r
(p_r sum t + t_r p_l)) and t_r's own 110 u, times e_i / z_r, rounded to its type."""
import numpy as np
import pytest
import torch

from oracle import scores as OS
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}


def inputs(rows, n, k, seed, dtype=torch.float32, T=1.0, masked=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = 2.0 * torch.randn(rows, n, device="cuda", generator=g)
    teacher = s + torch.randn(rows, n, device="cuda", generator=g)
    if masked and n > 8:
        off = torch.rand(rows, n, device="cuda", generator=g) < 0.1
        s[off], teacher[off] = float("-inf"), float("-inf")
    best = emr.log_probs(teacher, temperature=T, top=min(k, n))
    index, logp = torch.full((rows, k), -1, dtype=torch.int32, device="cuda"), torch.zeros(rows, k, device="cuda")
    index[:, :min(k, n)], logp[:, :min(k, n)] = best.top_index, best.top_logp
    return s.to(dtype), index, logp


def at(v, r):
    return float(v[r]) if isinstance(v, torch.Tensor) else float(np.float32(v))


def same(x, y):
    return torch.equal(torch.nan_to_num(x, 7.0), torch.nan_to_num(y, 7.0))


def check(s, index, l, T=1.0, tail=True, w=1.0, out=None, rows=None):
    ds, loss = emr.distill_grad(s, index, l, w, T, tail, out)
    again = emr.distill_grad(s, index, l, w, T, tail, out)
    assert same(ds, again[0]) and same(loss, again[1]) and same(loss, emr.distill(s, index, l, T, tail))
    assert ds.dtype == (out or s.dtype) and ds.shape == s.shape
    sn, xn, ln = s.double().cpu().numpy(), index.cpu().numpy(), l.double().cpu().numpy()
    for r in range(len(sn)) if rows is None else rows:
        heat, scale = at(T, r), at(w, r)
        want, g, size = OS.distill(sn[r], xn[r], ln[r], heat, tail)
        got, dg = float(loss[r]), ds[r].double().cpu().numpy()
        if not np.isfinite(want):
            assert np.isnan(want) and np.isnan(got) or want == got, (r, got, want)
        else:
            assert abs(got - want) <= 4e-5 * (1 + size), (r, got, want, size)
        assert np.array_equal(np.isnan(g), np.isnan(dg)), r
        if np.isnan(g).any():
            continue
        g = g * scale
        lp = OS.log_p(sn[r], heat)
        p = np.exp(lp)
        here = xn[r][xn[r] >= 0]
        listed = np.zeros(len(p), bool)
        listed[here] = True
        mag = 2 * p
        mag[listed] += 1.0
        p_rest = p[~listed].sum()
        t_sum = min(1.0, np.exp(ln[r][xn[r] >= 0]).sum()) if tail else 1.0
        if p_rest > 0:
            over = max(0.0, 1 - t_sum) if tail else 0.0
            mag[~listed] = p[~listed] / p_rest * (p_rest * t_sum + over * (1 - p_rest) + 0.4)
        tol = 2e-5 * mag * abs(scale) / heat + HALF[ds.dtype] * np.abs(g) + LEAST[ds.dtype]
        ok = np.abs(dg - g) <= tol
        assert ok.all(), (r, np.argmin(ok), dg[~ok][:3], g[~ok][:3])


# a warp's rows (many and short), a block's, a cluster's, slices of more than one piece of 131,072
SHAPES = [(1, 1, 1), (3, 2, 1), (5, 31, 4), (7, 1364, 16), (1300, 33, 8), (2000, 340, 50), (1220, 2047, 64), (1220, 2048, 65),
          (40, 5460, 50), (1, 4097, 256), (70, 8193, 64), (20, 20001, 100), (2, 87380, 256), (200, 30011, 10), (9, 349524, 100),
          (160, 140001, 20), (2, 1300001, 64)]


def some(rows):
    return range(rows) if rows <= 100 else list(range(0, rows, 97)) + [rows - 1]


@pytest.mark.parametrize("rows,n,k", SHAPES)
@pytest.mark.parametrize("T,tail", [(1.0, True), (0.7, True), (2.0, False)])
def test_distill(rows, n, k, T, tail):
    s, index, l = inputs(rows, n, k, 1, T=T)
    g = torch.Generator(device="cuda").manual_seed(2)
    check(s, index, l, T, tail, torch.rand(rows, device="cuda", generator=g), rows=some(rows))


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,k", [(1250, 341, 20), (9, 5461, 50), (3, 87381, 100)])
def test_types(dtype, out, rows, n, k):
    s, index, l = inputs(rows, n, k, 3, dtype)
    for kind in TYPES:
        check(s, index, l.to(kind), 1.0, True, 0.5, out, some(rows))
    check(s, index, 3 * l, 1.0, False, 0.5, out, some(rows))   # scores that are not normalised


@pytest.mark.parametrize("n", [40, 3000, 100001])
def test_the_same_entry_twice(n):
    """Each of its values counts, once in p_r, wherever the others stand."""
    s, index, l = inputs(6, n, 12, 4)
    index[:, 3] = index[:, 0]
    index[0, 11] = index[0, 0]
    index[1, 5:] = n - 1
    index[2] = 0
    l[2] = -3.0
    for tail in (True, False):
        check(s, index, l - 0.5, 1.0, tail)
        many = s.repeat(250, 1)
        check(many, index.repeat(250, 1), (l - 0.5).repeat(250, 1), 1.0, tail, rows=[0, 1, 2, 5, 1498, 1499])


@pytest.mark.parametrize("rows,n", [(16, 3000), (16, 100001), (1300, 300)])
@pytest.mark.parametrize("tail", [True, False])
def test_masked_rows_and_strange_values(rows, n, tail):
    s, index, l = inputs(rows, n, 6, 5)
    s[0] = float("-inf")                              # nothing left, a teacher that wants something
    s[1], index[1] = float("nan"), -1                 # nothing left and nothing wanted
    index[2] = -1                                     # nothing wanted
    s[3, int(index[3, 0])] = float("-inf")            # a wanted answer is masked
    l[4, 1] = float("-inf")                           # listed, without mass
    l[5, 2] = float("nan")
    index[6, 5] = n
    index[7, 0] = 2 ** 31 - 1
    s[8, 5] = s[8, 9] = float("inf")                  # only these two
    index[8, 0], index[8, 1:] = 5, -1
    s[9, int(index[9, 0])] = float("inf")
    s[10] = -3.4028234e38                             # a mask of the type's lowest value everywhere
    s[11, 1:] = -3.4028234e38
    s[11, 0] = 10.0
    l[12] = 0.0                                       # more than 1 in all
    s[13], s[13, :6] = float("-inf"), 1.0             # no entry that is not listed
    index[13] = torch.arange(6, dtype=torch.int32)
    index[14, 1:], l[14, 0] = -1, -30.0               # nearly all is left over
    s[15] = s[15] + 300.0
    check(s, index, l, 1.0, tail, rows=range(16))
    check(s.half(), index, l, 0.5, tail, rows=range(16))
    r = emr.distill_grad(s, index, l, 1.0, tail=tail)
    assert r[1][0] == np.inf and r[1][1] == 0 and r[1][2] == 0 and torch.isnan(r[1][5:8]).all() and torch.isnan(r[0][5:8]).all()
    assert not r[0][:3].any()


def test_far_rest():
    """The rest's softmax where its whole probability underflows: half of the teacher's mass pulls at it."""
    s = torch.full((1, 5000), -200.0, device="cuda")
    s[0, :3000] = torch.linspace(-201, -199, 3000, device="cuda")
    s[0, 4000] = 0.0
    index, l = torch.tensor([[4000]], dtype=torch.int32, device="cuda"), torch.tensor([[np.log(0.5)]], device="cuda", dtype=torch.float32)
    check(s, index, l)
    ds, loss = emr.distill_grad(s, index, l, 1.0)
    assert abs(float(ds[0, :4000].sum()) + 0.5 * 0.81) < 0.1 and 90 < float(loss) < 110


def test_parameters_for_each_row_and_strides():
    rows, n = 64, 2500
    s, index, l = inputs(rows, 2 * n, 20, 6)
    index = torch.where(index < n, index, -1)
    g = np.random.default_rng(7)
    f = lambda v: torch.from_numpy(g.choice(v, rows).astype(np.float32)).cuda()
    T, w = f([0.5, 1.0, 2.0, 0.0, -1.0]), f([0.0, 1.0, -2.0])
    bad = torch.isnan(emr.distill(s[:, :n], index, l, T))
    assert torch.equal(bad, T <= 0)
    T = T.abs().clamp_min(0.3)
    for v in (s[:, 3:n + 3], s[:, ::2], s[:1, :n].expand(rows, n)):
        check(v, index, l, T, True, w)
        check(v, index[:, ::2], l[:, ::2], T, False, w)
    ds, loss = emr.distill_grad(s[0], index[:1], l[:1], 1.0)
    assert ds.shape == (2 * n,) and loss.shape == (1,)


def test_a_student_like_its_teacher_has_no_loss():
    """KL of a distribution to itself: 0 within the tolerance above, gradient as well."""
    s, _, _ = inputs(50, 5460, 1, 8)
    best = emr.log_probs(s, temperature=0.8, top=100)
    ds, loss = emr.distill_grad(s, best.top_index, best.top_logp, 1.0, 0.8)
    assert float(loss.abs().max()) < 4e-5 and float(ds.abs().max()) < 4e-5


def test_refusals():
    s, index, l = inputs(4, 10, 3, 9)
    f = torch.ones(4, device="cuda")
    for call in (lambda: emr.distill(s.double(), index, l), lambda: emr.distill(s.cpu(), index, l), lambda: emr.distill(s, index.long(), l),
                 lambda: emr.distill(s, index[:3], l[:3]), lambda: emr.distill(s, index, l[:, :2]), lambda: emr.distill(s, index, l.double()),
                 lambda: emr.distill(s, index, l.cpu()), lambda: emr.distill(s, index, l, 0.0), lambda: emr.distill(s, index, l, f[:3]),
                 lambda: emr.distill(s, index[:, :0], l[:, :0]), lambda: emr.distill(s, index.repeat(1, 100), l.repeat(1, 100)),
                 lambda: emr.distill_grad(s, index, l, None), lambda: emr.distill_grad(s, index, l, f.half()),
                 lambda: emr.distill_grad(s, index, l, 1.0, out_dtype=torch.float64), lambda: emr.distill(s[:, :0], index, l)):
        with pytest.raises(ValueError):
            call()
    assert emr.distill_grad(s[:0], index[:0], l[:0], 1.0)[0].shape == (0, 10)
