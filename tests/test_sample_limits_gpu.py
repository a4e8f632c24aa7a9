"""Sampling where blocks of a row start apart, on rows longer than the sums of one step's 32 bits, and at the
edges of its filters, against the definition in float64 (oracle.sampling) or values worked out by hand."""
import numpy as np
import pytest
import torch

from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(), dict(top_k=40), dict(top_k=3000, top_p=0.9), dict(top_p=0.8, min_p=0.01)])
def test_rows_of_several_blocks_beside_other_work(kw):
    """Clusters of 2 to 8 blocks while another stream's kernels come and go on the same SMs, so that a row's
    blocks start apart: the same answers as alone."""
    g = torch.Generator(device="cuda").manual_seed(1)
    busy, side = torch.randn(2048, 2048, device="cuda", generator=g), torch.cuda.Stream()
    for rows, n in ((60, 4101), (30, 8300), (18, 16390), (5, 70001)):
        s = 2 * torch.randn(rows, n, device="cuda", generator=g)
        e = torch.empty(rows, n, device="cuda").exponential_(generator=g).clamp_min_(1e-30)
        want = emr.sample(s, e, **kw)
        side.wait_stream(torch.cuda.current_stream())
        got = []
        for _ in range(60):
            with torch.cuda.stream(side):
                busy @ busy
            got.append(emr.sample(s, e, **kw))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x in got for a, b in zip(x, want))


@pytest.mark.parametrize("rows,n,dtype", [(200, 700001, torch.bfloat16), (160, 1398100, torch.float16), (1, 9000000, torch.float32),
                                          (3, 12000001, torch.bfloat16)])
def test_top_p_of_long_rows_of_nearly_equal_scores(rows, n, dtype):
    """All scores but the first lie a little under 16 / 2047 or 16 / 4095 below it, the most that one step of the
    histogram spans: more of them in one step of one block than 32 bits hold the sum of. The prefix is the first
    entries by index; its end may be off by 1e-5 of the row (w is good to 4e-6 and a step's sum to 2^-20)."""
    for gap in (16 / 2047, 16 / 4095, 0.001):
        s = torch.zeros(1, n, dtype=dtype, device="cuda")
        s[0, 1:] = -0.98 * gap
        w = float(torch.exp(s[0, 1].double()))
        e = torch.ones(1, n, device="cuda")
        for p in (0.5, 0.9):
            kept = 1 + int(np.ceil((float(np.float32(p)) * (1 + (n - 1) * w) - 1) / w))
            for entry, stays in ((kept - 1 - n // 100000 - 1, True), (kept + n // 100000 + 1, False)):
                e[0, entry] = 1e-30
                index, _ = emr.sample(s.expand(rows, n), e.expand(rows, n), top_p=p)
                assert bool(((index == entry) == stays).all()), (gap, p, entry, kept, index)
                e[0, entry] = 1.0


def test_top_p_of_long_rows_of_many_scores():
    """A row of 9 million scores in the first few steps of the histogram, against a float64 sum in order."""
    n = 9000000
    g = torch.Generator(device="cuda").manual_seed(2)
    s = -0.012 * torch.rand(1, n, device="cuda", generator=g)
    order = torch.argsort(s[0], descending=True, stable=True)
    w = torch.exp(s[0, order].double() - s[0, order[0]].double())
    before = torch.cumsum(w, 0) - w
    for p in (0.3, 0.7):
        kept = int((before < float(np.float32(p)) * w.sum()).sum())
        for place, stays in ((kept - 91, True), (kept + 91, False)):     # 1e-5 of the row
            e = torch.ones(1, n, device="cuda")
            e[0, order[place]] = 1e-30
            index, _ = emr.sample(s, e, top_p=p)
            assert (int(index) == int(order[place])) == stays, (p, place, kept)


@pytest.mark.parametrize("n", [8, 9000])
@pytest.mark.parametrize("kw", [dict(), dict(top_k=7), dict(top_p=0.9999)])
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_what_min_p_keeps_is_what_the_probability_counts(kw, n, T):
    """One entry of w = 1 and three equal ones whose w min-p names to within two units in the last place: they stay
    or not, and if one is drawn, all that top-p leaves of the three are in the sum that its probability is taken of
    (log w good to 4e-6 and the end of top-p to 1e-5, as in test_sample_gpu.py)."""
    rows = 400
    g = np.random.default_rng(3)
    low = -g.uniform(0, 7, rows).astype(np.float32)
    s = torch.full((rows, n), -np.inf, device="cuda")
    s[:, 1] = 0.0
    s[:, [0, 3, n - 1]] = torch.from_numpy(low).cuda()[:, None]
    w = np.exp(low.astype(np.float64) / float(np.float32(T)))
    e = torch.ones(rows, n, device="cuda")
    e[:, 3] = 1e-20                                   # drawn whenever it stays
    for ulps in (-2, -1, 0, 1, 2):
        q = (w.astype(np.float32).view(np.int32) + ulps).view(np.float32)
        index, logp = emr.sample(s, e, T, min_p=torch.from_numpy(q).cuda(), **kw)
        index, logp = index.cpu().numpy(), logp.double().cpu().numpy()
        assert np.isin(index, (1, 3)).all()
        fits = np.zeros(rows, bool)
        for p in (kw.get("top_p", 2.0) * (1 + x) for x in (-1e-5, 0.0, 1e-5)):
            left = sum(1 + j * w < p * (1 + 3 * w) for j in range(3))        # of the three
            near = lambda want: np.abs(logp - want) <= 4e-6 + 2.0 ** -23 * np.abs(want)
            fits |= (index == 3) & (left >= 2) & near(np.log(w / (1 + left * w)))
            fits |= (index == 1) & (near(0.0 * w) | (left <= 1) & near(-np.log(1 + left * w)))
        assert fits.all(), (ulps, np.flatnonzero(~fits), index[~fits], logp[~fits])


@pytest.mark.parametrize("kw", [dict(), dict(min_p=0.3), dict(top_k=-3), dict(top_p=0.75)])
@pytest.mark.parametrize("score", [-0.0078125, -0.26, -1.0])
def test_probabilities_of_long_rows_of_equal_scores(score, kw):
    """A block adds up 1.4 million equal w: the probability is as good as a short row's (the bounds of
    test_sample_gpu.py; the end of top-p may be off by 1e-5 of the row, and its logarithm as much)."""
    rows, n = 160, 1398100
    s = torch.full((1, n), score, dtype=torch.bfloat16, device="cuda")
    s[0, 0] = 0.0
    w = float(torch.exp(s[0, 1].double()))
    e = torch.ones(1, n, device="cuda")
    e[0, 1000] = 1e-30
    kw = dict(kw, top_k=n - 3) if "top_k" in kw else kw
    index, logp = emr.sample(s.expand(rows, n), e.expand(rows, n), **kw)
    total = 1 + (n - 1) * w
    if "top_k" in kw:
        total -= 3 * w
    if "top_p" in kw:
        total = 1 + w * np.ceil((0.75 * total - 1) / w)
    want = np.log(w / total)
    assert bool((index == 1000).all())
    off = np.abs(logp.double().cpu().numpy() - want).max()
    assert off <= 4e-6 + 2.0 ** -23 * abs(want) + (1e-5 / 0.75 if "top_p" in kw else 0.0), off
