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
