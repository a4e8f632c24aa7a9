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
