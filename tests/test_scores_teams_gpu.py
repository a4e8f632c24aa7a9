"""Rows that are short and many belong to teams of 8 threads, four of which share a warp, or to single warps: log probabilities,
their gradient and distillation of such rows against their definitions in float64 (oracle.scores), with rows that take another
way through the kernel (infinities, nothing left, temperatures of 0 and below, answers past the row) beside ordinary ones of
the same warp. The numbers of rows follow the GPU's SMs as the kernels' choice of teams does, and fill no block.

Tolerances are those of the calls' own tests, from which the comparisons are taken."""
import numpy as np
import pytest
import torch
from test_distill_gpu import check as check_distill
from test_distill_gpu import inputs as lists
from test_log_probs_gpu import TYPES, check, check_gradient, inputs

from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu

HEATS = [0.5, 0.0, 1.0, 2.0, -1.0, 1.3, float("nan"), 0.7, float("inf")]


def many(rows_an_sm):
    return rows_an_sm * torch.cuda.get_device_properties(0).multi_processor_count


# teams of 8 (32 rows an SM, rows of up to 512), a warp for a row (16 rows an SM, up to 1024)
EIGHT = [(3, 5), (5, 45), (1, 340), (30, 512)]
WARP = [(3, 9), (6, 513), (1, 700), (7, 1024)]


def strange(rows, n, seed, dtype):
    """Scores and answers; of the first 64 rows every fourth is a strange one, at each place of four in turn, and so are the last two."""
    s, t = inputs(rows, n, seed, dtype)
    low = float(torch.finfo(dtype).min)
    for i in range(18):
        r = 4 * i + i % 4 if i < 16 else rows - 18 + i
        kind = i % 8
        if kind == 0:                                 # only two entries of +infinity count
            s[r, n // 2] = s[r, -1] = float("inf")
            t[r] = n // 2
        elif kind == 1:                               # nothing left
            s[r] = float("-inf")
        elif kind == 2:
            s[r] = float("nan")
        elif kind == 3:                               # one entry left
            s[r], s[r, -1], t[r] = float("-inf"), 3.0, n - 1
        elif kind == 4:                               # a masked answer beside one of +infinity
            s[r, 0], s[r, -1], t[r] = float("inf"), float("nan"), n - 1
        elif kind == 5:                               # a mask of the type's lowest value everywhere
            s[r] = low
        elif kind == 6:
            t[r] = n if i < 8 else 2 ** 31 - 1
        else:
            t[r] = -1
    return s, t


def looked_at(rows):
    return list(range(72)) + list(range(72, rows, 211)) + list(range(rows - 6, rows))


def heats(rows, seed):
    return torch.from_numpy(np.random.default_rng(seed).choice(HEATS, rows).astype(np.float32)).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("an_sm,more,n", [(32, *c) for c in EIGHT] + [(16, *c) for c in WARP])
def test_rows_that_part(an_sm, more, n, dtype):
    """A temperature for each row, some of them 0 and below, and one for all."""
    rows = many(an_sm) + more
    s, t = strange(rows, n, 21, dtype)
    g = torch.Generator(device="cuda").manual_seed(22)
    a, b = (torch.randn(rows, device="cuda", generator=g) for _ in range(2))
    for T in (heats(rows, 23), 0.8, 0.0):
        check(s, t, T, rows=looked_at(rows))
        check_gradient(s, t, a, b, T, rows=looked_at(rows))
    check_gradient(s, t, 1.0, None, 0.8, torch.float32, looked_at(rows))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("more,n", WARP)
def test_a_warps_best_answers(more, n, dtype):
    rows = many(16) + more
    s, t = strange(rows, n, 24, dtype)
    for T, top in ((heats(rows, 25), 5), (0.8, 32), (0.0, 3)):
        check(s, t, T, top, looked_at(rows))


def test_strided_rows_and_a_row_of_one_entry():
    rows = many(32) + 1
    s, t = strange(rows, 80, 26, torch.bfloat16)
    T = heats(rows, 27)
    for v in (s[:, 3:60], s[:, ::2], s[:1].expand(rows, 80)):
        check(v, t % 30, T, rows=looked_at(rows))
        check_gradient(v, t % 30, 0.5, -0.25, T, rows=looked_at(rows))
    one = s[:, :1].contiguous()
    check(one, t % 2, T, rows=looked_at(rows))
    check_gradient(one, t % 2, 1.0, 0.5, T, rows=looked_at(rows))


def strange_lists(rows, n, k, seed, dtype):
    """Students and lists; of the first 64 rows every fourth is a strange one, and so are the last two."""
    s, index, l = lists(rows, n, k, seed, dtype)
    for i in range(18):
        r = 4 * i + i % 4 if i < 16 else rows - 18 + i
        kind = i % 8
        if kind == 0:                                 # only two entries of +infinity count, one of them listed
            s[r, n // 2] = s[r, -1] = float("inf")
            index[r, 0], index[r, 1:] = n // 2, -1
        elif kind == 1:                               # nothing left
            s[r] = float("-inf")
        elif kind == 2:                               # an infinity among the rest
            s[r, (int(index[r].max()) + 1) % n] = float("inf")
        elif kind == 3:                               # a list of one entry, several times
            index[r], l[r] = n - 1, -3.0
        elif kind == 4:
            l[r, k // 2] = float("nan")
        elif kind == 5:
            index[r, 0] = n
        elif kind == 6:                               # nothing wanted
            index[r] = -1
        else:                                         # no entry that is not listed
            s[r], s[r, :k] = float("-inf"), 0.5
            index[r] = torch.arange(k, dtype=torch.int32)
    return s, index, l


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("more,n,k", [(3, 40, 6), (6, 513, 64), (1, 700, 33), (7, 1024, 64), (2, 1024, 1)])
def test_a_warps_distillation(more, n, k, dtype):
    rows = many(16) + more
    s, index, l = strange_lists(rows, n, k, 28, dtype)
    g = torch.Generator(device="cuda").manual_seed(29)
    w = torch.rand(rows, device="cuda", generator=g)
    T = torch.from_numpy(np.random.default_rng(30).choice([0.5, 1.0, 2.0], rows).astype(np.float32)).cuda()
    for tail in (True, False):
        check_distill(s, index, l, 1.0, tail, w, rows=looked_at(rows))
        check_distill(s, index, l.bfloat16(), 0.7, tail, 0.5, torch.float32, looked_at(rows))
    check_distill(s, index, l, T, False, w, rows=looked_at(rows))
    T[5], T[6] = 0.0, -1.0                            # no distribution
    loss = emr.distill(s, index, l, T)
    assert bool(torch.isnan(loss[5:7]).all())
