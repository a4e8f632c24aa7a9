"""What a teacher's list leaves over, 1 - sum t, where it is small: the gradient of entries that are not listed against its definition in
float64 (oracle.scores), with a student that is close to its teacher, whose gradient is a small difference.

Tolerance, in units u = 2^-24. Of an entry that is not listed the gradient is e_i / z_r (p_r sum t - t_r p_l): e_i / z_r, p_r and p_l are
good to 120 u relative (as log p's sums), sum t to 2 u, and t_r to 2 u relative and 2.2e-11 absolutely (the header of the kernel's e^l): 2e-5 of e_i / z_r
(p_r sum t + t_r p_l), and 2.5e-11 e_i / z_r, rounded to the gradient's type. Sums of t that are off by u give 6e-8 e_i / z_r and more."""
import numpy as np
import pytest
import torch

from oracle import scores as OS
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu

LEFT = [1e-2, 1e-4, 1e-5, 1e-6, 1e-7, 3e-8, 0.0]


def scene(rows, n, k, seed, near):
    """Lists that leave over about LEFT of the mass, and students with about as much (near: the same, else some multiples of it)."""
    g = np.random.default_rng(seed)
    index = np.stack([g.permutation(n)[:k] for _ in range(min(rows, 64))])
    index = index[np.arange(rows) % len(index)]
    left = np.array(LEFT)[np.arange(rows) % len(LEFT)][:, None]
    v = 2.5 * g.standard_normal((rows, k))
    t = np.exp(v - v.max(1, keepdims=True))
    l = np.log(t / t.sum(1, keepdims=True) * (1 - left)).astype(np.float32)
    s = np.log(np.maximum(left, 1e-8) / (n - k)) + 0.5 * g.standard_normal((rows, n)) + (0 if near else g.uniform(-3, 3, (rows, 1)))
    s[np.arange(rows)[:, None], index] = l + (0 if near else 0.3) * g.standard_normal((rows, k))
    return torch.from_numpy(s.astype(np.float32)).cuda(), torch.from_numpy(index.astype(np.int32)).cuda(), torch.from_numpy(l).cuda()


def compare(s, index, l, rows):
    ds, loss = emr.distill_grad(s, index, l, 1.0)
    sn, xn, ln, dn = s.double().cpu().numpy(), index.cpu().numpy(), l.double().cpu().numpy(), ds.double().cpu().numpy()
    for r in rows:
        want, g, size = OS.distill(sn[r], xn[r], ln[r])
        assert abs(float(loss[r]) - want) <= 4e-5 * (1 + size), r              # as in the loss's own tests
        p, t_sum = np.exp(OS.log_p(sn[r])), np.exp(ln[r]).sum()
        rest = np.ones(len(p), bool)
        rest[xn[r]] = False
        p_rest = p[rest].sum()
        share, over = p[rest] / p_rest, max(0.0, 1 - t_sum)
        tol = share * (2e-5 * (p_rest * t_sum + over * (1 - p_rest)) + 2.5e-11) + 2.0 ** -24 * np.abs(g[rest]) + 2.0 ** -126
        off = np.abs(dn[r][rest] - g[rest])
        assert (off <= tol).all(), (r, 1 - t_sum, p_rest, off.max(), tol[np.argmax(off - tol)])


# a block's rows, teams of 64, 32 and 128 threads (8, 16 and 4 rows an SM), a cluster's
@pytest.mark.parametrize("an_sm,more,n,k", [(0, 21, 340, 85), (0, 21, 1364, 256), (8, 3, 2047, 128), (16, 3, 340, 64), (16, 1, 90, 5), (4, 1, 5460, 200), (0, 14, 20001, 128),
                                            (0, 7, 140003, 256)])
@pytest.mark.parametrize("near", [True, False])
def test_small_remainders(an_sm, more, n, k, near):
    rows = an_sm * torch.cuda.get_device_properties(0).multi_processor_count + more
    compare(*scene(rows, n, k, 31, near), list(range(min(rows, 35))) + [rows - 1])


def test_one_answer_that_is_nearly_all():
    l = torch.tensor([[-1e-3], [-1e-5], [-1e-6], [-1e-7], [-3e-8], [-1e-12], [0.0], [1e-7], [1.0]], device="cuda")
    s = torch.full((len(l), 700), -20.0, device="cuda")
    s[:, 5] = 0.0
    compare(s, torch.full((len(l), 1), 5, dtype=torch.int32, device="cuda"), l, range(len(l)))


def test_lists_of_16_bits():
    """The definition is of the values that are given: bfloat16 ones add up to less or more than 1."""
    s, index, l = scene(35, 1364, 50, 32, False)
    for dtype in (torch.bfloat16, torch.float16):
        a, b = emr.distill_grad(s, index, l.to(dtype), 1.0), emr.distill_grad(s, index, l.to(dtype).float(), 1.0)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        compare(s, index, l.to(dtype).float(), range(35))
