"""Log probabilities, distillation and 4-bit products whose offsets pass 32 bits, and many rows with strange values (teams of 64
threads). Tolerances as in the calls' own tests."""
import numpy as np
import pytest
import torch

from oracle import q4 as OQ
from oracle import scores as OS
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def num(t):
    return t.double().cpu().numpy()


def check_rows(s, rows, out, ds):
    for r in rows:
        lp = OS.log_p(num(s[r]))
        t = int(out["target"][r])
        assert abs(float(out["logp"][r]) - lp[t]) <= 6e-6 + 2.4e-7 * abs(lp[t])
        assert np.array_equal(num(out["top"][r]), OS.best(num(s[r]), out["top"].shape[1]))
        g = OS.log_p_gradient(num(s[r]), t, 1.0, 0.0)
        assert np.all(np.abs(num(ds[r]) - g) <= 2e-5 * (np.exp(lp) + (np.arange(len(lp)) == t)) + HALF * np.abs(g) + 2.0 ** -126)


def test_scores():
    """More than 2^31 entries, and rows 2^30 entries apart."""
    rows, n = 24700, 87381
    s = torch.zeros(rows, n, device="cuda", dtype=torch.bfloat16)
    chosen = [0, 1, 12290, 24576, rows - 1]
    for r in chosen:
        s[r] = torch.randn(n, device="cuda").bfloat16() * 2
    target = torch.full((rows,), n - 1, dtype=torch.int32, device="cuda")
    a = emr.log_probs(s, target, top=4)
    ds, logp, _ = emr.log_probs_grad(s, target, 1.0)
    assert torch.equal(a.logp, logp)
    check_rows(s, chosen, {"target": target, "logp": logp, "top": a.top_index}, ds)
    assert abs(float(logp[7]) + np.log(n)) < 1e-4 and torch.equal(a.top_index[7].cpu(), torch.arange(4, dtype=torch.int32))
    del ds
    dd, loss = emr.distill_grad(s, a.top_index, a.top_logp, 1.0)
    for r in (chosen[1], rows - 1):
        want, g, size = OS.distill(num(s[r]), num(a.top_index[r]).astype(int), num(a.top_logp[r]))
        assert abs(float(loss[r]) - want) <= 4e-5 * (1 + size)
        assert np.all(np.abs(num(dd[r]) - g) <= 2e-5 * 4 + HALF * np.abs(g))
    del dd
    wide = s.view(-1).as_strided((3, 5000), (1 << 30, 1))
    for r in range(3):
        wide[r] = torch.randn(5000, device="cuda").bfloat16()
    target = torch.tensor([4999, 0, 17], dtype=torch.int32, device="cuda")
    a = emr.log_probs(wide, target, top=4)
    ds, logp, _ = emr.log_probs_grad(wide, target, 1.0)
    check_rows(wide, range(3), {"target": target, "logp": logp, "top": a.top_index}, ds)


@pytest.mark.parametrize("m", [4, 20])
def test_many_networks(m):
    """Codes of more than 2^31 bytes; one network's codes for all, with scales of their own."""
    nets, n, k, group = 280, 4096, 4096, 128
    g = np.random.default_rng(m)
    codes = torch.from_numpy(g.integers(-8, 8, (1, n, k)).astype(np.int8)).cuda()
    scales = torch.rand(nets, n, k // group, device="cuda").bfloat16() + 0.5
    q = emr.q4_pack(codes.expand(nets, n, k), scales, group)
    assert q.data.numel() > 1 << 31
    x = torch.randn(1, m, k, device="cuda").bfloat16()
    y = emr.q4_matmul(x, q, out_dtype=torch.bfloat16)
    for b in (0, 255, 256, nets - 1):
        z, mag = OQ.product(num(x[0]), num(codes[0, :200]), num(scales[b, :200]), group)
        tol = (k / 16 + 2 * k / 32 + 24) * 2.0 ** -23 * mag
        tol = tol + HALF * (np.abs(z) + tol)
        assert np.all(np.abs(num(y[b, :, :200]) - z) <= tol), b
    del y
    last = emr.q4_dequantize(q, torch.bfloat16)[nets - 1, -1]               # element 4.7e9 of its output
    assert torch.equal(last.float(), (codes[0, -1].float() * scales[nets - 1, -1].float().repeat_interleave(group)).bfloat16().float())


def test_many_rows_of_x():
    """Outputs of more than 2^31 entries."""
    m, n, k, group = 530000, 4096, 40, 32
    g = np.random.default_rng(2)
    codes = torch.from_numpy(g.integers(-8, 8, (1, n, k)).astype(np.int8)).cuda()
    scales = torch.rand(1, n, 2, device="cuda").bfloat16() + 0.5
    q = emr.q4_pack(codes, scales, group)
    x = torch.randn(1, m, k, device="cuda").bfloat16()
    y = emr.q4_matmul(x, q, out_dtype=torch.bfloat16)
    at = [0, 127, 128, 300000, 524287, 524288, m - 1]
    z, mag = OQ.product(num(x[0, at]), num(codes[0]), num(scales[0]), group)
    tol = (k / 16 + 2 * k / 32 + 24) * 2.0 ** -23 * mag
    assert np.all(np.abs(num(y[0, at]) - z) <= tol + HALF * (np.abs(z) + tol))


@pytest.mark.parametrize("n,dtype", [(45, torch.float32), (700, torch.bfloat16), (2999, torch.float32), (5461, torch.float16)])
@pytest.mark.parametrize("tail", [True, False])
def test_many_rows_with_strange_values(n, dtype, tail):
    rows, k = 1230, 30
    g = torch.Generator(device="cuda").manual_seed(n)
    s = (2 * torch.randn(rows, n, device="cuda", generator=g)).to(dtype)
    s[torch.rand(rows, n, device="cuda", generator=g) < 0.2] = float("-inf")
    s[0], s[1, 1:], s[2, n // 2], s[3, ::3], s[4] = float("-inf"), float("-inf"), float("inf"), float("nan"), 1.0
    s[5, 3], s[5, n - 1], s[6, 1:] = float("inf"), float("inf"), torch.finfo(dtype).min
    best = emr.log_probs(torch.randn(rows, n, device="cuda", generator=g), top=k)
    index, logp = best.top_index.clone(), best.top_logp.clone()
    index[7, 5:] = -1
    index[8, 1::2] = index[8, 0::2]                                         # each answer twice
    logp[8] -= 2
    index[9], index[10, 0], logp[11, 0] = -1, n, float("nan")
    index[12] = index[12, 0]                                                # one answer k times
    logp[12] = -6.0
    ds, loss = emr.distill_grad(s, index, logp, 1.0, 1.0, tail, torch.float32)
    target = torch.randint(0, n, (rows,), device="cuda", generator=g).int()
    a = emr.log_probs(s, target, top=8)
    dt, lp, h = emr.log_probs_grad(s, target, 1.0, 0.0, out_dtype=torch.float32)
    assert torch.equal(torch.nan_to_num(a.logp, 7.0), torch.nan_to_num(lp, 7.0)) and torch.equal(a.entropy, h)
    for r in list(range(13)) + [700, rows - 1]:
        sn = num(s[r])
        want, grad, size = OS.distill(sn, index[r].cpu().numpy(), num(logp[r]), 1.0, tail)
        got, dg = float(loss[r]), num(ds[r])
        if np.isfinite(want):
            assert abs(got - want) <= 4e-5 * (1 + size), (r, got, want)
        else:
            assert np.isnan(want) and np.isnan(got) or want == got, (r, got, want)
        assert np.array_equal(np.isnan(grad), np.isnan(dg)), r
        if not np.isnan(grad).any():
            assert np.abs(dg - grad).max() <= 2e-5 * 4, r                      # terms of at most 4 in all
        t = int(target[r])
        p = OS.log_p(sn)
        assert float(lp[r]) == p[t] or abs(float(lp[r]) - p[t]) <= 6e-6 + 2.4e-7 * abs(p[t]), r
        assert np.array_equal(num(a.top_index[r]), OS.best(sn, 8)), r
        g1 = OS.log_p_gradient(sn, t, 1.0, 0.0)
        assert np.all(np.abs(num(dt[r]) - g1) <= 2e-5 * (np.exp(p) + (np.arange(n) == t)) + 2.0 ** -126), r


def test_the_longest_row():
    """2^31 - 2^20 entries, all but four of them equal: sums known in closed form."""
    n = 2 ** 31 - 2 ** 20
    s = torch.full((1, n), -1.0, device="cuda", dtype=torch.bfloat16)
    places = [n // 2, n - 1, 2 ** 30 + 7, 0]
    values = np.array([5.0, 5.0, 4.0, 3.0])
    for i, v in zip(places, values):
        s[0, i] = v
    target = torch.tensor([n - 1], dtype=torch.int32, device="cuda")
    z = np.exp(values).sum() + (n - 4) * np.exp(-1.0)
    lp, low = values - np.log(z), -1.0 - np.log(z)
    h = -(np.exp(lp) * lp).sum() - (n - 4) * np.exp(low) * low
    a = emr.log_probs(s, target, top=4)
    assert a.top_index[0].tolist() == places
    tol = 6e-6 + 2.4e-7 * abs(lp)
    assert abs(float(a.logp[0]) - lp[1]) <= tol[1] and np.all(np.abs(num(a.top_logp[0]) - lp) <= tol) and abs(float(a.entropy[0]) - h) < 1e-5 * (1 + h)
    ds, logp, entropy = emr.log_probs_grad(s, target, -1.0)
    assert torch.equal(logp, a.logp) and torch.equal(entropy, a.entropy)
    at = [1, 5, 2 ** 30, n // 2 + 1, n - 2]
    assert np.all(np.abs(num(ds[0, at]) - np.exp(low)) <= (2e-5 + HALF) * np.exp(low))
    want = np.exp(lp) - np.array([0, 1, 0, 0])
    assert np.all(np.abs(num(ds[0, places]) - want) <= 2e-5 * (np.exp(lp) + [0, 1, 0, 0]) + HALF * np.abs(want))
    del ds
    index = torch.tensor([[n - 1, n // 2, 0]], dtype=torch.int32, device="cuda")
    t = np.array([0.4, 0.3, 0.2])
    l = torch.from_numpy(np.log(t)).float().cuda()[None]
    ds, loss = emr.distill_grad(s, index, l, 1.0)
    p, t = np.exp(lp[[1, 0, 3]]), np.exp(num(l[0]))
    t_r, p_r = 1 - t.sum(), 1 - p.sum()
    terms = np.append(t * (np.log(t) - np.log(p)), t_r * (np.log(t_r) - np.log(p_r)))
    assert abs(float(loss[0]) - terms.sum()) <= 4e-5 * (1 + np.abs(terms).sum())
    assert np.all(np.abs(num(ds[0, [n - 1, n // 2, 0]]) - (p - t)) <= 2e-5 * (p + t) + HALF * np.abs(p - t))
    e_z = np.exp(-1.0) / (z - np.exp(values[[0, 1, 3]]).sum())
    want = e_z * (p_r * t.sum() - t_r * p.sum())
    assert np.all(np.abs(num(ds[0, at]) - want) <= (2e-5 * 2 + 110 * 2.0 ** -24 + HALF) * abs(want) + 2e-5 * e_z)


@pytest.mark.parametrize("rows,n,dtype", [(700, 45, torch.bfloat16), (700, 701, torch.float32), (1300, 1365, torch.bfloat16), (640, 5461, torch.float16),
                                          (3700, 340, torch.float32), (3700, 1031, torch.bfloat16)])
@pytest.mark.parametrize("top", [33, 64, 65, 128, 129])
def test_long_lists_of_many_rows(rows, n, dtype, top):
    """The best of rows with masked and equal entries, and with fewer entries than are asked for."""
    g = torch.Generator(device="cuda").manual_seed(top)
    s = torch.randn(rows, n, device="cuda", generator=g).to(dtype)
    s[torch.rand(rows, n, device="cuda", generator=g) < 0.2] = float("-inf")
    s[0], s[1, 20:], s[2], s[3] = float("-inf"), float("-inf"), 0.5, torch.arange(n, device="cuda") / 64
    s[4] = -s[3]
    a = emr.log_probs(s, top=top)
    v = torch.nan_to_num(s.float(), neginf=-1e30)
    order = torch.sort(v, dim=1, descending=True, stable=True)
    k = min(top, n)
    want = torch.where(order.values[:, :k] > -1e29, order.indices[:, :k], -1)
    assert torch.equal(a.top_index[:, :k].long(), want) and bool((a.top_index[:, k:] == -1).all())
    z = torch.log_softmax(s.double(), 1).nan_to_num(nan=float("-inf"))
    lp = torch.where(want >= 0, z.gather(1, want.clamp(min=0)), float("-inf"))
    ok = (a.top_logp[:, :k].double() - lp).abs() <= 6e-6 + 2.4e-7 * lp.abs()
    assert bool((ok | (a.top_logp[:, :k] == lp)).all())
