"""Products with 4-bit weights against their definition in float64 (oracle.q4).

Tolerances: the quantised entries are equal bit for bit (the same 32-bit quotients). A product's terms code * x are exact; sums of 16 are
added by the instruction, which may cut off rather than round: 2^-23 of the running sum for each of k / 16 + the scalings and
joins of k / 32 groups, warps, blocks and parts: (k / 16 + 2 k / 32 + 24) 2^-23 of the sum of the terms' magnitudes; act is good to 2e-6 and its
slope at most 1; then the rounding to out's type."""
import numpy as np
import pytest
import torch

from oracle import dense as OD
from oracle import q4 as OQ
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def num(t):
    return t.double().cpu().numpy()


def weights(batch, n, k, group, seed):
    g = np.random.default_rng(seed)
    codes = np.clip(np.round(3 * g.standard_normal((batch, n, k))), -8, 7).astype(np.int8)
    codes[..., 0] = -8
    scales = np.exp(g.standard_normal((batch, n, (k + group - 1) // group))).astype(np.float32)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda().bfloat16()


def x_of(batch, m, k, seed, dtype):
    g = np.random.default_rng(seed)
    return torch.from_numpy((g.standard_normal((batch, m, k)) * np.exp(g.standard_normal((batch, m, 1)))).astype(np.float32)).cuda().to(dtype)


def check(x, codes, scales, group, b=None, act=0, out=torch.float32, q=None):
    q = q or emr.q4_pack(codes, scales, group)
    y = emr.q4_matmul(x, q, b, act, out)
    assert torch.equal(y, emr.q4_matmul(x, q, b, act, out)) and y.dtype == out
    k = codes.shape[-1]
    z, mag = OQ.product(num(x), num(codes), num(scales), group, num(b) if b is not None else None)
    name = OD.ACTS[act]
    with np.errstate(over="ignore"):
        want = OD.act(z, name)
    tol = (k / 16 + 2 * k / 32 + 24) * 2.0 ** -23 * mag + (2e-6 if act else 0)
    tol = tol + HALF[out] * (np.abs(want) + tol) + 2.0 ** -25 * (out == torch.float16)
    ok = np.abs(num(y) - want) <= tol
    assert y.shape == want.shape and ok.all(), (np.argwhere(~ok)[:3], num(y)[~ok][:3], want[~ok][:3])


# rows of x from one to several chunks of 64 (21 of float32); odd sizes; rows and columns of less than a unit; long contractions
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 5460, 1364), (2, 340, 85), (3, 17, 129), (5, 100, 4000), (7, 33, 131), (8, 2000, 1000),
                                   (9, 16, 128), (12, 48, 300), (16, 1000, 512), (17, 31, 700), (31, 250, 260), (33, 129, 1000), (64, 100, 515),
                                   (65, 40, 300), (130, 200, 333)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_product(m, n, k, group, dtype):
    check(x_of(1, m, k, 1, dtype), *weights(1, n, k, group, 2), group)


@pytest.mark.parametrize("m,n,k", [(1, 16, 131072), (3, 40, 70001), (8, 8192, 8192), (70, 20, 40000)])
def test_long_contractions(m, n, k):
    for dtype in TYPES:
        check(x_of(1, m, k, 3, dtype), *weights(1, n, k, 64, 4), 64)


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("act", range(6))
def test_bias_activation_and_types(act, out):
    codes, scales = weights(3, 77, 200, 32, 5)
    scales = (scales.float() * 0.01).bfloat16()
    g = torch.Generator(device="cuda").manual_seed(6)
    b = torch.randn(3, 77, device="cuda", generator=g)
    for dtype in TYPES:
        check(x_of(3, 5, 200, 7, dtype), codes, scales, 32, b, act, out)


def test_batches():
    codes, scales = weights(5, 90, 300, 64, 8)
    b = torch.randn(5, 90, device="cuda")
    check(x_of(1, 4, 300, 9, torch.float32), codes, scales, 64, b)          # x shared by all networks
    check(x_of(5, 20, 300, 10, torch.bfloat16), codes, scales, 64, b)
    one = codes[:1], scales[:1]
    check(x_of(5, 4, 300, 11, torch.float16), *one, 64, b)                  # weights shared
    many = weights(300, 20, 256, 128, 12)
    check(x_of(1, 2, 256, 13, torch.float32), *many, 128)
    assert torch.equal(emr.q4_matmul(x_of(1, 4, 300, 9, torch.float32)[0], emr.q4_pack(codes, scales, 64), b),
                       emr.q4_matmul(x_of(1, 4, 300, 9, torch.float32), emr.q4_pack(codes, scales, 64), b))


def test_strides_and_alignments():
    codes, scales = weights(2, 50, 260, 32, 14)
    wide = x_of(2, 9, 600, 15, torch.float32)
    for dtype in TYPES:
        v = wide.to(dtype)
        for x in (v[:, :, 1:261], v[:, :, 3:263], v[:, :, 4:264], v[:, :, :520:2], v[:, ::3, :260], v[:, 2:3, :260].expand(2, 6, 260),
                  v[:, :, :260].transpose(1, 2).contiguous().transpose(1, 2)):
            check(x, codes, scales, 32)
    padded = torch.zeros(2, 50, 300, dtype=torch.int8, device="cuda")
    padded[:, :, 7:267] = codes
    spread = scales.repeat_interleave(2, -1)
    q = emr.q4_pack(padded[:, :, 7:267], spread[..., ::2], 32)
    assert torch.equal(q.data, emr.q4_pack(codes, scales, 32).data)
    check(x_of(2, 3, 260, 16, torch.float32), codes, scales, 32, q=emr.Q4.of(q.data.clone(), 2, 50, 260, 32))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,n,k,group", [(1, 1, 1, 32), (2, 17, 129, 64), (1, 40, 1000, 128), (3, 33, 96, 32)])
def test_quantize(batch, n, k, group, dtype):
    g = np.random.default_rng(17)
    w = (g.standard_normal((batch, n, k)) * np.exp(3 * g.standard_normal((batch, n, 1)))).astype(np.float32)
    w[0, 0, : k // 2] = 0
    w = torch.from_numpy(w).cuda().to(dtype)
    q = emr.q4_quantize(w, group)
    codes, scales = OQ.quantized(num(w), group)
    assert np.array_equal(num(emr.q4_dequantize(q)), OQ.values(codes, scales, group))
    packed = emr.q4_pack(torch.from_numpy(codes.astype(np.int8)).cuda(), torch.from_numpy(scales).cuda().bfloat16(), group)
    assert torch.equal(q.data, packed.data)
    back = torch.from_numpy(OQ.values(codes, scales, group)).float().to(dtype)
    assert torch.equal(emr.q4_dequantize(q, dtype).cpu(), back)
    t = w.transpose(1, 2).contiguous().transpose(1, 2)                     # strides
    assert torch.equal(emr.q4_quantize(t, group).data, q.data)
    assert torch.equal(emr.q4_quantize(w[0], group).data, emr.q4_quantize(w[:1], group).data)


def test_quantized_extremes():
    w = torch.zeros(4, 128, device="cuda")
    w[0, 3], w[0, 40] = float("inf"), 1.0
    w[1, 5] = float("nan")
    w[2] = 1e-39
    w[2, 64] = 3.4e38
    w[3, :32] = 2.0 ** -126 * 6
    v = num(emr.q4_dequantize(emr.q4_quantize(w)))[0]
    assert np.isnan(v[0, :32]).all() and v[0, 40] == 7 * OQ.bf16(np.float32(1) / np.float32(7)) and np.isnan(v[1, :32]).all() and not v[1, 32:].any()
    assert not v[2, :64].any() and abs(v[2, 64] / 3.4e38 - 1) < 2.0 ** -8 and not v[3].any()
    y = emr.q4_matmul(torch.ones(1, 128, device="cuda"), emr.q4_quantize(w))
    assert torch.isnan(y[0, 0, :2]).all() and not torch.isnan(y[0, 0, 2:]).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan_stay_in_their_rows(dtype):
    codes, scales = weights(1, 60, 300, 32, 18)
    codes[codes == 0] = 1                                                  # 0 times infinity would be NaN
    x = x_of(1, 6, 300, 19, dtype)
    x[0, 1, 7], x[0, 2, 299], x[0, 4, 0], x[0, 4, 5] = float("inf"), float("nan"), float("inf"), float("nan")
    clean = x.clone()
    clean[0, 1, 7] = clean[0, 2, 299] = clean[0, 4, 0] = clean[0, 4, 5] = 0
    q = emr.q4_pack(codes, scales)
    y, z = emr.q4_matmul(x, q)[0], emr.q4_matmul(clean, q)[0]
    assert torch.equal(y[[0, 3, 5]], z[[0, 3, 5]]) and torch.isnan(y[[2, 4]]).all()
    assert torch.equal(y[1], torch.sign(codes[0, :, 7].float()) * float("inf"))


def test_all_bits_of_float32_count():
    """A value whose last bit alone is wanted: large terms cancel exactly, in groups of their own."""
    x = torch.zeros(1, 64, device="cuda")
    x[0, 0], x[0, 32] = 1 + 2.0 ** -23, 1.0
    codes = torch.zeros(1, 64, dtype=torch.int8, device="cuda")
    codes[0, 0], codes[0, 32] = 1, -1
    y = emr.q4_matmul(x, emr.q4_pack(codes, torch.ones(1, 2, device="cuda", dtype=torch.bfloat16)))
    assert float(y) == 2.0 ** -23
    x[0, 0], x[0, 32] = 3.4028234e38, 0.0
    assert float(emr.q4_matmul(x, emr.q4_pack(codes, torch.ones(1, 2, device="cuda", dtype=torch.bfloat16)))) == float(x[0, 0])


def test_refusals():
    x, (codes, scales) = x_of(2, 3, 100, 20, torch.float32), weights(2, 10, 100, 32, 21)
    q, b = emr.q4_pack(codes, scales), torch.zeros(2, 10, device="cuda")
    for call in (lambda: emr.q4_matmul(x[:, :, :99], q), lambda: emr.q4_matmul(x.double(), q), lambda: emr.q4_matmul(x.cpu(), q),
                 lambda: emr.q4_matmul(x.repeat(2, 1, 1)[:3], q), lambda: emr.q4_matmul(x, q, b[:1]), lambda: emr.q4_matmul(x, q, b.half()),
                 lambda: emr.q4_matmul(x, q, act=6), lambda: emr.q4_matmul(x, q, out_dtype=torch.float64), lambda: emr.q4_matmul(x[0, 0], q),
                 lambda: emr.q4_matmul(x, q, out=torch.empty(2, 3, 11, device="cuda")), lambda: emr.q4_pack(codes, scales, 48),
                 lambda: emr.q4_pack(codes, scales.float()), lambda: emr.q4_pack(codes.int(), scales), lambda: emr.q4_pack(codes, scales, 64),
                 lambda: emr.q4_quantize(x.double()), lambda: emr.q4_quantize(x, 16), lambda: emr.q4_dequantize(q, torch.int8),
                 lambda: emr.Q4.of(q.data[:-1], 2, 10, 100)):
        with pytest.raises(ValueError):
            call()
    assert emr.q4_matmul(x[:, :0], q).shape == (2, 0, 10)
    out = torch.full((2, 3, 10), 7.0, device="cuda")
    assert emr.q4_matmul(x, q, out=out) is out and torch.equal(out, emr.q4_matmul(x, q))


@pytest.mark.parametrize("m,k", [(17, 600), (33, 500), (129, 700), (70, 8200)])
def test_many_rows_of_batches(m, k):
    """The kernel of many rows with biases, activations, operands that all share, strides, and rows of W that fill no tile."""
    codes, scales = weights(3, 77, k, 32, 18)
    scales = (scales.float() * 0.01).bfloat16()
    b = torch.randn(3, 77, device="cuda")
    for act, dtype in enumerate(TYPES + TYPES):
        out = TYPES[(act + 1) % 3]
        check(x_of(3, m, k, 19, dtype), codes, scales, 32, b, act, out)
        check(x_of(1, m, k, 20, dtype), codes, scales, 32, b, act, out)
        check(x_of(3, m, k, 21, dtype), codes[:1], scales[:1], 32, b, act, out)
    wide = x_of(2, m, 2 * k + 5, 22, torch.float32)
    codes, scales = weights(2, 260, k, 128, 23)
    for dtype in TYPES:
        v = wide.to(dtype)
        for x in (v[:, :, 1:1 + k], v[:, :, :2 * k:2], v[:, :, 8:8 + k], v[:, :1, :k].expand(2, m, k)):
            check(x, codes, scales, 128)
