"""Dense substrate layers in 8-bit floating point against their definitions in float64 (oracle.dense).

Tolerances. The 8-bit values themselves are exact: scales are powers of two and codes are rounded to nearest
even on both sides. A product sums K exact terms in 32 bits in an order of its own, so it differs by at most
(K + 2) 2^-23 times the sum of the terms' magnitudes (2^-23 a step allows for truncation). Activations have
slopes of at most 1 and are computed to 2e-6; second derivatives are at most 2. Rounding to nearest with p
significant bits is off by at most 2^-p relative: 2^-8 for bfloat16, 2^-11 for float16 (there at least 2^-25)."""
import numpy as np
import pytest
import torch

from oracle import dense as OD
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
ULP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
ACT = dict(zip(OD.ACTS, range(6)))


def normal(seed, *shape, dtype=torch.float32, spread=1.0):
    g = np.random.default_rng(seed)
    v = g.standard_normal(shape) * np.exp(spread * g.standard_normal(shape[:-1] + (1,)))
    return torch.from_numpy(v.astype(np.float32)).cuda().to(dtype)


def f64(t):
    return t.double().cpu().numpy()


def back(q):
    return f64(emr.q8_dequantize(q))


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


@pytest.fixture(autouse=True)
def no_wait_gives_up():
    yield
    assert emr.device_error() == 0


# ---- the format -------------------------------------------------------------------------------------

@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 1, 127), (1, 3, 128), (2, 129, 129), (3, 40, 513), (1, 300, 1364)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_both_ways(shape, dtype):
    x = normal(1, *shape, dtype=dtype)
    q, qt = emr.Q8(*shape), emr.Q8(shape[0], shape[2], shape[1])
    emr.q8_quantize(x, q, qt)
    assert same(back(q), OD.held(f64(x)))
    assert same(back(qt), OD.held(np.swapaxes(f64(x), 1, 2)))
    q1, _ = emr.q8_quantize(x)                       # one way at a time gives the same
    assert same(back(q1), back(q))
    t1 = emr.Q8(*qt.shape)
    emr.q8_quantize(x, None, t1)
    assert same(back(t1), back(qt))
    assert torch.equal(q.values.view(shape[0], shape[1], -1)[:, :, shape[2]:].float().sum(), torch.tensor(0.).cuda())
    assert same(f64(emr.q8_dequantize(q, torch.bfloat16)), back(q))  # 4 bits and a power of two fit


@pytest.mark.parametrize("layout", ["transposed", "sliced", "stepped", "odd_start", "expanded"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_strides(layout, dtype):
    base = normal(2, 2, 150, 301, dtype=dtype)
    x = {"transposed": lambda: base.transpose(1, 2), "sliced": lambda: base[:, 3:140, 5:270],
         "stepped": lambda: base[:, ::3, ::2], "odd_start": lambda: base.view(-1)[1:1 + 2 * 100 * 131].view(2, 100, 131),
         "expanded": lambda: base[:1].expand(3, 150, 301)}[layout]()
    want = f64(x)
    q, qt = emr.Q8(*x.shape), emr.Q8(x.shape[0], x.shape[2], x.shape[1])
    emr.q8_quantize(x, q, qt)
    assert same(back(q), OD.held(want)) and same(back(qt), OD.held(np.swapaxes(want, 1, 2)))
    q1, _ = emr.q8_quantize(x)
    assert same(back(q1), back(q))


def test_quantize_extremes():
    """Zeros, subnormals, the largest values, block maxima at and beside 448 * 2^e, infinities and NaN."""
    x = torch.zeros(1, 12, 256)
    x[0, 1] = 1e-45
    x[0, 2, ::3] = 3e-39
    x[0, 3, 5] = 3.4e38
    x[0, 4, 7], x[0, 4, 200] = 448.0, float(np.nextafter(np.float32(448.0), np.float32(1e9)))
    x[0, 5] = torch.linspace(-1, 1, 256)
    x[0, 5, 9], x[0, 5, 130] = float("inf"), float("-inf")
    x[0, 6] = torch.linspace(-3, 3, 256)
    x[0, 6, 100] = float("nan")
    x[0, 7] = float("nan")
    x[0, 8] = torch.exp2(torch.linspace(-30, 0, 256))
    x[0, 9, 0], x[0, 9, 1:] = 448.0, torch.arange(1, 256) / 64 + 16.5    # ties between e4m3 neighbours
    x[0, 10, 128:] = -2.0 ** -126
    x[0, 11] = 2.0 ** 127
    x = x.cuda()
    q, qt = emr.Q8(1, 12, 256), emr.Q8(1, 256, 12)
    emr.q8_quantize(x, q, qt)
    with np.errstate(over="ignore"):                 # 3.4e38 is held as 2^128, which is infinite in 32 bits
        f32 = lambda v: v.astype(np.float32).astype(np.float64)
        assert same(back(q), f32(OD.held(f64(x))))
        assert same(back(qt), f32(OD.held(np.swapaxes(f64(x), 1, 2))))


def test_quantize_extremes_by_rows():
    """The rows of test_quantize_extremes that hold no finite value beyond 32 bits, at both alignments of a row."""
    x = torch.zeros(1, 9, 261)
    x[0, 1] = 1e-45
    x[0, 2, ::3] = 3e-39
    x[0, 3] = torch.linspace(-1, 1, 261)
    x[0, 3, 9], x[0, 3, 130] = float("inf"), float("-inf")
    x[0, 4] = torch.linspace(-3, 3, 261)
    x[0, 4, 100] = float("nan")
    x[0, 5] = float("nan")
    x[0, 6] = float("inf")
    x[0, 7, 0], x[0, 7, 1:] = 448.0, torch.arange(1, 261) / 64 + 16.5
    x[0, 8, 128:] = -2.0 ** -126
    for dtype in DTYPES:
        v = x.cuda().to(dtype)
        for w in (v, v[:, :, :256].contiguous(), v[:, 1:, 5:]):
            q, _ = emr.q8_quantize(w)
            assert same(back(q), OD.held(f64(w)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [1, 15, 16, 17, 112, 127, 128, 130, 300])
def test_quantize_rows_at_any_alignment(cols, dtype):
    """Rows that start at every element of 16 bytes, with NaN all around them: nothing but the row counts."""
    for start in range(16 // dtype.itemsize):
        for gap in (0, 1, 3, 8):
            base = torch.full((start + 7 * (cols + gap) + 64,), float("nan"), dtype=dtype, device="cuda")
            x = base[start:start + 7 * (cols + gap)].view(7, cols + gap)[:, :cols].unsqueeze(0)
            x.copy_(normal(start, 1, 7, cols, dtype=dtype))
            q, _ = emr.q8_quantize(x)
            assert same(back(q), OD.held(f64(x)))
    one = normal(3, 1, 1, cols, dtype=dtype).expand(2, 5, cols)  # one row in the place of all
    q, _ = emr.q8_quantize(one)
    assert same(back(q), OD.held(f64(one)))


@pytest.mark.parametrize("shape", [(1, 50001, 70), (3, 9000, 130), (30000, 3, 40), (1, 700, 20001)])
def test_quantize_rows_of_many_turns(shape):
    """More blocks than the device takes at a time; batches that end inside a turn."""
    x = normal(5, *shape, dtype=torch.float16)
    q, _ = emr.q8_quantize(x)
    assert same(back(q), OD.held(f64(x)))


@pytest.mark.parametrize("shape", [(1, 1, 5), (2, 130, 257), (1, 1000, 640)])
def test_transpose(shape):
    q, _ = emr.q8_quantize(normal(3, *shape, spread=3.0))
    assert same(back(emr.q8_transpose(q)), OD.held(np.swapaxes(back(q), 1, 2)))


@pytest.mark.parametrize("shape", [(1, 1, 5), (2, 130, 257), (1, 400, 640)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_held(shape, dtype):
    x = normal(3, *shape, spread=3.0, dtype=dtype)
    for v in (x, x.transpose(1, 2).contiguous().transpose(1, 2)):
        q, qt = emr.q8_quantize_held(v)
        assert same(back(q), OD.held(f64(x))) and same(back(qt), OD.held(np.swapaxes(back(q), 1, 2)))


# ---- the product --------------------------------------------------------------------------------------

def product_case(nets_a, nets_w, m, n, k, seed=4):
    a, _ = emr.q8_quantize(normal(seed, nets_a, m, k, spread=0.5))
    w, _ = emr.q8_quantize(normal(seed + 1, nets_w, n, k, spread=0.5) / np.sqrt(k))
    return a, w


SIZES = [(1, 1, 1, 1, 1), (1, 1, 1, 130, 128), (1, 1, 3, 5, 700), (1, 1, 8, 1364, 256), (1, 1, 9, 127, 129),
         (1, 1, 17, 129, 1364), (1, 1, 64, 333, 2048), (1, 1, 127, 128, 512), (1, 1, 129, 257, 640),
         (1, 1, 300, 1000, 131), (1, 1, 1000, 681, 1364), (3, 3, 20, 70, 200), (1, 5, 4, 340, 256), (4, 1, 33, 65, 300),
         (1, 1, 2500, 2600, 384)]


@pytest.mark.parametrize("nets_a,nets_w,m,n,k", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_product(nets_a, nets_w, m, n, k, dtype):
    a, w = product_case(nets_a, nets_w, m, n, k)
    out = f64(emr.q8_matmul(a, w, out_dtype=dtype))
    z, mag = OD.product(back(a), back(w))
    assert np.all(np.abs(out - z) <= (k + 2) * 2.0 ** -23 * mag + ULP[dtype] * np.abs(z) * 1.01 + 2.0 ** -25)


@pytest.mark.parametrize("nets,m,n,k", [(1, 65, 64, 300), (7, 5000, 45, 200), (40, 1500, 64, 130), (9, 2300, 30, 700), (3, 9000, 1, 90)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_product_of_few_columns(nets, m, n, k, dtype):
    """At most 64 columns and more tiles than there are SMs: the epilogue's warps take turns."""
    a, w = product_case(1, nets, m, n, k)
    out = f64(emr.q8_matmul(a, w, out_dtype=dtype))
    z, mag = OD.product(back(a), back(w))
    assert np.all(np.abs(out - z) <= (k + 2) * 2.0 ** -23 * mag + ULP[dtype] * np.abs(z) * 1.01 + 2.0 ** -25)


@pytest.mark.parametrize("act", OD.ACTS)
@pytest.mark.parametrize("m", [1, 6, 20, 150])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_product_bias_activation_and_slope(act, m, dtype):
    nets, n, k = 2, 203, 300
    a, w = product_case(1, nets, m, n, k)
    b = normal(9, nets, n, spread=0.0)
    d = emr.Q8(nets, m, n)
    out = f64(emr.q8_matmul(a, w, b, ACT[act], dtype, slope=d))
    plain = f64(emr.q8_matmul(a, w, b, ACT[act], dtype))
    assert m <= 16 or same(out, plain)               # keeping the slope changes nothing (few rows sum in another order)
    z, mag = OD.product(back(a), back(w), f64(b))
    dz = (k + 3) * 2.0 ** -23 * mag
    y = OD.act(z, act)
    for got in (out, plain):
        assert np.all(np.abs(got - y) <= dz + (2e-6 if act not in ("identity", "abs") else 0.0) + ULP[dtype] * np.abs(y) * 1.01 + 2.0 ** -25)
    s = OD.slope(z, act)
    got = back(d)
    scale = np.repeat(OD.block_scales(s), 128, -1)[..., :n]
    near = 2 * dz + 2e-6 if act != "identity" else 0.0
    if act == "abs":                                 # a sign is uncertain only where z is
        ok = (got == s) | (np.abs(z) <= dz)
        assert ok.all() and (np.abs(z) <= dz).mean() < 0.01
        return
    # half a step of e4m3: 2^-4 relative, or 2^-10 of twice the scale (near a scale's edge it may double)
    assert np.all(np.abs(got - s) <= near + 2.0 ** -4 * (np.abs(s) + near) + 2.0 ** -9 * scale)


@pytest.mark.parametrize("nets,m,n,k,total,slope", [(1, 3100, 2400, 2100, False, False), (3, 3100, 2400, 700, True, False),
                                                    (2, 1500, 2433, 3000, False, False), (1, 3100, 2400, 5100, False, True)])
def test_product_of_pairs(nets, m, n, k, total, slope):
    """Sizes that go to pairs of SMs, with odd numbers of row and column tiles."""
    a, w = product_case(nets, nets, m, n, k)
    b = None if total else normal(9, nets, n, spread=0.0)
    d = emr.Q8(nets, m, n) if slope else None
    act = emr.ACT_TANH if slope else emr.ACT_IDENTITY
    out = emr.q8_matmul(a, w, b, act, slope=d, sum_batch=total)
    assert torch.equal(out, emr.q8_matmul(a, w, b, act, slope=d, sum_batch=total))
    x, y = emr.q8_dequantize(a, torch.float32).double(), emr.q8_dequantize(w).double()
    z, mag = x @ y.mT, x.abs() @ y.abs().mT
    if b is not None:
        z, mag = z + b.double()[:, None], mag + b.double().abs()[:, None]
    if total:
        z, mag, k = z.sum(0, keepdim=True), mag.sum(0, keepdim=True), k * nets
    bound = (k + 3) * 2.0 ** -23 * mag + (2e-6 if slope else 0)
    assert bool(((out.double() - (torch.tanh(z) if slope else z)).abs() <= bound).all())
    if slope:
        s = OD.slope(z.cpu().numpy(), "tanh")
        scale = np.repeat(OD.block_scales(s), 128, -1)[..., :n]
        near = 2 * bound.cpu().numpy()
        assert np.all(np.abs(back(d) - s) <= near + 2.0 ** -4 * (s + near) + 2.0 ** -9 * scale)


@pytest.mark.parametrize("nets,shared", [(1, False), (3, False), (5, True)])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 40, 8192), (3, 333, 129), (4, 340, 256), (8, 70, 1024), (8, 130, 1300),
                                   (9, 100, 300), (16, 65, 512), (16, 200, 4000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layer_of_few_rows(nets, shared, m, n, k, dtype):
    """x quantised within the product, or before it; any strides of x."""
    w, b = normal(40, nets, n, k, spread=0.3) / np.sqrt(k), normal(41, nets, n, spread=0.0)
    x = normal(42, 1 if shared else nets, m, k, dtype=dtype)
    layer = emr.DenseLayer(w, b, emr.ACT_SIGMOID)
    y = layer.forward(x)
    z, mag = OD.product(OD.held(f64(x)), OD.held(f64(w)), f64(b))
    apart = emr.q8_matmul(emr.q8_quantize(x)[0], layer.w8, b, emr.ACT_SIGMOID)
    for got in (y, apart):                           # their sums may be in another order
        assert np.all(np.abs(f64(got) - OD.act(z, "sigmoid")) <= (k + 3) * 2.0 ** -23 * mag + 2e-6)
    assert torch.equal(y, layer.forward(x.transpose(1, 2).contiguous().transpose(1, 2)))


def test_product_of_few_rows_with_extreme_scales():
    x, w = normal(43, 1, 5, 300) * 2.0 ** 100, normal(44, 1, 33, 300) * 2.0 ** -110
    x[0, 2] *= 2.0 ** -120
    out = f64(emr.DenseLayer(w).forward(x))
    z, mag = OD.product(OD.held(f64(x)), OD.held(f64(w)))
    assert np.all(np.abs(out - z) <= 302 * 2.0 ** -23 * mag + 2.0 ** -149)


def test_product_sums_over_the_networks():
    a, w = product_case(6, 6, 140, 150, 300)
    out = f64(emr.q8_matmul(a, w, sum_batch=True))
    z, mag = OD.product(back(a), back(w))
    assert out.shape == (1, 140, 150)
    assert np.all(np.abs(out[0] - z.sum(0)) <= (6 * 300 + 2) * 2.0 ** -23 * mag.sum(0))


def test_product_precision_of_long_sums():
    """One large term and many that are 2^-20 of it: sums in fewer than 24 bits would drop them."""
    k, m, n = 8192, 4, 200
    for rows in (m, 200):
        x = torch.full((1, rows, k), 2.0 ** -10, device="cuda")
        w = torch.full((1, n, k), 2.0 ** -10, device="cuda")
        x[:, :, 0] = 1.0                             # its block's scale leaves 2^-10 representable (normal: 2^-14)
        w[:, :, 0] = 1.0
        out = f64(emr.q8_matmul(emr.q8_quantize(x)[0], emr.q8_quantize(w)[0]))
        want, _ = OD.product(OD.held(f64(x)), OD.held(f64(w)))
        assert np.abs(out / want - 1).max() < 64 * 8192 / 128 * 2.0 ** -24
        assert abs(want[0, 0, 0] - (1 + 8191 * 2.0 ** -20)) < 1e-12


def test_product_keeps_nan_to_its_row_and_column():
    x, w = normal(5, 1, 40, 300), normal(6, 1, 150, 300)
    x[0, 7, 130] = float("nan")
    x[0, 20, 3] = float("inf")
    w[0, 140, 299] = float("-inf")
    out = f64(emr.q8_matmul(emr.q8_quantize(x)[0], emr.q8_quantize(w)[0]))[0]
    bad = np.zeros((40, 150), bool)
    bad[[7, 20]] = True
    bad[:, 140] = True
    assert np.array_equal(np.isnan(out), bad)


def test_product_into_given_memory_writes_nothing_else():
    a, w = product_case(1, 1, 37, 131, 200)
    for dtype in DTYPES:
        room = torch.full((37 * 131 + 64,), 7.0, dtype=dtype, device="cuda")
        for at in (0, 1, 2, 3, 5):
            room.fill_(7.0)
            out = room[at:at + 37 * 131].view(1, 37, 131)
            emr.q8_matmul(a, w, out=out)
            assert same(f64(out), f64(emr.q8_matmul(a, w, out_dtype=dtype)))
            assert bool((room[:at] == 7).all()) and bool((room[at + 37 * 131:] == 7).all())


# ---- the layer ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("act", OD.ACTS)
@pytest.mark.parametrize("nets,shared,m,n,k", [(1, False, 1, 5, 3), (1, False, 200, 300, 150), (3, True, 70, 130, 90),
                                               (2, False, 260, 129, 257)])
def test_layer_gradients(act, nets, shared, m, n, k):
    w = normal(10, nets, n, k, spread=0.3) / np.sqrt(k)
    b = normal(11, nets, n, spread=0.0)
    x = normal(12, 1 if shared else nets, m, k, spread=0.3)
    dy = normal(13, nets, m, n, spread=0.5)
    layer = emr.DenseLayer(w, b, ACT[act], train=True)
    y, saved = layer.forward_train(x)
    assert m <= 16 or same(f64(y), f64(layer.forward(x)))
    dx, dw, db = layer.backward(dy, saved)
    xh, wh = OD.held(f64(x)), OD.held(f64(w))
    assert same(back(saved.xt), OD.held(np.swapaxes(xh, 1, 2)))
    z, _ = OD.product(xh, wh, f64(b))
    # the formulas, from the slopes that were kept
    d = back(saved.slope) if act != "identity" else np.ones_like(z)
    dz = np.float32(f64(dy)) * np.float32(d)         # one rounding in 32 bits, as kept
    dz = dz.astype(np.float64)
    assert np.all(np.abs(f64(db) - dz.sum(1)) <= (m + 2) * 2.0 ** -23 * np.abs(dz).sum(1))
    wt = OD.held(np.swapaxes(f64(w), 1, 2))
    want, mag = OD.product(OD.held(dz), wt)
    terms = n * (nets if shared else 1)
    if shared:
        want, mag = want.sum(0, keepdims=True), mag.sum(0, keepdims=True)
    assert dx.shape == x.shape and np.all(np.abs(f64(dx) - want) <= (terms + 2) * 2.0 ** -23 * mag)
    xt = OD.held(np.swapaxes(xh, 1, 2))
    want, mag = OD.product(OD.held(np.swapaxes(dz, 1, 2)), xt)
    assert dw.shape == w.shape and np.all(np.abs(f64(dw) - want) <= (m + 2) * 2.0 ** -23 * mag)
    # differences of the loss sum(dy y) in float64. Each factor is off by half a step of its 8-bit form: 2^-4
    # relative or 2^-10 of its block's scale (twice that where the scale is uncertain).
    full = f64(dy) * OD.slope(z, act)
    steep = np.abs(full) * 2.0 ** -4 + np.abs(f64(dy)) * np.repeat(OD.block_scales(OD.slope(z, act)), 128, -1)[..., :n] * 2.0 ** -9
    dzt_step = np.swapaxes(np.repeat(OD.block_scales(np.swapaxes(dz, 1, 2)), 128, -1)[..., :m], 1, 2)
    off = steep + (np.abs(full) + steep) * 2.0 ** -4 + dzt_step * 2.0 ** -9
    h = 1e-4
    rng = np.random.default_rng(3)

    def loss(wv, bv):
        return (f64(dy) * OD.act(OD.product(xh, wv, bv)[0], act)).sum()

    for _ in range(8):
        g, i, j = rng.integers(nets), rng.integers(n), rng.integers(k)
        step = np.zeros_like(wh)
        step[g, i, j] = h
        xg = xh[0 if shared else g]
        diff = (loss(wh + step, f64(b)) - loss(wh - step, f64(b))) / (2 * h)
        kink = np.abs(f64(dy)[g, :, i] * xg[:, j])[np.abs(z[g, :, i]) <= h * np.abs(xg[:, j])].sum() * 2 if act == "abs" else 0.0
        xt_off = np.abs(xg[:, j] - xt[0 if shared else g][j])
        bound = (off[g, :, i] * np.abs(xt[0 if shared else g][j])).sum() + (np.abs(full[g, :, i]) * xt_off).sum()
        assert abs(f64(dw)[g, i, j] - diff) <= bound + kink + 1e-5 * (1 + np.abs(f64(dy)[g, :, i] * xg[:, j]).sum())
        step = np.zeros_like(f64(b))
        step[g, i] = h
        diff = (loss(wh, f64(b) + step) - loss(wh, f64(b) - step)) / (2 * h)
        kink = np.abs(f64(dy)[g, :, i])[np.abs(z[g, :, i]) <= h].sum() * 2 if act == "abs" else 0.0
        assert abs(f64(db)[g, i] - diff) <= steep[g, :, i].sum() + kink + 1e-5 * (1 + np.abs(f64(dy)[g, :, i]).sum())


def test_slope_of_saturated_and_infinite_inputs():
    z = torch.tensor([[0.0, 1.0, -1.0, 8.0, -8.0, 30.0, -30.0, 100.0, -100.0, 400.0, -400.0]], device="cuda")
    one = emr.q8_quantize(torch.ones(1, 1, 1, device="cuda"))[0]
    w = emr.q8_quantize(torch.zeros(1, z.shape[1], 1, device="cuda"))[0]
    b = z.clone()
    for act in OD.ACTS:
        d = emr.Q8(1, 1, z.shape[1])
        y = f64(emr.q8_matmul(one, w, b, ACT[act], slope=d))
        assert np.allclose(y[0], OD.act(f64(z), act), rtol=2e-5, atol=2e-6)
        assert np.isfinite(back(d)).all()
    inf = torch.tensor([[float("inf"), float("-inf")]], device="cuda")
    w = emr.q8_quantize(torch.zeros(1, 2, 1, device="cuda"))[0]
    for act, want in (("sigmoid", [1, 0]), ("tanh", [1, -1]), ("gauss", [0, 0]), ("abs", [np.inf, np.inf])):
        d = emr.Q8(1, 1, 2)
        assert np.array_equal(f64(emr.q8_matmul(one, w, inf, ACT[act], slope=d))[0, 0], want)
        assert np.array_equal(back(d)[0, 0], [1, -1] if act == "abs" else [0, 0])


def test_layer_takes_the_materialised_outputs_of_a_genome():
    from paper_2608_27612_gb300 import workloads as W
    w = W.c2(D=3, P=6)
    dsc = emr.Discovery(w.pop, w.sources, w.D, w.theta, w.band, materialise=True)
    dsc.run_unfused()
    mats = dsc.out.view(dsc.P, dsc.S, -1).transpose(1, 2)          # [genome, position, slot]
    layer = emr.DenseLayer(mats, act=emr.ACT_TANH)
    x = normal(20, 7, dsc.S)
    y = f64(layer.forward(x))
    z, mag = OD.product(OD.held(f64(x)[None]), OD.held(f64(mats)))
    assert y.shape == (6, 7, dsc.grid.n_total)
    assert np.all(np.abs(y - np.tanh(z)) <= (dsc.S + 2) * 2.0 ** -23 * mag + 2e-6)


def test_layer_on_another_stream_and_after_an_update():
    w, x = normal(21, 300, 400) / 20, normal(22, 50, 400)
    layer = emr.DenseLayer(w, act=emr.ACT_SIN, train=True)
    want = layer.forward(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [layer.forward(x, stream=side) for _ in range(20)]
    side.synchronize()
    assert all(torch.equal(g, want) for g in got)
    layer.set_weights(2 * w)
    assert torch.equal(layer.forward(x), emr.DenseLayer(2 * w, act=emr.ACT_SIN).forward(x))
    assert layer.forward(x[:0]).shape == (1, 0, 300)


def test_same_call_twice_gives_the_same_bits():
    w, x, dy = normal(23, 500, 700), normal(24, 600, 700), normal(25, 600, 500)
    layer = emr.DenseLayer(w, act=emr.ACT_GAUSS, train=True)
    first = None
    for _ in range(3):
        y, saved = layer.forward_train(x)
        got = (y,) + layer.backward(dy, saved)
        if first is None:
            first = got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


# ---- refusals ---------------------------------------------------------------------------------------------

def test_refusals():
    x = normal(30, 2, 10, 20)
    q, _ = emr.q8_quantize(x)
    for call in (lambda: emr.q8_quantize(x, emr.Q8(2, 10, 21)), lambda: emr.q8_quantize(x, None, emr.Q8(2, 10, 20)),
                 lambda: emr.q8_transpose(q, emr.Q8(2, 10, 20)),
                 lambda: emr.q8_matmul(q, emr.Q8(3, 5, 20)), lambda: emr.q8_matmul(q, emr.Q8(2, 5, 19)),
                 lambda: emr.q8_matmul(q, q, act=6), lambda: emr.q8_matmul(q, q, act=emr.ACT_SIN, sum_batch=True),
                 lambda: emr.q8_matmul(q, q, slope=emr.Q8(2, 10, 11)),
                 lambda: emr.q8_slope(x, emr.Q8(2, 10, 21), emr.Q8(2, 10, 20)), lambda: emr.q8_slope(x, None)):
        with pytest.raises(emr.EmrError) as e:
            call()
        assert e.value.status == emr.EMR_ERR_ARG
    for call in (lambda: emr.q8_quantize(x.int()), lambda: emr.q8_quantize(x.cpu()), lambda: emr.q8_quantize(x[0, 0]),
                 lambda: emr.q8_matmul(q, q, bias=torch.zeros(2, 9, device="cuda")),
                 lambda: emr.q8_matmul(q, q, out_dtype=torch.float64),
                 lambda: emr.DenseLayer(x, act=9), lambda: emr.DenseLayer(x).forward(x[:, :, :19]),
                 lambda: emr.DenseLayer(x).forward_train(x), lambda: emr.DenseLayer(x).set_weights(x[:1]),
                 lambda: emr.DenseLayer(x, train=True).forward_train(x[:, :0])):
        with pytest.raises(ValueError):
            call()
