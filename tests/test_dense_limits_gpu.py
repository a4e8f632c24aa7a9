"""Dense layers at the edges of what their calls accept, against the same calls inside them or the definitions
(oracle.dense; the bounds are those of test_dense_gpu.py)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import dense as OD
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu


def normal(seed, *shape, dtype=torch.float32):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).cuda().to(dtype)


def f64(t):
    return t.double().cpu().numpy()


def f32(v):
    """v as 32 bits give it: 2^128 is infinite there."""
    with np.errstate(over="ignore"):
        return v.astype(np.float32).astype(np.float64)


def q8_at(offset, batch, rows, cols):
    """A Q8 whose buffers begin `offset` bytes after a multiple of 256, filled with a byte, and its memory."""
    n = sum(emr._q8_bytes(batch, rows, cols))
    room = torch.full((n + 512,), 0x5a, dtype=torch.uint8, device="cuda")
    start = -room.data_ptr() % 256 + offset
    return emr.Q8.of(room[start:start + n], batch, rows, cols), room, start


# few rows, single blocks' tiles, and pairs of SMs; a second batch of odd rows
@pytest.mark.parametrize("nets,m,n,k", [(1, 5, 40, 64), (2, 150, 203, 300), (1, 3100, 2400, 5100)])
@pytest.mark.parametrize("offset", [16, 48, 112, 240])
def test_slopes_at_every_multiple_of_16_bytes(nets, m, n, k, offset):
    a, w = (emr.q8_quantize(normal(s, nets, r, k) / np.sqrt(np.sqrt(k)))[0] for s, r in ((1, m), (2, n)))
    want = emr.Q8(nets, m, n)
    y = emr.q8_matmul(a, w, act=emr.ACT_TANH, slope=want)
    got, room, start = q8_at(offset, nets, m, n)
    assert got.values.data_ptr() % 32 == 16
    assert torch.equal(y, emr.q8_matmul(a, w, act=emr.ACT_TANH, slope=got))
    assert torch.equal(got.values, want.values)
    assert torch.equal(emr.q8_dequantize(got), emr.q8_dequantize(want))
    assert bool((room[:start] == 0x5a).all()) and bool((room[start + got.data.numel():] == 0x5a).all())
    assert emr.device_error() == 0


def test_training_step_into_memory_at_16_bytes():
    """emr_dense_forward with x8, xt and slope at 16 bytes after a multiple of 32, and its backward pass."""
    nets, m, n, k = 2, 70, 130, 90
    layer = emr.DenseLayer(normal(3, nets, n, k) / 9, act=emr.ACT_GAUSS, train=True)
    x, dy = normal(4, nets, m, k), normal(5, nets, m, n)
    y, saved = layer.forward_train(x)
    L, sizes = emr.lib(), [C.c_size_t() for _ in range(4)]
    assert L.emr_dense_forward_room(layer._ref, nets, m, 1, *[C.byref(s) for s in sizes[:3]]) == emr.EMR_OK
    assert L.emr_dense_backward_room(layer._ref, nets, m, C.byref(sizes[3])) == emr.EMR_OK
    rooms = [torch.empty(s.value + 256, dtype=torch.uint8, device="cuda") for s in sizes]
    x8, xt, slope, ws = (r.data_ptr() + (16 - r.data_ptr()) % 32 for r in rooms)
    out, stream = torch.empty_like(y), torch.cuda.current_stream().cuda_stream
    assert L.emr_dense_forward(layer._ref, x.data_ptr(), 0, nets, m, *x.stride(), out.data_ptr(), 0, 1, x8, xt, slope, stream) == emr.EMR_OK
    dx, dw, db = (torch.empty(s, device="cuda") for s in ((nets, m, k), (nets, n, k), (nets, n)))
    assert L.emr_dense_backward(layer._ref, dy.data_ptr(), 0, nets, m, xt, slope, dx.data_ptr(), dw.data_ptr(), db.data_ptr(), 0, ws,
                                sizes[3], stream) == emr.EMR_OK
    assert torch.equal(out, y)
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), layer.backward(dy, saved)))


@pytest.mark.parametrize("large", [3e4, 1e9, 1e13, 3e30, float("inf")])
@pytest.mark.parametrize("m", [1, 20, 150])
def test_sin_of_large_values_beside_nan(large, m):
    """A column of NaN leaves the columns before and after it as they are: sin and its slope of a large value stay those
    of the full range (to 2e-6; the slope in 8 bits to half a step, 2^-4 relative or 2^-10 of its block's scale)."""
    n = 70
    x, w = emr.q8_quantize(torch.zeros(1, m, 1, device="cuda"))[0], emr.q8_quantize(torch.zeros(1, n, 1, device="cuda"))[0]
    b = torch.linspace(-3, 3, n, device="cuda")[None]
    b[0, [2, 40]], b[0, [3, 41, 69]] = large, float("nan")
    layer = emr.DenseLayer(torch.zeros(1, n, 1, device="cuda"), b, emr.ACT_SIN)
    z = f64(b)[0]
    with np.errstate(invalid="ignore"):
        y, s = np.sin(z), np.cos(z)
    d = emr.Q8(1, m, n)
    for out in (layer.forward(torch.zeros(1, m, 1, device="cuda")), emr.q8_matmul(x, w, b, emr.ACT_SIN),
                emr.q8_matmul(x, w, b, emr.ACT_SIN, slope=d)):
        got = f64(out)[0]
        assert np.array_equal(np.isnan(got), np.broadcast_to(np.isnan(y), got.shape))
        assert np.nanmax(np.abs(got - y)) <= 2e-6
    got = f64(emr.q8_dequantize(d))[0]
    scale = OD.block_scales(np.nan_to_num(s))[0]
    assert np.array_equal(np.isnan(got), np.broadcast_to(np.isnan(s), got.shape))
    assert np.nanmax(np.abs(got - s) - 2.0 ** -4 * np.abs(s)) <= 4e-6 + 2.0 ** -10 * scale


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_transpose_of_the_largest_values(dtype):
    """Values that are held as 2^128, which 32 bits do not have, are held as that in the transpose, too: only infinities
    and NaN become NaN there."""
    top = float(torch.finfo(dtype).max)
    x = torch.zeros(2, 150, 261)
    x[0, 3, 1], x[0, 7, 2], x[0, 100, 2], x[0, 140, 255], x[1, 0, 0] = -top, top, 1e37, 3.3e38, -3.2e38
    x[1, 5], x[1, 9, 4], x[1, 130, 4], x[1, 131, 4] = top, float("inf"), -top, float("nan")
    x = x.cuda().to(dtype)
    once = OD.held(f64(x))
    want = f32(OD.held(np.swapaxes(once, 1, 2)))
    q, qt = emr.q8_quantize_held(x)
    assert np.array_equal(f64(emr.q8_dequantize(q)), f32(once), equal_nan=True)
    assert np.array_equal(f64(emr.q8_dequantize(qt)), want, equal_nan=True)
    assert np.array_equal(f64(emr.q8_dequantize(emr.q8_transpose(q))), want, equal_nan=True)
    # the values themselves are there: times 2^-120 they fit
    w = emr.q8_quantize(torch.full((2, 1, 150), 2.0 ** -120, device="cuda"))[0]
    got = f64(emr.q8_matmul(qt, w))[..., 0]
    sums = np.swapaxes(once, 1, 2).sum(-1) * 2.0 ** -120
    assert np.array_equal(np.isnan(got), np.isnan(sums)) and np.nanmax(np.abs(got - sums)) <= 152 * 2.0 ** -23 * 256 * 150


def taken(n, ptr):
    """Eight pieces of memory of n bytes, overwritten; none of them is the one at ptr."""
    junk = [torch.full((n,), 0x38, dtype=torch.uint8, device="cuda") for _ in range(8)]
    assert all(j.data_ptr() != ptr for j in junk)
    return junk


def late(side):
    """Work given to `side` after this begins some 50 ms later."""
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)


def test_a_layer_may_go_while_another_stream_uses_it():
    w, b, x = normal(6, 1, 300, 400) / 20, normal(7, 1, 300), normal(8, 1, 50, 400)
    want = emr.DenseLayer(w, b, emr.ACT_TANH).forward(x)
    side = torch.cuda.Stream()
    layer = emr.DenseLayer(w, b, emr.ACT_TANH)
    late(side)
    got = layer.forward(x, stream=side)
    n, ptr = layer.w8.data.numel(), layer.w8.data.data_ptr()
    del layer
    taken(n, ptr)
    side.synchronize()
    assert torch.equal(got, want)


def test_what_a_step_keeps_may_go_while_another_stream_uses_it():
    w, x, dy = normal(9, 1, 300, 400) / 20, normal(10, 1, 200, 400), normal(11, 1, 200, 300)
    layer, side = emr.DenseLayer(w, act=emr.ACT_GAUSS, train=True), torch.cuda.Stream()
    _, saved = layer.forward_train(x)
    want = layer.backward(dy, saved)
    late(side)
    got = layer.backward(dy, saved, stream=side)
    kept = (saved._data.numel(), saved._data.data_ptr()), (layer.w8t.data.numel(), layer.w8t.data.data_ptr())
    del saved, layer
    for n, ptr in kept:
        taken(n, ptr)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("nets,shared,m,n,k", [(1, False, 4, 60, 200), (6, True, 40, 130, 90), (1, False, 700, 900, 1300)])
def test_a_step_and_a_draw_in_a_captured_graph(nets, shared, m, n, k):
    """An update of the weights, a training step, a forward pass and a draw, captured once and replayed on new
    inputs: the same bits as the calls by themselves."""
    def inputs(seed):
        return (normal(seed, nets, n, k) / np.sqrt(k), normal(seed + 1, nets, n), normal(seed + 2, 1 if shared else nets, m, k),
                normal(seed + 3, nets, m, n), torch.rand(nets * m, n, device="cuda") + 1e-3)

    def step(w, b, x, dy, e):
        layer.set_weights(w, b)
        y, saved = layer.forward_train(x)
        scores = layer.forward(x)
        return (y, scores) + layer.backward(dy, saved) + emr.sample(scores.view(nets * m, n), e, top_k=20, top_p=0.9)

    held = inputs(20)
    layer = emr.DenseLayer(held[0], held[1], emr.ACT_SIGMOID, train=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                     # what is asked of the device once is asked before
        step(*held)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*held)
    for seed in (30, 40):
        new = inputs(seed)
        for a, v in zip(held, new):
            a.copy_(v)
        graph.replay()
        out = [t.clone() for t in got]
        want = step(*new)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
