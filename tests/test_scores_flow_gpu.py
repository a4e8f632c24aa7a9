"""The calls together, as a small substrate learns from a large one and is served: a teacher's layer, its best answers, distillation into
a student's layer, the student's weights in 4 bits, draws and their probabilities; in a captured graph, on another stream, and
with a bystander's memory around."""
import numpy as np
import pytest
import torch

from oracle import scores as OS
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu


def scene(nets, m, k, n, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)
    noise = torch.empty(nets * m, n, device="cuda").exponential_(generator=g).clamp_min_(1e-30)
    return {"x": r(1, m, k), "big": r(nets, n, k) / k ** 0.5 * 3, "small": r(nets, n, k) / k ** 0.5, "b": 0.1 * r(nets, n), "noise": noise}


def teach(s, top=16, T=1.5):
    """Every output of one round of all calls."""
    nets, n, k = s["small"].shape
    m = s["x"].shape[1]
    teacher = emr.DenseLayer(s["big"], s["b"])
    best = emr.log_probs(teacher.forward(s["x"]).view(nets * m, n), temperature=T, top=top)
    student = emr.DenseLayer(s["small"], s["b"], train=True)
    y, saved = student.forward_train(s["x"])
    dy, loss = emr.distill_grad(y.view(nets * m, n), best.top_index, best.top_logp, T * T / (nets * m), T)
    dx, dw, db = student.backward(dy.view(nets, m, n), saved)
    w = s["small"] - 20 * dw
    served = emr.q4_quantize(w, 64)
    z = emr.q4_matmul(s["x"], served, s["b"]).view(nets * m, n)
    index, logp = emr.sample(z, s["noise"], temperature=0.9)
    again = emr.log_probs(z, index, 0.9, top=3)
    grad, lp, h = emr.log_probs_grad(z, index, -1.0 / (nets * m), 0.01)
    after = emr.distill(z, best.top_index, best.top_logp, T)
    return [best.top_index, best.top_logp, best.entropy, loss, dy, dx, dw, db, served.data, z, index, logp, again.logp, again.top_index, grad, lp,
            h, after, y]


SCENES = [(3, 5, 200, 340), (2, 40, 129, 1364), (1, 30, 300, 9001)]


@pytest.mark.parametrize("nets,m,k,n", SCENES)
def test_a_round(nets, m, k, n):
    s = scene(nets, m, k, n)
    out = teach(s)
    for x, y in zip(out, teach(s)):
        assert torch.equal(x, y)
    best_i, best_l, _, loss, dy, _, _, _, data, z, index, logp, again, _, _, _, _, after, y = out
    assert torch.allclose(again, logp, atol=2e-5)                       # the draw's own answer
    zn, yn = z.double().cpu().numpy(), y.view(nets * m, n).double().cpu().numpy()
    w = emr.q4_dequantize(emr.Q4.of(data, nets, n, k, 64)).double()
    want = (s["x"].double() @ w.mT + s["b"].double()[:, None]).reshape(nets * m, n)
    mag = (s["x"].double().abs() @ w.abs().mT).reshape(nets * m, n) + 1
    assert bool(((z.double() - want).abs() <= (k / 8 + 24) * 2.0 ** -23 * mag).all())        # as the product's own tests
    for r in (0, nets * m - 1):
        for got, scores in ((after, zn), (loss, yn)):
            want, grad, size = OS.distill(scores[r], best_i[r].cpu().numpy(), best_l[r].double().cpu().numpy(), 1.5)
            assert abs(float(got[r]) - want) <= 4e-5 * (1 + size)
        grad *= 1.5 ** 2 / (nets * m)                                   # of y: entries of at most 2 terms of 1 / 1.5 of that
        assert np.abs(dy[r].double().cpu().numpy() - grad).max() <= 2e-5 * 4 * 1.5 / (nets * m) + 1e-30


@pytest.mark.parametrize("nets,m,k,n", SCENES)
def test_captured_and_replayed(nets, m, k, n):
    """Two graphs of the same calls, replayed in turn with new inputs, give the calls' own bits."""
    s, other = scene(nets, m, k, n), scene(nets, m, k, n, 1)
    first, second = teach(s), teach(other)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(teach(s))
        graphs.append(g)
    originals = {name: v.clone() for name, v in s.items()}
    for turn in range(2):
        for inputs, want in ((other, second), (originals, first)):
            for name, v in inputs.items():
                s[name].copy_(v)
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            for out in outs:
                assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_on_another_stream():
    """Made, used and freed on streams of their own, with the default stream's allocations in between."""
    s = scene(2, 33, 200, 1364)
    want = teach(s)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for stream in streams:
        with torch.cuda.stream(stream):
            outs.append(teach(s))
    q = emr.q4_quantize(s["small"], 64)
    late = emr.q4_matmul(s["x"], q, s["b"], stream=streams[0])          # memory of the default stream, used on another
    torch.cuda.current_stream().wait_stream(streams[0])
    del q
    filler = [torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for out in outs for x, y in zip(out, want)) and len(filler) == 4
    assert torch.equal(late, emr.q4_matmul(s["x"], emr.q4_quantize(s["small"], 64), s["b"]))
    streams[1].wait_stream(torch.cuda.current_stream())
    t = torch.zeros(33, dtype=torch.int32, device="cuda")
    a = emr.log_probs(late[0], t, top=4, stream=streams[1])
    b = emr.distill_grad(late[0], a.top_index, a.top_logp, 1.0, stream=streams[1])
    torch.cuda.synchronize()
    assert torch.equal(a.logp, emr.log_probs(late[0], t).logp) and torch.equal(b[1], emr.distill(late[0], a.top_index, a.top_logp))
    assert emr.device_error() == 0


@pytest.mark.parametrize("rows,n,dtype", [(3, 7, torch.bfloat16), (5200, 45, torch.float16), (2500, 700, torch.float32), (700, 3001, torch.bfloat16), (1250, 3001, torch.float16),
                                          (9, 5461, torch.float32), (2, 40003, torch.bfloat16), (2, 140001, torch.float16)])
def test_neighbours_are_neither_counted_nor_touched(rows, n, dtype):
    """Rows in the middle of a larger buffer: huge values around them change nothing, and gradients written with a row stride of
    their own through the C ABI leave what lies between as it was. Both sides may be off as the calls' own tests say, so twice that: 2e-5 for
    log p, 3e-4 for gradients whose terms have magnitudes of up to 7."""
    wide = torch.full((rows + 2, n + 21), float("inf"), device="cuda", dtype=dtype)
    s = torch.randn(rows, n, device="cuda").to(dtype)
    v = wide[1:-1, 5:5 + n]
    v.copy_(s)
    t = torch.randint(0, n, (rows,), device="cuda", dtype=torch.int32)
    a, b = emr.log_probs(s, t, top=min(n, 9)), emr.log_probs(v, t, top=min(n, 9))
    assert torch.allclose(a.logp, b.logp, atol=2e-5) and torch.equal(a.top_index, b.top_index) and torch.allclose(a.entropy, b.entropy, atol=1e-4)
    L, pitch = emr.lib(), n + 13
    out = torch.full((rows, pitch), 7.0, device="cuda")
    raw = torch.cuda.current_stream().cuda_stream
    kind = emr._DTYPES[dtype]
    assert L.emr_log_probs_grad(v.data_ptr(), kind, rows, n, v.stride(0), t.data_ptr(), None, 1.0, None, 1.0, None, 0.5, None, None, out.data_ptr(),
                                emr.EMR_F32, pitch, raw) == 0
    want = emr.log_probs_grad(s, t, 1.0, 0.5, out_dtype=torch.float32)[0]
    assert torch.allclose(out[:, :n], want, atol=3e-4) and bool((out[:, n:] == 7).all())
    out.fill_(7.0)
    assert L.emr_distill(v.data_ptr(), kind, rows, n, v.stride(0), a.top_index.data_ptr(), a.top_logp.data_ptr(), emr.EMR_F32, a.top_index.shape[1],
                         None, 1.0, 1, None, 1.0, None, out.data_ptr(), emr.EMR_F32, pitch, raw) == 0
    want = emr.distill_grad(s, a.top_index, a.top_logp, 1.0, out_dtype=torch.float32)[0]
    assert torch.allclose(out[:, :n], want, atol=3e-4) and bool((out[:, n:] == 7).all())
    half = torch.full((rows, pitch), 7.0, device="cuda", dtype=torch.bfloat16)
    assert L.emr_log_probs_grad(v.data_ptr(), kind, rows, n, v.stride(0), t.data_ptr(), None, 1.0, None, 1.0, None, 0.0, None, None, half.data_ptr(),
                                emr.EMR_BF16, pitch, raw) == 0
    assert bool((half[:, n:] == 7).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_products_write_their_outputs_alone(dtype):
    """What lies before and behind an output, and behind its last rows, stays as it was: rows and columns that fill no tile."""
    for m, n, k in ((1, 17, 40), (7, 33, 300), (21, 140, 257), (40, 15, 130), (101, 129, 129)):
        q = emr.q4_quantize(torch.randn(2, n, k, device="cuda"), 32)
        x = torch.randn(2, m, k, device="cuda").to(dtype)
        want = emr.q4_matmul(x, q)
        room = torch.full((2 * m * n + 64,), 7.0, device="cuda")
        emr.q4_matmul(x, q, out=room[32:32 + 2 * m * n].view(2, m, n))
        assert torch.equal(room[32:-32].view(2, m, n), want) and bool((room[:32] == 7).all()) and bool((room[-32:] == 7).all())
        wide = torch.full((2, m, k + 9), float("nan"), device="cuda").to(dtype)
        wide[:, :, 3:3 + k] = x
        assert torch.equal(emr.q4_matmul(wide[:, :, 3:3 + k], q), want)
