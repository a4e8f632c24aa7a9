"""Measured cases of the dense-layer and sampling operators.

Three operators, which a dense substrate layer uses one after the other:

product  y = act(x W^T + b) with x and W held in 8-bit floating point (e4m3), one power-of-two scale for
         each block of 128 along the contraction, sums in 32 bits.
step     a training step of such a layer: the forward pass keeps x and act'(z) in 8 bits, and the backward
         pass takes dx, dW and db from those.
sample   one index for each row of scores, with temperature, top-k, top-p and min-p, from given
         exponential random numbers.

`run` computes them in plain 32-bit torch operations, or with the framework's calls where `own` is true.
"""
import math

import torch

own = False

BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ("identity", "sigmoid", "tanh", "gauss", "sin", "abs")


# ---- cases ---------------------------------------------------------------------------------------

def listed():
    return [
        # one pattern through a layer from the plane of depths 0..4 to the plane of depths 0..5: a single
        # answer, where the time of a launch counts
        {"name": "product one pattern", "op": "product", "nets": 1, "shared": False, "m": 1, "n": 5460, "k": 1364,
         "act": "tanh", "dtype": "f32", "out": "f32"},
        # a few patterns through a wide layer: every weight is read for eight rows
        {"name": "product eight patterns", "op": "product", "nets": 1, "shared": False, "m": 8, "n": 8192, "k": 8192,
         "act": "sigmoid", "dtype": "bf16", "out": "bf16"},
        # 150 networks with weights of their own answer the same four patterns
        {"name": "product population", "op": "product", "nets": 150, "shared": True, "m": 4, "n": 1364, "k": 256,
         "act": "tanh", "dtype": "f32", "out": "f32"},
        # an ordinary batch, no size a multiple of a tile
        {"name": "product thousand", "op": "product", "nets": 1, "shared": False, "m": 1000, "n": 5460, "k": 1364,
         "act": "gauss", "dtype": "bf16", "out": "bf16"},
        # a whole data set of 94,464 samples through a hidden layer
        {"name": "product data set", "op": "product", "nets": 1, "shared": False, "m": 94464, "n": 1364, "k": 1364,
         "act": "sin", "dtype": "f16", "out": "f16"},
        # 64 small networks trained on the same patterns: the gradient of x sums over the networks
        {"name": "step population", "op": "step", "nets": 64, "shared": True, "m": 250, "n": 340, "k": 256,
         "act": "sigmoid", "dtype": "f32", "out": "bf16"},
        # an ordinary training batch with odd widths
        {"name": "step ordinary", "op": "step", "nets": 1, "shared": False, "m": 2000, "n": 5460, "k": 1364,
         "act": "tanh", "dtype": "bf16", "out": "bf16"},
        # the largest: bound by the matrix products
        {"name": "step large", "op": "step", "nets": 1, "shared": False, "m": 8192, "n": 8192, "k": 8192,
         "act": "gauss", "dtype": "bf16", "out": "bf16"},
        # one answer of a network whose outputs are the plane of depths 0..4
        {"name": "sample one row", "op": "sample", "rows": 1, "n": 1364, "dtype": "f32", "temperature": 0.8,
         "top_k": 0, "top_p": 0.95, "min_p": 0.0},
        # a population's answers over the plane of depths 0..5, nothing filtered: every random number is used
        {"name": "sample population", "op": "sample", "rows": 1000, "n": 5460, "dtype": "f32", "temperature": 1.0,
         "top_k": 0, "top_p": 1.0, "min_p": 0.0},
        # answers over the plane of depths 0..7, all filters on
        {"name": "sample depth 7", "op": "sample", "rows": 256, "n": 87380, "dtype": "bf16", "temperature": 0.7,
         "top_k": 50, "top_p": 0.9, "min_p": 0.02},
        # few rows over the plane of depths 0..8: a long axis, and a set of many thousands kept
        {"name": "sample depth 8", "op": "sample", "rows": 24, "n": 349524, "dtype": "f32", "temperature": 1.3,
         "top_k": 0, "top_p": 0.9, "min_p": 0.0},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["product", "product", "step", "sample"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op == "sample":
        rows, n = _log(rng, 1, 1000), _log(rng, 4, 349524)
        n = max(4, min(n, 22_000_000 // rows))
        return {"op": op, "rows": rows, "n": n, "dtype": dtype, "temperature": rng.choice([0.5, 0.7, 1.0, 1.3]),
                "top_k": rng.choice([0, 0, 1, 20, 50, 1000]), "top_p": rng.choice([1.0, 0.95, 0.9, 0.5]),
                "min_p": rng.choice([0.0, 0.0, 0.02, 0.1])}
    act, out = rng.choice(ACTS), rng.choice(["bf16", "f16"])
    nets = rng.choice([1, 1, 1, _log(rng, 2, 150)])
    shared = nets > 1 and rng.random() < 0.5
    if op == "product":
        m, n, k = _log(rng, 1, 94464), _log(rng, 16, 8192), _log(rng, 32, 8192)
        m = max(1, min(m, 170_000_000_000 // (nets * n * k), 130_000_000 // (nets * max(n, k))))
        while nets * n * k > 67_000_000:
            n, k = max(16, n // 2), max(32, k // 2 + 1)
    else:
        m, n, k = _log(rng, 32, 8192), _log(rng, 32, 8192), _log(rng, 32, 8192)
        while nets * max(m * n, n * k, m * k) > 67_000_000:
            m, n, k = m // 2 + 1, n // 2 + 1, k // 2 + 1
    return {"op": op, "nets": nets, "shared": shared, "m": m, "n": n, "k": k, "act": act, "dtype": dtype, "out": out}


# ---- inputs ----------------------------------------------------------------------------------------

def _rand(case, seed):
    """x, w, b, dy of a dense layer, on the GPU: activations with some rows and columns larger than others,
    weights of different size for different outputs."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, nets, m, n, k = TYPES[case["dtype"]], case["nets"], case["m"], case["n"], case["k"]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    x = normal(1 if case["shared"] else nets, m, k)
    x *= torch.exp(0.5 * normal(x.shape[0], m, 1))
    x *= torch.exp(0.5 * normal(1, 1, k))
    w = normal(nets, n, k)
    w *= torch.exp(0.5 * normal(nets, n, 1)) / math.sqrt(2.0 * k)
    b = 0.1 * normal(nets, n)
    s = {"x": x.to(dt), "w": w.to(dt), "b": b}
    if case["op"] == "step":
        dy = normal(nets, m, n)
        dy *= torch.exp(normal(nets, m, 1)) / m
        s["dy"] = dy.to(TYPES[case["out"]])
    return s


def _scores(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rows, n = case["rows"], case["n"]
    scores = 2.5 * torch.randn(rows, n, device="cuda", generator=g)
    noise = torch.empty(rows, n, device="cuda").exponential_(generator=g).clamp_min_(1e-30)
    return {"scores": scores.to(TYPES[case["dtype"]]), "noise": noise}


def prepare(case, seed):
    if case["op"] == "sample":
        return {"case": case, **_scores(case, seed)}
    s = {"case": case, **_rand(case, seed)}
    if own:
        from paper_2608_27612_gb300 import emr
        s["layer"] = emr.DenseLayer(s["w"], s["b"], act=ACTS.index(case["act"]), train=case["op"] == "step")
    elif case["op"] == "product":  # the weights as a program keeps them: codes and one scale for each block
        s["w8"], s["ws"] = _codes(s["w"].float())
    return s


# ---- plain forms -----------------------------------------------------------------------------------

def _codes(v):
    """e4m3 codes [.., blocks, 128] and scales [.., blocks, 1] of v, blocks of 128 along its last axis."""
    c = v.shape[-1]
    v = torch.nn.functional.pad(v, (0, -c % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = v.abs().amax(-1, keepdim=True)
    bits = top.view(torch.int32)
    e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000).int()  # the least e with top <= 448 * 2^e
    e = torch.where(top == 0, torch.zeros_like(e), e.clamp(-126, 127))
    scale = ((e + 127) << 23).view(torch.float32)
    return (v * (1.0 / scale)).to(torch.float8_e4m3fn), scale


def _values(codes, scale, c):
    return (codes.float() * scale).flatten(-2)[..., :c]


def _q8(v):
    """What v is held as: 8-bit values with blocks along the last axis, in 32 bits."""
    return _values(*_codes(v), v.shape[-1])


def _act(z, act):
    """act(z) and act'(z)."""
    if act == "sigmoid":
        y = torch.sigmoid(z)
        return y, y * (1 - y)
    if act == "tanh":
        y = torch.tanh(z)
        return y, 1 - y * y
    if act == "gauss":
        y = torch.exp(-z * z)
        return y, -2 * z * y
    if act == "sin":
        return torch.sin(z), torch.cos(z)
    if act == "abs":
        return z.abs(), torch.sign(z)
    return z, None


def _plain_product(s):
    c = s["case"]
    w = _values(s["w8"], s["ws"], c["k"])
    z = torch.matmul(_q8(s["x"].float()), w.transpose(-1, -2)) + s["b"].unsqueeze(-2)
    return _act(z, c["act"])[0].to(TYPES[c["out"]])


def _plain_step(s):
    c = s["case"]
    out = TYPES[c["out"]]
    w, dy = s["w"].float(), s["dy"].float()
    x = _q8(s["x"].float())
    z = torch.matmul(x, _q8(w).transpose(-1, -2)) + s["b"].unsqueeze(-2)
    y, d = _act(z, c["act"])
    dz = dy if d is None else dy * _q8(d)
    dx = torch.matmul(_q8(dz), _q8(w.transpose(-1, -2)).transpose(-1, -2))
    if c["shared"]:
        dx = dx.sum(0, keepdim=True)
    xt = _q8(x.transpose(-1, -2))
    dw = torch.matmul(_q8(dz.transpose(-1, -2)), xt.transpose(-1, -2))
    return {"y": y.to(out), "dx": dx.to(out), "dw": dw.to(out), "db": dz.sum(-2).to(out)}


def _plain_sample(s):
    c = s["case"]
    v, n = s["scores"].float(), c["n"]
    v, order = torch.sort(v, dim=-1, descending=True, stable=True)
    w = torch.exp((v - v[:, :1]) / c["temperature"])
    keep = torch.ones_like(w, dtype=torch.bool)
    if 0 < c["top_k"] < n:
        keep &= torch.arange(n, device=v.device) < c["top_k"]
    if c["top_p"] < 1:
        mass = torch.where(keep, w, 0.0)
        before = torch.cumsum(mass, -1) - mass
        keep &= before < c["top_p"] * mass.sum(-1, keepdim=True)
    keep &= w >= c["min_p"]
    key = torch.where(keep, w / s["noise"].gather(-1, order), -1.0)
    at = key.argmax(-1, keepdim=True)
    logp = torch.log(w.gather(-1, at) / torch.where(keep, w, 0.0).sum(-1, keepdim=True))
    return {"index": order.gather(-1, at).squeeze(-1).int(), "logp": logp.squeeze(-1)}


def run(state):
    c = state["case"]
    if own:
        from paper_2608_27612_gb300 import emr
        if c["op"] == "sample":
            index, logp = emr.sample(state["scores"], state["noise"], temperature=c["temperature"],
                                     top_k=c["top_k"], top_p=c["top_p"], min_p=c["min_p"])
            return {"index": index, "logp": logp}
        layer, out = state["layer"], TYPES[c["out"]]
        if c["op"] == "product":
            return layer.forward(state["x"], out_dtype=out)
        layer.set_weights(state["w"], state["b"])  # a step follows an update of the weights
        y, saved = layer.forward_train(state["x"], out_dtype=out)
        dx, dw, db = layer.backward(state["dy"], saved, out_dtype=out)
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    if c["op"] == "sample":
        return _plain_sample(state)
    return _plain_product(state) if c["op"] == "product" else _plain_step(state)


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if case["op"] == "sample":
        rows, n, k = case["rows"], case["n"], case["top_k"]
        used = min(n, k) if k else n  # random numbers of what may be kept
        return {"bytes": rows * (n * size[case["dtype"]] + used * 4 + 8), "flops": rows * n * 4}
    nets, m, n, k = case["nets"], case["m"], case["n"], case["k"]
    xs = 1 if case["shared"] else nets
    i, o = size[case["dtype"]], size[case["out"]]
    flops = 2 * nets * m * n * k
    if case["op"] == "product":  # the weights are kept in 8 bits with their scales
        return {"bytes": xs * m * k * i + nets * (n * k * (1 + 1 / BLOCK) + n * 4 + m * n * o), "flops": flops}
    return {"bytes": xs * m * k * (i + o) + nets * (n * k * (i + o) + n * (4 + o) + 2 * m * n * o), "flops": 3 * flops}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _held(v):
    """The 8-bit value of each element of v (64 bits), rounded to nearest even by arithmetic."""
    c = v.shape[-1]
    out = torch.empty_like(v)
    for at in range(0, c, BLOCK):
        u = v[..., at:at + BLOCK]
        top = u.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 448.0))
        e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)
        e = torch.where(top <= 448.0 * torch.exp2(e - 1), e - 1, e)
        scale = torch.exp2(torch.where(top > 0, e.clamp(-126, 127), torch.zeros_like(e)))
        t = u / scale
        _, p = torch.frexp(t)
        step = torch.exp2((p - 1).clamp_min(-6).double() - 3)
        out[..., at:at + BLOCK] = torch.round(t / step) * step * scale
    return out


def _exact_layer(case, seed):
    s = _rand(case, seed)
    x, w = _held(s["x"].double()), s["w"].double()
    z = x @ _held(w).mT + s["b"].double().unsqueeze(-2)
    act = case["act"]
    f = {"identity": lambda t: t, "sigmoid": lambda t: 1 / (1 + torch.exp(-t)), "tanh": torch.tanh,
         "gauss": lambda t: torch.exp(-t ** 2), "sin": torch.sin, "abs": torch.abs}[act]
    y = f(z)
    if case["op"] == "product":
        return y
    dz = s["dy"].double()
    if act != "identity":
        slope = {"sigmoid": lambda t: torch.exp(-t.abs()) / (1 + torch.exp(-t.abs())) ** 2,
                 "tanh": lambda t: 1 / torch.cosh(t) ** 2, "gauss": lambda t: -2 * t * torch.exp(-t ** 2),
                 "sin": torch.cos, "abs": torch.sign}[act]
        dz = dz * _held(slope(z))
    dx = _held(dz) @ _held(w.mT.contiguous()).mT
    dw = _held(dz.mT.contiguous()) @ _held(x.mT.contiguous()).mT
    return {"y": y, "dx": dx.sum(0, keepdim=True) if case["shared"] else dx, "dw": dw, "db": dz.sum(-2)}


def _exact_sample(case, seed):
    s = _scores(case, seed)
    index, logp = [], []
    for v, noise in zip(s["scores"].double(), s["noise"].double()):
        order = torch.argsort(v, descending=True, stable=True)
        p = torch.softmax(v / case["temperature"], 0)[order]
        if case["top_k"]:
            p = p[:case["top_k"]]
        p = p / p.sum()
        if case["top_p"] < 1:
            p = p[:max(1, int((torch.cumsum(p, 0) - p < case["top_p"]).sum()))]
        p = p[p >= case["min_p"] * p[0]]
        order = order[:len(p)]
        at = torch.argmax(p / noise[order])
        index.append(order[at])
        logp.append(torch.log(p[at] / p.sum()))
    return {"index": torch.stack(index).int(), "logp": torch.stack(logp)}


def exact(case, seed):
    return _exact_sample(case, seed) if case["op"] == "sample" else _exact_layer(case, seed)
