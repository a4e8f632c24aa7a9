"""Measured cases of the operators on scores and of the product with 4-bit weights.

Four operators, which follow one another when a large substrate teaches a small one and that one is served:

logp       log probabilities of given answers from rows of scores, the rows' entropies, and the best answers.
logp_step  the gradient of given log probabilities and entropies with respect to the scores, and their values.
distill    the loss of a student's scores against the best answers of a teacher, and its gradient.
q4         y = act(x W^T + b) with W in 4 bits, one scale for each group of its columns, sums in 32 bits.

`run` computes them in plain 32-bit torch operations, or with the framework's calls where `own` is true.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ("identity", "sigmoid", "tanh", "gauss", "sin", "abs")


# ---- cases ---------------------------------------------------------------------------------------

def listed():
    return [
        # one answer over the plane of depths 0..4 and its five best alternatives: the time of a launch
        {"name": "logp one row", "op": "logp", "rows": 1, "n": 1364, "dtype": "f32", "temperature": 1.0, "top": 5},
        # a population's answers over the plane of depths 0..5 with the alternatives that a teacher keeps
        {"name": "logp population", "op": "logp", "rows": 4000, "n": 5460, "dtype": "f32", "temperature": 0.7, "top": 20},
        # few rows over the plane of depths 0..8: a long axis, and many equal scores in 16 bits
        {"name": "logp depth 8", "op": "logp", "rows": 24, "n": 349524, "dtype": "bf16", "temperature": 1.0, "top": 100},
        # 64 networks trained on 250 patterns: many short rows
        {"name": "logp step short rows", "op": "logp_step", "rows": 16000, "n": 340, "dtype": "bf16", "temperature": 1.0,
         "entropy": False},
        # long rows with an entropy term, the largest of the gradients in 32 bits
        {"name": "logp step depth 7", "op": "logp_step", "rows": 512, "n": 87380, "dtype": "f32", "temperature": 1.3,
         "entropy": True},
        # a small student and 16 answers of its teacher
        {"name": "distill small", "op": "distill", "rows": 250, "n": 1364, "k": 16, "dtype": "f32", "temperature": 2.0,
         "tail": False},
        # an ordinary batch
        {"name": "distill ordinary", "op": "distill", "rows": 2000, "n": 5460, "k": 50, "dtype": "bf16", "temperature": 1.0,
         "tail": True},
        # long rows, the whole of what the teacher left out as one answer
        {"name": "distill depth 7", "op": "distill", "rows": 1000, "n": 87380, "k": 64, "dtype": "f16", "temperature": 1.5,
         "tail": True},
        # one pattern from the plane of depths 0..4 to that of depths 0..5
        {"name": "q4 one pattern", "op": "q4", "nets": 1, "shared": False, "m": 1, "n": 5460, "k": 1364, "group": 32,
         "act": "tanh", "dtype": "f32", "out": "f32"},
        # 150 networks with weights of their own answer the same four patterns
        {"name": "q4 population", "op": "q4", "nets": 150, "shared": True, "m": 4, "n": 1364, "k": 256, "group": 64,
         "act": "sigmoid", "dtype": "f16", "out": "f32"},
        # a few patterns through a wide layer
        {"name": "q4 eight patterns", "op": "q4", "nets": 1, "shared": False, "m": 8, "n": 8192, "k": 8192, "group": 128,
         "act": "gauss", "dtype": "bf16", "out": "bf16"},
        # an odd number of rows, the most for which reading the weights counts
        {"name": "q4 hundred patterns", "op": "q4", "nets": 1, "shared": False, "m": 101, "n": 16384, "k": 8192, "group": 128,
         "act": "identity", "dtype": "bf16", "out": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logp", "logp_step", "distill", "q4"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op == "q4":
        nets = rng.choice([1, 1, _log(rng, 2, 150)])
        m, n, k = _log(rng, 1, 101), _log(rng, 16, 16384), _log(rng, 32, 8192)
        while nets * n * k > 134_000_000:
            n, k = max(16, n // 2), max(32, k // 2 + 1)
        m = max(1, min(m, 13_000_000_000 // (nets * n * k)))
        return {"op": op, "nets": nets, "shared": nets > 1 and rng.random() < 0.5, "m": m, "n": n, "k": k,
                "group": rng.choice([32, 64, 128]), "act": rng.choice(ACTS), "dtype": dtype,
                "out": rng.choice(["f32", "bf16", "f16"])}
    rows, n = _log(rng, 1, 16000), _log(rng, 4, 349524)
    rows = max(1, min(rows, {"logp": 21_000_000, "logp_step": 44_000_000, "distill": 87_000_000}[op] // n))
    case = {"op": op, "rows": rows, "n": n, "dtype": dtype, "temperature": rng.choice([0.5, 0.7, 1.0, 1.3, 2.0])}
    if op == "logp":
        case["top"] = min(n, rng.choice([0, 1, 5, 20, 100]))
    elif op == "logp_step":
        case["entropy"] = rng.random() < 0.5
    else:
        case["k"], case["tail"] = min(max(1, n // 4), _log(rng, 1, 128)), rng.random() < 0.6
    return case


# ---- inputs ----------------------------------------------------------------------------------------

def _scores(case, g):
    """Rows of scores; a quarter of the rows ends early: what lies past their end is masked."""
    rows, n = case["rows"], case["n"]
    v = 2.5 * torch.randn(rows, n, device="cuda", generator=g)
    end = torch.randint((n + 1) // 2, 4 * n, (rows, 1), device="cuda", generator=g)
    masked = torch.arange(n, device="cuda") >= end
    return v.masked_fill_(masked, -math.inf), masked


def _loss_scale(case):
    """A mean over the rows; gradients of type f16 are taken of a loss scaled up, as they would be 0 without that."""
    return 256.0 if case["dtype"] == "f16" else 1.0 / case["rows"]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["op"] == "q4":
        dt, nets, m, n, k = TYPES[case["dtype"]], case["nets"], case["m"], case["n"], case["k"]
        x = torch.randn(1 if case["shared"] else nets, m, k, device="cuda", generator=g)
        x *= torch.exp(0.5 * torch.randn(x.shape[0], m, 1, device="cuda", generator=g))
        codes = torch.randn(nets, n, k, device="cuda", generator=g).mul_(3).round_().clamp_(-8, 7).to(torch.int8)
        groups = (k + case["group"] - 1) // case["group"]
        scales = torch.exp(0.5 * torch.randn(nets, n, groups, device="cuda", generator=g)) / (3 * math.sqrt(k))
        return {"x": x.to(dt), "codes": codes, "scales": scales.to(torch.bfloat16),
                "b": 0.1 * torch.randn(nets, n, device="cuda", generator=g)}
    rows, n = case["rows"], case["n"]
    v, masked = _scores(case, g)
    s = {"scores": v.to(TYPES[case["dtype"]])}
    if case["op"] == "distill":  # the teacher's scores are like the student's
        t = v * 1.2 + torch.randn(rows, n, device="cuda", generator=g)
        l = t / case["temperature"]
        l = l - torch.logsumexp(l, -1, keepdim=True)
        s["logp"], index = torch.topk(l, case["k"], -1)
        s["index"] = index.int()
        s["dloss"] = torch.rand(rows, device="cuda", generator=g) * _loss_scale(case)
        return s
    # given answers: among the likely ones of a row
    pick = v.clone().add_(torch.empty_like(v).exponential_(generator=g).clamp_min_(1e-30).log_(), alpha=-2.0)
    s["targets"] = pick.argmax(-1).int()
    if case["op"] == "logp_step":
        s["dlogp"] = torch.randn(rows, device="cuda", generator=g) * _loss_scale(case)
        s["dentropy"] = 0.1 * torch.rand(rows, device="cuda", generator=g) * _loss_scale(case) if case["entropy"] else None
    return s


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if own and case["op"] == "q4":
        from paper_2608_27612_gb300 import emr
        s["w"] = emr.q4_pack(s.pop("codes"), s.pop("scales"), case["group"])
    return s


# ---- plain forms -----------------------------------------------------------------------------------

def _act(z, act):
    if act == "sigmoid":
        return torch.sigmoid(z)
    if act == "tanh":
        return torch.tanh(z)
    if act == "gauss":
        return torch.exp(-z * z)
    if act == "sin":
        return torch.sin(z)
    return z.abs() if act == "abs" else z


def _plain_q4(s):
    c = s["case"]
    scale = torch.repeat_interleave(s["scales"].float(), c["group"], -1)[..., :c["k"]]
    w = s["codes"].float() * scale
    z = torch.matmul(s["x"].float(), w.transpose(-1, -2)) + s["b"].unsqueeze(-2)
    return _act(z, c["act"]).to(TYPES[c["out"]])


def _log_softmax(scores, T):
    d = scores.float()
    d = (d - d.amax(-1, keepdim=True)) / T
    return d - torch.log(torch.exp(d).sum(-1, keepdim=True))


def _terms(w, l):
    """w times l, 0 where w is."""
    return torch.where(w > 0, w * l, 0.0)


def _plain_logp(s):
    c = s["case"]
    l = _log_softmax(s["scores"], c["temperature"])
    p = torch.exp(l)
    out = {"logp": l.gather(-1, s["targets"].long().unsqueeze(-1)).squeeze(-1), "entropy": -_terms(p, l).sum(-1)}
    if c["op"] == "logp":
        if c["top"]:
            v, order = torch.sort(s["scores"], dim=-1, descending=True, stable=True)
            order = order[:, :c["top"]]
            kept = v[:, :c["top"]] > -math.inf
            out["top_index"] = torch.where(kept, order, -1).int()
            out["top_logp"] = l.gather(-1, order)
        return out
    d = -s["dlogp"].unsqueeze(-1) * p
    if c["entropy"]:
        d = d - s["dentropy"].unsqueeze(-1) * _terms(p, l + out["entropy"].unsqueeze(-1))
    d = d.scatter_add(-1, s["targets"].long().unsqueeze(-1), s["dlogp"].unsqueeze(-1))
    out["dscores"] = (d / c["temperature"]).to(s["scores"].dtype)
    return out


def _plain_distill(s):
    """The loss is a small difference of sums of about 1, and what a teacher leaves over one of two: those are taken in 64 bits."""
    c = s["case"]
    index = s["index"].long()
    scores = s["scores"].float()
    top = scores.amax(-1, keepdim=True)
    e = torch.exp((scores - top) / c["temperature"])
    z = e.sum(-1, keepdim=True, dtype=torch.float64)
    lp = (scores.gather(-1, index).double() - top.double()) / c["temperature"] - torch.log(z)
    lt = s["logp"].double()
    if not c["tail"]:
        lt = lt - torch.log(torch.exp(lt).sum(-1, keepdim=True))
    t = torch.exp(lt)
    loss = _terms(t, lt - lp).sum(-1, keepdim=True)
    mass = t.sum(-1, keepdim=True)
    if c["tail"]:
        rest = e.scatter(-1, index, 0.0)
        z_rest = rest.sum(-1, keepdim=True, dtype=torch.float64)
        t_rest = torch.where(z_rest > 0, (1 - mass).clamp_min(0.0), 0.0)
        loss = loss + _terms(t_rest, torch.log(t_rest) - torch.log(z_rest) + torch.log(z))
        over = torch.where(t_rest > 0, t_rest / z_rest, 0.0)
        grad = ((mass + t_rest) / z).float() * e - over.float() * rest
    else:
        grad = (mass / z).float() * e
    grad = grad.scatter_add(-1, index, -t.float()) * (s["dloss"].unsqueeze(-1) / c["temperature"])
    return {"loss": loss.squeeze(-1).float(), "dscores": grad.to(s["scores"].dtype)}


def run(state):
    c = state["case"]
    if own:
        from paper_2608_27612_gb300 import emr
        if c["op"] == "q4":
            return emr.q4_matmul(state["x"], state["w"], state["b"], act=ACTS.index(c["act"]), out_dtype=TYPES[c["out"]])
        T = c["temperature"]
        if c["op"] == "distill":
            dscores, loss = emr.distill_grad(state["scores"], state["index"], state["logp"], state["dloss"], temperature=T,
                                             tail=c["tail"])
            return {"loss": loss, "dscores": dscores}
        if c["op"] == "logp_step":
            dscores, logp, entropy = emr.log_probs_grad(state["scores"], state["targets"], state["dlogp"], state["dentropy"],
                                                        temperature=T)
            return {"logp": logp, "entropy": entropy, "dscores": dscores}
        r = emr.log_probs(state["scores"], state["targets"], temperature=T, top=c["top"])
        out = {"logp": r.logp, "entropy": r.entropy}
        if c["top"]:
            out["top_index"], out["top_logp"] = r.top_index, r.top_logp
        return out
    if c["op"] == "q4":
        return _plain_q4(state)
    return _plain_distill(state) if c["op"] == "distill" else _plain_logp(state)


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    i = size[case["dtype"]]
    if case["op"] == "q4":
        nets, m, n, k, g = case["nets"], case["m"], case["n"], case["k"], case["group"]
        xs = 1 if case["shared"] else nets
        weights = nets * n * (k / 2 + 2 * ((k + g - 1) // g) + 4)
        return {"bytes": xs * m * k * i + weights + nets * m * n * size[case["out"]], "flops": 2 * nets * m * n * k}
    rows, n = case["rows"], case["n"]
    if case["op"] == "logp":
        return {"bytes": rows * (n * i + 12 + 8 * case["top"]), "flops": 6 * rows * n}
    if case["op"] == "logp_step":
        return {"bytes": rows * (2 * n * i + 20), "flops": 10 * rows * n}
    return {"bytes": rows * (2 * n * i + 8 + 8 * case["k"]), "flops": 9 * rows * n}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _exact_q4(case, s):
    f = {"identity": lambda t: t, "sigmoid": lambda t: 1 / (1 + torch.exp(-t)), "tanh": torch.tanh,
         "gauss": lambda t: torch.exp(-t ** 2), "sin": torch.sin, "abs": torch.abs}[case["act"]]
    x, g, k = s["x"].double(), case["group"], case["k"]
    y = []
    for net in range(case["nets"]):
        z = s["b"][net].double()
        for j in range(0, k, 16 * g):  # sixteen groups of columns at a time
            w = s["codes"][net, :, j:j + 16 * g].double()
            w = torch.nn.functional.pad(w, (0, -w.shape[1] % g)).unflatten(1, (-1, g))
            w = (w * s["scales"][net, :, j // g:j // g + 16, None].double()).flatten(1)[:, :min(k - j, 16 * g)]
            z = z + x[0 if case["shared"] else net, :, j:j + 16 * g] @ w.T
        y.append(f(z))
    return torch.stack(y)


def _exact_rows(case, s):
    T = case["temperature"]
    found = {}

    def add(**row):
        for name, v in row.items():
            found.setdefault(name, []).append(v)

    for r in range(case["rows"]):
        v = s["scores"][r].double()
        l = torch.log_softmax(v / T, 0)
        p = torch.softmax(v / T, 0)
        if case["op"] == "distill":
            at, lt = s["index"][r].long(), s["logp"][r].double()
            hot = torch.zeros_like(p)
            if case["tail"]:
                t = lt.exp()
                over = torch.ones_like(p, dtype=torch.bool)
                over[at] = False
                t_rest, rest = (1 - t.sum()).clamp(min=0), torch.where(over, p, torch.zeros_like(p))
                loss = torch.special.xlogy(t, t).sum() - (t * l[at]).nan_to_num(0.0).sum()
                if t_rest > 0:
                    loss = loss + t_rest * (t_rest.log() - torch.logsumexp(torch.where(over, l, -math.inf), 0))
                    hot = t_rest * rest / rest.sum()
                mass = t.sum() + t_rest
            else:
                t, mass = torch.softmax(lt, 0), 1.0
                loss = (torch.special.xlogy(t, t) - (t * l[at]).nan_to_num(0.0)).sum()
            hot[at] += t
            add(loss=loss, dscores=s["dloss"][r].double() * (mass * p - hot) / T)
            continue
        t = int(s["targets"][r])
        entropy = torch.special.entr(p).sum()
        add(logp=l[t], entropy=entropy)
        if case["op"] == "logp":
            if case["top"]:
                order = torch.argsort(v, descending=True, stable=True)[:case["top"]]
                add(top_index=torch.where(v[order] > -math.inf, order, -1).int(), top_logp=l[order])
            continue
        a, b = s["dlogp"][r].double(), s["dentropy"][r].double() if case["entropy"] else 0.0
        d = -a * p + b * (torch.special.entr(p) - p * entropy)
        d[t] += a
        add(dscores=d / T)
    return {name: torch.stack(v) for name, v in found.items()}


def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_q4(case, s) if case["op"] == "q4" else _exact_rows(case, s)
