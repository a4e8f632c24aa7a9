"""A dense HyperNEAT substrate, answered with and trained.

Every genome of a small population gets a network whose weights are its CPPN's outputs: sources on y = -1
connect to every position of a hidden plane, and every hidden position to every position of an answer plane
(emr_eval materialises both weight matrices). The networks run as dense layers in 8-bit floating point, an
answer is a position drawn from the last layer's scores, and some steps of gradient descent then move
every network's answers toward a given position for each pattern.

    python examples/dense_substrate.py
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2608_27612_gb300 import emr  # noqa: E402
from paper_2608_27612_gb300 import workloads as W  # noqa: E402


def positions(depth: int) -> np.ndarray:
    """Coordinates [n, 2] of the grid's positions of depths 0 .. depth, by global index."""
    xy = []
    for g in range(emr.grid_build(depth).n_total):
        d, i, j = emr.index_to_ij(g)
        xy.append(((2 * i + 1) / 2 ** (d + 1) - 1, (2 * j + 1) / 2 ** (d + 1) - 1))
    return np.array(xy, np.float32)


def weights(pop, nodes: np.ndarray, depth: int) -> torch.Tensor:
    """CPPN outputs from every node to every position of a plane: [genome, node, position]."""
    slots = np.concatenate([nodes, np.full((len(nodes), 1), W.SIDE_OUT)], 1)
    dsc = emr.Discovery(pop, W.shared_sources(slots), depth, 0.03, 0.3, materialise=True)
    dsc.run_unfused()
    return dsc.out.view(dsc.P, dsc.S, -1)


def run(genomes: int = 12, patterns: int = 64, steps: int = 30, hidden_depth: int = 1, answer_depth: int = 2, rate: float = 0.5,
        seed: int = 0):
    """Mean log probability of the wanted answers before each step, and the answers drawn last."""
    pop = W.c2(D=answer_depth, P=genomes).pop
    sources = np.stack([np.linspace(-1, 1, 8), np.full(8, -1.0)], 1).astype(np.float32)
    w1 = weights(pop, sources, hidden_depth).transpose(1, 2)                    # [genome, hidden, source]: a view
    w2 = weights(pop, positions(hidden_depth), answer_depth).transpose(1, 2)    # [genome, answer, hidden]
    w1, w2 = w1.clamp(-3, 3).contiguous(), w2.clamp(-3, 3).contiguous()
    b1, b2 = (torch.zeros(w.shape[:2], device="cuda") for w in (w1, w2))
    first = emr.DenseLayer(w1, b1, emr.ACT_TANH, train=True)
    last = emr.DenseLayer(w2, b2, emr.ACT_IDENTITY, train=True)

    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(1, patterns, len(sources), device="cuda", generator=g)      # shared by all networks
    wanted = torch.randint(0, w2.shape[1], (patterns,), device="cuda", generator=g).expand(genomes, patterns)
    history = []
    for _ in range(steps):
        h, kept1 = first.forward_train(x)
        scores, kept2 = last.forward_train(h)
        p = torch.softmax(scores, -1)
        history.append(float(torch.log(p.gather(-1, wanted[..., None])).mean()))
        dy = p.scatter_add(-1, wanted[..., None], torch.full_like(p[..., :1], -1.0)) / patterns
        dh, dw2, db2 = last.backward(dy, kept2)
        _, dw1, db1 = first.backward(dh, kept1)
        for v, d in ((w1, dw1), (b1, db1), (w2, dw2), (b2, db2)):
            v.sub_(rate * d)
        first.set_weights(w1, b1)
        last.set_weights(w2, b2)

    scores = last.forward(first.forward(x)).view(genomes * patterns, -1)
    noise = torch.empty_like(scores).exponential_(generator=g).clamp_min_(1e-30)
    index, logp = emr.sample(scores, noise, temperature=0.7, top_k=20, top_p=0.95)
    return history, index.view(genomes, patterns), logp.view(genomes, patterns), wanted


if __name__ == "__main__":
    history, index, logp, wanted = run()
    print("mean log probability of the wanted answers: %.3f before, %.3f after %d steps" % (history[0], history[-1], len(history)))
    print("drawn answers that are the wanted ones: %.0f%%" % (100 * float((index == wanted).float().mean())))
