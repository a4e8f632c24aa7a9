"""Substrates that learn from larger ones and are served with 4-bit weights.

Every genome of a small population gets two networks, as in dense_substrate.py: a teacher whose hidden plane is
fine and a student whose hidden plane is coarse, with the same sources and the same answer plane. The
teachers' best answers to a set of patterns, with their log probabilities, are kept; the students learn
from those lists alone, and what the lists leave over counts as one more answer. Each student's weights are
then laid down in 4 bits, its answers are drawn from the scores of 4-bit products, and the draws' log
probabilities and entropies are reported.

    python examples/taught_substrate.py
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for path in (ROOT, os.path.join(ROOT, "examples")):
    if path not in sys.path:
        sys.path.insert(0, path)

from dense_substrate import positions, weights  # noqa: E402
from paper_2608_27612_gb300 import emr  # noqa: E402
from paper_2608_27612_gb300 import workloads as W  # noqa: E402


def substrate(pop, sources: np.ndarray, hidden_depth: int, answer_depth: int, train: bool):
    """Both weight matrices of every genome and their two layers."""
    w1 = weights(pop, sources, hidden_depth).transpose(1, 2).clamp(-3, 3).contiguous()
    w2 = weights(pop, positions(hidden_depth), answer_depth).transpose(1, 2).clamp(-3, 3).contiguous()
    return w1, w2, emr.DenseLayer(w1, None, emr.ACT_TANH, train=train), emr.DenseLayer(w2, None, emr.ACT_IDENTITY, train=train)


def serve(w1, w2, group: int = 32):
    """A function that answers patterns with 4-bit copies of the weights."""
    q1, q2 = emr.q4_quantize(w1, group), emr.q4_quantize(w2, group)
    return lambda x: emr.q4_matmul(emr.q4_matmul(x, q1, act=emr.ACT_TANH), q2)


def run(genomes: int = 8, patterns: int = 48, steps: int = 20, top: int = 12, temperature: float = 2.0, rate: float = 0.3, seed: int = 0):
    """Mean loss before each step, the loss of the 4-bit students, and the drawn answers with their log probabilities and entropies."""
    pop = W.c2(D=3, P=genomes).pop
    sources = np.stack([np.linspace(-1, 1, 8), np.full(8, -1.0)], 1).astype(np.float32)
    _, _, first, last = substrate(pop, sources, 2, 3, False)
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(1, patterns, len(sources), device="cuda", generator=g)      # shared by all networks
    rows = genomes * patterns
    best = emr.log_probs(last.forward(first.forward(x)).view(rows, -1), temperature=temperature, top=top)

    w1, w2, first, last = substrate(pop, sources, 1, 3, True)
    history = []
    for _ in range(steps):
        h, kept1 = first.forward_train(x)
        scores, kept2 = last.forward_train(h)
        dy, loss = emr.distill_grad(scores.view(rows, -1), best.top_index, best.top_logp, temperature ** 2 / patterns, temperature)
        history.append(float(loss.mean()))
        dh, dw2, _ = last.backward(dy.view_as(scores), kept2)
        _, dw1, _ = first.backward(dh, kept1)
        for layer, w, d in ((first, w1, dw1), (last, w2, dw2)):
            w.sub_(rate * d)
            layer.set_weights(w)

    scores = serve(w1, w2)(x).view(rows, -1)
    loss = emr.distill(scores, best.top_index, best.top_logp, temperature)
    noise = torch.empty_like(scores).exponential_(generator=g).clamp_min_(1e-30)
    index, logp = emr.sample(scores, noise)
    of = emr.log_probs(scores, index)
    return history, float(loss.mean()), index.view(genomes, patterns), of.logp.view(genomes, patterns), of.entropy.view(genomes, patterns), logp


if __name__ == "__main__":
    history, served, index, logp, entropy, _ = run()
    print("mean divergence from the teachers: %.3f before, %.3f in the last step, %.3f with 4-bit weights" % (history[0], history[-1], served))
    print("mean log probability of the drawn answers %.2f, mean entropy %.2f" % (float(logp.mean()), float(entropy.mean())))
