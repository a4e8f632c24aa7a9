"""The example of substrates that learn from larger ones and are served in 4 bits, end to end, and the gradient of its loss."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import scores as OS
from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("taught_substrate", os.path.join(ROOT, "examples", "taught_substrate.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_runs():
    history, served, index, logp, entropy, drawn = example().run(steps=4)
    assert len(history) == 4 and np.isfinite(history).all() and np.isfinite(served) and min(history) > 0
    assert index.shape == logp.shape == entropy.shape and int(index.min()) >= 0 and int(index.max()) < 340
    assert bool((logp <= 0).all()) and bool((entropy >= 0).all()) and float(entropy.max()) <= np.log(340) + 1e-4
    assert torch.allclose(logp.view(-1), drawn, atol=2e-5)


def test_gradient_of_a_step():
    """The scores' gradient against central differences of the loss in float64, in random directions: the example's own sizes."""
    g = torch.Generator(device="cuda").manual_seed(3)
    scores = torch.randn(48, 340, device="cuda", generator=g)
    best = emr.log_probs(torch.randn(48, 340, device="cuda", generator=g) * 2, temperature=2.0, top=12)
    dy, loss = emr.distill_grad(scores, best.top_index, best.top_logp, 4.0 / 48, 2.0)
    s, i, l = scores.double().cpu().numpy(), best.top_index.cpu().numpy(), best.top_logp.double().cpu().numpy()
    rng = np.random.default_rng(0)
    for r in (0, 17, 47):
        v = rng.standard_normal(340)
        h = 1e-5
        up, down = (OS.distill(s[r] + d * v, i[r], l[r], 2.0)[0] for d in (h, -h))
        # differences: h^2 third derivatives (|v|^3 / 8 < 1,000) and 1e-15 / h; the kernel: 2e-5 * 3 / 2 an entry
        assert abs(float(dy[r].double().cpu().numpy() @ v) * 12 - (up - down) / (2 * h)) <= 3e-5 * np.abs(v).sum() + 1e-6
