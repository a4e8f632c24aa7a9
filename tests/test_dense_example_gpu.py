"""The dense substrate example end to end: CPPN outputs as weights, answers drawn, gradient steps."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle
from paper_2608_27612_gb300 import workloads as W

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("dense_substrate", os.path.join(ROOT, "examples", "dense_substrate.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_weights_are_the_oracles_outputs():
    m = example()
    pop = W.c2(D=1, P=4).pop
    nodes = m.positions(0)
    assert nodes.shape == (4, 2) and np.all(np.abs(nodes) == 0.5)
    got = m.weights(pop, nodes, 1).cpu().numpy()
    slots = W.shared_sources([(x, y, W.SIDE_OUT) for x, y in nodes])
    ora = oracle.discover(pop, slots, 1, 0.03, 0.3, fields=("w", "w_err"))
    want, err = ora["w"].reshape(got.shape), ora["w_err"].reshape(got.shape)
    assert np.all(np.abs(got - want) <= 1e-5 + 1e-4 * np.abs(want) + err)


def test_steps_raise_the_probability_of_the_wanted_answers():
    history, index, logp, wanted = example().run(steps=20)
    assert np.isfinite(history).all() and history[-1] > history[0] + 0.2
    assert index.shape == wanted.shape and int(index.min()) >= 0 and int(index.max()) < 84
    assert bool((logp <= 0).all()) and bool(torch.isfinite(logp).all())
