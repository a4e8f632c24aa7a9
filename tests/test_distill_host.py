"""Distillation without a GPU: refusals of the C ABI, and the float64 definition by hand and by differences."""
import numpy as np
import pytest

from oracle import scores as OS
from paper_2608_27612_gb300 import emr

FAKE = 1 << 20
#     scores     rows n  stride index teacher    k     T        tail dloss     loss  dscores
OK = [FAKE, 0, 4, 10, 10, FAKE, FAKE, 0, 5, None, 1.0, 1, None, 1.0, FAKE, 2 * FAKE, 0, 10, None]


@pytest.mark.parametrize("i,v,want", [
    (0, None, emr.EMR_ERR_ARG), (0, FAKE + 2, emr.EMR_ERR_ARG), (1, 3, emr.EMR_ERR_ARG), (2, 0, emr.EMR_ERR_ARG),
    (2, 2 ** 27 + 1, emr.EMR_ERR_RANGE), (3, 0, emr.EMR_ERR_ARG), (4, -1, emr.EMR_ERR_ARG), (5, None, emr.EMR_ERR_ARG),
    (5, FAKE + 2, emr.EMR_ERR_ARG), (6, None, emr.EMR_ERR_ARG), (6, FAKE + 2, emr.EMR_ERR_ARG), (7, 4, emr.EMR_ERR_ARG),
    (8, 0, emr.EMR_ERR_ARG), (8, 257, emr.EMR_ERR_RANGE), (9, FAKE + 1, emr.EMR_ERR_ARG), (10, 0.0, emr.EMR_ERR_ARG),
    (10, float("nan"), emr.EMR_ERR_ARG), (12, FAKE + 2, emr.EMR_ERR_ARG), (14, FAKE + 2, emr.EMR_ERR_ARG),
    (15, 2 * FAKE + 2, emr.EMR_ERR_ARG), (15, FAKE + 100, emr.EMR_ERR_ARG), (16, 3, emr.EMR_ERR_ARG), (17, 9, emr.EMR_ERR_ARG)])
def test_refusals_come_before_any_launch(i, v, want):
    args = list(OK)
    args[i] = v
    assert emr.lib().emr_distill(*args) == want


def test_nothing_asked_for_is_refused():
    args = list(OK)
    args[14] = args[15] = None
    assert emr.lib().emr_distill(*args) == emr.EMR_ERR_ARG


def test_by_hand():
    s = np.log([1.0, 1.0, 2.0, 4.0])
    loss, g, _ = OS.distill(s, [3, 0, -1], np.log([0.5, 0.25, 9.0]))
    assert np.isclose(loss, 0.25 * np.log(2) + 0.25 * np.log(0.25 / 0.375))
    assert np.allclose(g, [0.125 - 0.25, 0.125 * (1 - 0.25 / 0.375), 0.25 * (1 - 0.25 / 0.375), 0.0])
    loss, g, _ = OS.distill(s, [3, 0], np.log([4.0, 1.0]), tail=False)
    assert np.isclose(loss, 0.8 * np.log(0.8 / 0.5) + 0.2 * np.log(0.2 / 0.125))
    assert np.allclose(g, [0.125 - 0.2, 0.125, 0.25, 0.5 - 0.8])
    assert OS.distill(s, [-1, -1], [0.0, 0.0])[0] == 0 and np.isnan(OS.distill(s, [4], [0.0])[0])


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [1.0, 0.6])
def test_gradients_are_differences(tail, T):
    g = np.random.default_rng(0)
    s = 2 * g.standard_normal(9)
    s[3] = -np.inf
    index, l = [5, 1, 5, -1, 7], np.log([0.3, 0.2, 0.1, 0.5, 0.05])
    want = np.zeros(9)
    for i in range(9):
        if i != 3:
            e = np.zeros(9)
            e[i] = 1e-6
            want[i] = (OS.distill(s + e, index, l, T, tail)[0] - OS.distill(s - e, index, l, T, tail)[0]) / 2e-6
    assert np.allclose(OS.distill(s, index, l, T, tail)[1], want, atol=1e-8)
