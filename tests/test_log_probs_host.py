"""Log probabilities without a GPU: refusals of the C ABI, and the float64 definitions against values worked out by hand."""
import ctypes as C

import numpy as np
import pytest

from oracle import scores as OS
from paper_2608_27612_gb300 import emr

FAKE = 1 << 20
OK = [FAKE, 0, 4, 10, 10, FAKE, None, 1.0, 5, FAKE, FAKE, FAKE, FAKE, None]
GRAD = [FAKE, 0, 4, 10, 10, FAKE, None, 1.0, None, 1.0, None, 0.0, FAKE, FAKE, 2 * FAKE, 0, 10, None]


@pytest.mark.parametrize("i,v,want", [
    (0, None, emr.EMR_ERR_ARG), (0, FAKE + 2, emr.EMR_ERR_ARG), (1, 3, emr.EMR_ERR_ARG), (2, 0, emr.EMR_ERR_ARG),
    (2, 2 ** 27 + 1, emr.EMR_ERR_RANGE), (3, 0, emr.EMR_ERR_ARG), (3, 2 ** 31, emr.EMR_ERR_RANGE), (4, -1, emr.EMR_ERR_ARG),
    (5, None, emr.EMR_ERR_ARG), (5, FAKE + 1, emr.EMR_ERR_ARG), (6, FAKE + 2, emr.EMR_ERR_ARG), (8, -1, emr.EMR_ERR_ARG),
    (8, 257, emr.EMR_ERR_RANGE), (9, FAKE + 1, emr.EMR_ERR_ARG), (10, FAKE + 1, emr.EMR_ERR_ARG), (11, FAKE + 2, emr.EMR_ERR_ARG),
    (12, FAKE + 3, emr.EMR_ERR_ARG)])
def test_refusals_come_before_any_launch(i, v, want):
    args = list(OK)
    args[i] = v
    assert emr.lib().emr_log_probs(*args) == want


def test_nothing_asked_for_is_refused():
    args = list(OK)
    args[8], args[9], args[10] = 0, None, None
    assert emr.lib().emr_log_probs(*args) == emr.EMR_ERR_ARG


@pytest.mark.parametrize("i,v,want", [
    (0, None, emr.EMR_ERR_ARG), (5, None, emr.EMR_ERR_ARG), (8, FAKE + 1, emr.EMR_ERR_ARG), (10, FAKE + 1, emr.EMR_ERR_ARG),
    (14, None, emr.EMR_ERR_ARG), (14, FAKE, emr.EMR_ERR_ARG), (14, FAKE + 156, emr.EMR_ERR_ARG), (14, FAKE - 156, emr.EMR_ERR_ARG),
    (14, 2 * FAKE + 2, emr.EMR_ERR_ARG), (15, 3, emr.EMR_ERR_ARG), (16, 9, emr.EMR_ERR_ARG), (3, 2 ** 31, emr.EMR_ERR_RANGE)])
def test_refusals_of_the_gradient(i, v, want):
    """Also a gradient that would be written over the scores."""
    args = list(GRAD)
    args[i] = v
    if i == 3:
        args[16] = v
    assert emr.lib().emr_log_probs_grad(*args) == want


def test_by_hand():
    s = np.log([1.0, 2.0, 5.0])
    lp = OS.log_p(s)
    assert np.allclose(lp, np.log([0.125, 0.25, 0.625]))
    assert np.isclose(OS.entropy(lp), 0.125 * np.log(8) + 0.25 * np.log(4) + 0.625 * np.log(1.6))
    assert OS.best([1, 3, 3, -np.inf, np.nan, 2], 5).tolist() == [1, 2, 5, 0, -1]
    assert OS.best([0, np.inf, 5, np.inf], 3).tolist() == [1, 3, -1]
    assert OS.log_p([7, 9, 9], 0.0).tolist() == [-np.inf, 0, -np.inf]
    assert np.allclose(OS.log_p_gradient(s, 1, 2.0, 0.0, 0.5), 4 * (np.array([0, 1, 0]) - np.array([1, 4, 25]) / 30))
    assert OS.log_p_gradient([-np.inf, np.nan], 0, 1.0, 1.0).tolist() == [0, 0]


def test_gradients_are_differences():
    g = np.random.default_rng(0)
    s = 2 * g.standard_normal(9)
    s[3] = -np.inf
    for T, t, a, b in ((1.0, 2, 1.0, 0.0), (0.7, 0, -0.5, 0.3), (1.9, -1, 1.0, 1.0), (1.0, 3, 0.0, -2.0)):
        def f(x):
            lp = OS.log_p(x, T)
            return (a * lp[t] if t >= 0 and a else 0.0) + b * OS.entropy(lp)
        want = np.zeros(9)
        for i in range(9):
            if i != 3:
                e = np.zeros(9)
                e[i] = 1e-6
                want[i] = (f(s + e) - f(s - e)) / 2e-6
        assert np.allclose(OS.log_p_gradient(s, t, a, b, T), want, atol=1e-8)
