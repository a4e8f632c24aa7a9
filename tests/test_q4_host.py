"""4-bit weights without a GPU: sizes and refusals of the C ABI, and the float64 definition by hand."""
import ctypes as C

import numpy as np
import pytest

from oracle import q4 as OQ
from paper_2608_27612_gb300 import emr

FAKE = 1 << 20


def sizes(batch, rows, cols, group):
    n = C.c_size_t()
    return emr.lib().emr_q4_size(batch, rows, cols, group, C.byref(n)), n.value


def test_sizes():
    assert sizes(1, 1, 1, 32) == (emr.EMR_OK, 1152)
    assert sizes(3, 17, 257, 64) == (emr.EMR_OK, 3 * 2 * 3 * 1088)
    assert sizes(2, 32, 128, 128) == (emr.EMR_OK, 2 * 2 * 1056)
    for bad in ((0, 1, 1, 32), (1, 0, 1, 32), (1, 1, 0, 32), (1, 1, 1, 16), (1, 1, 1, 0)):
        assert sizes(*bad)[0] == emr.EMR_ERR_ARG
    assert sizes(1, 2 ** 31, 1, 32)[0] == sizes(1, 1, 2 ** 31, 32)[0] == emr.EMR_ERR_RANGE
    assert sizes(2 ** 30, 2 ** 30, 2 ** 30, 32)[0] == emr.EMR_ERR_RANGE


def q4(batch=1, rows=4, cols=5, group=32, data=FAKE):
    return emr.Q4C(batch, group, rows, cols, data)


def test_refusals_come_before_any_launch():
    L = emr.lib()
    bad = [q4(batch=0), q4(rows=0), q4(cols=0), q4(group=48), q4(data=None), q4(data=FAKE + 8)]
    for q in bad:
        assert L.emr_q4_quantize(FAKE, 0, 20, 5, 1, C.byref(q), None) == emr.EMR_ERR_ARG
        assert L.emr_q4_pack(FAKE, 20, 5, 1, FAKE, 4, 1, 1, C.byref(q), None) == emr.EMR_ERR_ARG
        assert L.emr_q4_dequantize(C.byref(q), FAKE, 0, None) == emr.EMR_ERR_ARG
        assert L.emr_q4_matmul(FAKE, 0, 1, 2, 10, 5, 1, C.byref(q), None, 0, FAKE, 0, None, 0, None) == emr.EMR_ERR_ARG
    ref = C.byref(q4())
    far = 3 * FAKE
    for args in ((None, 0, 20, 5, 1), (far, 3, 20, 5, 1), (far + 2, 0, 20, 5, 1), (far, 0, -1, 5, 1), (far, 0, 20, -5, 1), (far, 0, 20, 5, -1),
                 (FAKE + 16, 0, 20, 5, 1), (FAKE - 56, 0, 20, 5, 1)):
        assert L.emr_q4_quantize(*args, ref, None) == emr.EMR_ERR_ARG
    for args in ((None, 20, 5, 1, far, 4, 1, 1), (far, 20, 5, 1, None, 4, 1, 1), (far, 20, 5, 1, far + 1, 4, 1, 1), (far, 20, -5, 1, far, 4, 1, 1),
                 (far, 20, 5, 1, far, 4, -1, 1), (FAKE, 20, 5, 1, far, 4, 1, 1), (far, 20, 5, 1, FAKE, 4, 1, 1)):
        assert L.emr_q4_pack(*args, ref, None) == emr.EMR_ERR_ARG
    assert L.emr_q4_dequantize(ref, None, 0, None) == L.emr_q4_dequantize(ref, far, 7, None) == emr.EMR_ERR_ARG
    assert L.emr_q4_dequantize(ref, far + 1, 1, None) == L.emr_q4_dequantize(ref, FAKE, 0, None) == emr.EMR_ERR_ARG


OK = [3 * FAKE, 0, 3, 2, 10, 5, 1, q4(batch=3), None, 0, 2 * FAKE, 0, None, 0, None]


@pytest.mark.parametrize("i,v,want", [
    (0, None, emr.EMR_ERR_ARG), (0, 3 * FAKE + 2, emr.EMR_ERR_ARG), (1, 3, emr.EMR_ERR_ARG), (2, 0, emr.EMR_ERR_ARG), (2, 2, emr.EMR_ERR_ARG),
    (3, 0, emr.EMR_ERR_ARG), (3, 2 ** 31, emr.EMR_ERR_RANGE), (4, -1, emr.EMR_ERR_ARG), (5, -1, emr.EMR_ERR_ARG), (6, -1, emr.EMR_ERR_ARG),
    (8, FAKE + 2, emr.EMR_ERR_ARG), (9, 6, emr.EMR_ERR_ARG), (9, -1, emr.EMR_ERR_ARG), (10, None, emr.EMR_ERR_ARG), (10, 2 * FAKE + 2, emr.EMR_ERR_ARG), (10, 3 * FAKE + 116, emr.EMR_ERR_ARG), (10, 3 * FAKE - 92, emr.EMR_ERR_ARG),
    (10, FAKE, emr.EMR_ERR_ARG), (10, FAKE - 4, emr.EMR_ERR_ARG),
    (11, -1, emr.EMR_ERR_ARG)])
def test_refusals_of_the_product(i, v, want):
    """Also an output that lies in x or w."""
    args = list(OK)
    args[i] = v
    args[7] = C.byref(args[7])
    assert emr.lib().emr_q4_matmul(*args) == want


def room(dtype, rows, x=FAKE, row_stride=8, q=None):
    n = C.c_size_t()
    q = q or q4()
    return emr.lib().emr_q4_matmul_room(x, dtype, 1, rows, 0, row_stride, 1, C.byref(q), C.byref(n)), n.value


def test_room():
    """Nothing for few rows; else x in tiles of rows rounded up to 16, whole blocks of 128 columns, three parts of float32."""
    assert room(emr.EMR_F32, 16) == room(emr.EMR_BF16, 32, row_stride=5) == room(emr.EMR_F32, 8, q=q4(cols=513)) == (emr.EMR_OK, 0)
    assert room(emr.EMR_F16, 16, q=q4(cols=513)) == (emr.EMR_OK, 0) and room(emr.EMR_F16, 17, q=q4(cols=513)) == (emr.EMR_OK, 5 * 32 * 256)
    assert room(emr.EMR_F32, 17) == (emr.EMR_OK, 3 * 32 * 256) and room(emr.EMR_F32, 9, q=q4(cols=513)) == (emr.EMR_OK, 5 * 3 * 16 * 256) and room(emr.EMR_F32, 65) == (emr.EMR_OK, 2 * 3 * 48 * 256)
    assert room(emr.EMR_BF16, 100, row_stride=5) == room(emr.EMR_F16, 100) == (emr.EMR_OK, 112 * 256)
    assert room(emr.EMR_F16, 129, q=q4(cols=129)) == (emr.EMR_OK, 2 * 2 * 80 * 256)
    assert room(emr.EMR_F32, 0)[0] == room(3, 1)[0] == room(0, 1, q=q4(group=1))[0] == emr.EMR_ERR_ARG
    args = list(OK)
    args[3] = 100
    args[7] = C.byref(args[7])
    assert emr.lib().emr_q4_matmul(*args) == emr.EMR_ERR_ARG              # no workspace
    args[12], args[13] = FAKE, 100
    assert emr.lib().emr_q4_matmul(*args) == emr.EMR_ERR_CAPACITY
    args[12] = FAKE + 8
    assert emr.lib().emr_q4_matmul(*args) == emr.EMR_ERR_ARG


def test_by_hand():
    w = np.zeros(70)
    w[:4] = 7.0, -7.0, 1.5, 2.5
    w[40] = -3.5
    codes, scales = OQ.quantized(w, 32)
    assert scales.tolist() == [1.0, 0.5, 0.0] and codes[:4].tolist() == [7, -7, 2, 2] and codes[40] == -7
    assert OQ.bf16(1 + 2.0 ** -8) == 1 and OQ.bf16(1 + 3 * 2.0 ** -8) == 1 + 2.0 ** -6
    w[1], w[69] = np.inf, 1e-39
    codes, scales = OQ.quantized(w, 32)
    assert np.isnan(scales[0]) and scales[2] == 0 and not codes[:32].any() and codes[69] == 0
    z, mag = OQ.product(np.array([[1.0, 2.0]]), np.array([[3.0, -4.0]]), np.array([[0.5]]), 32, np.array([1.0]))
    assert z == [[-1.5]] and mag == [[6.5]]
