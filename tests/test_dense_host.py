"""Dense layers in 8-bit floating point without a GPU: sizes and refusals of the C ABI, and the float64
definitions themselves against values worked out by hand."""
import ctypes as C

import numpy as np
import pytest

from oracle import dense as OD
from paper_2608_27612_gb300 import emr


def sizes(batch, rows, cols):
    v, s = C.c_size_t(), C.c_size_t()
    return emr.lib().emr_q8_size(batch, rows, cols, C.byref(v), C.byref(s)), v.value, s.value


def test_sizes():
    assert sizes(1, 1, 1) == (emr.EMR_OK, 128, 512)
    assert sizes(3, 128, 512) == (emr.EMR_OK, 3 * 128 * 512, 3 * 512)
    assert sizes(2, 129, 513) == (emr.EMR_OK, 2 * 129 * 640, 2 * 2 * 2 * 512)
    assert sizes(0, 1, 1)[0] == emr.EMR_ERR_ARG and sizes(1, 0, 1)[0] == emr.EMR_ERR_ARG
    assert sizes(1, 1, 2 ** 31)[0] == emr.EMR_ERR_RANGE
    assert sizes(2 ** 30, 2 ** 30, 2 ** 30)[0] == emr.EMR_ERR_RANGE
    n = C.c_size_t()
    assert emr.lib().emr_q8_slope_workspace_size(2, 129, 7, C.byref(n)) == emr.EMR_OK and n.value == 2 * 2 * 7 * 4
    assert emr.lib().emr_q8_slope_workspace_size(1, 1, 0, C.byref(n)) == emr.EMR_ERR_ARG


def test_refusals_come_before_any_launch():
    L, fake = emr.lib(), C.c_void_p(1 << 20)
    q = emr.Q8C(1, 0, 4, 4, 1 << 20, 1 << 20)
    bad = emr.Q8C(1, 0, 4, 4, (1 << 20) + 8, 1 << 20)
    none = emr.Q8C(1, 0, 4, 4, None, 1 << 20)
    big = emr.Q8C(1, 0, 4, 2 ** 31, 1 << 20, 1 << 20)
    quant = lambda src=fake, dt=0, b=1, r=4, c=4, rs=4, cs=1, q=q, qt=None: L.emr_q8_quantize(
        src, dt, b, r, c, 16, rs, cs, C.byref(q) if q else None, C.byref(qt) if qt else None, None)
    for kw in (dict(src=None), dict(dt=3), dict(b=0), dict(r=0), dict(c=-1), dict(rs=-4), dict(q=None), dict(q=bad),
               dict(q=none), dict(r=5), dict(src=C.c_void_p((1 << 20) + 2))):
        assert quant(**kw) == emr.EMR_ERR_ARG, kw
    assert quant(c=2 ** 31) == emr.EMR_ERR_RANGE
    mm = lambda a=q, w=q, act=0, out=fake, dt=0: L.emr_q8_matmul(C.byref(a), C.byref(w), None, act, 0, out, dt, None, None)
    for kw in (dict(a=bad), dict(w=none), dict(act=-1), dict(act=6), dict(out=None), dict(dt=5), dict(a=big, w=big),
               dict(out=C.c_void_p((1 << 20) + 1))):
        assert mm(**kw) == emr.EMR_ERR_ARG, kw
    assert L.emr_q8_slope(fake, 0, 1, 4, 4, None, C.byref(q), None, fake, 0, fake, 0, None) == emr.EMR_ERR_CAPACITY
    assert L.emr_q8_slope(fake, 0, 1, 4, 4, None, None, None, None, 0, None, 0, None) == emr.EMR_ERR_ARG
    assert L.emr_q8_transpose(C.byref(q), C.byref(none), None) == emr.EMR_ERR_ARG
    assert L.emr_q8_dequantize(C.byref(q), None, 0, None) == emr.EMR_ERR_ARG
    assert L.emr_device_error(None, None) == emr.EMR_ERR_ARG


@pytest.mark.parametrize("v,want", [(0.0, 0.0), (1.0, 1.0), (1.0625, 1.0), (1.1875, 1.25), (17.0, 16.0), (19.0, 20.0),
                                    (447.0, 448.0), (-432.0, -448.0), (-431.0, -416.0), (2.0 ** -9, 2.0 ** -9),
                                    (2.0 ** -10, 0.0), (3 * 2.0 ** -10, 2.0 ** -8), (2.0 ** -6 * 1.0625, 2.0 ** -6)])
def test_e4m3_rounding_by_hand(v, want):
    assert OD.e4m3(v) == want


def test_every_e4m3_value_is_its_own_rounding():
    codes = np.arange(127)                            # 0 .. 0x7e: the finite non-negative codes
    e, f = codes >> 3, codes & 7
    vals = np.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * 2.0 ** (e - 7.0))
    assert vals[-1] == 448.0 and np.array_equal(OD.e4m3(vals), vals) and np.array_equal(OD.e4m3(-vals), -vals)
    mid = (vals[1:] + vals[:-1]) / 2                  # ties go to the even code
    assert np.array_equal(OD.e4m3(mid), vals[(codes[:-1] + 1) // 2 * 2])


def test_block_scales_by_hand():
    x = np.zeros(300)
    x[0], x[130], x[299] = 448.0, -449.0, 1.0
    assert np.array_equal(OD.block_scales(x), [1.0, 2.0, 2.0 ** -8])
    assert np.array_equal(OD.block_scales(np.zeros(5)), [1.0])
    assert np.array_equal(OD.block_scales(np.array([1e-300])), [2.0 ** -126])
    assert np.array_equal(OD.block_scales(np.array([np.inf, 896.0, np.nan])), [2.0])
    h = OD.held(np.array([np.inf, 896.0, np.nan, 33.0]))
    assert np.isnan(h[0]) and np.isnan(h[2]) and h[1] == 896.0 and h[3] == 32.0


def test_slopes_are_differences():
    z = np.linspace(-4, 4, 41) + 0.01
    for name in OD.ACTS:
        d = (OD.act(z + 1e-6, name) - OD.act(z - 1e-6, name)) / 2e-6
        assert np.allclose(d, OD.slope(z, name), atol=1e-8)
