"""The 4-bit product without a GPU: outputs that lie in memory that the call still reads."""
import ctypes as C

import pytest

from paper_2608_27612_gb300 import emr

FAKE = 1 << 20


# x [3][2][5], w 3 of [4][5], bias [3][4] (48 bytes), out [3][2][4] (96 bytes of float32, 48 of bfloat16)
@pytest.mark.parametrize("dtype,size", [(emr.EMR_F32, 96), (emr.EMR_BF16, 48)])
@pytest.mark.parametrize("rows", [2, 1])
def test_a_bias_in_the_output_is_refused(dtype, size, rows):
    q = emr.Q4C(3, 32, 4, 5, FAKE)
    call = lambda bias, ws=None: emr.lib().emr_q4_matmul(3 * FAKE, 0, 3, rows, 10, 5, 1, C.byref(q), bias, 0, 2 * FAKE, dtype, ws, 0, None)
    for bias in (2 * FAKE, 2 * FAKE + 4, 2 * FAKE - 44, 2 * FAKE + size * rows // 2 - 4):
        assert call(bias) == emr.EMR_ERR_ARG
