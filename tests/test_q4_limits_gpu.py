"""4-bit weights at the edges of what their calls accept."""
import ctypes as C

import pytest
import torch
from test_dense_limits_gpu import late, normal, taken

from paper_2608_27612_gb300 import emr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("product", [False, True])
@pytest.mark.parametrize("given", [False, True])
def test_weights_may_go_while_another_stream_uses_them(given, product):
    x, w, side = normal(41, 1, 3, 400), normal(42, 1, 3000, 400), torch.cuda.Stream()
    codes, scales = torch.ones(1, 3000, 400, dtype=torch.int8, device="cuda"), torch.ones(1, 3000, 13, dtype=torch.bfloat16, device="cuda")
    q = emr.q4_pack(codes, scales) if given else emr.q4_quantize(w)
    call = (lambda **k: emr.q4_matmul(x, q, **k)) if product else lambda **k: emr.q4_dequantize(q, **k)
    want = call()
    late(side)
    got = call(stream=side)
    n, ptr = q.data.numel(), q.data.data_ptr()
    del q, call
    taken(n, ptr)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,n,k", [(33, 77, 500), (17, 300, 600), (100, 140, 513), (129, 2000, 640), (40, 90, 2000)])
def test_what_the_workspace_held_changes_nothing(m, n, k, dtype):
    """The product's bits, whatever stands in the parts of the workspace that no row of x fills: zeros, NaN, the largest values."""
    q, x, b = emr.q4_quantize(normal(43, 2, n, k), 32), normal(44, 2, m, k, dtype=dtype), normal(45, 2, n)
    args, room = (x.data_ptr(), emr._DTYPES[dtype], 2, m, *x.stride(), q.ref), C.c_size_t()
    assert emr.lib().emr_q4_matmul_room(*args, C.byref(room)) == 0 and room.value > 0
    ws = torch.empty(room.value, dtype=torch.uint8, device="cuda")
    raw = torch.cuda.current_stream().cuda_stream
    for act in range(6):
        outs = []
        for byte in (0, 255, 0x7f, 0x7b):
            ws.fill_(byte)
            outs.append(torch.empty(2, m, n, device="cuda"))
            assert emr.lib().emr_q4_matmul(*args, b.data_ptr(), act, outs[-1].data_ptr(), emr.EMR_F32, ws.data_ptr(), room.value, raw) == 0
        outs.append(emr.q4_matmul(x, q, b, act))
        assert all(torch.equal(outs[0], y) for y in outs[1:]), act
    assert emr.device_error() == 0
