"""4-bit weights at the edges of what their calls accept."""
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
