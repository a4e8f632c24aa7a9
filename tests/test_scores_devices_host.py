"""Log probabilities, distillation and 4-bit products on a GPU that is not the current one, without a GPU: the calls make the
tensors' GPU current before they allocate or launch, and refuse operands and streams of different GPUs."""
import ctypes as C

import pytest
import torch
from test_dense_devices_host import Entered, Stream, second_gpu, tensor  # noqa: F401

from paper_2608_27612_gb300 import emr

I = torch.int32


def q4(batch, rows, cols, gpu=1):
    q = emr.Q4.__new__(emr.Q4)
    q.batch, q.rows, q.cols, q.group, q.data, q._home = batch, rows, cols, 32, tensor(8, gpu=gpu, dtype=torch.uint8), None
    q.c = emr.Q4C()
    q.ref = C.byref(q.c)
    return q


CALLS = {
    "log_probs": lambda **k: emr.log_probs(tensor(3, 4), tensor(3, dtype=I), tensor(3), 2, **k),
    "log_probs_grad": lambda **k: emr.log_probs_grad(tensor(3, 4), tensor(3, dtype=I), tensor(3), tensor(3), **k),
    "distill": lambda **k: emr.distill(tensor(3, 4), tensor(3, 2, dtype=I), tensor(3, 2), **k),
    "distill_grad": lambda **k: emr.distill_grad(tensor(3, 4), tensor(3, 2, dtype=I), tensor(3, 2), tensor(3), **k),
    "q4_quantize": lambda **k: emr.q4_quantize(tensor(1, 3, 4), **k),
    "q4_pack": lambda **k: emr.q4_pack(tensor(1, 3, 4, dtype=torch.int8), tensor(1, 3, 1, dtype=torch.bfloat16), **k),
    "q4_dequantize": lambda **k: emr.q4_dequantize(q4(1, 3, 4), **k),
    "q4_matmul": lambda **k: emr.q4_matmul(tensor(1, 3, 4), q4(1, 5, 4), tensor(1, 5), **k),
}


@pytest.mark.parametrize("name", CALLS)
def test_the_tensors_gpu_is_made_current(second_gpu, name):  # noqa: F811
    with pytest.raises(Entered) as e:
        CALLS[name]()
    assert e.value.args == (torch.device("cuda", 1),)


@pytest.mark.parametrize("name", CALLS)
def test_a_stream_of_the_tensors_gpu_is_entered(second_gpu, name):  # noqa: F811
    stream = Stream("cuda:1")
    with pytest.raises(Entered) as e:
        CALLS[name](stream=stream)
    assert e.value.args == (stream,)


@pytest.mark.parametrize("name", CALLS)
def test_a_stream_of_another_gpu_is_refused(second_gpu, name):  # noqa: F811
    with pytest.raises(ValueError, match="stream"):
        CALLS[name](stream=Stream("cuda:0"))


def test_operands_on_different_gpus_are_refused(second_gpu):  # noqa: F811
    for call in (lambda: emr.log_probs(tensor(3, 4), tensor(3, gpu=0, dtype=I)), lambda: emr.log_probs(tensor(3, 4), temperature=tensor(3, gpu=0)),
                 lambda: emr.log_probs_grad(tensor(3, 4), tensor(3, dtype=I), tensor(3, gpu=0)),
                 lambda: emr.distill(tensor(3, 4), tensor(3, 2, gpu=0, dtype=I), tensor(3, 2)),
                 lambda: emr.distill(tensor(3, 4), tensor(3, 2, dtype=I), tensor(3, 2, gpu=0)),
                 lambda: emr.distill_grad(tensor(3, 4), tensor(3, 2, dtype=I), tensor(3, 2), tensor(3, gpu=0)),
                 lambda: emr.q4_pack(tensor(1, 3, 4, dtype=torch.int8), tensor(1, 3, 1, gpu=0, dtype=torch.bfloat16)),
                 lambda: emr.q4_matmul(tensor(1, 3, 4), q4(1, 5, 4, gpu=0)), lambda: emr.q4_matmul(tensor(1, 3, 4), q4(1, 5, 4), tensor(1, 5, gpu=0)),
                 lambda: emr.q4_matmul(tensor(1, 3, 4), q4(1, 5, 4), out=tensor(1, 3, 5, gpu=0))):
        with pytest.raises(ValueError):
            call()


def test_operands_in_host_memory_are_refused():
    host = emr.Q4.of(torch.zeros(1152, dtype=torch.uint8), 1, 3, 4)
    for call in (lambda: emr.q4_dequantize(host), lambda: emr.log_probs(torch.zeros(3, 4)), lambda: emr.q4_quantize(torch.zeros(3, 4)),
                 lambda: emr.distill(torch.zeros(3, 4), torch.zeros(3, 2, dtype=I), torch.zeros(3, 2)),
                 lambda: emr.q4_matmul(torch.zeros(3, 4), host)):
        with pytest.raises(ValueError):
            call()
