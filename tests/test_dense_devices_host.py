"""Dense layers and sampling on a GPU that is not the current one, without a GPU: the calls make the tensors' GPU current
before they allocate or launch, and refuse operands and streams of different GPUs. The tensors have a device
but no memory."""
import pytest
import torch

from paper_2608_27612_gb300 import emr


class Entered(Exception):
    pass


class Context:
    def __init__(self, what):
        self.what = what

    def __enter__(self):
        raise Entered(self.what)

    def __exit__(self, *exc):
        return False


class Stream:
    def __init__(self, device):
        self.device, self.cuda_stream = torch.device(device), 1


@pytest.fixture
def second_gpu(monkeypatch):
    """GPU 0 is current; entering a device or a stream raises Entered, any call of the library fails."""
    def launched(*a, **k):
        raise AssertionError("a call before the tensors' GPU was made current")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream("cuda:0"))
    monkeypatch.setattr(torch.cuda, "device", Context)
    monkeypatch.setattr(torch.cuda, "stream", Context)
    monkeypatch.setattr(emr, "lib", launched)
    monkeypatch.setattr(emr, "_lib", None)


class Shell(torch.Tensor):
    """A tensor of a shape, type and device, on which nothing can be computed."""
    @staticmethod
    def __new__(cls, shape, dtype, device):
        return torch.Tensor._make_wrapper_subclass(cls, shape, dtype=dtype, device=device)

    @classmethod
    def __torch_dispatch__(cls, call, types, args=(), kwargs=None):
        raise AssertionError("%s before the tensors' GPU was made current" % call)


def tensor(*shape, gpu=1, dtype=torch.float32):
    return Shell(shape, dtype, "cuda:%d" % gpu)


def q8(batch, rows, cols, gpu=1):
    q = emr.Q8.__new__(emr.Q8)
    q.batch, q.rows, q.cols, q.data = batch, rows, cols, tensor(8, gpu=gpu, dtype=torch.uint8)
    return q


def layer(gpu=1):
    made = emr.DenseLayer.__new__(emr.DenseLayer)
    made.nets, made.n, made.k, made.act, made.train, made.device = 1, 5, 4, emr.ACT_TANH, True, torch.device("cuda", gpu)
    made._room, made._kept, made._back = {}, {}, {}
    return made


CALLS = {
    "q8_quantize": lambda **k: emr.q8_quantize(tensor(1, 3, 4), **k),
    "q8_quantize_held": lambda **k: emr.q8_quantize_held(tensor(1, 3, 4), **k),
    "q8_transpose": lambda **k: emr.q8_transpose(q8(1, 3, 4), **k),
    "q8_dequantize": lambda **k: emr.q8_dequantize(q8(1, 3, 4), **k),
    "q8_matmul": lambda **k: emr.q8_matmul(q8(1, 3, 4), q8(1, 5, 4), tensor(1, 5), **k),
    "q8_slope": lambda **k: emr.q8_slope(tensor(1, 3, 4), q8(1, 3, 4), q8(1, 3, 4), **k),
    "DenseLayer": lambda **k: emr.DenseLayer(tensor(1, 5, 4), **k),
    "set_weights": lambda **k: layer().set_weights(tensor(1, 5, 4), tensor(1, 5), **k),
    "forward": lambda **k: layer().forward(tensor(1, 3, 4), **k),
    "forward_train": lambda **k: layer().forward_train(tensor(1, 3, 4), **k),
    "backward": lambda **k: (lambda made: made.backward(tensor(1, 3, 5), emr.Saved(made, 1, 3, tensor(64, dtype=torch.uint8), 0), **k))(layer()),
    "sample": lambda **k: emr.sample(tensor(3, 4), tensor(3, 4), **k),
}


@pytest.mark.parametrize("name", CALLS)
def test_the_tensors_gpu_is_made_current(second_gpu, name):
    with pytest.raises(Entered) as e:
        CALLS[name]()
    assert e.value.args == (torch.device("cuda", 1),)


@pytest.mark.parametrize("name", CALLS)
def test_a_stream_of_the_tensors_gpu_is_entered(second_gpu, name):
    stream = Stream("cuda:1")
    with pytest.raises(Entered) as e:
        CALLS[name](stream=stream)
    assert e.value.args == (stream,)


@pytest.mark.parametrize("name", CALLS)
def test_a_stream_of_another_gpu_is_refused(second_gpu, name):
    with pytest.raises(ValueError, match="stream"):
        CALLS[name](stream=Stream("cuda:0"))


def test_operands_on_different_gpus_are_refused(second_gpu):
    for call in (lambda: emr.q8_quantize(tensor(1, 3, 4), q8(1, 3, 4, gpu=0)), lambda: emr.q8_quantize(tensor(1, 3, 4), None, q8(1, 4, 3, gpu=0)),
                 lambda: emr.q8_transpose(q8(1, 3, 4), q8(1, 4, 3, gpu=0)), lambda: emr.q8_matmul(q8(1, 3, 4), q8(1, 5, 4, gpu=0)),
                 lambda: emr.q8_matmul(q8(1, 3, 4), q8(1, 5, 4), slope=q8(1, 3, 5, gpu=0)),
                 lambda: emr.q8_slope(tensor(1, 3, 4), q8(1, 3, 4, gpu=0), q8(1, 3, 4)),
                 lambda: emr.q8_slope(tensor(1, 3, 4), None, q8(1, 3, 4, gpu=0)), lambda: emr.q8_slope(tensor(1, 3, 4), None, None, q8(1, 4, 3, gpu=0))):
        with pytest.raises(ValueError, match="one GPU"):
            call()


def test_operands_in_host_memory_are_refused():
    host = emr.Q8.of(torch.zeros(4096, dtype=torch.uint8), 1, 3, 4)
    for call in (lambda: emr.q8_transpose(host), lambda: emr.q8_dequantize(host), lambda: emr.q8_matmul(host, host)):
        with pytest.raises(ValueError, match="one GPU"):
            call()
