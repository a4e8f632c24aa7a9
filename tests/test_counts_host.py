"""Rows and batches of more than 2^31 - 1, which the library counts in 32 bits: refused before anything is allocated or launched, not
taken as another number. Without a GPU: the tensors have a device but no memory."""
import pytest
import torch
from test_dense_devices_host import tensor
from test_scores_devices_host import q4

from paper_2608_27612_gb300 import emr

I, MANY = torch.int32, 2 ** 32 + 1


@pytest.fixture(autouse=True)
def nothing_runs(monkeypatch):
    def launched(*a, **k):
        raise AssertionError("a call of the library")
    emr.lib()
    monkeypatch.setattr(emr, "lib", launched)
    monkeypatch.setattr(emr, "strerror", lambda status: str(status))
    monkeypatch.setattr(emr, "_away", lambda dev, stream: None)


@pytest.mark.parametrize("call", [
    lambda: emr.log_probs(tensor(MANY, 4), tensor(MANY, dtype=I)), lambda: emr.log_probs(tensor(MANY, 4), top=3),
    lambda: emr.log_probs_grad(tensor(MANY, 4), tensor(MANY, dtype=I), 1.0),
    lambda: emr.distill(tensor(MANY, 4), tensor(MANY, 2, dtype=I), tensor(MANY, 2)),
    lambda: emr.distill_grad(tensor(2 ** 31, 4), tensor(2 ** 31, 2, dtype=I), tensor(2 ** 31, 2), 1.0),
    lambda: emr.sample(tensor(MANY, 4), tensor(MANY, 4)),
    lambda: emr.Q4(MANY, 3, 4, device="cpu"), lambda: emr.Q4.of(torch.zeros(1152, dtype=torch.uint8), MANY, 3, 4),
    lambda: emr.q4_quantize(tensor(MANY, 3, 4)), lambda: emr.q4_matmul(tensor(MANY, 3, 4), q4(1, 5, 4))])
def test_counts_that_do_not_fit(call):
    with pytest.raises(emr.EmrError) as e:
        call()
    assert e.value.status == emr.EMR_ERR_RANGE
