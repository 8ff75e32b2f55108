"""The binding's own refusals for the training-step operators, without a GPU: MistError, before the library is called."""
import types

import pytest

from paper_2503_19050_amd import mist


@pytest.fixture(scope="module")
def torch():
    return mist._torch()


def refused(call):
    with pytest.raises(mist.MistError) as e:
        call()
    assert e.value.status == mist.E_INVALID and str(e.value)


def test_host_tensors_are_refused(torch):
    ids, table, grad = torch.zeros(2, 3, dtype=torch.int64), torch.zeros(5, 8), torch.zeros(2, 3, 8)
    for call in (lambda: mist.embed(ids, table), lambda: mist.embed(ids, table, out=grad), lambda: mist.embed(ids, table, pos=grad[0]),
                 lambda: mist.embed_grad(ids, grad, table), lambda: mist.TensorList([table]),
                 lambda: mist.StepRecord(device="cpu")):
        refused(call)


def test_a_step_count_below_zero_is_refused(torch):
    """Its bias correction would divide by 1 - beta^0 or less."""
    refused(lambda: mist.StepRecord(step=-1))


def test_a_stream_of_another_device_is_refused(torch):
    here, there = torch.device("cuda", 0), torch.device("cuda", 1)
    stream = types.SimpleNamespace(device=there, cuda_stream=64)
    refused(lambda: mist._stream_of(torch, stream, here))
    assert mist._stream_of(torch, stream, there) == (64, stream)


def test_a_lookup_that_autograd_would_lose_is_refused(torch):
    """The result has no graph: a table or positions that require a gradient are taken where none is recorded."""
    ids, table, pos = torch.zeros(2, 3, dtype=torch.int64), torch.zeros(5, 8, requires_grad=True), torch.zeros(3, 8, requires_grad=True)
    for call in (lambda: mist.embed(ids, table), lambda: mist.embed(ids, table.detach(), pos=pos)):
        with pytest.raises(mist.MistError, match="no_grad"):
            call()
        with torch.no_grad(), pytest.raises(mist.MistError, match="on one GPU"):  # the next check
            call()
