"""Tensor lists around a graph's capture (GPU)."""
import gc

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "a GPU is required"
    torch.cuda.set_device(0)
    return torch


@pytest.mark.parametrize("allocator", ["torch", None])
def test_lists_closed_during_a_capture(torch, allocator):
    """The capture goes on, the graph's replays are right, and the tables are freed afterwards."""
    from paper_2503_19050_amd import mist
    g = torch.randn(5000, device="cuda")
    kept, closed, dropped = (mist.TensorList([g], allocator=allocator) for _ in range(3))
    rec, other = mist.StepRecord(), mist.StepRecord()
    for x in (kept, closed, dropped):
        mist.grad_norm(x, other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        closed.close()
        mist.grad_norm(kept, rec)
        del dropped, x
        gc.collect()
        with pytest.raises(mist.MistError, match="captured"):
            mist.TensorList([g])
        mist.grad_clip(kept, rec)
    assert len(mist._closed) == 2
    with pytest.raises(mist.MistError, match="closed"):
        mist.grad_norm(closed, other)
    for k in range(4):
        g.normal_()
        total = (g.double() ** 2).sum()
        graph.replay()
        torch.cuda.synchronize()
        assert abs(float(rec.total) - float(total)) <= 5000 * 2.0 ** -51 * float(total) and int(rec.step) == k + 1
        torch.randn(1 << 20, device="cuda").sum().item()
    with mist.TensorList([g]) as T:
        assert len(mist._closed) == 0
        mist.grad_norm(T, other)
    assert len(mist._closed) == 0
