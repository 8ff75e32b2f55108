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


def test_tensors_that_overlap_are_read_and_not_written(torch):
    """One parameter under two names: its norm counts it twice, clipping and steps into it are refused."""
    from paper_2503_19050_amd import mist
    x = torch.full((5000,), 2.0, device="cuda")
    twice, part = mist.TensorList([x, x]), mist.TensorList([x[:4000], x[3999:]])
    apart = [mist.TensorList([torch.zeros(5000, device="cuda") for _ in range(2)]) for _ in range(4)]
    rec = mist.StepRecord()
    mist.grad_norm(twice, rec, max_norm=100.0)
    assert float(rec.total) == 2 * 5000 * 4.0
    for call in (lambda: mist.grad_clip(twice, rec), lambda: mist.grad_clip(apart[0], rec, twice), lambda: mist.grad_clip(part, rec),
                 lambda: mist.adam_step(twice, *apart[:3], rec, lr=0.1), lambda: mist.adam_step(apart[0], twice, *apart[1:3], rec, lr=0.1),
                 lambda: mist.adam_step(*apart[:2], twice, apart[2], rec, lr=0.1),
                 lambda: mist.adam_step(*apart, rec, lr=0.1, weights=twice)):
        with pytest.raises(mist.MistError, match="overlap") as e:
            call()
        assert e.value.status == -1
    mist.grad_clip(twice, rec, apart[0])
    assert (x == 2.0).all() and all(torch.equal(t, apart[0].tensors[0]) for t in apart[0].tensors) and float(apart[0].tensors[0][0]) == 1.0
