"""Cases of the kept activations beyond the grids of test_gpu_kept.py."""
import math
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "a GPU is required"
    torch.cuda.set_device(0)
    return torch


@pytest.mark.parametrize("form", ["silu", "gelu"])
@pytest.mark.parametrize("width", [8, 129, 1000])
def test_f16_at_its_largest_value(torch, form, width):
    """65504 is kept as 64 times 1024, past the type: the backward pass takes the value that a load gives, so the activation formed again
    and the gradients are those at the type's largest value."""
    from paper_2503_19050_amd import mist
    print("largest", form, width, file=sys.stderr, flush=True)
    top = 65504.0
    x = torch.full((3, width), 1.0, device="cuda", dtype=torch.float16)
    x[0], x[1, ::2] = top, -top
    one = torch.ones_like(x)
    d = torch.full_like(x, 2.0 ** -10)
    for up, gate in ((x, None), (one, x), (x, one)):
        r = mist.mlp_act(up, gate, kind=form, save=True)
        loaded = [None if c is None else mist.checkpoint_load(c) for c in (r.up, r.gate)]
        assert bool(r.out.isfinite().all()) and bool(loaded[0].isfinite().all())
        again = torch.full_like(x, math.nan)
        dup, dgate = mist.mlp_act_grad(d, r.up, r.gate, kind=form, out=again)
        # at what is loaded, in 64 bits; a result is of at most ten roundings of 2^-24 and one of 2^-11, with 2^-24 for subnormals
        u, g = (None if t is None else t.double() for t in loaded)
        z = (u if g is None else g).requires_grad_()
        a = torch.nn.functional.silu(z) if form == "silu" else torch.nn.functional.gelu(z, approximate="tanh")
        slope, = torch.autograd.grad(a.sum(), z)
        a = a.detach()
        want = [a, d.double() * slope] if g is None else [a * u, d.double() * a, d.double() * u * slope]
        for got, w in zip([again, dup] + ([] if g is None else [dgate]), want):
            assert bool(got.isfinite().all())
            assert bool(((got.double() - w).abs() <= (2.0 ** -11 + 2.0 ** -20) * w.abs() + 2.0 ** -24).all())


def test_a_checkpoint_of_a_stream(torch):
    """A checkpoint made for another stream, given as a torch stream or as its handle, and for the default one."""
    from paper_2503_19050_amd import mist
    side = torch.cuda.Stream()
    x = torch.randn(5, 300, device="cuda").bfloat16()
    want = mist.checkpoint_store(x)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream, 0, None):
        for device in ("cuda", x.device):
            c = mist.Checkpoint((5, 300), torch.bfloat16, device, stream=stream)
            assert c.values.device == x.device
            assert mist.checkpoint_store(x, c, stream=stream) is c
            torch.cuda.synchronize()
            assert torch.equal(c.values, want.values) and torch.equal(c.exponents, want.exponents)


def test_a_place_for_a_gate_that_is_not_there(torch):
    from paper_2503_19050_amd import mist
    x = torch.zeros(4, 200, device="cuda", dtype=torch.bfloat16)
    a, b = (mist.Checkpoint((4, 200), torch.bfloat16) for _ in range(2))
    with pytest.raises(mist.MistError, match="gate"):
        mist.mlp_act(x, save=(a, b))
    r = mist.mlp_act(x, save=(a, None))
    assert r.up is a and r.gate is None
