"""The Adam step's constants and its verdict on the GPU: what the weight decay and the betas are worth in fp32.

A single value cannot show an error far below its last place, the mean over many can: rounding one
result errs by up to half an ulp either way, evenly where the low bits are spread evenly, so the mean of N
of them is within 6 ulp / sqrt(12 N) of none (six deviations of N evenly spread errors).  Added to it below: the largest
error that the other roundings of the formula could share.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

N = 1 << 20


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "a GPU is required"
    torch.cuda.set_device(0)
    return torch


def lists(mist, *tensors):
    return [mist.TensorList([t]) for t in tensors]


def mean_bound(ulp):
    return 6 * ulp / math.sqrt(12 * N)


@pytest.mark.parametrize("lr, decay", [(1e-6, 0.01), (1e-5, 0.01), (3e-7, 0.1), (3e-4, 0.1)])
def test_small_weight_decay_is_kept(torch, lr, decay):
    """Weights in [2^-7, 2^-6) (one ulp of 2^-30) under updates of either sign: their mean moves by lr * decay * mean(p)."""
    from paper_2503_19050_amd import mist
    gen = torch.Generator("cuda").manual_seed(3)
    p = torch.empty(N, device="cuda").uniform_(2.0 ** -7, 2.0 ** -6, generator=gen)
    p.clamp_(2.0 ** -7 + 2 * lr, 2.0 ** -6 - 2 * lr)
    m = torch.empty(N, device="cuda").uniform_(-1.0, 1.0, generator=gen)
    v, g = torch.ones(N, device="cuda"), torch.zeros(N, device="cuda")
    was, t = [x.double() for x in (p, m, v)], 1001
    rec = mist.StepRecord(step=t - 1)
    P, M, V, G = lists(mist, p, m, v, g)
    mist.grad_norm(G, rec)
    mist.adam_step(P, M, V, G, rec, lr=lr, betas=(0.9, 0.95), eps=1e-8, weight_decay=decay)
    update = 0.9 * was[1] / (1 - 0.9 ** t) / ((0.95 * was[2] / (1 - 0.95 ** t)).sqrt() + 1e-8)
    want = was[0] - lr * (update + decay * was[0])
    error = float((p.double() - want).mean())
    # the update's roundings: 24 2^-24 of lr * 1, were they all of one sign
    assert abs(error) <= mean_bound(2.0 ** -30) + 24 * 2.0 ** -24 * lr, (error, lr * decay * float(was[0].mean()))


@pytest.mark.parametrize("beta", [0.999, 0.99999, 1 - 1e-6])
@pytest.mark.parametrize("which", ["m", "v"])
def test_slow_averages_decay_at_their_rate(torch, which, beta):
    """Averages in [1, 2) (one ulp of 2^-23) decay by 1 - beta, whatever beta rounds to in fp32."""
    from paper_2503_19050_amd import mist
    gen = torch.Generator("cuda").manual_seed(4)
    p = torch.zeros(N, device="cuda")
    m, v, g = (torch.empty(N, device="cuda").uniform_(1.0, 2.0, generator=gen) for _ in range(3))
    span = 8 * 2.0 ** -23 / (1 - beta)   # terms that move the average by several ulps at the least, evenly
    if which == "m":
        g.uniform_(-max(1.0, span), max(1.0, span), generator=gen)
    else:
        g.uniform_(0.0, max(1.0, span), generator=gen).sqrt_()
    old, x = (m if which == "m" else v).double(), g.double()
    P, M, V, G = lists(mist, p, m, v, g)
    rec = mist.StepRecord(step=99)
    mist.grad_norm(G, rec)
    mist.adam_step(P, M, V, G, rec, lr=0.0, betas=(beta, 0.9) if which == "m" else (0.9, beta))
    term = x if which == "m" else x * x
    want = beta * old + (1 - beta) * term
    error = float(((m if which == "m" else v).double() - want).mean())
    shared = 4 * 2.0 ** -24 * (1 - beta) * float(term.abs().max())
    assert abs(error) <= mean_bound(2.0 ** -23) + shared, (error, beta)


def test_infinite_averages_stay(torch):
    """An average that has left fp32 (a gradient past 1.8e19) stays inf and gives no NaN."""
    from paper_2503_19050_amd import mist
    p, m, v, g = (torch.ones(1000, device="cuda") for _ in range(4))
    v.fill_(float("inf"))
    P, M, V, G = lists(mist, p, m, v, g)
    rec = mist.StepRecord()
    for betas in ((0.9, 0.999), (0.0, 0.5)):
        mist.grad_norm(G, rec)
        mist.adam_step(P, M, V, G, rec, lr=0.1, betas=betas)
        assert v.isinf().all() and (p == 1).all() and m.isfinite().all()


def test_constants_past_fp32_are_refused(torch):
    """lr and weight_decay that are finite in 64 bits and infinite in the kernel's 32."""
    from paper_2503_19050_amd import mist
    L = lists(mist, *(torch.ones(5, device="cuda") for _ in range(4)))
    rec = mist.StepRecord()
    mist.grad_norm(L[3], rec)
    for bad in (dict(lr=1e39), dict(lr=0.1, weight_decay=1e39)):
        with pytest.raises(mist.MistError) as e:
            mist.adam_step(*L, rec, **bad)
        assert e.value.status == -1
    assert all((x.tensors[0] == 1).all() for x in L)


def test_norm_past_fp32_changes_nothing(torch):
    """The record's norm is fp32: where it is inf, so is the verdict, though the sum of squares in 64 bits is finite."""
    from paper_2503_19050_amd import mist
    for grads, scale in (([3e38, 3e38], 1.0), ([1e30, 0.0], 1e10)):
        g = torch.tensor(grads, device="cuda")
        rec = mist.StepRecord(step=2)
        G = mist.TensorList([g])
        mist.grad_norm(G, rec, max_norm=1.0, grad_scale=scale)
        assert math.isfinite(float(rec.total)) and float(rec.norm) == math.inf
        assert (int(rec.applied), int(rec.step), int(rec.skipped)) == (0, 2, 1)
        out = torch.empty_like(g)
        mist.grad_clip(G, rec, mist.TensorList([out]))
        assert torch.equal(out, g)
    g = torch.tensor([3e38, 0.0], device="cuda")   # the largest that has a norm: a subnormal factor
    rec, out = mist.StepRecord(), torch.empty_like(g)
    mist.grad_norm(mist.TensorList([g]), rec, max_norm=1.0)
    mist.grad_clip(mist.TensorList([g]), rec, mist.TensorList([out]))
    coef = 1.0 / float(g[0].double())
    assert int(rec.applied) == 1 and abs(float(rec.coef) - coef) <= 2.0 ** -23 * coef + 2.0 ** -150
    assert abs(float(out[0]) - 1.0) <= 2.0 ** -150 / coef + 2.0 ** -22 and float(out[1]) == 0.0


def test_step_without_a_norm(torch):
    """grad_finish on a total of zero forms a factor of grad_scale and counts the step: no pass over the gradients."""
    from paper_2503_19050_amd import mist
    g = torch.full((777,), 2.0, device="cuda")
    p, m, v = (torch.zeros(777, device="cuda") for _ in range(3))
    rec = mist.StepRecord()
    L = lists(mist, p, m, v, g)
    for k in range(2):
        rec.total.zero_()
        mist.grad_finish(rec, grad_scale=0.5)
        mist.adam_step(*L, rec, lr=0.25, betas=(0.5, 0.5))
        assert (int(rec.applied), int(rec.step), float(rec.coef)) == (1, k + 1, 0.5)
        # g' = 1 in every step: both averages are 1 after bias correction, the update is lr
        assert torch.equal(m, torch.full_like(m, 1 - 0.5 ** (k + 1)))
        assert ((p + 0.25 * (k + 1)).abs() <= 1e-6).all()
