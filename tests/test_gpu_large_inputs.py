"""The forms that large inputs take, on the GPU, against the definition in 64 bits (there too, by elementary operations):
lookups with several tokens a wave, lists of more pieces than blocks, calls of several launches, sums over large batches.

Tolerances as in test_gpu_embed.py and test_gpu_step.py; those of sums over large batches stand with their test.
"""
import math
import sys

import pytest

pytestmark = pytest.mark.gpu

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -149}
E24 = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "a GPU is required"
    torch.cuda.set_device(0)
    return torch


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def types(torch):
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def within(got, want, slack, what):
    bad = ~((got.double() - want).abs() <= slack)
    assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:3].tolist(), got[bad][:3], want[bad][:3])


# batch, seq, vocab, hidden: 2, 3 or 16 tokens a wave with positions, in waves that hold parts of several
# positions or several of a position's sequences; eights, fours and odd widths
LOOKUPS = [(2, 20000, 500, 8), (3, 5500, 1000, 1032), (5, 1101, 700, 4104), (1, 270001, 300, 8), (40, 7001, 300, 12),
           (3, 100003, 50, 7), (17, 1901, 2000, 4097), (64, 4099, 300, 24), (16384, 17, 99, 40), (300001, 1, 99, 8)]


@pytest.mark.parametrize("act, weight", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("shape", LOOKUPS, ids=str)
def test_lookup_with_positions_of_many_tokens(torch, shape, act, weight):
    from paper_2503_19050_amd import mist
    batch, seq, vocab, hidden = shape
    say("lookup", shape, act, weight)
    T, gen = types(torch), torch.Generator("cuda").manual_seed(batch + seq)
    ids = torch.randint(-3, vocab + 3, (batch, seq), device="cuda", generator=gen, dtype=torch.int32 if seq % 2 else torch.int64)
    table = torch.empty(vocab, hidden, device="cuda").normal_(generator=gen).to(T[weight])
    pos = torch.empty(seq, hidden, device="cuda").normal_(generator=gen).to(T[weight])
    out = torch.full((batch, seq, hidden), float("nan"), device="cuda", dtype=T[act])
    mist.embed(ids, table, scale=3.7, pos=pos, out=out)
    inside = (ids >= 0) & (ids < vocab)
    scale = float(torch.tensor(3.7, dtype=torch.float32))
    at = max(1, (1 << 25) // (seq * hidden))      # sequences at a time
    for b in range(0, batch, at):
        x = torch.where(inside[b:b + at, :, None], table.double()[ids[b:b + at].clamp(0, vocab - 1).long()] * scale, 0.0)
        p = pos.double()[None]
        within(out[b:b + at], x + p, UNIT[act] * (x + p).abs() + 2.0 ** -22 * (x.abs() + p.abs()) + TINY[act], "lookup")


def test_lookup_of_more_tokens_than_a_launch_takes(torch):
    """2^25 waves of four tokens a launch: past 2^27 tokens there are two."""
    from paper_2503_19050_amd import mist
    n = (1 << 27) + 4099
    table = torch.randn(200, 1, device="cuda").bfloat16()
    ids = torch.randint(0, 200, (1, n), device="cuda", dtype=torch.int32)
    out = torch.full((1, n, 1), float("nan"), device="cuda", dtype=torch.bfloat16)
    mist.embed(ids, table, scale=2.0, out=out)
    for lo in range(0, n, 1 << 26):
        want = (table.float() * 2.0).bfloat16()[ids[0, lo:lo + (1 << 26)].long()]   # exact products
        assert torch.equal(out[0, lo:lo + (1 << 26)], want)


@pytest.mark.parametrize("act, weight", [("bf16", "f32"), ("f32", "f32"), ("f16", "bf16")])
@pytest.mark.parametrize("batch, seq, hidden", [(4097, 3, 24), (131072, 1, 8), (1 << 20, 1, 8), (20000, 2, 7), (1000, 1, 8),
                                                (1000, 1, 520), (9001, 16, 12)])
def test_positions_of_a_large_batch(torch, batch, seq, hidden, act, weight):
    """Terms of one sign that a long sum's last place does not hold: sums of at most 64 terms are added up, so that
    the error is that of 64 + batch / 64 roundings, not of batch."""
    from paper_2503_19050_amd import mist
    say("positions", batch, seq, hidden, act, weight)
    T, gen = types(torch), torch.Generator("cuda").manual_seed(batch)
    grad = torch.empty(batch, seq, hidden, device="cuda", dtype=T[act])
    grad[:] = (1.00276 if act == "f32" else 1.0 + 2.0 ** -7) * 2.0 ** (torch.arange(hidden, device="cuda") % 3 - 1)
    ids = torch.randint(0, 50, (batch, seq), device="cuda", generator=gen)
    want = grad.double().sum(0)
    for old in (0.0, 3.0):
        dtable, dpos = torch.zeros(50, hidden, device="cuda", dtype=T[weight]), torch.full((seq, hidden), old, device="cuda", dtype=T[weight])
        mist.embed_grad(ids, grad, dtable, dpos=dpos, accumulate=old > 0)
        x = want + old
        within(dpos, x, UNIT[weight] * x + (64 + batch / 64 + 3) * E24 * x + TINY[weight], "dpos")


LISTS = {"one": [9000001], "two": [12000007, 8000009], "many": [5000 + 7 * k % 9001 for k in range(2600)],
         "mixed": [11000003] + [1 + k % 5000 for k in range(3000)]}


def views(torch, sizes, dtype, std, shift, gen):
    flat = torch.full((sum(sizes) + shift + 16,), 77.0, device="cuda", dtype=dtype)
    part = flat[shift:shift + sum(sizes)]
    part.copy_(torch.empty(sum(sizes), device="cuda").normal_(0.0, std, generator=gen))
    return flat, part, list(part.split(sizes))


def untouched(flat, part, shift):
    assert (flat[:shift] == 77.0).all() and (flat[shift + part.numel():] == 77.0).all()


@pytest.mark.parametrize("g, w, shift", [("bf16", "bf16", 0), ("f32", "bf16", 1), ("f16", "f32", 3)])
@pytest.mark.parametrize("sizes", LISTS, ids=str)
def test_lists_of_more_pieces_than_blocks(torch, sizes, g, w, shift):
    """Norm, clipping and step; the norm's blocks take two pieces and more."""
    from paper_2503_19050_amd import mist
    say("list", sizes, g, w, shift)
    S, T, gen = LISTS[sizes], types(torch), torch.Generator("cuda").manual_seed(shift)
    gf, grad, grads = views(torch, S, T[g], 0.01, shift, gen)
    state = [views(torch, S, torch.float32, 0.01, shift, gen) for _ in range(3)]
    state[2][1].square_()
    wf, weight, weights = views(torch, S, T[w], 1.0, shift, gen)
    G, W = mist.TensorList(grads), mist.TensorList(weights)
    x = grad.double()
    total = float((x * x).sum())
    rec = mist.StepRecord(step=10)
    mist.grad_norm(G, rec, kind="max")
    assert float(rec.total) == float(x.abs().max())
    mist.grad_norm(G, rec, max_norm=1.0)
    assert abs(float(rec.total) - total) <= len(x) * 2.0 ** -51 * total   # both sums are rounded
    norm = math.sqrt(total)
    coef = 1.0 / norm if norm > 1.0 else 1.0
    mist.grad_clip(G, rec, W)
    within(weight, coef * x, (UNIT[w] + 2.0 ** -22) * (coef * x).abs() + TINY[w], "clip")
    was = [s[1].double() for s in state]
    mist.adam_step(*(mist.TensorList(s[2]) for s in state), G, rec, lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, weights=W)
    gx, t = coef * x, 12
    size = 0.9 * was[1].abs() + 0.1 * gx.abs()
    m, v = 0.9 * was[1] + (1 - 0.9) * gx, 0.95 * was[2] + (1 - 0.95) * gx * gx
    down = (v / (1 - 0.95 ** t)).sqrt() + 1e-8
    p = was[0] - 3e-3 * (m / (1 - 0.9 ** t) / down + 0.1 * was[0])
    within(state[1][1], m, 6 * E24 * size + TINY["f32"], "m")
    within(state[2][1], v, 8 * E24 * v + TINY["f32"], "v")
    within(state[0][1], p, 4 * E24 * was[0].abs() + 3e-3 * 24 * E24 * size / (1 - 0.9 ** t) / down + TINY["f32"], "p")
    assert torch.equal(weight, state[0][1].to(T[w]))
    for flat, part in [(gf, grad), (wf, weight)] + [(s[0], s[1]) for s in state]:
        untouched(flat, part, shift)
