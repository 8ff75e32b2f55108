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


LISTS = {"one": [9000001], "two": [12000007, 8000009], "many": [5000 + 7 * k % 9001 for k in range(2600)],
         "mixed": [11000003] + [1 + k % 5000 for k in range(3000)]}


def views(torch, sizes, dtype, std, shift, gen):
    flat = torch.full((sum(sizes) + shift + 16,), 77.0, device="cuda", dtype=dtype)
    part = flat[shift:shift + sum(sizes)]
    part.copy_(torch.empty(sum(sizes), device="cuda").normal_(0.0, std, generator=gen))
    return flat, part, list(part.split(sizes))


def untouched(flat, part, shift):
    assert (flat[:shift] == 77.0).all() and (flat[shift + part.numel():] == 77.0).all()
