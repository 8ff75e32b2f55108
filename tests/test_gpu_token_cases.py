"""Cases of the token operators beyond the grids of test_gpu_token.py, against the same definition and with its tolerances."""
import math
import sys

import pytest

from test_gpu_token import Truth, alternatives, types, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "a GPU is required"
    torch.cuda.set_device(0)
    return torch


def say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.mark.parametrize("kind, rows", [("bf16", 37001), ("bf16", 57349), ("f16", 45071), ("bf16", 70013), ("f16", 131079), ("f32", 18501), ("f32", 28675),
                                        ("f32", 33003), ("bf16", 4003), ("bf16", 20013), ("f32", 1001), ("f32", 9999)])
def test_alternatives_at_the_end_of_a_row(torch, kind, rows):
    """The last values of a row, or of its first chunk, that fill no whole vector, and values that the thread behind them looks through,
    are alternatives together, each once; also where that thread has a NaN."""
    from paper_2503_19050_amd import mist
    per = 4 if kind == "f32" else 8   # of a vector
    chunk = 512 * 16 * per
    for off in (0, 1, per - 1):   # of the row from a multiple of 16 bytes
        for nan in (0, 64, 256, 512):
            say("end of a row", kind, rows, off, nan)
            g = torch.Generator("cuda").manual_seed(rows + off)
            room = torch.empty(1, 3, rows + (-rows) % per + per, device="cuda").normal_(0.0, 1.0, generator=g).to(types(torch)[kind])
            x = room[..., off:off + rows]
            head = (-off) % per
            for n in {rows, min(rows, chunk)}:
                tail = n - (n - head) % per
                x[..., tail:n] = torch.arange(40, 40 - (n - tail), -1, device="cuda", dtype=x.dtype)
                back = tail - 512 * per
                if back >= 0:
                    x[..., back:back + per] = torch.arange(20, 20 - per, -1, device="cuda", dtype=x.dtype)
                if nan and tail - nan * per >= 0:
                    x[:, 1, tail - nan * per + 1] = math.nan
            x[..., 5] = 9
            for top in (1, 2, 3, 12, 40):
                r = mist.token_logprob(x, top=top)
                ids = alternatives(torch, x, top)
                assert torch.equal(r.top_ids.reshape(ids.shape), ids), (off, nan, top)
                p = mist.token_part(x, torch.zeros(1, 3, device="cuda", dtype=torch.int64), vocab_begin=7, top=top)
                assert torch.equal(p.top_ids.reshape(ids.shape), ids + 7), (off, nan, top)


@pytest.mark.parametrize("kind, chunk", [("bf16", 65536), ("f16", 65536), ("f32", 32768)])
@pytest.mark.parametrize("more", [1, 4000, 70003])
def test_chunks_of_the_lowest_value(torch, kind, chunk, more):
    """Every value of a first chunk at the type's lowest, as masks have it, ordinary ones after it."""
    from paper_2503_19050_amd import mist
    say("lowest chunk", kind, chunk, more)
    rows = chunk + more
    g = torch.Generator("cuda").manual_seed(rows)
    x = torch.empty(1, 4, rows, device="cuda").normal_(0.0, 2.0, generator=g).to(types(torch)[kind])
    x[..., :chunk] = torch.finfo(x.dtype).min
    x[0, 1, 3] = 1.0
    x[0, 2, chunk:-1] = torch.finfo(x.dtype).min
    t = torch.tensor([[rows - 1, 3, rows - 1, -1]], device="cuda")
    for scale in (1.0, 0.75):
        w = Truth(torch, x, t, scale)
        r = mist.token_logprob(x, t, scale=scale, entropy=True, top=3)
        part = mist.token_part(x, t, vocab_begin=0, scale=scale)
        for got in (r, mist.token_join(part.stats[None], t, entropy=True)):
            within(got.lse, w.lse, w.e_lse, "lse")
            within(got.logp, w.logp, w.e_logp, "logp")
            within(got.entropy, w.entropy, w.e_entropy, "entropy")
        d = torch.tensor([[1.0, -1.0, 0.5, 2.0]], device="cuda")
        got = mist.token_grad(x, t, r.lse, dlogp=d, entropy=r.entropy, dentropy=-d, scale=scale)
        want, slack = w.grad(torch, d, -d, scale, kind)
        within(got, want, slack, "gradient")
        logp, got = mist.token_loss(x, t, -d, scale=scale)
        want, slack = w.grad(torch, d, torch.zeros_like(d), scale, kind)
        within(logp, w.logp, w.e_logp, "logp")
        within(got, want, slack, "loss")


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows", [9, 5000, 50257, 70000])
@pytest.mark.parametrize("scale", [0.75, 0.9, 1.0 / 3.0, 1.25, 2.0 ** -70, 3e-39, 1e30])
def test_scaled_values_of_any_size(torch, kind, rows, scale):
    """Rows of one value, whatever its size and the scale, are uniform: entropy log n, a gradient of weight / n, and log
    probabilities that are none above 0.  Beside the largest value others have none."""
    from paper_2503_19050_amd import mist
    say("sizes", kind, rows, scale)
    T = types(torch)[kind]
    scale = float(torch.tensor(scale, dtype=torch.float32))
    top, tiny = float(torch.finfo(torch.float32).max), 2.0 ** -100
    values = [v for v in (float(torch.finfo(T).min), -1.23e10, -7e8, -3.3, 0.0, 1.7, 1e5, 3.1e37) if abs(v) <= float(torch.finfo(T).max)]
    x = torch.tensor(values, device="cuda", dtype=T)[None, :, None].expand(1, len(values), rows).contiguous()
    z = x[0, :, 0].double() * scale
    t = torch.full((1, len(values)), rows - 1, device="cuda")
    r = mist.token_logprob(x, t, scale=scale, entropy=True, top=2)
    logp, d = mist.token_loss(x, t, 0.5, scale=scale)
    grad = mist.token_grad(x, t, r.lse, dlogp=torch.ones(1, len(values), device="cuda"), entropy=r.entropy, dentropy=torch.ones(1, len(values), device="cuda"), scale=scale)
    for k, v in enumerate(z.tolist()):
        if v < -top:      # masked out
            assert r.lse[0, k] == -math.inf and r.entropy[0, k] == 0 and r.logp[0, k] == -math.inf and not d[0, k].any() and not grad[0, k].any(), v
            continue
        if v > top:
            assert r.lse[0, k].isnan() and r.logp[0, k].isnan() and r.entropy[0, k].isnan() and d[0, k].isnan().all(), v
            continue
        # a sum of ones is exact below 2^24; the logarithm, at most 11.2, is off by two of its ulps of 2^-20
        assert abs(float(r.entropy[0, k]) - math.log(rows)) <= 2.0 ** -19, v
        assert abs(float(r.lse[0, k]) - v) <= math.log(rows) + 2.0 ** -22 * (abs(v) + 20), v
        assert -math.log(rows) - 2.0 ** -22 * (abs(v) + 20) <= float(r.logp[0, k]) <= 0.0 and r.logp[0, k] == logp[0, k], v
        assert r.top_ids[0, k].tolist() == [0, 1] and bool((r.top_logp[0, k] == r.logp[0, k]).all()), v
        if 4 * scale * (1 + math.log(rows)) > float(torch.finfo(T).max):   # the gradient's own factors pass the type
            continue
        p = d[0, k].double() / (0.5 * scale)
        # of p c0: roundings of p (2^-22 of it), of the factor and of the output
        unit = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[kind] + 2.0 ** -21
        small = {"bf16": 2.0 ** -133, "f16": 2.0 ** -24, "f32": 2.0 ** -148}[kind] / (0.5 * scale)
        assert bool(((p[:-1] - 1 / rows).abs() <= unit / rows + small).all()) and abs(float(p[-1]) - 1 / rows + 1) <= unit + small, v
        assert bool(grad[0, k].isfinite().all()), v
    y = x.clone()
    y[..., 0] = torch.where(x[..., 0] < 0, x[..., 0] / 2, x[..., 0] * 2 + 1)
    far = (y[0, :, 0].double() - x[0, :, 0].double()) * scale > 200
    r = mist.token_logprob(y, torch.zeros_like(t), scale=scale, entropy=True)
    one = far & (y[0, :, 0].double() * scale <= top) & (y[0, :, 0].double() * scale >= -top)
    assert bool((r.logp[0][one] == 0).all()) and bool((r.entropy[0][one].abs() < tiny).all())


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("ranks", [1, 2, 4, 30])
def test_joined_alternatives_past_fp32(torch, kind, ranks):
    """Finite logits whose scaled value is below fp32's range are alternatives of -inf, from parts as from the whole vocabulary; a masked one is none."""
    from paper_2503_19050_amd import mist
    low = torch.finfo(types(torch)[kind]).min
    x = torch.full((1, 3, 60), low, device="cuda", dtype=types(torch)[kind])
    x[0, 1, 44] = 1.0
    x[0, 2] = -math.inf
    x[0, 2, 31] = low
    t = torch.full((1, 3), 44, device="cuda")
    whole = mist.token_logprob(x, t, scale=1.5, top=3)
    assert whole.top_ids.tolist() == [[[0, 1, 2], [44, 0, 1], [31, -1, -1]]]
    per = 60 // ranks
    parts = [mist.token_part(x[..., k * per:(k + 1) * per], t, vocab_begin=k * per, scale=1.5, top=3) for k in range(ranks)]
    r = mist.token_join(torch.stack([p.stats for p in parts]), t, top_ids=torch.stack([p.top_ids for p in parts]), top_z=torch.stack([p.top_z for p in parts]))
    assert torch.equal(r.top_ids, whole.top_ids) and torch.equal(r.top_logp, whole.top_logp) and torch.equal(r.logp, whole.logp)


def test_joined_alternatives_of_one_scaled_value(torch):
    """fp32 logits that differ and have one z: by logit in a part and in the whole vocabulary, by id where parts are joined."""
    from paper_2503_19050_amd import mist
    scale = float(torch.tensor(0.6))
    high = torch.tensor([2.0 - k * 2.0 ** -23 for k in range(1, 9)], device="cuda")
    z = high * torch.tensor(scale, device="cuda")
    k = int((z[:-1] == z[1:]).nonzero()[0])
    x = torch.zeros(1, 1, 20, device="cuda")
    x[0, 0, 3], x[0, 0, 17] = high[k + 1], high[k]
    t = torch.zeros(1, 1, device="cuda", dtype=torch.int64)
    assert mist.token_logprob(x, t, scale=scale, top=3).top_ids.tolist() == [[[17, 3, 0]]]
    part = mist.token_part(x, t, vocab_begin=0, scale=scale, top=3)
    assert part.top_ids.tolist() == [[[17, 3, 0]]] and part.top_z[0, 0, 0] == part.top_z[0, 0, 1] == z[k]
    r = mist.token_join(part.stats[None], t, top_ids=part.top_ids[None], top_z=part.top_z[None])
    assert r.top_ids.tolist() == [[[3, 17, 0]]]
