"""The gradient norm, clipping and the Adam step over lists of tensors (mist_grad_norm, mist_grad_clip,
mist_adam_step) on the GPU against the definition in 64 bits on the CPU.

Tolerances, fixed before the first run (u, tiny: of the output type, as half an ulp of 1 and half the
smallest subnormal).  Constants of the call are rounded to fp32 once each.
  total  sums of squares in 64 bits: n 2^-52
  norm, coef: one rounding to fp32 of a 64-bit value: 2^-23
  clip   one product in fp32, one rounding: u |x| + 2^-22 |x| + tiny
  m      6 2^-24 (beta1 |m| + (1 - beta1) |g'|) + tiny;   v  8 2^-24 (beta2 v + (1 - beta2) g'^2) + tiny
  p      4 2^-24 |p| + lr 24 2^-24 (beta1 |m| + (1 - beta1) |g'|) / bc1 / (sqrt(v / bc2) + eps) + tiny;   w  u |p| more
"""
import gc
import math
import sys

import numpy as np
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


def kind(torch, name):
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


SIZES = {
    "one": [1], "empty": [0, 0], "some-empty": [0, 3, 0, 1000, 0], "small": [1, 2, 3, 7, 8, 9, 63, 64, 65, 255, 256, 257],
    "chunks": [8191, 8192, 8193, 16384, 16385, 1], "large": [3000001], "many": [5 + k % 40 for k in range(700)],
    "layers": [256, 256 * 768, 768, 256 * 256, 256, 256, 256, 256 * 1024, 1024, 1024 * 256, 256] * 4,
}


def tensors(torch, rng, sizes, dtype, std, shift, apart=0):
    """Views of one flat buffer that starts `shift` elements past its allocation, `apart` elements between them;
    what lies between holds a value that must stay."""
    n = sum(sizes) + apart * len(sizes) + shift + 8
    flat = torch.full((n,), 77.0, dtype=kind(torch, dtype), device="cuda")
    views, at = [], shift
    for k in sizes:
        views.append(flat[at:at + k])
        views[-1].copy_(torch.tensor(rng.standard_normal(k) * std))
        at += k + apart
    return flat, views


def as64(views):
    return np.concatenate([v.double().cpu().numpy() for v in views]) if views else np.zeros(0)


def untouched(torch, flat, views):
    rest = torch.ones_like(flat, dtype=torch.bool)
    at0 = flat.data_ptr()
    for v in views:
        if v.numel():
            at = (v.data_ptr() - at0) // flat.element_size()
            rest[at:at + v.numel()] = False
    assert (flat[rest] == 77.0).all()


def within(got, want, slack, what):
    bad = ~(np.abs(got - want) <= slack)
    assert not np.any(bad), (what, int(np.sum(bad)), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3])


@pytest.mark.parametrize("shift", [0, 1, 8])
@pytest.mark.parametrize("g, o", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("f16", "bf16")])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_norm_and_clip(torch, sizes, g, o, shift):
    from paper_2503_19050_amd import mist
    say("clip", sizes, g, o, shift)
    rng = np.random.default_rng(len(sizes) + shift)
    flat, grads = tensors(torch, rng, SIZES[sizes], g, 0.3, shift, apart=shift)
    out_flat, out = tensors(torch, rng, SIZES[sizes], o, 1.0, 8 - shift, apart=3)
    x = as64(grads)
    norm = math.sqrt(float(np.sum(x * x)))
    G, O = mist.TensorList(grads), mist.TensorList(out)
    for most, scale in ((0.5, 1.0), (1e9, 1.0), (float("inf"), -0.25), (0.25, 1.0 / 1024)):
        rec = mist.StepRecord(step=6)
        mist.grad_norm(G, rec, max_norm=most, grad_scale=scale)
        mist.grad_clip(G, rec, O)
        within(np.array(float(rec.total)), np.array(norm ** 2), max(len(x), 4) * 2.0 ** -52 * norm ** 2, "total")
        n = abs(scale) * norm
        within(np.array(float(rec.norm)), np.array(n), 2.0 ** -23 * n, "norm")
        coef = scale * (most / n if n > most else 1.0)
        within(np.array(float(rec.coef)), np.array(coef), 2.0 ** -23 * abs(coef), "coef")
        assert (int(rec.step), int(rec.applied), int(rec.skipped)) == (7, 1, 0)
        want = coef * x
        within(as64(out), want, (UNIT[o] + 2.0 ** -22) * np.abs(want) + TINY[o], "clip")
        untouched(torch, out_flat, out)
        first = [v.clone() for v in out]
        mist.grad_norm(G, rec, max_norm=most, grad_scale=scale)
        mist.grad_clip(G, rec, O)
        assert all(torch.equal(a, b) for a, b in zip(first, out)) and int(rec.step) == 8
    untouched(torch, flat, grads)
    # in place
    rec = mist.StepRecord()
    mist.grad_norm(G, rec, max_norm=0.5)
    mist.grad_clip(G, rec)
    coef = 0.5 / norm if norm > 0.5 else 1.0
    within(as64(grads), coef * x, (UNIT[g] + 2.0 ** -22) * np.abs(coef * x) + TINY[g], "in place")
    untouched(torch, flat, grads)


@pytest.mark.parametrize("g", ["bf16", "f16", "f32"])
def test_largest_magnitude(torch, g):
    from paper_2503_19050_amd import mist
    rng = np.random.default_rng(4)
    for name in ("one", "some-empty", "chunks", "many"):
        flat, grads = tensors(torch, rng, SIZES[name], g, 0.3, 1)
        rec = mist.StepRecord()
        G = mist.TensorList(grads)
        mist.grad_norm(G, rec, max_norm=0.01, kind="max")
        top = np.abs(as64(grads)).max()
        assert float(rec.total) == top and float(rec.norm) == np.float32(top)
        within(np.array(float(rec.coef)), np.array(0.01 / top if top > 0.01 else 1.0), 2.0 ** -23, "coef")
        last = grads[-1] if grads[-1].numel() else grads[-2]
        for bad in (float("nan"), float("-inf")):
            last[-1] = bad
            mist.grad_norm(G, rec, kind="max")
            assert int(rec.applied) == 0 and int(rec.step) == 1


def test_several_lists_and_ranks(torch):
    """Lists of different types joined into one norm; totals of ranks added before the step is finished."""
    from paper_2503_19050_amd import mist
    rng = np.random.default_rng(8)
    _, a = tensors(torch, rng, SIZES["layers"], "bf16", 0.1, 1)
    _, b = tensors(torch, rng, SIZES["small"], "f32", 0.1, 0)
    A, B = mist.TensorList(a), mist.TensorList(b)
    total = float((as64(a) ** 2).sum() + (as64(b) ** 2).sum())
    rec = mist.StepRecord()
    mist.grad_norm(A, rec, finish=False)
    assert int(rec.step) == 0
    mist.grad_norm(B, rec, accumulate=True, max_norm=2.0)
    within(np.array(float(rec.norm)), np.array(math.sqrt(total)), 2.0 ** -23 * math.sqrt(total), "norm")
    one, two = mist.StepRecord(step=3), mist.StepRecord()
    mist.grad_norm(A, one, finish=False)
    mist.grad_norm(B, two, finish=False)
    one.total += two.total
    mist.grad_finish(one, max_norm=2.0)
    assert float(one.norm) == float(rec.norm) and float(one.coef) == float(rec.coef) and int(one.step) == 4


def test_squares_past_the_range_of_fp32(torch):
    """Gradients whose squares leave fp32's range, both ways, have a norm."""
    from paper_2503_19050_amd import mist
    for size in (1e25, 1e-25):
        g = torch.full((1000,), size, device="cuda")
        rec = mist.StepRecord()
        mist.grad_norm(mist.TensorList([g]), rec, max_norm=size)
        want = math.sqrt(1000) * float(g[0].double())
        within(np.array(float(rec.norm)), np.array(want), 2.0 ** -23 * want, "norm")
        assert int(rec.applied) == 1


def adam(p, m, v, g, t, lr, b1, b2, eps, decay):
    size = b1 * np.abs(m) + (1 - b1) * np.abs(g)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    down = np.sqrt(v / (1 - b2 ** t)) + eps
    new = p - lr * ((m / (1 - b1 ** t)) / down + decay * p)
    slack = 4 * E24 * np.abs(p) + lr * 24 * E24 * size / (1 - b1 ** t) / down
    return new, m, v, slack + TINY["f32"], 6 * E24 * size + TINY["f32"], 8 * E24 * v + TINY["f32"]


@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("g, w, step", [("bf16", "bf16", 0), ("f16", "f16", 99), ("f32", "f32", 5), ("f32", "bf16", 1 << 20),
                                        ("bf16", None, 1), ("f16", "bf16", 0), ("f32", None, 0)])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_adam(torch, sizes, g, w, step, shift):
    from paper_2503_19050_amd import mist
    say("adam", sizes, g, w, step, shift)
    rng = np.random.default_rng(step % 1000 + shift)
    S = SIZES[sizes]
    pf, p = tensors(torch, rng, S, "f32", 0.5, shift)
    mf, m = tensors(torch, rng, S, "f32", 0.01, shift, apart=shift)
    vf, v = tensors(torch, rng, S, "f32", 0.01, 0 if shift == 4 else shift)
    gf, grads = tensors(torch, rng, S, g, 0.3, shift)
    wf, weights = tensors(torch, rng, S, w or "f32", 1.0, shift)
    for a, b in zip(m, v):
        if step:
            b.square_()
        else:
            a.zero_(), b.zero_()
    hyper = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1 if shift else 0.0)
    lists = [mist.TensorList(x) for x in (p, m, v, grads)]
    W = mist.TensorList(weights) if w else None
    rec = mist.StepRecord(step=step)
    for k in range(2):
        x = as64(grads)
        was = as64(p), as64(m), as64(v)
        mist.grad_norm(lists[3], rec, max_norm=1.0, grad_scale=0.5)
        norm = 0.5 * math.sqrt(float((x * x).sum()))
        x = x * (0.5 * (1.0 / norm if norm > 1.0 else 1.0))
        mist.adam_step(*lists, rec, weights=W, **hyper)
        assert int(rec.step) == step + 1 + k
        new, nm, nv, sp, sm, sv = adam(*was, x, step + 1 + k, 3e-3, 0.9, 0.95, 1e-8, hyper["weight_decay"])
        within(as64(m), nm, sm, "m")
        within(as64(v), nv, sv, "v")
        within(as64(p), new, sp, "p")
        if w:
            assert all(torch.equal(a, b.to(a.dtype)) for a, b in zip(weights, p))
        for f, views in ((pf, p), (mf, m), (vf, v), (gf, grads), (wf, weights)):
            untouched(torch, f, views)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_non_finite_gradients_change_nothing(torch, bad):
    """One inf or NaN anywhere: the step is skipped and counted as skipped, and the next one goes on from there."""
    from paper_2503_19050_amd import mist
    rng = np.random.default_rng(9)
    S = SIZES["layers"]
    views = [tensors(torch, rng, S, t, 0.1, 1)[1] for t in ("f32", "f32", "f32", "f16", "bf16")]
    for t in views[2]:
        t.square_()
    lists = [mist.TensorList(x) for x in views]
    rec = mist.StepRecord(step=4)
    for where in (0, len(S) // 2, len(S) - 1):
        keep = views[3][where][-1].clone()
        views[3][where][-1] = bad
        before = [[t.clone() for t in x] for x in views]
        mist.grad_norm(lists[3], rec, max_norm=1.0, grad_scale=2.0)
        mist.adam_step(*lists[:4], rec, lr=0.1, weights=lists[4], weight_decay=0.1)
        assert int(rec.applied) == 0 and int(rec.step) == 4
        for x, y in zip(views, before):
            assert all(torch.equal(a.view(torch.int16 if a.element_size() == 2 else torch.int32),
                                   b.view(torch.int16 if b.element_size() == 2 else torch.int32)) for a, b in zip(x, y))
        out = [torch.empty_like(t, dtype=torch.float32) for t in views[3]]
        mist.grad_clip(lists[3], rec, mist.TensorList(out))
        assert all(torch.equal(a.nan_to_num(7.0), b.float().nan_to_num(7.0)) for a, b in zip(out, views[3]))
        views[3][where][-1] = keep
    assert int(rec.skipped) == 3
    mist.grad_norm(lists[3], rec, max_norm=1.0)
    mist.adam_step(*lists[:4], rec, lr=0.1, weights=lists[4])
    assert int(rec.applied) == 1 and int(rec.step) == 5
    assert all(t.isfinite().all() for x in views for t in x)


def test_zero_gradients(torch):
    from paper_2503_19050_amd import mist
    g = torch.zeros(1000, device="cuda")
    p, m, v = torch.ones(1000, device="cuda"), torch.zeros(1000, device="cuda"), torch.zeros(1000, device="cuda")
    lists = [mist.TensorList([t]) for t in (p, m, v, g)]
    rec = mist.StepRecord()
    mist.grad_norm(lists[3], rec, max_norm=1.0)
    mist.adam_step(*lists, rec, lr=0.5)
    assert float(rec.norm) == 0.0 and float(rec.coef) == 1.0 and (p == 1).all() and (m == 0).all() and (v == 0).all()


def test_streams_and_graphs(torch):
    """A whole step captured once and replayed, with other work between the replays, against the same steps made
    one by one; and on a stream of the caller's."""
    from paper_2503_19050_amd import mist
    rng = np.random.default_rng(12)
    S = SIZES["layers"] + [100003]

    def state():
        r = np.random.default_rng(13)
        return [tensors(torch, r, S, t, 0.1, 1)[1] for t in ("f32", "f32", "f32", "bf16", "bf16")]

    def step(lists, rec, stream=None):
        mist.grad_norm(lists[3], rec, max_norm=1.0, stream=stream)
        mist.grad_clip(lists[3], rec, stream=stream)
        mist.adam_step(*lists[:4], rec, lr=0.01, weights=lists[4], stream=stream)

    A, B = state(), state()
    for x in A[2] + B[2]:
        x.square_()
    LA, LB = [mist.TensorList(x) for x in A], [mist.TensorList(x) for x in B]
    ra, rb = mist.StepRecord(step=1), mist.StepRecord(step=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(LA, ra)
    step(LB, rb, side)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(A, B) for a, b in zip(x, y))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(LB, rb)
    for k in range(4):
        for a, b in zip(A[3], B[3]):
            a.normal_(0.0, 0.1 * (k + 1))
            b.copy_(a)
        if k == 2:
            A[3][0][0] = B[3][0][0] = float("nan")
        graph.replay()
        torch.cuda.synchronize()
        step(LA, ra)
        assert all(torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0)) for x, y in zip(A, B) for a, b in zip(x, y))
        assert int(ra.step) == int(rb.step) == 3 + k - (k >= 2)
        torch.randn(1 << 20, device="cuda").sum().item()


def test_refusals(torch):
    from paper_2503_19050_amd import mist
    f = [torch.zeros(5, device="cuda") for _ in range(6)]
    with pytest.raises(mist.MistError):
        mist.TensorList([])
    with pytest.raises(mist.MistError):
        mist.TensorList([f[0], f[1].half()])
    with pytest.raises(mist.MistError):
        mist.TensorList([f[0].cpu()])
    with pytest.raises(mist.MistError):
        mist.TensorList([torch.zeros(5, 6, device="cuda").t()])
    with pytest.raises(mist.MistError):
        mist.TensorList([f[0].double()])
    P, M, V, G, X = (mist.TensorList([t]) for t in f[:5])
    other, half = mist.TensorList([torch.zeros(6, device="cuda")]), mist.TensorList([f[5].half()])
    rec = mist.StepRecord()
    bad = [lambda: mist.grad_norm(G, rec, max_norm=0.0), lambda: mist.grad_norm(G, rec, max_norm=float("nan")),
           lambda: mist.grad_norm(G, rec, grad_scale=0.0), lambda: mist.grad_norm(G, rec, grad_scale=float("inf")),
           lambda: mist.grad_norm(G, rec, kind="l1"), lambda: mist.grad_clip(G, rec, other),
           lambda: mist.adam_step(P, M, V, other, rec, lr=0.1), lambda: mist.adam_step(P, M, half, G, rec, lr=0.1),
           lambda: mist.adam_step(P, M, M, G, rec, lr=0.1), lambda: mist.adam_step(P, M, V, G, rec, lr=-1.0),
           lambda: mist.adam_step(P, M, V, G, rec, lr=0.1, betas=(1.0, 0.9)),
           lambda: mist.adam_step(P, M, V, G, rec, lr=0.1, eps=-1.0), lambda: mist.adam_step(P, M, V, G, rec, lr=0.1, eps=0.0),
           lambda: mist.adam_step(P, M, V, G, rec, lr=0.1, eps=1e-60), lambda: mist.adam_step(P, M, V, G, rec, lr=0.1, weights=P),
           lambda: mist.adam_step(P, M, V, G, rec, lr=float("nan")), lambda: mist.grad_finish(rec, max_norm=-1.0)]
    for call in bad:
        with pytest.raises(mist.MistError) as e:
            call()
        assert e.value.status == -1 and str(e.value)
    X.close()
    with pytest.raises(mist.MistError):
        mist.grad_norm(X, rec)
    assert int(rec.step) == 0 and mist.load().mist_grad_norm(G.h, None, 0, 1, rec.data.data_ptr(), None, 0, None) == -1


def test_list_without_device_memory(torch):
    """An allocator that has nothing: MIST_E_NOMEM, no list, nothing freed that was not given."""
    import ctypes
    from paper_2503_19050_amd import mist
    L, freed = mist.load(), []
    cb = mist.ALLOC_FN(lambda n, s, c: None), mist.FREE_FN(lambda p, c: freed.append(p))
    t = torch.ones(5, device="cuda")
    out = ctypes.c_void_p(1)
    rc = L.mist_tensors_create((ctypes.c_void_p * 1)(t.data_ptr()), (ctypes.c_int64 * 1)(5), 1, 0,
                               ctypes.byref(mist.Allocator(cb[0], cb[1], None)), ctypes.byref(out))
    assert rc == -2 and not out.value and not freed and L.mist_last_error()


@pytest.mark.parametrize("allocator", ["torch", None])
def test_lists_come_and_go(torch, allocator):
    """A list's tables are returned when it is closed; the tensors stay."""
    from paper_2503_19050_amd import mist
    t = [torch.full((1000,), float(k), device="cuda") for k in range(50)]
    gc.collect()  # what earlier tests left
    before = torch.cuda.memory_allocated()
    for _ in range(3):
        with mist.TensorList(t, allocator=allocator) as T:
            rec = mist.StepRecord()
            mist.grad_norm(T, rec)
            assert float(rec.total) == sum(1000.0 * k * k for k in range(50)) and len(T) == 50
        del rec
    gc.collect()
    assert torch.cuda.memory_allocated() == before
    assert all((x == k).all() for k, x in enumerate(t))
