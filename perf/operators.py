"""Timed cases of the training-step operators: the embedding and its gradient, the global gradient
norm with clipping, and the Adam step, over the shapes of the models that the tuner plans for.

    embed       look up a microbatch's tokens in one vocabulary shard (scaled, with learned positions)
    embed_grad  the gradient of the shard's rows and of the positions
    clip        global norm of a stage's gradients, and the clipped gradients
    adam        global norm, then the Adam step of a stage's parameters with the clip factor

A stage's tensors are those of its layers (as the cost model counts them) in flat buffers.
"""

from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
GPT, LLAMA = "gpt", "llama"

MOST_CELLS = 1 << 29       # tokens x hidden of a drawn embedding case, at most (the largest listed one has 2^30, of 16 bits)
MOST_TABLE = 270_000_000   # values of a drawn case's table shard, at most
MOST_PARAMS = 540_000_000  # parameters of a drawn stage, at most (the largest listed one: 6.3e8, of fewer bytes each)
BETA1, BETA2, EPS = 0.9, 0.95, 1e-8


def _embed(name, op, batch, seq, vocab, hidden, shards=1, shard=0, pos=False, scale=1.0, dtype="bf16", grad="",
           ids="i64", pad=0.0, accumulate=False):
    c = dict(op=op, batch=batch, seq=seq, vocab=vocab, hidden=hidden, shards=shards, shard=shard, pos=pos,
             scale=scale, dtype=dtype, grad=grad or dtype, ids=ids, pad=pad, accumulate=accumulate)
    return dict(name=name, **c) if name else c


def _stage(name, op, arch, layers, hidden, ffn, kv=0, tp=1, vocab=0, seq=0, grad="bf16", out="bf16", shift=0,
           max_norm=1.0, size=3e-4, step=100, decay=0.1):
    c = dict(op=op, arch=arch, layers=layers, hidden=hidden, ffn=ffn, kv=kv or hidden, tp=tp, vocab=vocab, seq=seq,
             grad=grad, out=out, shift=shift, max_norm=max_norm, size=size, step=step, decay=decay)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # One short sequence of a small model: launches and latency count.
        _embed("embed-tiny-1x128", "embed", 1, 128, 1000, 256, pos=True),
        # The largest microbatch of the ordinary query's model, learned positions.
        _embed("embed-gpt2.7b-32x2048", "embed", 32, 2048, 50257, 2560, pos=True),
        # One of eight vocabulary shards of the largest model: most tokens lie in other shards and give zeros.
        _embed("embed-llama42b-tp8-4x8192", "embed", 4, 8192, 32000, 8192, shards=8, shard=0, scale=90.5, ids="i32"),
        # One microbatch of a small model in 32 bits.
        _embed("grad-tiny-1x256", "embed_grad", 1, 256, 2048, 512, dtype="f32"),
        # One sequence added to 32-bit gradients that gather over microbatches: only the rows that occur change.
        _embed("grad-llama7b-1x4095-add", "embed_grad", 1, 4095, 32000, 4096, grad="f32", accumulate=True),
        # The ordinary query's largest microbatch, overwriting 16-bit gradients, with positions.
        _embed("grad-gpt2.7b-32x2048", "embed_grad", 32, 2048, 50257, 2560, pos=True),
        # The largest: 16 sequences of 8192 tokens, a quarter of them padding.
        _embed("grad-llama42b-16x8192", "embed_grad", 16, 8192, 32000, 8192, ids="i32", pad=0.25),
        # Every tensor of a small model: many tensors of which most are small.
        _stage("clip-tiny-l4", "clip", GPT, 4, 256, 1024, vocab=1000, seq=128, grad="f32", out="f32"),
        # Six layers of the 1.3B model; 32-bit gathered gradients to the 16 bits that are sent on.
        _stage("clip-gpt1.3b-l6", "clip", GPT, 6, 2048, 8192, grad="f32", out="bf16"),
        # A small model's whole step.
        _stage("adam-tiny-l6", "adam", LLAMA, 6, 512, 1408, kv=128, vocab=2048),
        # One layer's shard, which starts at an odd element (a ZeRO rank's share), gradients within the bound.
        _stage("adam-llama13b-l1-tp8", "adam", LLAMA, 1, 5120, 13824, tp=8, grad="f16", out="f16", shift=1,
               max_norm=100.0),
        # Eight layers of the 2.7B model: a pipeline stage of the ordinary query's plans.
        _stage("adam-gpt2.7b-l8", "adam", GPT, 8, 2560, 10240),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _hidden(rng):
    """Mostly a multiple of 8, as heads of 16 to 128 make it, sometimes odd."""
    return 40 * _log_int(rng, 2, 204) if rng.random() < 0.8 else 2 * _log_int(rng, 33, 4095) + 1


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "clip", "adam"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("embed", "embed_grad"):
        while True:
            batch, seq = _log_int(rng, 1, 32), rng.choice([1 << rng.randrange(14), 2 * _log_int(rng, 1, 4096) - 1])
            hidden = _hidden(rng)
            vocab, shards = 2 * _log_int(rng, 250, 25128) + 1, rng.choice([1, 1, 2, 8])
            if batch * seq * hidden <= MOST_CELLS and vocab // shards * hidden <= MOST_TABLE:
                break
        grad = rng.choice([dtype, "f32"])
        return _embed(None, op, batch, seq, vocab, hidden, shards=shards, shard=rng.randrange(shards),
                      pos=rng.random() < 0.5, scale=rng.choice([1.0, round(math.sqrt(hidden), 3)]), dtype=dtype,
                      grad=grad if op == "embed_grad" else dtype, ids=rng.choice(["i32", "i64"]),
                      pad=rng.choice([0.0, 0.0, round(rng.uniform(0.0, 0.9), 3)]),
                      accumulate=op == "embed_grad" and rng.random() < 0.5)
    while True:
        arch = rng.choice([GPT, LLAMA])
        hidden = _hidden(rng)
        c = _stage(None, op, arch, _log_int(rng, 1, 8), hidden, 40 * _log_int(rng, hidden / 20, hidden / 10),
                   kv=hidden // rng.choice([1, 1, 4]), tp=rng.choice([1, 1, 2, 8]),
                   vocab=rng.choice([0, 0, 2 * _log_int(rng, 250, 16000) + 1]), seq=rng.choice([0, 128, 2048]), grad=dtype,
                   out=rng.choice([dtype, "bf16"]), shift=rng.choice([0, 0, 1, 8]),
                   max_norm=rng.choice([0.5, 1.0, 100.0]), size=rng.choice([1e-5, 3e-4, 1e-2]),
                   step=rng.choice([0, 1, 100, 20000]), decay=rng.choice([0.0, 0.1]))
        if sum(_sizes(c)) <= MOST_PARAMS:
            return c


def _sizes(c):
    """Elements of each tensor of a stage: per layer the norms, the attention's and the MLP's weights (and, for
    GPT, their biases), shards over tp rounded up; then the embedding and its positions, if the stage has them."""
    h, f, kv, tp = c["hidden"], -(-c["ffn"] // c["tp"]), -(-c["kv"] // c["tp"]), c["tp"]
    a = -(-h // tp)
    if c["arch"] == GPT:
        layer = [h, h, h * 3 * a, 3 * a, a * h, h, h, h, h * f, f, f * h, h]
    else:
        layer = [h, h * a, h * kv, h * kv, a * h, h, h * f, h * f, f * h]
    top = [-(-c["vocab"] // tp) * h] if c["vocab"] else []
    return layer * c["layers"] + top + ([c["seq"] * h] if c["arch"] == GPT and c["seq"] else [])


def _shard(c):
    rows = -(-c["vocab"] // c["shards"])
    begin = rows * c["shard"]
    return begin, max(1, min(rows, c["vocab"] - begin))


def _ids(c, seed):
    """Tokens as text has them: the k-th of the vocabulary about 1/k as often as the first; padding is -1.  One
    more token a sequence than is looked up, as a loader hands them (the targets are shifted by one)."""
    g = torch.Generator("cuda").manual_seed(seed)
    shape = (c["batch"], c["seq"] + 1)
    u = torch.rand(shape, device="cuda", dtype=torch.float64, generator=g)
    ids = (torch.exp(u * math.log(c["vocab"] + 1)) - 1).long().clamp_(0, c["vocab"] - 1)
    if c["pad"]:
        ids[torch.rand(shape, device="cuda", generator=g) < c["pad"]] = -1
    return ids.to(torch.int32 if c["ids"] == "i32" else torch.int64)[:, :-1], g


def _views(flat, sizes, shift):
    return list(flat[shift:shift + sum(sizes)].split(sizes))


def prepare(case, seed):
    c = case
    if c["op"] in ("embed", "embed_grad"):
        ids, g = _ids(c, seed)
        begin, rows = _shard(c)

        def normal(*shape, std, dtype):
            return torch.empty(shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=g)

        s = dict(c=c, ids=ids, begin=begin, rows=rows)
        if c["op"] == "embed":
            s["table"] = normal(rows, c["hidden"], std=0.02, dtype=TYPES[c["dtype"]])
            s["pos"] = normal(c["seq"], c["hidden"], std=0.02, dtype=TYPES[c["dtype"]]) if c["pos"] else None
            s["out"] = torch.empty(c["batch"], c["seq"], c["hidden"], device="cuda", dtype=TYPES[c["dtype"]])
        else:
            s["dout"] = normal(c["batch"], c["seq"], c["hidden"], std=1e-2, dtype=TYPES[c["dtype"]])
            kind = TYPES[c["grad"]]
            s["dtable"] = normal(rows, c["hidden"], std=1e-2, dtype=kind)
            s["dpos"] = normal(c["seq"], c["hidden"], std=1e-2, dtype=kind) if c["pos"] else None
        return s
    sizes, g = _sizes(c), torch.Generator("cuda").manual_seed(seed)
    n, shift = sum(sizes), c["shift"]

    def flat(std, dtype):
        return torch.empty(n + shift, device="cuda", dtype=dtype).normal_(0.0, std, generator=g)

    s = dict(c=c, sizes=sizes, n=n, grad=flat(c["size"], TYPES[c["grad"]]))
    s["out"] = torch.zeros(n + shift, device="cuda", dtype=TYPES[c["out"]])
    if c["op"] == "adam":
        s["master"] = flat(0.02, torch.float32)
        s["m"] = flat(c["size"], torch.float32) if c["step"] else torch.zeros(n + shift, device="cuda")
        s["v"] = flat(c["size"], torch.float32).square_() if c["step"] else torch.zeros(n + shift, device="cuda")
    s["step"] = torch.full((), c["step"], device="cuda", dtype=torch.int64)
    if own:
        from paper_2503_19050_amd import mist
        s["record"] = mist.StepRecord(step=c["step"])
        s["lists"] = {k: mist.TensorList(_views(s[k], sizes, shift)) for k in ("grad", "out", "master", "m", "v")
                      if k in s}
    return s


def _embed_plain(s):
    c = s["c"]
    row = s["ids"].long() - s["begin"]
    inside = (row >= 0) & (row < s["rows"])
    x = s["table"][row.clamp(0, s["rows"] - 1)].float() * c["scale"]
    x = torch.where(inside[..., None], x, torch.zeros((), device=x.device))
    if s["pos"] is not None:
        x = x + s["pos"].float()
    s["out"].copy_(x)
    return s["out"]


def _embed_grad_plain(s):
    c = s["c"]
    row = (s["ids"].long() - s["begin"]).reshape(-1)
    inside = (row >= 0) & (row < s["rows"])
    d = s["dout"].float()
    total = torch.zeros(s["rows"], c["hidden"], device=d.device)
    total.index_add_(0, row[inside], d.reshape(-1, c["hidden"])[inside])
    total = total * c["scale"]
    s["dtable"].copy_(s["dtable"].float() + total if c["accumulate"] else total)
    if s["dpos"] is None:
        return [s["dtable"]]
    total = d.sum(0)
    s["dpos"].copy_(s["dpos"].float() + total if c["accumulate"] else total)
    return [s["dtable"], s["dpos"]]


def _norm_plain(s):
    norm = s["g"].square().sum().sqrt()
    most = s["c"]["max_norm"]
    return norm, torch.where(norm > most, most / norm, torch.ones_like(norm))


def _step_plain(s):
    c = s["c"]
    part = slice(c["shift"], c["shift"] + s["n"])
    s["g"] = s["grad"][part].float()
    norm, coef = _norm_plain(s)
    g = s.pop("g") * coef
    if c["op"] == "clip":
        s["out"][part].copy_(g)
        return [s["out"], norm]
    s["step"] += 1
    t = s["step"].double()
    bc1, bc2 = (1 - BETA1 ** t).float(), (1 - BETA2 ** t).float()
    p, m, v = s["master"][part], s["m"][part], s["v"][part]
    m.copy_(BETA1 * m + (1 - BETA1) * g)
    v.copy_(BETA2 * v + (1 - BETA2) * g * g)
    p.copy_(p - 1e-4 * ((m / bc1) / ((v / bc2).sqrt() + EPS) + c["decay"] * p))
    s["out"][part].copy_(p)
    return [s["master"], s["m"], s["v"], s["out"], norm]


def run(state):
    s, c = state, state["c"]
    if not own:
        return {"embed": _embed_plain, "embed_grad": _embed_grad_plain}.get(c["op"], _step_plain)(s)
    from paper_2503_19050_amd import mist
    if c["op"] == "embed":
        return mist.embed(s["ids"], s["table"], scale=c["scale"], pos=s["pos"], vocab_begin=s["begin"], out=s["out"])
    if c["op"] == "embed_grad":
        mist.embed_grad(s["ids"], s["dout"], s["dtable"], scale=c["scale"], dpos=s["dpos"], vocab_begin=s["begin"],
                        accumulate=c["accumulate"])
        return [s["dtable"]] if s["dpos"] is None else [s["dtable"], s["dpos"]]
    lists, record = s["lists"], s["record"]
    mist.grad_norm(lists["grad"], record, max_norm=c["max_norm"])
    if c["op"] == "clip":
        mist.grad_clip(lists["grad"], record, out=lists["out"])
        return [s["out"], record.norm]
    mist.adam_step(lists["master"], lists["m"], lists["v"], lists["grad"], record, lr=1e-4, betas=(BETA1, BETA2),
                   eps=EPS, weight_decay=c["decay"], weights=lists["out"])
    return [s["master"], s["m"], s["v"], s["out"], record.norm]


def exact(case, seed):
    s, c = prepare(case, seed), case
    ids = s["ids"].reshape(-1).tolist() if "ids" in s else []
    if c["op"] == "embed":
        zero = torch.zeros(1, c["hidden"], device="cuda", dtype=torch.float64)
        table = torch.cat([s["table"].double() * c["scale"], zero])   # the last row: tokens of no row here
        at = [i - s["begin"] if 0 <= i - s["begin"] < s["rows"] else s["rows"] for i in ids]
        out = table.index_select(0, torch.tensor(at, device="cuda")).reshape(c["batch"], c["seq"], c["hidden"])
        return out if s["pos"] is None else out.add_(s["pos"].double()[None])
    if c["op"] == "embed_grad":
        # sums of runs of equal ids: differences of a running sum would cancel, so the runs are summed one by one
        # level at a time, by halving: rows of the same id are paired until each id has one.
        d = s["dout"].reshape(-1, c["hidden"])
        key = torch.tensor(ids, device="cuda") - s["begin"]
        order = torch.argsort(key, stable=True)
        order = order[(key[order] >= 0) & (key[order] < s["rows"])]
        out = torch.zeros(s["rows"], c["hidden"], device="cuda", dtype=torch.float64)
        for lo in range(0, c["hidden"], 1024):
            x, k = d[:, lo:lo + 1024][order].double(), key[order]
            while len(k):
                start = torch.ones(len(k), device="cuda", dtype=torch.bool)
                start[1:] = k[1:] != k[:-1]
                first = torch.where(start, torch.arange(len(k), device="cuda"), 0).cummax(0).values
                odd = (torch.arange(len(k), device="cuda") - first) % 2 == 1
                if not bool(odd.any()):
                    break
                at = odd.nonzero()[:, 0]
                x[at - 1] += x[at]
                x, k = x[~odd], k[~odd]
            out[k, lo:lo + 1024] = x
        out *= c["scale"]
        pos = s["dout"].double().sum(0) if s["dpos"] is not None else None
        if c["accumulate"]:
            out += s["dtable"].double()
            pos = None if pos is None else pos + s["dpos"].double()
        return [out] if pos is None else [out, pos]
    a, b = c["shift"], c["shift"] + s["n"]
    total = math.fsum(float(x.double().pow(2).sum()) for x in s["grad"][a:b].split(1 << 24))
    norm = math.sqrt(total)
    factor = c["max_norm"] / norm if norm > c["max_norm"] else 1.0
    out = s["out"].double()
    said = torch.tensor(norm, dtype=torch.float64)
    if c["op"] == "clip":
        out[a:b] = s["grad"][a:b].double() * factor
        return [out, said]
    got = [s[k].double() for k in ("master", "m", "v")] + [out]
    t = c["step"] + 1
    for lo in range(a, b, 1 << 25):
        r = slice(lo, min(b, lo + (1 << 25)))
        p, m, v = (x[r] for x in got[:3])
        g = s["grad"][r].double() * factor
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g ** 2
        change = m / (1 - BETA1 ** t) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
        p = p * (1 - 1e-4 * c["decay"]) - 1e-4 * change
        for x, y in zip(got, (p, m, v, p)):
            x[r] = y
    return got + [said]


def _distinct(c):
    """Rows of the shard that occur, as expected of the tokens' distribution."""
    begin, rows = _shard(c)
    n, top = c["batch"] * c["seq"] * (1 - c["pad"]), math.log(c["vocab"] + 1)
    k = torch.arange(begin, begin + rows, dtype=torch.float64)
    p = torch.log1p(1 / (k + 1)) / top
    return float((1 - torch.exp(n * torch.log1p(-p))).sum())


def work(case):
    c = case
    if c["op"] in ("embed", "embed_grad"):
        n, h, e, rows = c["batch"] * c["seq"], c["hidden"], BYTES[c["dtype"]], _shard(c)[1]
        ids = n * (4 if c["ids"] == "i32" else 8)
        used = min(_distinct(c), rows)
        if c["op"] == "embed":
            return {"bytes": ids + (n + used + c["pos"] * c["seq"]) * h * e, "flops": (1 + c["pos"]) * n * h}
        w = BYTES[c["grad"]]
        table = 2 * used if c["accumulate"] else rows
        pos = c["pos"] * c["seq"] * (2 if c["accumulate"] else 1)
        # without positions, the gradients of tokens outside the shard are not needed
        begin, top = _shard(c)[0], math.log(c["vocab"] + 1)
        share = 1.0 if c["pos"] else (1 - c["pad"]) * (math.log(begin + rows + 1) - math.log(begin + 1)) / top
        return {"bytes": ids + n * share * h * e + (table + pos) * h * w, "flops": (1 + c["pos"]) * n * share * h}
    n = sum(_sizes(c))
    if c["op"] == "clip":
        return {"bytes": n * (BYTES[c["grad"]] + BYTES[c["out"]]), "flops": 3 * n}
    return {"bytes": n * (BYTES[c["grad"]] + 24 + BYTES[c["out"]]), "flops": 17 * n}
