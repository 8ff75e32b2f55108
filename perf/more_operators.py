"""Timed cases of the operators beside a stage's matrix products: the last stage's loss and token log
probabilities, the norms around a block, and activations kept in 8 bits for the backward pass, over the
shapes of the models that the tuner plans for.

    logprob  log probabilities of given tokens, entropies and the most probable alternatives
    loss     log probabilities of a training microbatch and the logits' gradient of their weighted sum
    shard    one rank's share of the vocabulary: partial results, the ranks' results joined, the gradient of the
             log probabilities and entropies
    norm     the residual's sum with a block's (normed, gated) output, and the next block's norm
    norm_bwd the same with its gradients: a training pass
    ckpt     a tensor stored in 8 bits and loaded again
    act      the MLP's activation with its inputs kept in 8 bits, and its gradients from these: a training pass
"""

from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
GROUP = 128          # values that share a scale in a checkpoint
EPS = 1e-5

MOST_LOGITS = 800_000_000   # logits of a drawn case, at most (the listed ones: up to 1.65e9)
MOST_VALUES = 250_000_000   # tokens x width of a drawn norm or activation, at most (the listed ones: up to 2.7e8)


def _tokens(name, op, batch, seq, vocab, dtype="bf16", pad=0.0, scale=1.0, entropy=False, top=0, shards=1, shard=0, ids="i64"):
    c = dict(op=op, batch=batch, seq=seq, vocab=vocab, dtype=dtype, pad=pad, scale=scale, entropy=entropy, top=top,
             shards=shards, shard=shard, ids=ids)
    return dict(name=name, **c) if name else c


def _block(name, op, batch, seq, hidden, kind="rms", bias=False, post=False, gate="", dtype="bf16", res="", weights="",
           res_scale=1.0, block_scale=1.0):
    c = dict(op=op, batch=batch, seq=seq, hidden=hidden, kind=kind, bias=bias, post=post, gate=gate, dtype=dtype,
             res=res or dtype, weights=weights or dtype, res_scale=res_scale, block_scale=block_scale)
    return dict(name=name, **c) if name else c


def _kept(name, op, tokens, width, dtype="bf16", kind="silu", gated=True, fused=False, again=False):
    c = dict(op=op, tokens=tokens, width=width, dtype=dtype, kind=kind, gated=gated, fused=fused, again=again)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # One token being answered: its log probability, the entropy and twenty alternatives.
        _tokens("logprob-one-50257", "logprob", 1, 1, 50257, scale=1.25, entropy=True, top=20),
        # Scoring of sequences whose last position predicts nothing.
        _tokens("logprob-gpt2.7b-8x2047", "logprob", 8, 2047, 50257, entropy=True, top=8),
        # A small model's loss in 32 bits, some targets padding.
        _tokens("loss-tiny-1x128", "loss", 1, 128, 1000, dtype="f32", pad=0.1),
        # The ordinary query's model, a microbatch of sixteen sequences.
        _tokens("loss-gpt2.7b-16x2048", "loss", 16, 2048, 50257, pad=0.02),
        # One of eight vocabulary shards of the largest model, with an entropy term as reinforcement learning has it.
        _tokens("shard-llama42b-tp8-4x8192", "shard", 4, 8192, 32000, shards=8, shard=3, entropy=True, ids="i32"),
        # The norm before a block for one token being answered.
        _block("norm-one-4096", "norm", 1, 1, 4096),
        # The largest model's residual and next norm.
        _block("norm-llama42b-4x8192", "norm", 4, 8192, 8192),
        # Norms before and after the block, gates by sequence, odd sizes.
        _block("norm_bwd-odd-3x511", "norm_bwd", 3, 511, 1025, kind="layer", bias=True, post=True, gate="sequence",
               dtype="f16", res="f32", weights="f32", res_scale=0.75, block_scale=1.5),
        # The ordinary query's largest microbatch, layer norms with biases.
        _block("norm_bwd-gpt2.7b-32x2048", "norm_bwd", 32, 2048, 2560, kind="layer", bias=True),
        # The input of a recomputed layer of the largest model, kept in 8 bits.
        _kept("ckpt-llama42b-32768", "ckpt", 32768, 8192),
        # A small model's MLP.
        _kept("act-tiny-128x1024", "act", 128, 1024, dtype="f32", kind="gelu", gated=False),
        # Two sequences of the 13B model, gate and up from one product; the activation is formed again for the gradient of its projection.
        _kept("act-llama13b-8192x13824", "act", 8192, 13824, fused=True, again=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, most=8192):
    """Mostly a multiple of 8, as heads of 16 to 128 make it, sometimes odd."""
    return 8 * _log_int(rng, 8, most // 8) if rng.random() < 0.75 else 2 * _log_int(rng, 33, most // 2) - 1


def draw(rng):
    op = rng.choice(["logprob", "loss", "shard", "norm", "norm_bwd", "norm_bwd", "ckpt", "act"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("logprob", "loss", "shard"):
        while True:
            batch, seq = _log_int(rng, 1, 16), _log_int(rng, 1, 8192)
            vocab, shards = _log_int(rng, 100, 130000), rng.choice([2, 4, 8]) if op == "shard" else 1
            if batch * seq * (vocab // shards) <= MOST_LOGITS:
                break
        return _tokens(None, op, batch, seq, vocab, dtype=dtype, pad=rng.choice([0.0, 0.1, 0.5]),
                       scale=rng.choice([1.0, 1.0, 0.5, 1.25]), entropy=op == "shard" or rng.random() < 0.5,
                       top=rng.choice([0, 1, 5, 20]) if op == "logprob" else 0, shards=shards, shard=rng.randrange(shards),
                       ids=rng.choice(["i32", "i64"]))
    while True:
        tokens, width = _log_int(rng, 1, 65536), _width(rng, 8192 if op in ("norm", "norm_bwd") else 24576)
        if tokens * width <= MOST_VALUES // (3 if op == "act" else 1):
            break
    if op in ("ckpt", "act"):
        return _kept(None, op, tokens, width, dtype=dtype, kind=rng.choice(["silu", "gelu"]), gated=rng.random() < 0.5,
                     fused=rng.random() < 0.5, again=rng.random() < 0.5)
    batch, res = rng.choice([1, 2, 5, 8]), rng.choice([dtype, "f32"])
    return _block(None, op, batch, -(-tokens // batch), width, kind=rng.choice(["rms", "layer"]), bias=rng.random() < 0.5,
                  post=rng.random() < 0.5, gate=rng.choice(["", "", "all", "sequence"]), dtype=dtype,
                  res=res, weights=rng.choice([dtype, res]), res_scale=rng.choice([1.0, 1.0, 0.75]),
                  block_scale=rng.choice([1.0, 1.0, 0.5]))


def _shard(c):
    rows = -(-c["vocab"] // c["shards"])
    begin = rows * c["shard"]
    return begin, max(1, min(rows, c["vocab"] - begin))


def _prepare_tokens(c, g):
    """Logits as a trained model has them: most targets well above the rest, a few not; one more position a sequence
    than is scored (its target is not known), targets with one more at the front, as a loader hands them."""
    b, s, dtype = c["batch"], c["seq"], TYPES[c["dtype"]]
    begin, rows = _shard(c)
    logits = torch.empty(b, s + 1, rows, device="cuda", dtype=dtype).normal_(0.0, 2.0, generator=g)
    ids = torch.randint(0, c["vocab"], (b, s + 1), device="cuda", generator=g)
    at = ids[:, 1:] - begin
    here = (at >= 0) & (at < rows)
    lift = torch.rand(b, s, device="cuda", generator=g) * 14
    logits[:, :s].scatter_add_(2, at.clamp(0, rows - 1)[..., None], torch.where(here, lift, torch.zeros_like(lift))[..., None].to(dtype))
    if c["pad"]:
        ids[torch.rand(b, s + 1, device="cuda", generator=g) < c["pad"]] = -1
    ids = ids.to(torch.int32 if c["ids"] == "i32" else torch.int64)
    st = dict(c=c, logits=logits[:, :s], targets=ids[:, 1:])
    if c["op"] == "loss":
        valid = (st["targets"] >= 0)
        st["weights"] = (valid.float() / valid.sum().clamp(min=1)).contiguous()
        st["dlogits"] = torch.empty(b, s, rows, device="cuda", dtype=dtype)
    if c["op"] == "shard":
        st["begin"] = begin
        st["dlogits"] = torch.empty(b, s, rows, device="cuda", dtype=dtype)
        st["dlogp"] = torch.empty(b, s, device="cuda").normal_(0.0, 1.0, generator=g)
        st["dentropy"] = torch.full((b, s), 1e-2, device="cuda")
        # what the other ranks send: largest logit, sum of exponentials, sum of exponentials times logits above it, the
        # target's logit (-inf: not theirs)
        other = torch.empty(c["shards"], b, s, 64, device="cuda").normal_(0.0, 2.0, generator=g) * c["scale"]
        most = other.max(-1).values
        d = other - most[..., None]
        stats = torch.stack([most, d.exp().sum(-1), (d.exp() * d).sum(-1), torch.full_like(most, -math.inf)], -1)
        owner = torch.div(st["targets"].long(), -(-c["vocab"] // c["shards"]), rounding_mode="floor")
        theirs = torch.arange(c["shards"], device="cuda")[:, None, None] == owner
        stats[..., 3] = torch.where(theirs, other[..., 0], stats[..., 3])
        st["stats"] = stats
    return st


def _prepare_block(c, g):
    b, s, h = c["batch"], c["seq"], c["hidden"]
    dtype, res, wt = TYPES[c["dtype"]], TYPES[c["res"]], TYPES[c["weights"]]

    def normal(*shape, std, dtype, mean=0.0):
        return torch.empty(shape, device="cuda", dtype=dtype).normal_(mean, std, generator=g)

    st = dict(c=c, x=normal(b, s, h, std=1.5, dtype=res, mean=0.1), block=normal(b, s, h, std=0.5, dtype=dtype))
    st["weight"] = normal(h, std=0.1, dtype=wt, mean=1.0)
    st["bias"] = normal(h, std=0.1, dtype=wt) if c["bias"] else None
    st["post_weight"] = normal(h, std=0.1, dtype=wt, mean=1.0) if c["post"] else None
    st["post_bias"] = normal(h, std=0.1, dtype=wt) if c["post"] and c["bias"] else None
    st["gate"] = normal(*((b, h) if c["gate"] == "sequence" else (h,)), std=0.3, dtype=wt, mean=0.5) if c["gate"] else None
    if c["op"] == "norm_bwd":
        st["dh"] = normal(b, s, h, std=1e-2, dtype=dtype)
        st["dy"] = normal(b, s, h, std=1e-2, dtype=res)
        for k in ("weight", "bias", "post_weight", "post_bias", "gate"):
            if st[k] is not None:
                st["d" + k] = torch.empty(st[k].shape, device="cuda", dtype=wt)
    return st


def _prepare_kept(c, g):
    n, w, dtype = c["tokens"], c["width"], TYPES[c["dtype"]]

    def normal(*shape, std):
        return torch.empty(shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=g)

    if c["op"] == "ckpt":
        # a residual stream: a few channels are far larger than the others
        x = normal(n, w, std=1.0)
        x[:, torch.randint(0, w, (max(1, w // 512),), device="cuda", generator=g)] *= 12
        return dict(c=c, x=x, out=torch.empty_like(x))
    st = dict(c=c, dout=normal(n, w, std=1e-2), gate=None)
    if c["gated"] and c["fused"]:
        both = normal(n, 2 * w, std=1.5)
        st["gate"], st["up"] = both[:, :w], both[:, w:]
    else:
        st["up"] = normal(n, w, std=1.5)
        if c["gated"]:
            st["gate"] = normal(n, w, std=1.5)
    return st


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    kind = {"norm": _prepare_block, "norm_bwd": _prepare_block, "ckpt": _prepare_kept, "act": _prepare_kept}
    return kind.get(case["op"], _prepare_tokens)(case, g)


# ---- plain forms ---------------------------------------------------------------------------------
def _stats_plain(z):
    most = z.max(-1).values
    d = z - most[..., None]
    e = d.exp()
    return most, e.sum(-1), (e * d).sum(-1)


def _target_plain(z, targets, begin):
    at = targets.long() - begin
    here = (at >= 0) & (at < z.shape[-1])
    found = z.gather(-1, at.clamp(0, z.shape[-1] - 1)[..., None])[..., 0]
    return torch.where(here, found, torch.full_like(found, -math.inf)), at, here


def _logprob_plain(s):
    c = s["c"]
    z = s["logits"].float() * c["scale"]
    most, total, moment = _stats_plain(z)
    lse = most + total.log()
    found, _, _ = _target_plain(z, s["targets"], 0)
    out = [torch.where(s["targets"] >= 0, found - lse, torch.zeros_like(lse)), lse]
    if c["entropy"]:
        out.append(total.log() - moment / total)
    if c["top"]:
        del z
        # distinct keys in the logits' order, the lower index first among equals
        bits = (s["logits"].float() + 0.0).view(torch.int32).long()
        order = torch.where(bits >= 0, bits, -2147483648 - bits)
        key = order * (1 << 32) + (0xFFFFFFFF - torch.arange(bits.shape[-1], device=bits.device))
        del bits, order
        ids = 0xFFFFFFFF - (torch.topk(key, c["top"]).values & 0xFFFFFFFF)
        values = s["logits"].gather(-1, ids).float() * c["scale"] - lse[..., None]
        out += [ids.int(), values]
    return out


def _loss_plain(s):
    c = s["c"]
    z = s["logits"].float() * c["scale"]
    most, total, _ = _stats_plain(z)
    lse = most + total.log()
    found, at, _ = _target_plain(z, s["targets"], 0)
    valid = s["targets"] >= 0
    w = torch.where(valid, s["weights"], torch.zeros_like(lse)) * c["scale"]
    d = (z - lse[..., None]).exp_().mul_(w[..., None])
    d.scatter_add_(-1, at.clamp(min=0)[..., None], -w[..., None])
    s["dlogits"].copy_(d)
    return [torch.where(valid, found - lse, torch.zeros_like(lse)), s["dlogits"]]


def _shard_plain(s):
    c = s["c"]
    z = s["logits"].float() * c["scale"]
    most, total, moment = _stats_plain(z)
    found, at, here = _target_plain(z, s["targets"], s["begin"])
    stats = s["stats"].clone()
    stats[c["shard"]] = torch.stack([most, total, moment, found], -1)
    m = stats[..., 0].max(0).values
    f = (stats[..., 0] - m).exp()
    total = (f * stats[..., 1]).sum(0)
    moment = (f * (stats[..., 2] + (stats[..., 0] - m) * stats[..., 1])).sum(0)
    lse = m + total.log()
    entropy = total.log() - moment / total
    valid = s["targets"] >= 0
    logp = torch.where(valid, stats[..., 3].max(0).values - lse, torch.zeros_like(lse))
    dlogp = torch.where(valid, s["dlogp"], torch.zeros_like(lse))
    lp = z - lse[..., None]
    d = lp.exp() * (-dlogp[..., None] - s["dentropy"][..., None] * (lp + entropy[..., None]))
    d.scatter_add_(-1, at.clamp(0, z.shape[-1] - 1)[..., None], torch.where(here, dlogp, torch.zeros_like(dlogp))[..., None])
    s["dlogits"].copy_(d * c["scale"])
    return [logp, entropy, s["dlogits"]]


def _normed_plain(x, kind):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _affine_plain(x, weight, bias):
    x = x * weight.float()
    return x if bias is None else x + bias.float()


def _block_plain(s):
    c = s["c"]
    x, b = s["x"].float(), s["block"].float()
    gate = None if s["gate"] is None else s["gate"].float()
    if c["gate"] == "sequence":
        gate = gate[:, None]
    v = b
    if c["post"]:
        bn, br = _normed_plain(b, c["kind"])
        v = _affine_plain(bn, s["post_weight"], s["post_bias"])
    gated = v if gate is None else v * gate
    y = c["res_scale"] * x + c["block_scale"] * gated
    yn, yr = _normed_plain(y, c["kind"])
    h = _affine_plain(yn, s["weight"], s["bias"])
    out = dict(y=y.to(s["x"].dtype), h=h.to(s["block"].dtype))
    if c["op"] == "norm":
        return out

    def back(d, n, r):
        m = d.mean(-1, keepdim=True) if c["kind"] == "layer" else 0.0
        return r * (d - m - n * (d * n).mean(-1, keepdim=True))

    dh = s["dh"].float()
    s["dweight"].copy_((dh * yn).sum((0, 1)))
    if c["bias"]:
        s["dbias"].copy_(dh.sum((0, 1)))
    d = s["dy"].float() + back(dh * s["weight"].float(), yn, yr)
    out["dx"] = (c["res_scale"] * d).to(s["x"].dtype)
    d = c["block_scale"] * d
    if gate is not None:
        s["dgate"].copy_((d * v).sum(1) if c["gate"] == "sequence" else (d * v).sum((0, 1)))
        d = d * gate
    if c["post"]:
        s["dpost_weight"].copy_((d * bn).sum((0, 1)))
        if c["bias"]:
            s["dpost_bias"].copy_(d.sum((0, 1)))
        d = back(d * s["post_weight"].float(), bn, br)
    out["dblock"] = d.to(s["block"].dtype)
    out.update({k: s[k] for k in ("dweight", "dbias", "dpost_weight", "dpost_bias", "dgate") if k in s})
    return out


def _power_of_two(e):
    return ((e + 1023) << 52).view(torch.float64)


def _kept_plain(x):
    """x as its checkpoint holds it: groups of 128 along the row, each with the least power of two under which the largest
    magnitude is at most 127, values rounded to whole multiples of it."""
    n, w = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -w % GROUP)).view(n, -1, GROUP)
    most = x.abs().amax(-1, keepdim=True).double()
    _, e = torch.frexp(most / 127.0)
    e = e.long() - (most <= 127.0 * _power_of_two(e.long() - 1)).long()
    step = _power_of_two(e.clamp(-126, 121)).float()
    return ((x / step).round() * step).view(n, -1)[:, :w]


def _act_plain(x, kind):
    """The activation and its derivative."""
    if kind == "silu":
        p = 1 / (1 + (-x).exp())
        return x * p, p * (1 + x * (1 - p))
    k = 2 * math.sqrt(2 / math.pi)
    p = 1 / (1 + (-k * (x + 0.044715 * x * x * x)).exp())
    return x * p, p + x * p * (1 - p) * k * (1 + 3 * 0.044715 * x * x)


def _acts_plain(s):
    c, dtype = s["c"], s["up"].dtype

    def joined(up, gate):
        return _act_plain(up, c["kind"])[0] if gate is None else _act_plain(gate, c["kind"])[0] * up

    up, gate = s["up"], s["gate"]
    out = [joined(up.float(), None if gate is None else gate.float()).to(dtype)]
    up, gate, d = _kept_plain(up), None if gate is None else _kept_plain(gate), s["dout"].float()
    a, da = _act_plain(up if gate is None else gate, c["kind"])
    out += [(d * da).to(dtype)] if gate is None else [(d * a).to(dtype), (d * up * da).to(dtype)]
    if c["again"]:
        out.append(joined(up, gate).to(dtype))
    return out


def _ckpt_plain(s):
    s["out"].copy_(_kept_plain(s["x"]))
    return s["out"]


# ---- the framework's calls -----------------------------------------------------------------------
def _tokens_own(s, mist):
    c = s["c"]
    if c["op"] == "logprob":
        r = mist.token_logprob(s["logits"], s["targets"], scale=c["scale"], entropy=c["entropy"], top=c["top"])
        return [x for x in (r.logp, r.lse, r.entropy, r.top_ids, r.top_logp) if x is not None]
    if c["op"] == "loss":
        logp, dlogits = mist.token_loss(s["logits"], s["targets"], s["weights"], scale=c["scale"], dlogits=s["dlogits"])
        return [logp, dlogits]
    # the exchange between ranks: this rank's place in what they all gather
    mist.token_part(s["logits"], s["targets"], vocab_begin=s["begin"], scale=c["scale"], stats=s["stats"][c["shard"]])
    r = mist.token_join(s["stats"], s["targets"], entropy=True)
    mist.token_grad(s["logits"], s["targets"], r.lse, dlogp=s["dlogp"], entropy=r.entropy, dentropy=s["dentropy"],
                    vocab_begin=s["begin"], scale=c["scale"], dlogits=s["dlogits"])
    return [r.logp, r.entropy, s["dlogits"]]


def _block_own(s, mist):
    c = s["c"]
    how = dict(weight=s["weight"], post_weight=s["post_weight"], post_bias=s["post_bias"], gate=s["gate"], kind=c["kind"],
               res_scale=c["res_scale"], block_scale=c["block_scale"])
    r = mist.block_norm(s["x"], s["block"], bias=s["bias"], eps=EPS, stored=False, **how)  # of the sum, as the plain form has it
    out = dict(y=r.y, h=r.h)
    if c["op"] == "norm":
        return out
    grads = {k: s[k] for k in ("dweight", "dbias", "dpost_weight", "dpost_bias", "dgate") if k in s}
    dx, dblock = mist.block_norm_grad(r.y, r.stats, s["dh"], block=s["block"], dy=s["dy"], **how, **grads)
    return dict(out, dx=dx, dblock=dblock, **grads)


def _kept_own(s, mist):
    c = s["c"]
    if c["op"] == "ckpt":
        return mist.checkpoint_load(mist.checkpoint_store(s["x"]), out=s["out"])
    r = mist.mlp_act(s["up"], s["gate"], kind=c["kind"], save=True)
    again = torch.empty_like(r.out) if c["again"] else None
    dup, dgate = mist.mlp_act_grad(s["dout"], r.up, r.gate, kind=c["kind"], out=again)
    return [x for x in (r.out, dup, dgate, again) if x is not None]


def run(state):
    op = state["c"]["op"]
    if own:
        from paper_2503_19050_amd import mist
        return {"norm": _block_own, "norm_bwd": _block_own, "ckpt": _kept_own, "act": _kept_own}.get(op, _tokens_own)(state, mist)
    return {"logprob": _logprob_plain, "loss": _loss_plain, "shard": _shard_plain, "ckpt": _ckpt_plain,
            "act": _acts_plain}.get(op, _block_plain)(state)


# ---- in 64 bits ----------------------------------------------------------------------------------
def _exact_tokens(s, c):
    b, n = s["logits"].shape[:2]
    v = s["logits"].shape[2]
    begin = s.get("begin", 0)
    logits = s["logits"].reshape(b * n, v)
    targets = s["targets"].reshape(-1).long()
    logp, lse, ent = (torch.zeros(b * n, device="cuda", dtype=torch.float64) for _ in range(3))
    ids = torch.zeros(b * n, max(1, c["top"]), device="cuda", dtype=torch.int32)
    values = torch.zeros(b * n, max(1, c["top"]), device="cuda", dtype=torch.float64)
    grad = torch.empty(b * n, v, device="cuda", dtype=torch.float64) if c["op"] != "logprob" else None
    step = max(1, (1 << 27) // v)
    for lo in range(0, b * n, step):
        r = slice(lo, min(b * n, lo + step))
        z = logits[r].double() * c["scale"]
        t = targets[r]
        rows = torch.arange(len(t), device="cuda")
        local = torch.logsumexp(z, -1)
        p = torch.softmax(z, -1)
        mean = torch.where(p > 0, p * z, torch.zeros_like(z)).sum(-1)
        mine = (t >= begin) & (t < begin + v)
        zt = torch.full_like(local, -math.inf)
        zt[mine] = z[rows[mine], t[mine] - begin]
        if c["op"] == "shard":
            q = s["stats"].reshape(c["shards"], b * n, 4)[:, r].double()
            parts = q[..., 0] + torch.log(q[..., 1])
            means = q[..., 0] + q[..., 2] / q[..., 1]
            parts[c["shard"]], means[c["shard"]] = local, mean
            q[c["shard"], :, 3] = zt
            all_ = torch.logsumexp(parts, 0)
            mean = (torch.exp(parts - all_) * means).sum(0)
            zt, local = q[..., 3].amax(0), all_
        lse[r], ent[r] = local, local - mean
        logp[r] = torch.where(t >= 0, zt - local, torch.zeros_like(local))
        if c["op"] == "logprob" and c["top"]:
            # the largest in turn; equal ones by their lowest place
            left = logits[r].double()
            for k in range(c["top"]):
                best = left.amax(-1, keepdim=True)
                at = (left == best).to(torch.uint8).argmax(-1)
                ids[r, k], values[r, k] = at.int(), z[rows, at] - local
                left[rows, at] = -math.inf
        if grad is not None:
            p = torch.exp(z - local[:, None])
            if c["op"] == "loss":
                w = s["weights"].reshape(-1)[r].double()
                up = torch.where(t >= 0, -w, torch.zeros_like(w))
                d = -p * up[:, None]
            else:
                up = torch.where(t >= 0, s["dlogp"].reshape(-1)[r].double(), torch.zeros_like(local))
                slope = s["dentropy"].reshape(-1)[r].double()
                d = -p * (up[:, None] + slope[:, None] * (z - mean[:, None]))
            d[rows[mine], t[mine] - begin] += up[mine]
            grad[r] = d * c["scale"]
    shape = (b, n)
    if c["op"] == "loss":
        return [logp.view(shape), grad.view(b, n, v)]
    if c["op"] == "shard":
        return [logp.view(shape), ent.view(shape), grad.view(b, n, v)]
    out = [logp.view(shape), lse.view(shape)] + ([ent.view(shape)] if c["entropy"] else [])
    return out + ([ids.view(b, n, -1), values.view(b, n, -1)] if c["top"] else [])


def _exact_block(s, c):
    b, n, h = s["x"].shape
    wide = {k: s[k].double() for k in ("weight", "bias", "post_weight", "post_bias", "gate") if s[k] is not None}
    y = torch.empty(b, n, h, device="cuda", dtype=torch.float64)
    out = dict(y=y, h=torch.empty_like(y))
    train = c["op"] == "norm_bwd"
    if train:
        out.update(dx=torch.empty_like(y), dblock=torch.empty_like(y))
        out.update({"d" + k: torch.zeros_like(v) for k, v in wide.items()})
    step = max(1, (1 << 26) // h)
    for i in range(b):
        for lo in range(0, n, step):
            r = slice(lo, min(n, lo + step))
            x, f = s["x"][i, r].double(), s["block"][i, r].double()
            gate = wide.get("gate", torch.ones((), device="cuda", dtype=torch.float64))
            gate = gate[i] if c["gate"] == "sequence" else gate

            def stats(t):
                mu = t.mean(-1, keepdim=True) if c["kind"] == "layer" else torch.zeros_like(t[:, :1])
                return mu, 1 / torch.sqrt(((t - mu) ** 2).mean(-1, keepdim=True) + EPS)

            v = f
            if c["post"]:
                mu_f, r_f = stats(f)
                hat_f = (f - mu_f) * r_f
                v = hat_f * wide["post_weight"] + wide.get("post_bias", 0.0)
            yy = c["res_scale"] * x + c["block_scale"] * gate * v
            mu, rr = stats(yy)
            hat = (yy - mu) * rr
            y[i, r], out["h"][i, r] = yy, hat * wide["weight"] + wide.get("bias", 0.0)
            if not train:
                continue

            def through(d, hat, rr):
                proj = hat * (d * hat).sum(-1, keepdim=True) / h
                if c["kind"] == "layer":
                    proj = proj + d.sum(-1, keepdim=True) / h
                return (d - proj) * rr

            dh = s["dh"][i, r].double()
            out["dweight"] += (dh * hat).sum(0)
            if "bias" in wide:
                out["dbias"] += dh.sum(0)
            dy = s["dy"][i, r].double() + through(dh * wide["weight"], hat, rr)
            out["dx"][i, r] = dy * c["res_scale"]
            dv = dy * c["block_scale"]
            if "gate" in wide:
                (out["dgate"][i] if c["gate"] == "sequence" else out["dgate"]).add_((dv * v).sum(0))
            dv = dv * gate
            if c["post"]:
                out["dpost_weight"] += (dv * hat_f).sum(0)
                if "post_bias" in wide:
                    out["dpost_bias"] += dv.sum(0)
                dv = through(dv * wide["post_weight"], hat_f, r_f)
            out["dblock"][i, r] = dv
    return out


def _exact_kept(x):
    out = torch.empty(x.shape, device="cuda", dtype=torch.float64)
    steps = torch.tensor([2.0 ** e for e in range(-126, 122)], device="cuda", dtype=torch.float64)
    for lo in range(0, x.shape[1], GROUP):
        part = x[:, lo:lo + GROUP].double()
        most = part.abs().amax(-1, keepdim=True)
        at = torch.searchsorted(127.0 * steps, most.reshape(-1)).clamp(max=len(steps) - 1)
        step = steps[at][:, None]
        out[:, lo:lo + GROUP] = torch.round(part / step) * step
    return out


def _exact_acts(s, c):
    def act(x):
        if c["kind"] == "silu":
            p = torch.sigmoid(x)
            return x * p, p + x * p * torch.sigmoid(-x)
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (x + 0.044715 * x ** 3))
        return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 3 * 0.044715 * x ** 2)

    def both(up, gate):
        return act(up)[0] if gate is None else act(gate)[0] * up

    up, gate = s["up"], s["gate"]
    out = [both(up.double(), None if gate is None else gate.double())]
    up, gate, d = _exact_kept(up), None if gate is None else _exact_kept(gate), s["dout"].double()
    a, slope = act(up if gate is None else gate)
    out += [d * slope] if gate is None else [d * a, d * up * slope]
    return out + ([both(up, gate)] if c["again"] else [])


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "norm_bwd"):
        return _exact_block(s, case)
    if case["op"] == "ckpt":
        return _exact_kept(s["x"])
    if case["op"] == "act":
        return _exact_acts(s, case)
    return _exact_tokens(s, case)


def work(case):
    c = case
    if c["op"] in ("logprob", "loss", "shard"):
        n, (_, rows), e = c["batch"] * c["seq"], _shard(c), BYTES[c["dtype"]]
        ids = n * (4 if c["ids"] == "i32" else 8)
        if c["op"] == "logprob":
            return {"bytes": n * rows * e + ids + n * (8 + 4 * c["entropy"] + 8 * c["top"]), "flops": 5 * n * rows}
        if c["op"] == "loss":
            return {"bytes": 2 * n * rows * e + ids + 8 * n, "flops": 7 * n * rows}
        return {"bytes": 2 * n * rows * e + ids + n * (16 * c["shards"] + 16), "flops": 10 * n * rows}
    if c["op"] in ("norm", "norm_bwd"):
        n, h, e, r, w = c["batch"] * c["seq"], c["hidden"], BYTES[c["dtype"]], BYTES[c["res"]], BYTES[c["weights"]]
        gates = {"": 0, "all": 1, "sequence": c["batch"]}[c["gate"]]
        params = (1 + c["bias"]) * (1 + c["post"]) + gates
        # x and the block's output in, y and h out; the gradients of y and h in, of x and the block's output out
        bwd = c["op"] == "norm_bwd"
        return {"bytes": (2 + 2 * bwd) * n * h * (e + r) + params * h * w * (1 + bwd), "flops": (8 + 5 * c["post"]) * (3 if bwd else 1) * n * h}
    n, w, e = c["tokens"], c["width"], BYTES[c["dtype"]]
    kept = n * (w + -(-w // GROUP))  # bytes of one checkpoint
    if c["op"] == "ckpt":
        return {"bytes": 2 * n * w * e + 2 * kept, "flops": 4 * n * w}
    k = 1 + c["gated"]
    return {"bytes": n * w * e * (2 * k + 2 + c["again"]) + 2 * k * kept, "flops": (30 + 10 * k) * n * w}
