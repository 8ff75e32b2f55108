"""Runs the ends of a planned training step on the current device: what the operator database leaves out.

The tuner's plan gives every stage its layers, its microbatch and its parallelism; the layers' GEMMs are
in the operator database (calibrate.py), the step's ends are not.  For the first stage of a workload's
plan this program allocates the tensors of one rank, the first of its tensor-parallel group: the parameters that
the cost model counts, which has no biases of the projections (the vocabulary shard and the positions, the
layers' shards), and fp32 master weights with Adam's m and v of the rank's ZeRO share.  It makes training steps
with synthetic data: per microbatch the embedding lookup and its gradient, then the gradient norm, the
clip factor and the Adam step of the rank's share.  Weights and gradients are whole and the norm is of all the
rank's gradients, for ZeRO-2 and ZeRO-3 too, which split them; nothing is exchanged with other ranks.
The embedding learns random targets, so its loss falls; the layers' gradients are random.  It prints each
operator's time and its bytes per second.

For the last stage (--stage last) it runs a training step of one rank's last MLP, the norms around it, the head
and the loss: the MLP's inputs are kept in 8 bits for the backward pass, the norms take the residual's sum
with them, and the loss leaves the logits' gradient in the logits' place.  The residual that comes in and the targets are synthetic; the
rank's vocabulary shard counts as the whole vocabulary, and its share of the MLP as the whole.

    python -m paper_2503_19050_amd.step --workload gpt2.7b-d16 --out step.json
    python -m paper_2503_19050_amd.step --workload gpt2.7b-d16 --stage last
"""
from __future__ import annotations

import argparse
import json
import math
import sys

from paper_2503_19050_amd import mist
from paper_2503_19050_amd import workloads as W


def stage_tensors(model: dict, tp: int, layers: int, first: bool = False, last: bool = False) -> list[tuple[str, tuple]]:
    """(name, shape) of one rank's tensors of a stage: the parameters the cost model counts (per layer the
    query, key/value and output projections, the MLP and the norms; the vocabulary shard and, for GPT, the
    positions on the first stage; the head and the last norm on the last)."""
    h, f, heads, kv = model["hidden"], model["ffn"], model["heads"], model["kv_heads"]
    gpt = model["arch"] == W.GPT
    d = h // heads
    kv_r = kv // tp * d if tp <= kv else d
    rows = -(-model["vocab"] // tp)
    norms = [(n, (h,)) for n in (("norm1.w", "norm1.b", "norm2.w", "norm2.b") if gpt else ("norm1.w", "norm2.w"))]
    mlp = [("up", (f // tp, h)), ("down", (h, f // tp))] + ([] if gpt else [("gate", (f // tp, h))])
    layer = [("q", (h // tp, h)), ("kv", (2 * kv_r, h)), ("o", (h, h // tp))] + mlp + norms
    out = [("embed", (rows, h))] + ([("positions", (model["seq"], h))] if gpt else []) if first else []
    out += [("layer%d.%s" % (i, n), s) for i in range(layers) for n, s in layer]
    if last:
        out += [("head", (rows, h)), ("norm.w", (h,))] + ([("norm.b", (h,))] if gpt else [])
    return out


class Timer:
    """Device times of named parts over the steps."""

    def __init__(self, torch):
        self.torch, self.events = torch, {}

    def __call__(self, name, fn, *args, **kw):
        a, b = (self.torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        r = fn(*args, **kw)
        b.record()
        self.events.setdefault(name, []).append((a, b))
        return r

    def ms(self) -> dict:
        self.torch.cuda.synchronize()
        times = {k: sorted(a.elapsed_time(b) for a, b in v) for k, v in self.events.items()}
        return {k: v[len(v) // 2] for k, v in times.items()}


def run(model: dict, stage: dict, steps: int = 4, microbatches: int = 2, max_norm: float = 1.0, lr: float = 1e-3,
        seed: int = 0) -> dict:
    """Training steps of one rank of the stage (a plan's stage: keys b, tp, dp, zero, l).  Returns the losses, the
    norms and the median time of each part."""
    import torch
    gen = torch.Generator("cuda").manual_seed(seed)
    b, tp, dp, seq, h = stage["b"], stage["tp"], stage["dp"], model["seq"], model["hidden"]
    named = stage_tensors(model, tp, stage["l"], first=True)
    sizes = [math.prod(s) for _, s in named]
    total = sum(sizes)
    weights = torch.empty(total, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02, generator=gen)
    grads = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
    w = {n: x.view(s) for (n, s), x in zip(named, weights.split(sizes))}
    g = {n: x.view(s) for (n, s), x in zip(named, grads.split(sizes))}
    # The rank's share of the optimizer: all of it, or one of dp contiguous ranges, cut where tensors end or not.
    share = -(-total // dp) if stage["zero"] else total
    cuts, at = [], 0
    for n in sizes:
        if at < share:
            cuts.append(min(n, share - at))
        at += n
    master = weights[:share].float()
    m, v = torch.zeros_like(master), torch.zeros_like(master)

    def lists(flat):
        return mist.TensorList(flat[:share].split(cuts))

    everything = mist.TensorList(grads.split(sizes))   # the norm is over all gradients, the step over the share
    P, M, V, G, X = lists(master), lists(m), lists(v), lists(grads), lists(weights)
    record = mist.StepRecord()
    rows = named[0][1][0]
    tokens = [torch.randint(0, model["vocab"], (b, seq), device="cuda", generator=gen) for _ in range(microbatches)]
    target = torch.empty(b, seq, h, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.1, generator=gen)
    pos, dpos = w.get("positions"), g.get("positions")
    table, dtable = w["embed"], g["embed"]
    ends = dtable.numel() + (0 if dpos is None else dpos.numel())
    scale = math.sqrt(h)
    out = torch.empty_like(target)
    timer, losses, norms = Timer(torch), [], []
    for k in range(steps):
        grads[ends:].normal_(0.0, 1e-6, generator=gen)   # the layers' gradients stand in for a backward pass
        loss = torch.zeros((), device="cuda")
        for i, ids in enumerate(tokens):
            timer("embed", mist.embed, ids, table, scale=scale, pos=pos, out=out)
            diff = (out - target).div_(ids.numel())
            loss = loss + diff.float().square().sum() * ids.numel() / 2
            timer("embed_grad", mist.embed_grad, ids, diff, dtable, scale=scale, dpos=dpos, accumulate=i > 0)
        timer("grad_norm", mist.grad_norm, everything, record, max_norm=max_norm)
        timer("adam_step", mist.adam_step, P, M, V, G, record, lr=lr, weights=X)
        losses.append(loss)
        norms.append(record.norm.clone())
    ms = timer.ms()
    n = b * seq
    e = 2  # bytes of weights, gradients and activations
    moved = {"embed": 8 * n + 2 * n * h * e, "embed_grad": 8 * n + n * h * e + (rows + (0 if dpos is None else seq)) * h * e,
             "grad_norm": total * e, "adam_step": share * (2 * e + 24)}
    return {"stage": stage, "parameters": total, "share": share, "steps": int(record.step), "skipped": int(record.skipped),
            "losses": [float(x) for x in losses], "norms": [float(x) for x in norms], "ms": ms,
            "bytes": moved, "bytes_per_s": {k: moved[k] / (1e-3 * t) for k, t in ms.items() if t > 0}}


class LastMlp:
    """The end of a last stage on one rank: norm, MLP, residual with the last norm, head, loss.  params and grads: {name:
    tensor} of the tensors that stage_tensors calls norm2, up, gate, down, norm and head."""

    def __init__(self, model: dict, params: dict, grads: dict, timer=None):
        self.gpt = model["arch"] == W.GPT
        self.p, self.g = params, grads
        self.how = dict(kind="layer" if self.gpt else "rms")
        self.act = "gelu" if self.gpt else "silu"
        self.timer = timer or (lambda name, fn, *args, **kw: fn(*args, **kw))

    def microbatch(self, x, targets, weight: float, accumulate: bool):
        """Log probabilities of the targets, and the residual's gradient, for x [batch, seq, hidden]; the parameters' gradients of
        -weight * (the log probabilities' sum) are overwritten, or added to."""
        import torch
        p, g, t = self.p, self.g, self.timer

        def product(name, rows, columns):   # the gradient of a weight of rows' outputs and columns' inputs
            d, c = rows.reshape(-1, rows.shape[-1]), columns.reshape(-1, columns.shape[-1])
            if accumulate:
                g[name].addmm_(d.t(), c)
            else:
                torch.mm(d.t(), c, out=g[name])

        before = t("norm", mist.block_norm, x, weight=p["norm2.w"], bias=p.get("norm2.b"), dtype=p["up"].dtype, **self.how)
        up, gate = before.h @ p["up"].t(), None if self.gpt else before.h @ p["gate"].t()
        kept = t("mlp_act", mist.mlp_act, up, gate, kind=self.act, save=True, out=up)   # up and gate are in 8 bits from here on
        del up, gate
        block = kept.out @ p["down"].t()
        last = t("norm_residual", mist.block_norm, x, block, weight=p["norm.w"], bias=p.get("norm.b"), **self.how)
        logits = last.h @ p["head"].t()
        logp, dlogits = t("token_loss", mist.token_loss, logits, targets, weight, dlogits=logits)
        dh = dlogits @ p["head"]
        product("head", dlogits, last.h)
        del logits, dlogits
        dy, dblock = t("norm_residual_grad", mist.block_norm_grad, last.y, last.stats, dh, block=block, weight=p["norm.w"], dweight=g["norm.w"],
                       dbias=g.get("norm.b"), accumulate=accumulate, dblock=dh, **self.how)
        again = torch.empty_like(kept.out)
        dup, dgate = t("mlp_act_grad", mist.mlp_act_grad, dblock @ p["down"], kept.up, kept.gate, kind=self.act, out=again)
        product("down", dblock, again)
        dh = dup @ p["up"]
        product("up", dup, before.h)
        if dgate is not None:
            dh += dgate @ p["gate"]
            product("gate", dgate, before.h)
        dx, _ = t("norm_grad", mist.block_norm_grad, x, before.stats, dh, dy=dy, weight=p["norm2.w"], dweight=g["norm2.w"], dbias=g.get("norm2.b"),
                  accumulate=accumulate, dx=dy, **self.how)
        return logp, dx


def run_last(model: dict, stage: dict, steps: int = 4, microbatches: int = 2, max_norm: float = 1.0, lr: float = 1e-3, seed: int = 0) -> dict:
    """Training steps of the end of a last stage on one rank.  Returns what run does."""
    import torch
    gen = torch.Generator("cuda").manual_seed(seed)
    b, tp, seq, h = stage["b"], stage["tp"], model["seq"], model["hidden"]
    end = "layer%d." % (stage["l"] - 1)
    named = [(n.replace(end, ""), s) for n, s in stage_tensors(model, tp, stage["l"], last=True)]
    named = [(n, s) for n, s in named if n in ("up", "gate", "down", "head") or n.startswith("norm2.") or n.startswith("norm.")]
    sizes = [math.prod(s) for _, s in named]
    weights, grads = (torch.zeros(sum(sizes), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = {n: x.view(s) for (n, s), x in zip(named, weights.split(sizes))}
    g = {n: x.view(s) for (n, s), x in zip(named, grads.split(sizes))}
    for n, x in w.items():
        if n.endswith(".w"):
            x.fill_(1.0)
        elif not n.endswith(".b"):
            x.normal_(0.0, 0.02, generator=gen)
    master = weights.float()
    m, v = torch.zeros_like(master), torch.zeros_like(master)
    P, M, V, G, X = (mist.TensorList(flat.split(sizes)) for flat in (master, m, v, grads, weights))
    record = mist.StepRecord()
    rows = w["head"].shape[0]
    xs = [torch.empty(b, seq, h, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=gen) for _ in range(microbatches)]
    targets = [torch.randint(0, rows, (b, seq), device="cuda", generator=gen) for _ in range(microbatches)]
    timer = Timer(torch)
    mlp = LastMlp(model, w, g, timer)
    losses, norms = [], []
    for k in range(steps):
        loss = torch.zeros((), device="cuda")
        for i, (x, t) in enumerate(zip(xs, targets)):
            logp, _ = mlp.microbatch(x, t, 1.0 / (t.numel() * microbatches), i > 0)
            loss = loss - logp.mean() / microbatches
        timer("grad_norm", mist.grad_norm, G, record, max_norm=max_norm)
        timer("adam_step", mist.adam_step, P, M, V, G, record, lr=lr, weights=X)
        losses.append(loss)
        norms.append(record.norm.clone())
    ms = timer.ms()
    n, f, e, gated = b * seq, w["up"].shape[0], 2, model["arch"] != W.GPT
    k, kept = 1 + gated, n * (f + -(-f // mist.KEPT_GROUP))
    moved = {"norm": 2 * n * h * e, "norm_residual": 4 * n * h * e, "norm_residual_grad": 4 * n * h * e, "norm_grad": 4 * n * h * e,
             "mlp_act": (k + 1) * n * f * e + k * kept, "mlp_act_grad": (k + 2) * n * f * e + k * kept, "token_loss": 2 * n * rows * e,
             "grad_norm": sum(sizes) * e, "adam_step": sum(sizes) * (2 * e + 24)}
    return {"stage": stage, "parameters": sum(sizes), "share": sum(sizes), "steps": int(record.step), "skipped": int(record.skipped),
            "losses": [float(x) for x in losses], "norms": [float(x) for x in norms], "ms": ms,
            "bytes": moved, "bytes_per_s": {k: moved[k] / (1e-3 * t) for k, t in ms.items() if t > 0}}


def planned_stage(name: str, last: bool = False) -> tuple[dict, dict]:
    """The model of a workload and the first or last stage of its plan."""
    wl = W.workload(name)
    with mist.from_workload(wl) as S:
        S.eval()
        plan = S.plan()
        if plan is None:
            raise RuntimeError("%s: no plan fits the memory" % name)
        c = S.decode(plan["stages"][-1 if last else 0]["id"])
    return wl["model"], {k: c[k] for k in ("b", "tp", "dp", "zero", "l")}


def first_stage(name: str) -> tuple[dict, dict]:
    """The model of a workload and the first stage of its plan."""
    return planned_stage(name)


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workload", default="gpt2.7b-d16", choices=W.WORKLOADS + ["tiny", "tiny_llama"])
    ap.add_argument("--stage", default="first", choices=["first", "last"])
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--microbatches", type=int, default=2)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--out", default="")
    args = ap.parse_args()
    import torch
    if not torch.cuda.is_available():
        print("the step needs a GPU", file=sys.stderr)
        return 2
    model, stage = planned_stage(args.workload, args.stage == "last")
    print("%s stage of %s: %s" % (args.stage, args.workload, stage), flush=True)
    r = (run_last if args.stage == "last" else run)(model, stage, args.steps, args.microbatches, args.max_norm)
    print("%d parameters on the rank, %d of them stepped; loss %.4g -> %.4g, norm %.4g -> %.4g"
          % (r["parameters"], r["share"], r["losses"][0], r["losses"][-1], r["norms"][0], r["norms"][-1]), flush=True)
    for k, t in r["ms"].items():
        print("  %-18s %9.3f ms  %7.1f GB/s" % (k, t, r["bytes_per_s"][k] / 1e9), flush=True)
    if args.out:
        with open(args.out, "w") as f:
            json.dump(dict(r, workload=args.workload, device=torch.cuda.get_device_name(0)), f, indent=1)
        print("wrote", args.out, flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
