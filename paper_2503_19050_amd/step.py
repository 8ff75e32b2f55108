"""Runs the two ends of a planned training step on the current device: what the operator database leaves out.

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

    python -m paper_2503_19050_amd.step --workload gpt2.7b-d16 --out step.json
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


def first_stage(name: str) -> tuple[dict, dict]:
    """The model of a workload and the first stage of its plan."""
    wl = W.workload(name)
    with mist.from_workload(wl) as S:
        S.eval()
        plan = S.plan()
        if plan is None:
            raise RuntimeError("%s: no plan fits the memory" % name)
        c = S.decode(plan["stages"][0]["id"])
    return wl["model"], {k: c[k] for k in ("b", "tp", "dp", "zero", "l")}


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workload", default="gpt2.7b-d16", choices=W.WORKLOADS + ["tiny", "tiny_llama"])
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--microbatches", type=int, default=2)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--out", default="")
    args = ap.parse_args()
    import torch
    if not torch.cuda.is_available():
        print("the step needs a GPU", file=sys.stderr)
        return 2
    model, stage = first_stage(args.workload)
    print("first stage of %s: %s" % (args.workload, stage), flush=True)
    r = run(model, stage, args.steps, args.microbatches, args.max_norm)
    print("%d parameters on the rank, %d of them stepped; loss %.4g -> %.4g, norm %.4g -> %.4g"
          % (r["parameters"], r["share"], r["losses"][0], r["losses"][-1], r["norms"][0], r["norms"][-1]), flush=True)
    for k, t in r["ms"].items():
        print("  %-11s %9.3f ms  %7.1f GB/s" % (k, t, r["bytes_per_s"][k] / 1e9), flush=True)
    if args.out:
        with open(args.out, "w") as f:
            json.dump(dict(r, workload=args.workload, device=torch.cuda.get_device_name(0)), f, indent=1)
        print("wrote", args.out, flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
