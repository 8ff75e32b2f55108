"""The end of a last stage's step (step.py): norms, MLP with kept activations, head and loss together, against autograd in 64 bits."""
import math

import pytest

from paper_2503_19050_amd import step
from paper_2503_19050_amd import workloads as W

pytestmark = pytest.mark.gpu


def reference(torch, model, p, x, targets, weight, kept):
    """(logp, gradients) in 64 bits; the activation's backward pass is at the kept values, as defined."""
    gpt = model["arch"] == W.GPT

    def act(v):
        return torch.nn.functional.gelu(v, approximate="tanh") if gpt else torch.nn.functional.silu(v)

    class Act(torch.autograd.Function):
        @staticmethod
        def forward(ctx, up, gate):
            return act(up) if gpt else act(gate) * up

        @staticmethod
        def backward(ctx, d):
            u, g = kept
            with torch.enable_grad():
                v = (u if gpt else g).detach().requires_grad_()
                slope, = torch.autograd.grad(act(v).sum(), v)
            return (d * slope, None) if gpt else (d * act(g), d * u * slope)

    class Down(torch.autograd.Function):   # the projection's gradient takes the activation at the kept values
        @staticmethod
        def forward(ctx, a, w):
            ctx.save_for_backward(w)
            return a @ w.t()

        @staticmethod
        def backward(ctx, d):
            w, = ctx.saved_tensors
            a = act(kept[0]) if gpt else act(kept[1]) * kept[0]
            return d @ w, d.reshape(-1, d.shape[-1]).t() @ a.reshape(-1, a.shape[-1])

    def norm(v, name):
        if gpt:
            v = v - v.mean(-1, keepdim=True)
        return v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt() * q[name + ".w"] + (q[name + ".b"] if gpt else 0.0)

    q = {k: v.double().detach().requires_grad_() for k, v in p.items()}
    x = x.double().detach().requires_grad_()
    h = norm(x, "norm2")
    up = h @ q["up"].t()
    a = Act.apply(up, up.detach() if gpt else h @ q["gate"].t())
    z = norm(x + Down.apply(a, q["down"]), "norm") @ q["head"].t()
    logp = torch.log_softmax(z, -1).gather(-1, targets.clamp(min=0)[..., None])[..., 0]
    logp = torch.where(targets >= 0, logp, 0.0)
    (-weight * logp.sum()).backward()
    return logp.detach(), dict({k: v.grad for k, v in q.items()}, x=x.grad)


@pytest.mark.parametrize("name", ["tiny", "tiny_llama"])
def test_gradients(name):
    """fp32 sums of at most 2048 terms in each product and chain of products: 1e-5 of a tensor's norm is over a hundred roundings
    (2^-24 each, of random sign) of its largest sum."""
    import torch
    from paper_2503_19050_amd import mist
    model = W.workload(name)["model"]
    gpt = model["arch"] == W.GPT
    gen = torch.Generator("cuda").manual_seed(1)
    named = [(n.replace("layer0.", ""), s) for n, s in step.stage_tensors(model, 1, 1, last=True)]
    p = {n: torch.empty(s, device="cuda").normal_(1.0 if n.endswith(".w") else 0.0, 0.1 if "." in n else s[-1] ** -0.5, generator=gen)
         for n, s in named if n in ("up", "gate", "down", "head") or n.startswith(("norm2.", "norm."))}
    g = {n: torch.full_like(v, math.nan) for n, v in p.items()}
    xs = [torch.empty(2, 33, model["hidden"], device="cuda").normal_(0.0, 1.0, generator=gen) for _ in range(2)]
    ts = [torch.randint(0, model["vocab"], (2, 33), device="cuda", generator=gen) for _ in range(2)]
    ts[0][0, 3:7] = -1
    mlp = step.LastMlp(model, p, g)
    total = None
    for i, (x, t) in enumerate(zip(xs, ts)):
        h = mist.block_norm(x, weight=p["norm2.w"], bias=p.get("norm2.b"), kind="layer" if gpt else "rms").h
        kept = [None if n not in p else mist.checkpoint_load(mist.checkpoint_store(h @ p[n].t())).double() for n in ("up", "gate")]
        logp, dx = mlp.microbatch(x.clone(), t, 0.01, i > 0)
        want, grads = reference(torch, model, p, x, t, 0.01, kept)
        assert float((logp - want).abs().max()) < 1e-5 * float(want.abs().max())
        dwant = grads.pop("x")
        assert float((dx - dwant).norm()) < 1e-5 * float(dwant.norm())
        total = grads if total is None else {k: v + grads[k] for k, v in total.items()}
    for k, v in total.items():
        assert float((g[k] - v).norm()) < 1e-5 * float(v.norm()), k


@pytest.mark.parametrize("stage", [dict(b=2, tp=1, dp=1, zero=0, l=2), dict(b=1, tp=4, dp=3, zero=1, l=1)], ids=str)
@pytest.mark.parametrize("name", ["tiny", "tiny_llama"])
def test_steps(name, stage):
    r = step.run_last(W.workload(name)["model"], stage, steps=3)
    assert r["steps"] == 3 and r["skipped"] == 0
    assert all(math.isfinite(x) for x in r["losses"] + r["norms"])
    assert set(r["ms"]) == {"norm", "mlp_act", "norm_residual", "token_loss", "norm_residual_grad", "mlp_act_grad", "norm_grad", "grad_norm", "adam_step"}
    assert min(r["ms"].values()) > 0 and set(r["bytes"]) == set(r["ms"])


def test_plan_to_step(capsys, monkeypatch, tmp_path):
    """From a workload's plan to its last stage's step, through the command."""
    out = tmp_path / "s.json"
    monkeypatch.setattr("sys.argv", ["step", "--workload", "tiny_llama", "--stage", "last", "--steps", "2", "--out", str(out)])
    assert step.main() == 0
    assert "token_loss" in capsys.readouterr().out and out.exists()
