"""The step program: its tensors are the cost model's parameters (CPU), and its steps learn (GPU)."""
import math

import pytest

from paper_2503_19050_amd import step
from paper_2503_19050_amd import workloads as W


@pytest.mark.parametrize("name", W.WORKLOADS + ["tiny", "tiny_llama"])
@pytest.mark.parametrize("tp", [1, 2, 4])
def test_tensors_are_the_cost_models_parameters(name, tp):
    m = W.workload(name)["model"]
    h, f, V, gpt = m["hidden"], m["ffn"], m["vocab"], m["arch"] == W.GPT
    d = h // m["heads"]
    kv = m["kv_heads"] * d
    kv_r = kv // tp if tp <= m["kv_heads"] else d
    layer = (2 * h * h + (2 if gpt else 3) * h * f) // tp + 2 * h * kv_r + (4 if gpt else 2) * h
    rows = -(-V // tp)

    def count(*a, **k):
        return sum(math.prod(s) for _, s in step.stage_tensors(m, tp, *a, **k))

    assert count(3) == 3 * layer
    assert count(0, first=True) == rows * h + (m["seq"] * h if gpt else 0)
    assert count(1, last=True) == layer + rows * h + (2 if gpt else 1) * h
    assert len({n for n, _ in step.stage_tensors(m, tp, 5, True, True)}) == len(step.stage_tensors(m, tp, 5, True, True))


@pytest.mark.gpu
@pytest.mark.parametrize("stage", [dict(b=2, tp=1, dp=1, zero=0, l=2), dict(b=1, tp=4, dp=3, zero=1, l=1)], ids=str)
@pytest.mark.parametrize("name", ["tiny", "tiny_llama"])
def test_steps_learn(name, stage):
    r = step.run(W.workload(name)["model"], stage, steps=8, lr=3e-3, max_norm=0.5)
    assert r["steps"] == 8 and r["skipped"] == 0
    assert all(math.isfinite(x) for x in r["losses"] + r["norms"])
    assert r["share"] == (r["parameters"] if stage["zero"] == 0 else -(-r["parameters"] // stage["dp"]))
    assert r["losses"][-1] < r["losses"][0]
    assert set(r["ms"]) == {"embed", "embed_grad", "grad_norm", "adam_step"} and min(r["ms"].values()) > 0


@pytest.mark.gpu
def test_plan_to_step(capsys, monkeypatch, tmp_path):
    """From a workload's plan to its first stage's step, through the command."""
    out = tmp_path / "s.json"
    monkeypatch.setattr("sys.argv", ["step", "--workload", "tiny_llama", "--steps", "3", "--out", str(out)])
    assert step.main() == 0
    assert "adam_step" in capsys.readouterr().out and out.exists()
