"""The example's training loop: it learns, and one of its steps is what plain 64-bit arithmetic makes of the same gradients."""
from __future__ import annotations

import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_lists", os.path.join(ROOT, "examples", "train_lists.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_learns(example):
    history = example.main(40)
    first, last = history[0]["loss"], history[-1]["loss"]
    assert abs(first - math.log(example.VOCAB)) < 1.0 and last < 0.6 * first
    assert all(math.isfinite(h["norm"]) and h["next_b"] <= example.B_MAX for h in history)
    assert all(b["next_b"] >= a["next_b"] for a, b in zip(history, history[1:]))
    # two ways to the norm of the mean: the list's and the step's own
    assert all(abs(h["norm"] ** 2 - h["gbar_sq"]) <= 1e-5 * h["gbar_sq"] for h in history)


def test_one_step_in_64_bits(example):
    t = example.Trainer(seed=3)
    t.step()
    seen, backward = [], t.backward
    t.backward = lambda: (backward(), seen.append([p.grad.double().clone() for p in t.params]))[0]
    w, m, v = ([x.double() for x in xs] for xs in (t.w, t.m, t.v))
    out = t.step()
    M = example.MICRO_STEPS
    assert len(seen) == example.WORKERS * M
    mean = [sum(g[i] for g in seen) / len(seen) for i in range(len(t.params))]
    norm = math.sqrt(sum(float(g.square().sum()) for g in mean))
    assert abs(out["norm"] - norm) <= 1e-5 * norm and out["clipped"] == (norm > example.MAX_NORM)
    factor = min(1.0, example.MAX_NORM / (norm + 1e-6))
    lr, wd, b1, b2, k = 2e-3, 0.01, 0.9, 0.95, 2
    for i, g in enumerate(mean):
        em = b1 * m[i] + (1 - b1) * factor * g
        ev = b2 * v[i] + (1 - b2) * (factor * g) ** 2
        ew = (1 - lr * wd) * w[i] - lr * (em / (1 - b1 ** k)) / ((ev / (1 - b2 ** k)).sqrt() + 1e-8)
        # the mean is an fp32 sum of eight terms, which may cancel: 1e-5 of the tensor's root mean square, and AdamW's step is at most some lr
        for got, want, scale in ((t.m[i], em, 0.0), (t.v[i], ev, 0.0), (t.w[i], ew, lr)):
            rms = float(want.square().mean().sqrt())
            assert float((got.double() - want).abs().max()) <= 1e-5 * (float(want.abs().max()) + rms + 10 * scale)
        assert torch.equal(t.params[i].detach(), t.w[i].to(torch.bfloat16))
