"""The training example's low-precision layers: their gradients from the formulas, in 64 bits on the codes that they multiply, and that a few steps run."""
import importlib.util
import os

import mx_reference as R
import numpy as np
import pytest
import torch

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
spec = importlib.util.spec_from_file_location("train_lists", os.path.join(os.path.dirname(HERE), "examples", "train_lists.py"))
E = importlib.util.module_from_spec(spec)
spec.loader.exec_module(E)

DEV = "cuda:0"
NEAR = 2.0 ** -9 + 1e-4      # a bf16 result's rounding, half a step at most, and the 8-bit products' sums


def near(got, want, more=0.0):
    return np.linalg.norm(R.wide(got) - want) <= (NEAR + more) * np.linalg.norm(want)


def quantized(x, noise=None):
    return R.quantized(x, R.E4M3, noise is not None, noise)


@pytest.mark.parametrize("tokens", [1, 65])
@pytest.mark.parametrize("residual", [False, True])
def test_gradients(tokens, residual):
    torch.manual_seed(3)
    layer = E.NormLinear4(96, 200, DEV)
    layer.gain.data += 0.1 * torch.randn_like(layer.gain)
    x, r = (torch.randn(tokens, 96, device=DEV).to(torch.bfloat16).requires_grad_() for _ in range(2))
    d, dsum = (torch.randn(tokens, n, device=DEV).to(torch.bfloat16) for n in (200, 96))
    out, total = layer(x, r if residual else None)
    state = torch.cuda.get_rng_state(DEV)
    torch.autograd.backward([out, total], [d, dsum])
    torch.cuda.set_rng_state(state, DEV)
    noise = torch.randint(256, d.shape, dtype=torch.uint8, device=DEV).cpu().numpy()
    h = R.wide(total)
    assert near(total, R.wide(x) + (R.wide(r) if residual else 0.0))
    rstd = 1 / np.sqrt((h ** 2).mean(1, keepdims=True) + 1e-5)
    gain, w = R.wide(layer.gain), R.wide(layer.weight)
    y = h * rstd * gain
    # fp32 values of y a rounding away from a border may fall on its other side: a step of 1/8 of a value, few of them
    assert near(out, quantized(y) @ R.quantized(w, R.E2M1).T, 1e-3)
    y16 = torch.from_numpy(y).to(torch.bfloat16)
    assert near(layer.weight.grad, quantized(R.wide(d).T, noise.T) @ quantized(R.wide(y16).T).T, 1e-3)
    dy = R.wide(torch.from_numpy(quantized(R.wide(d), noise) @ R.quantized(w.T, R.E2M1).T).to(torch.bfloat16))
    g, hat = dy * gain, h * rstd
    dx = R.wide(dsum) + rstd * (g - hat * (g * hat).mean(1, keepdims=True))
    assert near(x.grad, dx, 2.0 ** -9) and near(layer.gain.grad, (dy * hat).sum(0), 2.0 ** -9)
    if residual:
        assert torch.equal(r.grad, x.grad)


def test_gradients_without_norm():
    torch.manual_seed(4)
    layer = E.Linear4(128, 70, DEV)
    x, d = torch.randn(33, 128, device=DEV).to(torch.bfloat16).requires_grad_(), torch.randn(33, 70, device=DEV).to(torch.bfloat16)
    out = layer(x)
    state = torch.cuda.get_rng_state(DEV)
    out.backward(d)
    torch.cuda.set_rng_state(state, DEV)
    noise = torch.randint(256, d.shape, dtype=torch.uint8, device=DEV).cpu().numpy()
    w = R.wide(layer.weight)
    assert near(out, quantized(R.wide(x)) @ R.quantized(w, R.E2M1).T)
    assert near(x.grad, quantized(R.wide(d), noise) @ R.quantized(w.T, R.E2M1).T)
    assert near(layer.weight.grad, quantized(R.wide(d).T, noise.T) @ quantized(R.wide(x).T).T)


def test_runs():
    trainer = E.Trainer(mx=True)
    for _ in range(3):
        s = trainer.step()
        assert all(np.isfinite(s[k]) for k in ("loss", "norm", "T"))
    for layer in trainer.net.modules():
        if isinstance(layer, E.Linear4):      # what the next step multiplies is the new weight
            assert np.array_equal(R.numbers(layer.forth), R.quantized(R.wide(layer.weight), R.E2M1))
