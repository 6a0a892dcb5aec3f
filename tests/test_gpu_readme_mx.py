"""The README's recipe for low-precision layers, run as it stands there: what it leaves in the gradients."""
import os
import re

import mx_reference as R
import numpy as np
import pytest
import torch

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md"), encoding="utf-8") as f:
    RECIPE = re.search(r"## Low-precision layers.*?```python\n(.*?)```", f.read(), re.S).group(1)
TOKENS, FEATURES, OUT = 64, 96, 40


def inputs(seed):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen).to(DEV)   # noqa: E731
    half = lambda *s: r(*s).to(torch.bfloat16)              # noqa: E731
    empty = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)   # noqa: E731
    return dict(B=B, torch=torch, tokens=TOKENS, features=FEATURES, out_features=OUT, micro_batches=4, master=0.1 * r(OUT, FEATURES),
                norm_weight=1 + 0.1 * r(FEATURES), x=half(TOKENS, FEATURES), r=half(TOKENS, FEATURES), dy=half(TOKENS, OUT), dh=half(TOKENS, FEATURES),
                h=empty(TOKENS, FEATURES), xn=empty(TOKENS, FEATURES), y=empty(TOKENS, OUT), dxn=empty(TOKENS, FEATURES), dx=empty(TOKENS, FEATURES),
                rstd=torch.empty(TOKENS, device=DEV), weight_grad=torch.zeros(OUT, FEATURES, device=DEV), norm_grad=torch.zeros(FEATURES, device=DEV))


def test_gradients_are_rounded_without_bias(monkeypatch):
    """Over all bytes, the mean of what the two products read is the gradient."""
    s = inputs(1)
    sums = np.zeros((TOKENS, OUT)), np.zeros((OUT, TOKENS))
    for byte in range(256):
        with monkeypatch.context() as m:
            m.setattr(torch, "randint", lambda high, size, **k: torch.full(size, byte, **k))
            exec(RECIPE, s)
        for total, name in zip(sums, ("G8", "G8t")):
            total += R.numbers(s[name])
    wide = R.wide(s["dy"])
    for total, want, mx in zip(sums, (wide, wide.T), (s["G8"], s["G8t"])):
        blocks = -(-mx.cols // 32)
        scale = np.exp2(mx.scales.cpu().numpy()[:, :blocks].astype(float) - 127).repeat(32, 1)[:, :mx.cols]
        a = np.abs(want) / scale
        step = np.diff(R.GRID[R.E4M3])[np.minimum(np.searchsorted(R.GRID[R.E4M3], a, side="right") - 1, 125)] * scale
        assert (np.abs(total / 256 - want) <= step / 512 * (1 + 1e-9)).all()


def test_gradients_are_means_of_the_micro_batches():
    """The weight's and the norm's gradient of a few micro-batches, added up in what the recipe is given, against 64 bits."""
    s = inputs(2)
    want_w, want_n, size_w, size_n = 0.0, 0.0, 0.0, 0.0
    for k in range(s["micro_batches"]):
        s.update({name: value for name, value in inputs(3 + k).items() if name in ("x", "r", "dy", "dh")})
        exec(RECIPE, s)
        turned, y = R.numbers(s["G8t"]), R.numbers(s["X8t"])
        term = R.wide(s["dxn"]) * R.wide(s["h"]) * R.wide(s["rstd"])[:, None]
        want_w, size_w = want_w + turned @ y.T, size_w + np.abs(turned) @ np.abs(y).T
        want_n, size_n = want_n + term.sum(0), size_n + np.abs(term).sum(0)
    n = s["micro_batches"]
    # fp32 sums: for a micro-batch, two instructions' 32 tokens and the joins of parts, a cut of 2^-23 each (some 18), or 64 rows' additions and products
    # of 2^-24 each (some 80), and two roundings as it is scaled and added to the others
    assert (np.abs(R.wide(s["weight_grad"]) - want_w / n) <= 24 * 2.0 ** -23 * size_w / n).all()
    assert (np.abs(R.wide(s["norm_grad"]) - want_n / n) <= 96 * 2.0 ** -24 * size_n / n).all()
