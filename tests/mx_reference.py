"""Microscaled matrices in 64 bits on the host: quantisation by search among a format's numbers, and codes to numbers by table.  Written from
the definition in the header, without the library."""
from __future__ import annotations

import numpy as np
import torch

E2M1, E4M3 = 0, 1
GRID = {
    E2M1: np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]),
    E4M3: np.array([m / 512 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1]),
}
TOP = {E2M1: 2, E4M3: 8}   # exponent of the largest number
BYTES = {E2M1: 16, E4M3: 32}


def wide(t: torch.Tensor) -> np.ndarray:
    return t.detach().double().cpu().numpy()


def _blocks(x):
    rows, cols = x.shape
    pad = -cols % 32
    return np.pad(x, ((0, 0), (0, pad))).reshape(rows, -1, 32)


def quantize(x: np.ndarray, form: int, fit: bool = False, noise=None):
    """(codes' numbers before scaling, scale bytes): arrays (rows, blocks, 32) and (rows, blocks)."""
    grid = GRID[form]
    b = _blocks(x)
    top = np.abs(b).max(-1)
    fine = np.isfinite(top)
    top = np.where(fine, top, 0.0)
    e = np.frexp(top)[1] - 1                       # 2^e <= top < 2^(e + 1)
    s = np.where(top > 0, e - TOP[form], -127)
    if fit:
        s = s + (top > grid[-1] * np.exp2(s.astype(float)))
    s = np.clip(s, -127, 127)
    with np.errstate(invalid="ignore"):
        a = np.minimum(np.abs(b) * np.exp2(-s.astype(float))[..., None], grid[-1])
    a = np.where(fine[..., None], a, 0.0)
    below = np.searchsorted(grid, a, side="right") - 1
    above = np.minimum(below + 1, len(grid) - 1)
    gap = np.where(above > below, grid[above] - grid[below], 1.0)
    share = (a - grid[below]) / gap
    if noise is None:
        up = (share > 0.5) | ((share == 0.5) & (below % 2 == 1))
    else:
        up = _blocks(noise.astype(float)) + 0.5 < 256 * share
    out = np.where(up, grid[above], grid[below]) * np.sign(np.where(np.isfinite(b), b, 0.0))
    return out, np.where(fine, s + 127, 255).astype(np.uint8)


def values(grid, scales, cols):
    """The numbers that (codes' numbers, scale bytes) stand for."""
    by = np.where(scales < 255, np.exp2(scales.astype(float) - 127), np.nan)
    return (grid * by[..., None]).reshape(grid.shape[0], -1)[:, :cols]


def quantized(x, form, fit=False, noise=None):
    return values(*quantize(x, form, fit, noise), x.shape[1])


def decode(codes: np.ndarray, form: int):
    """Codes' numbers, (rows, blocks, 32)."""
    grid = GRID[form]
    if form == E2M1:
        code = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
        table = np.concatenate([grid, -grid])
    else:
        code = codes
        table = np.concatenate([grid, [np.nan], -grid, [np.nan]])
    return table[code].reshape(codes.shape[0], -1, 32)


def numbers(mx) -> np.ndarray:
    """What an MxTensor on the device stands for."""
    blocks = -(-mx.cols // 32)
    codes = mx.codes.cpu().numpy()[:, :blocks * BYTES[mx.format]]
    return values(decode(codes, mx.format), mx.scales.cpu().numpy()[:, :blocks], mx.cols)
