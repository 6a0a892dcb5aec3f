"""Calls on lists of tensors in forms that a list of one group, or of one kind of tensor, does not reach."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import test_gpu_tensor_lists as L
from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("G", [(1 << 20) + 3, (1 << 21) + 5])
def test_norms_of_very_many_groups(G):
    """Groups without elements beside those of four tensors, in runs of two and three items."""
    ids = [0, (1 << 20) - 1, 1 << 20, G - 1]
    x = [torch.full((n,), 2.0, device=DEV) for n in (5, 9000, 4097, 3)]
    lst = B.make_tensor_list(x, groups=ids)
    views = B.norm_views(B.normtest_grad_norm(lst, max_norm=1.0))
    norm = torch.zeros(ids[-1] + 1, device=DEV)
    for t, g in zip(x, ids):
        norm[g] = 2.0 * math.sqrt(t.numel())
    assert bool(((views["norm"] - norm).abs() <= 1e-7 * norm).all())
    assert torch.equal(views["flags"][:, 0] == B.NT_STATUS_ZERO_GRAD_NORM, norm == 0) and torch.equal(views["flags"][:, 1] == 1, norm > 0)


# whole and part items, rows, split rows, and groups that meet inside a run of tensors
MIXED = [(12_288,), (10_001,), (50, 70), (3,), (3, 5001), (4097,), (0,)]
GROUPS = [2, 0, 1, 0, 2, 1, 1]


def by_group(types, seed):
    """Gradients whose groups have norms far apart, so that no two factors are alike."""
    x, untouched = L.carve(MIXED, L.cycle(types, MIXED), seed, offset=1, extra=3)
    for t, g in zip(x, GROUPS):
        t.mul_(4.0 ** g)
    return x, untouched, B.make_tensor_list(x, groups=GROUPS)


def factors(norms, scale=1.0):
    """In 64 bits, of every group; all of them clip."""
    r = B.read_norms(norms)
    assert all(q.clipped for q in r) and len({q.factor for q in r}) == 3
    return [scale * q.coef for q in r]


@pytest.mark.parametrize("types", L.TYPES, ids=str)
@pytest.mark.parametrize("to", [None, (F32,), (BF16, F16)], ids=str)
def test_clip_by_group(types, to):
    x, untouched, lst = by_group(types, 80)
    old = [L.wide(t) for t in x]
    out, out_untouched = (x, untouched) if to is None else L.carve(MIXED, L.cycle(to, MIXED), 81, offset=2)
    norms = B.normtest_clip_grad_norm(lst, 0.5, grad_scale=0.25, out=None if to is None else B.make_tensor_list(out, like=lst))
    f = factors(norms, 0.25)
    for y, a, g in zip(out, old, GROUPS):
        L.check_written(y, a, np.zeros_like(a), 0.0, f[g])
    untouched()
    out_untouched()


@pytest.mark.parametrize("types", L.TYPES, ids=str)
def test_adamw_by_group(types):
    x, _, lst = by_group(types, 82)
    (w, m, v), checks = L.state(MIXED, extra=1)
    before = [np.concatenate([L.wide(t) for t in ts]) for ts in (w, m, v)]
    norms = B.normtest_grad_norm(lst, max_norm=0.5, grad_scale=0.25)
    h = L.hyper()
    B.normtest_adamw_tensors(lst, *[B.make_tensor_list(t, like=lst) for t in (w, m, v)], h, norms=norms, grad_scale=3.0)
    f = factors(norms, 0.25)
    per_element = np.concatenate([np.full(t.numel(), 3.0 * f[g]) for t, g in zip(x, GROUPS)])
    L.check_adamw([np.concatenate([L.wide(t) for t in ts]) for ts in (w, m, v)], before, np.concatenate([L.wide(t) for t in x]), h, per_element)
    for check in checks:
        check()


# Mostly dense tensors, so that AdamW's blocks are kept in step, and beside them rows: whole and split ones, with ends of one to three elements.
DENSE_AND_ROWS = [(45_000_001,), (3001, 5003), (2000, 1001), (7,)]


def test_long_lists_of_dense_tensors_and_rows():
    L.test_long_lists_have_the_bits_of_short_ones(DENSE_AND_ROWS)


def test_adamw_by_group_of_a_long_list():
    x, untouched = L.carve(DENSE_AND_ROWS, [BF16, F32, F16, F32], 83, offset=1, extra=3)
    groups = [1, 0, 2, 0]
    lst = B.make_tensor_list(x, groups=groups)
    (w, m, v), checks = L.state(DENSE_AND_ROWS, extra=2)
    before = [[t.double() for t in ts] for ts in (w, m, v)]
    norms = B.normtest_grad_norm(lst, max_norm=0.5)
    h = L.hyper()
    B.normtest_adamw_tensors(lst, *[B.make_tensor_list(t, like=lst) for t in (w, m, v)], h, norms=norms)
    f = factors(norms)
    want = [[], [], []]
    for i, g in enumerate(groups):
        a = f[g] * x[i].double()
        w0, m0, v0 = (ts[i] for ts in before)
        m1, v1 = h.beta1 * m0 + (1 - h.beta1) * a, h.beta2 * v0 + (1 - h.beta2) * a * a
        w1 = w0 * (1 - h.lr * h.weight_decay) - h.lr * (m1 / (1 - h.beta1 ** h.step)) / ((v1 / (1 - h.beta2 ** h.step)).sqrt() + h.eps)
        for to, t in zip(want, (w1, m1, v1)):
            to.append(t)
    for got, wanted in zip((w, m, v), want):
        rms = math.sqrt(sum(float(t.square().sum()) for t in wanted) / sum(t.numel() for t in wanted))
        for a, b in zip(got, wanted):
            assert bool(((a.double() - b).abs() <= 1e-6 * b.abs().clamp(min=rms)).all())
    untouched()
    for check in checks:
        check()


def test_calls_on_several_streams_that_are_ordered():
    """One call at a time may use a plan: streams that wait for each other share it, and its counters are at zero in the end."""
    x, _ = L.carve([(1 << 20,), (777_777,), (300, 4000)], [BF16, F32, F16], 84, extra=2)
    groups = [0, 1, 0]
    lst = B.make_tensor_list(x, groups=groups)
    image = lst.plan.image[:lst.plan.record.upload_bytes].clone()
    norms = B.make_norms(lst)
    streams = [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(30):
        streams[k % 3].wait_stream(streams[(k - 1) % 3])
        with torch.cuda.stream(streams[k % 3]):
            B.normtest_grad_norm(lst, norms, max_norm=1.0)
    torch.cuda.synchronize()
    L.check_norms(norms, x, groups, 2, max_norm=1.0)
    assert torch.equal(lst.plan.image[:lst.plan.record.upload_bytes], image)
