"""Calls on lists of tensors in forms that a list of one group, or of one kind of tensor, does not reach."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def test_norms_of_more_groups_than_a_launch_has_blocks():
    """Groups without elements beside the first, the last and those at the seam between two launches."""
    ids = [0, (1 << 20) - 1, 1 << 20, (1 << 20) + 2]
    x = [torch.full((n,), 2.0, device=DEV) for n in (5, 9000, 4097, 3)]
    lst = B.make_tensor_list(x, groups=ids)
    views = B.norm_views(B.normtest_grad_norm(lst, max_norm=1.0))
    norm = torch.zeros(ids[-1] + 1, device=DEV)
    for t, g in zip(x, ids):
        norm[g] = 2.0 * math.sqrt(t.numel())
    assert bool(((views["norm"] - norm).abs() <= 1e-7 * norm).all())
    assert torch.equal(views["flags"][:, 0] == B.NT_STATUS_ZERO_GRAD_NORM, norm == 0) and torch.equal(views["flags"][:, 1] == 1, norm > 0)
