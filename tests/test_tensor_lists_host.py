"""CPU checks of the calls on lists of tensors: the plan covers every element once, and arguments are refused before the GPU is touched."""
import ctypes
import math
import random
import struct

import numpy as np
import pytest
import torch

from paper_2412_21124_amd import binding as B

ITEM, ROWS = 4096, 1 << 31


def plan_of(shapes, groups=None, G=None):
    """(nt_plan, image bytes) of tensors with these (rows, cols)."""
    groups = [0] * len(shapes) if groups is None else groups
    G = max(groups, default=0) + 1 if G is None else G
    records = (B.nt_tensor * len(shapes))(*[B.nt_tensor(0x1000, r, c, c + 8, B.NT_F32, g) for (r, c), g in zip(shapes, groups)])
    plan = B.nt_plan()
    assert B.lib().normtest_plan_make(records, len(shapes), G, ctypes.byref(plan), None, 0) == B.NT_OK
    image = np.zeros(max(8, plan.upload_bytes), dtype=np.uint8)
    assert B.lib().normtest_plan_make(records, len(shapes), G, ctypes.byref(plan), image.ctypes.data, image.size) == B.NT_OK
    return plan, image


def slab_shift(slots):
    shift = 4
    while shift < 8 and slots >> (2 * shift):
        shift += 1
    return 7 if slots <= 128 else shift


def cuts_of(plan, image):
    """The image's parts: per cut (items, groups, counters) as arrays, and the shapes."""
    at = 0

    def take(n, dtype):
        nonlocal at
        size = n * np.dtype(dtype).itemsize
        part = image[at:at + size].view(dtype) if size else np.zeros(0, dtype)
        at += (size + 63) // 64 * 64
        return part
    shapes = take(plan.tensors, np.dtype([("rows", "i8"), ("cols", "i8"), ("per_row", "u4", 2), ("rows_per_item", "u4", 2)]))
    cuts = []
    for k in range(2):
        here = plan.items[k] > 0
        items = take(plan.items[k], np.dtype([("tensor", "u4"), ("idx", "u4"), ("group", "u4"), ("count", "u4")]))
        groups = take(plan.groups if here else 0, np.dtype([("item0", "u4"), ("slot0", "u4"), ("slots", "u4"), ("slab0", "u4"),
                                                            ("elements", "i8"), ("pad", "i8")]))
        counters = take(16 * (plan.slabs[k] + plan.groups) if here else 0, "u4")
        if here:
            cuts.append((items, groups, counters))
    assert at == plan.upload_bytes
    scratch = sum((8 * n + 63) // 64 * 64 for n in (*plan.slots, *plan.slabs))
    assert plan.bytes == plan.upload_bytes + scratch
    return shapes, cuts


def covered(shape, item, k, size):
    """(row, column, number) of every group of up to four elements that the threads of an item's block take."""
    rows, cols = int(shape["rows"]), int(shape["cols"])
    idx, count = int(item["idx"]), int(item["count"])
    out = []
    for q in range(size // 4):
        if not count & ROWS:
            r, c, left = 0, idx * size + 4 * q, count - 4 * q
        elif shape["per_row"][k]:
            per_row = int(shape["per_row"][k])
            r, c = idx // per_row, (idx % per_row) * size + 4 * q
            left = min((idx % per_row + 1) * size, cols) - c
        else:
            quads = -(-cols // 4)
            r, c = q // quads, 4 * (q % quads)
            left = cols - c if r < count & ~ROWS else 0
            r += idx * int(shape["rows_per_item"][k])
        if left > 0:
            out.append((r, c, min(4, left)))
    return out


SHAPES = [
    [(1, 0)], [(1, 1)], [(1, 3)], [(1, 4096)], [(1, 4097)], [(1, 12288), (1, 5), (1, 0), (1, 4096)],
    [(7, 3)], [(1000, 1)], [(33, 33)], [(3, 5000)], [(2, 4096)], [(5, 4095)], [(1025, 4)], [(4, 8193)], [(2000, 31), (1, 77), (1, 9)],
]


@pytest.mark.parametrize("shapes", SHAPES, ids=str)
@pytest.mark.parametrize("long_list", [False, True])
def test_every_element_is_in_one_item(shapes, long_list):
    # a tensor of 2^23 elements makes the list long (2^21 do), which has a second cut of longer items
    shapes = shapes + ([(1, 1 << 23)] if long_list else [])
    plan, image = plan_of(shapes)
    held, cuts = cuts_of(plan, image)
    assert len(cuts) == (2 if long_list else 1) and plan.elements == sum(r * c for r, c in shapes)
    for k, (items, groups, counters) in enumerate(cuts):
        size = [ITEM, 8192][k]
        seen = [np.zeros((r, c), np.int32) if r * c < 1 << 20 else None for r, c in shapes]
        for item in items:
            if item["count"] and seen[item["tensor"]] is not None:
                for r, c, n in covered(held[item["tensor"]], item, k, size):
                    seen[item["tensor"]][r, c:c + n] += 1
        assert all((s == 1).all() for s in seen if s is not None)
        if long_list:
            last = items[items["tensor"] == len(shapes) - 1]
            assert (last["count"] == size).all() and (last["idx"] == np.arange((1 << 23) // size)).all()
        assert not counters.any()


@pytest.mark.parametrize("seed", range(12))
def test_slots_and_slabs_are_a_groups_own(seed):
    """The blocks' walk over the items as the kernels make it: every part that a block leaves has a slot of its own inside its group's, and
    the counters of slabs and groups are counted up as often as the last block expects."""
    rng = random.Random(seed)
    shapes = [rng.choice([(1, 0), (1, rng.randrange(1, 40000)), (rng.randrange(2, 300), rng.randrange(1, 900))]) for _ in range(rng.choice([1, 40, 300]))]
    if seed % 2:
        shapes += [(1, rng.randrange(1 << 23, 1 << 26)), (1 << 12, rng.randrange(100, 9000))]
    G = rng.choice([1, 3, 50])
    groups = [rng.randrange(G) for _ in shapes]
    plan, image = plan_of(shapes, groups, G)
    _, cuts = cuts_of(plan, image)
    assert len(cuts) == (2 if plan.elements >= 1 << 21 else 1)
    for k, (items, grps, _) in enumerate(cuts):
        rows = 2 * sum(r * c for r, c in shapes if r > 1) > plan.elements
        run = [1, 0 if plan.items[1] >= 1024 * G else 1 if rows else 2][k]
        shift = slab_shift(plan.slots[k])
        assert (np.diff(items["group"].astype(np.int64)) >= 0).all() and set(items["group"]) == set(range(G))
        parts = {}   # group -> slots in the order of their blocks
        for b in range(-(-len(items) // run) if run else min(1024, len(items))):
            mine = items["group"][b * run:(b + 1) * run] if run else items["group"][b::1024]
            for g in np.unique(mine):
                item0 = int(grps["item0"][g])
                parts.setdefault(int(g), []).append(b - item0 // run if run else (b - item0) % 1024)
        slot0 = slab0 = 0
        for g in range(G):
            assert grps["elements"][g] == sum(r * c for (r, c), h in zip(shapes, groups) if h == g)
            assert (int(grps["slot0"][g]), int(grps["slab0"][g])) == (slot0, slab0)
            assert sorted(parts[g]) == list(range(grps["slots"][g]))
            slot0 += int(grps["slots"][g])
            slab0 += ((int(grps["slots"][g]) - 1) >> shift) + 1
        assert (slot0, slab0) == (plan.slots[k], plan.slabs[k])
        for item in items:
            if item["count"]:
                assert groups[item["tensor"]] == item["group"]


def test_sizes_that_a_plan_refuses():
    make = B.lib().normtest_plan_make
    plan = B.nt_plan()

    def rc(*tensors, G=1, N=None):
        records = (B.nt_tensor * len(tensors))(*[B.nt_tensor(0x1000, *t) for t in tensors])
        return make(records, len(tensors) if N is None else N, G, ctypes.byref(plan), None, 0)
    assert rc() == B.NT_OK and plan.elements == 0 and plan.items[0] == 1
    assert rc((1, 5, 5, 0, 0), (3, 5, 7, 1, 1), G=2) == B.NT_OK
    for bad in [(-1, 5, 5, 0, 0), (1, -5, 5, 0, 0), (2, 5, 4, 0, 0), (1, 5, 5, 0, 1), (1, 5, 5, 0, -1)]:
        assert rc(bad) == B.NT_ERR_BAD_ARG
    assert rc(G=0) == B.NT_ERR_BAD_ARG and rc(N=-1) == B.NT_ERR_BAD_ARG
    assert make(None, 1, 1, ctypes.byref(plan), None, 0) == B.NT_ERR_BAD_ARG and make(None, 0, 1, None, None, 0) == B.NT_ERR_BAD_ARG
    assert rc((1, (1 << 43) + 1, 0, 0, 0)) == B.NT_ERR_TOO_LARGE and rc((1 << 40, 1 << 40, 1 << 40, 0, 0)) == B.NT_ERR_TOO_LARGE
    records = (B.nt_tensor * 1)(B.nt_tensor(0x1000, 1, 5, 5, 0, 0))
    buf = np.zeros(64, np.uint8)
    assert make(records, 1, 1, ctypes.byref(plan), buf.ctypes.data, 64) == B.NT_ERR_WORKSPACE_TOO_SMALL


def test_lists_that_the_check_refuses():
    def rc(t, like=(1, 5, 5), dtypes=B.ANY_DTYPE):
        a = (B.nt_tensor * 1)(B.nt_tensor(*t))
        b = (B.nt_tensor * 1)(B.nt_tensor(0x1000, *like, 0, 0))
        return B.lib().normtest_list_check(a, b, 1, dtypes)
    assert rc((0x1000, 1, 5, 0, B.NT_F32, 0)) == B.NT_OK and rc((0x1002, 1, 5, 0, B.NT_F16, 9)) == B.NT_OK
    assert rc((None, 1, 0, 0, B.NT_F32, 0), (1, 0, 0)) == B.NT_OK
    assert rc((0x1000, 2, 5, 8, B.NT_F32, 0), (2, 5, 5)) == B.NT_OK
    for t, like in [((0x1002, 1, 5, 5, B.NT_F32, 0), (1, 5, 5)), ((0x1001, 1, 5, 5, B.NT_BF16, 0), (1, 5, 5)), ((None, 1, 5, 5, 0, 0), (1, 5, 5)),
                    ((0x1000, 1, 6, 6, 0, 0), (1, 5, 5)), ((0x1000, 5, 1, 1, 0, 0), (1, 5, 5)), ((0x1000, 2, 5, 4, 0, 0), (2, 5, 5))]:
        assert rc(t, like) == B.NT_ERR_BAD_ARG
    assert rc((0x1000, 1, 5, 5, 3, 0)) == B.NT_ERR_UNSUPPORTED and rc((0x1000, 1, 5, 5, -1, 0)) == B.NT_ERR_UNSUPPORTED
    assert rc((0x1000, 1, 5, 5, B.NT_BF16, 0), dtypes=1 << B.NT_F32) == B.NT_ERR_UNSUPPORTED


def test_calls_refuse_bad_arguments_before_any_launch():
    L = B.lib()
    plan, _ = plan_of([(1, 5)])
    plan.image = 0x10000
    ok = ctypes.byref(plan)
    hy = B.make_hyper()
    nan, inf = math.nan, math.inf
    bad = B.NT_ERR_BAD_ARG
    norm = lambda p=ok, g=0x1000, kind=0, mx=1.0, s=1.0, n=0x2000: L.normtest_grad_norm(p, g, kind, mx, s, n, None)   # noqa: E731
    for kw in [dict(p=None), dict(g=None), dict(g=0x1004), dict(kind=2), dict(kind=-1), dict(mx=nan), dict(s=nan), dict(s=inf), dict(n=None),
               dict(n=0x2004)]:
        assert norm(**kw) == bad, kw
    clip = lambda g=0x1000, o=None, n=0x2000: L.normtest_clip_grads(ok, g, o, n, None)   # noqa: E731
    for kw in [dict(g=None), dict(o=0x1004), dict(n=None), dict(n=0x2004)]:
        assert clip(**kw) == bad, kw
    acc = lambda d=0x1000, s=0x3000, beta=1.0, scale=1.0, sn=None, kind=0, mx=1.0, gs=1.0, n=0x2000: \
        L.normtest_accumulate(ok, d, s, beta, scale, sn, kind, mx, gs, n, None)   # noqa: E731
    for kw in [dict(d=None), dict(s=None), dict(beta=nan), dict(scale=inf), dict(sn=0x2004), dict(kind=7), dict(mx=nan), dict(gs=inf), dict(n=0x2004)]:
        assert acc(**kw) == bad, kw
    adam = lambda g=0x1000, w=0x1000, m=0x1000, v=0x1000, c=None, h=ctypes.byref(hy), s=1.0, n=None, f=0: \
        L.normtest_adamw_tensors(ok, g, w, m, v, c, h, s, n, f, None)   # noqa: E731
    for kw in [dict(g=None), dict(w=None), dict(m=None), dict(v=0x1004), dict(c=0x1001), dict(h=None), dict(s=nan), dict(n=0x2004), dict(f=2), dict(f=1)]:
        assert adam(**kw) == bad, kw
    for wrong in [dict(step=0), dict(lr=-1.0), dict(lr=inf), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(eps=nan), dict(weight_decay=inf)]:
        assert adam(h=ctypes.byref(B.make_hyper(**wrong))) == bad, wrong
    for spoil in [dict(magic=0), dict(image=None), dict(image=0x10008), dict(groups=0), dict(tensors=-1)]:
        other, _ = plan_of([(1, 5)])
        other.image = 0x10000
        for k, x in spoil.items():
            setattr(other, k, x)
        assert norm(p=ctypes.byref(other)) == bad, spoil


def test_records_have_the_headers_layout():
    assert ctypes.sizeof(B.nt_tensor) == 40 and ctypes.sizeof(B.nt_norm) == B.NORM_BYTES == 40 and ctypes.sizeof(B.nt_plan) == 72
    raw = struct.pack("ddffIiq", 3.0, 0.5, 3.0, 0.25, 1, 1, 7)
    norms = torch.frombuffer(bytearray(raw * 2), dtype=torch.uint8)
    assert [r.as_dict() for r in B.read_norms(norms)] == [dict(norm=3.0, coef=0.5, norm32=3.0, factor=0.25, status=1, clipped=1, elements=7)] * 2
    views = B.norm_views(norms)
    assert views["norm"].tolist() == [3.0, 3.0] and views["factor"].tolist() == [0.25, 0.25] and views["flags"].tolist() == [[1, 1], [1, 1]]


def test_layouts_in_memory():
    z = torch.zeros
    for t, want in [(z(3, 4), (1, 12, 12, None)), (z(3, 4).t(), (1, 12, 12, (1, 0))), (z(5, 9)[:, 2:5], (5, 3, 9, None)), (z(()), (1, 1, 1, None)),
                    (z(0, 3), (1, 0, 0, None)), (z(10)[::2], (5, 1, 2, None)), (z(2, 3, 4)[:, :, 1:3], (6, 2, 4, None)),
                    (z(4, 5, 6).permute(2, 0, 1), (1, 120, 120, (1, 2, 0))), (z(4, 1, 6)[:, :, :3], (4, 3, 6, None)), (z(1, 7)[:, 2:4], (1, 2, 2, None))]:
        assert B._rows_of(t) == want
    for t in [z(3, 1).expand(3, 4), z(4, 5, 6)[:, 1:3, 2:4], torch.as_strided(z(20), (3, 4), (2, 1))]:
        with pytest.raises(ValueError):
            B._rows_of(t)


def test_lists_refuse_what_is_not_on_the_device():
    with pytest.raises(ValueError, match="no CPU path"):
        B.make_tensor_list([torch.zeros(3)])
    with pytest.raises(TypeError):
        B.make_tensor_list([torch.zeros(3, dtype=torch.float64)])
    with pytest.raises(ValueError, match="device"):
        B.make_tensor_list([])
    for call in (lambda: B.normtest_grad_norm([torch.zeros(3)]), lambda: B.normtest_clip_grads([], None), lambda: B.normtest_accumulate([], []),
                 lambda: B.normtest_adamw_tensors([], [], [], [], B.make_hyper())):
        with pytest.raises(TypeError, match="make_tensor_list"):
            call()


def test_scalars_that_fp32_does_not_hold_are_refused():
    """The kernels multiply in fp32: a finite double past its range would be infinite there, and make NaN of a zero."""
    L = B.lib()
    plan, _ = plan_of([(1, 5)])
    plan.image = 0x10000
    ok, bad = ctypes.byref(plan), B.NT_ERR_BAD_ARG
    for x in (1e39, -1e39, 1e300):
        assert L.normtest_grad_norm(ok, 0x1000, 0, 1.0, x, 0x2000, None) == bad
        assert L.normtest_accumulate(ok, 0x1000, 0x3000, x, 1.0, None, 0, 1.0, 1.0, None, None) == bad
        assert L.normtest_accumulate(ok, 0x1000, 0x3000, 1.0, x, None, 0, 1.0, 1.0, None, None) == bad
        assert L.normtest_accumulate(ok, 0x1000, 0x3000, 1.0, 1.0, None, 0, 1.0, x, 0x2000, None) == bad
        assert L.normtest_adamw_tensors(ok, 0x1000, 0x1000, 0x1000, 0x1000, None, ctypes.byref(B.make_hyper()), x, None, 0, None) == bad
    for wrong in [dict(lr=1e39), dict(lr=1e38, beta1=0.99), dict(lr=1e20, weight_decay=1e20)]:
        hyper = ctypes.byref(B.make_hyper(**wrong))
        assert L.normtest_adamw_tensors(ok, 0x1000, 0x1000, 0x1000, 0x1000, None, hyper, 1.0, None, 0, None) == bad, wrong


@pytest.mark.parametrize("seed", range(8))
def test_the_check_finds_shared_elements(seed):
    """Against the sets of bytes: few tensors of any rows, strides and types in little memory, so that about half of the lists share some."""
    rng = random.Random(seed)
    found = [0, 0]
    for _ in range(400):
        tensors, held, shared = [], set(), False
        for _ in range(rng.choice([2, 2, 3, 5])):
            dtype = rng.choice([B.NT_F32, B.NT_BF16, B.NT_F16])
            size = 4 if dtype == B.NT_F32 else 2
            rows, cols = rng.choice([(1, rng.randrange(40)), (rng.randrange(1, 12), rng.randrange(0, 9))])
            ld = cols + rng.choice([0, 1, 7, rng.randrange(40), 30 - cols])
            at = 0x1000 + size * rng.randrange(600)
            tensors.append(B.nt_tensor(at, rows, cols, ld, dtype, 0))
            mine = {at + size * (r * ld + c) + b for r in range(rows) for c in range(cols) for b in range(size)}
            shared |= bool(mine & held)
            held |= mine
        records = (B.nt_tensor * len(tensors))(*tensors)
        rc = B.lib().normtest_list_check(records, records, len(tensors), B.ANY_DTYPE)
        assert rc == (B.NT_ERR_SHARED_MEMORY if shared else B.NT_OK)
        found[shared] += 1
    assert min(found) > 50
    far = (B.nt_tensor * 2)(B.nt_tensor(0x1000, 2, 5, 1 << 62, 0, 0), B.nt_tensor(0x2000, 1, 5, 5, 0, 0))
    assert B.lib().normtest_list_check(far, far, 2, B.ANY_DTYPE) == B.NT_ERR_BAD_ARG


def test_a_list_of_something_else_than_tensors():
    """The first entry like any other: a gradient that backward() has not made is None."""
    for bad in ([None], [None, torch.zeros(3)], [3.0], [torch.zeros(3).numpy()]):
        with pytest.raises(TypeError, match="torch tensors"):
            B.make_tensor_list(bad)
