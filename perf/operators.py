"""Timing cases of the operators over lists of tensors: gradient norm, clipping, accumulation and clipped AdamW.

One case is a plain dict:

    op       "norm"        norms of a gradient list
             "clip"        norms, then the scaled gradients into a list of their own (the raw ones stay for the batch-size test)
             "accumulate"  a micro-batch's gradients added to a list, with the norm of what is stored
             "adamw"       norm, then AdamW on the clipped gradient
    n        elements in all tensors together (about);  tensors  how many tensors, in the proportions of a decoder's parameters
    dtype    of the gradients: "bf16", "f16" (with a loss scale), "f32", or "mixed" (matrices bf16, vectors f32)
    to       type of the list that "clip" or "accumulate" writes;  beta  of "accumulate" (0: a gather)
    copy     "adamw" writes a bf16 copy of the weights too
    groups   norms of "all" tensors together, of "each" tensor, or of matrices and vectors apart ("kinds")
    kind     "l2" or "max"
    layout   "padded" (every tensor starts at a multiple of 64 elements), "packed" (one right behind the other, so at any element) or
             "strided" (column slices of wider matrices, as tensor parallelism leaves them)

The tensors of a list are views of one buffer per type, and outputs are those buffers whole: what lies between the tensors has to stay
as it was.  Weights and moments are updated in place by every pass.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
LOSS_SCALE = 1024.0
MAX_NORM = 1.0
HYPER = dict(lr=4e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=10)
_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_GAP = 7.0           # what lies between tensors
_CHUNK = 1 << 27     # elements widened to 64 bits at a time


def _case(name, op, n, tensors, dtype, *, to="f32", beta=1.0, copy=False, groups="all", kind="l2", layout="padded"):
    c = {"op": op, "n": n, "tensors": tensors, "dtype": dtype, "to": to, "beta": beta, "copy": copy, "groups": groups, "kind": kind,
         "layout": layout}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a probe's or an adapter's few parameters of odd size: launches and latency
        _case("norm_small_odd", "norm", 100_003, 12, "f32", layout="packed"),
        # the largest magnitude of every tensor of a mid-sized model, the table that a monitor draws
        _case("norm_each_max", "norm", 30_000_001, 75, "f16", groups="each", kind="max", layout="packed"),
        # the global norm of the headline model's gradients
        _case("norm_1p5b", "norm", 1_500_000_000, 300, "bf16"),
        # the smallest clipped step of the benchmark's tiny size
        _case("clip_tiny", "clip", 1 << 20, 12, "f32"),
        # the 148-tensor GPT-2-small-sized model, raw gradients kept for the test
        _case("clip_gpt2", "clip", 124_439_808, 148, "bf16", to="bf16"),
        # a tensor-parallel rank's slices, matrices and vectors clipped apart, to fp32
        _case("clip_slices", "clip", 30_000_001, 75, "mixed", groups="kinds", layout="strided"),
        # an adapter's gradients gathered into a row of the step's matrix
        _case("gather_small_odd", "accumulate", 100_003, 12, "bf16", beta=0.0, layout="packed"),
        # one micro-batch of the 148-tensor model added to its fp32 sums
        _case("accumulate_gpt2", "accumulate", 124_439_808, 148, "bf16"),
        # the paper's 304.6M-parameter model, accumulated in the gradients' own type
        _case("accumulate_300m", "accumulate", 304_600_000, 148, "bf16", to="bf16"),
        # the clipped update of the benchmark's tiny size
        _case("adamw_tiny", "adamw", 1 << 20, 12, "f32"),
        # one of eight shards of the 1.1B-parameter model under a loss scale, with the weights' copy for the next forward pass
        _case("adamw_shard", "adamw", 137_500_000, 156, "f16", copy=True, layout="packed"),
        # the whole 1.1B-parameter model on one GPU
        _case("adamw_1p1b", "adamw", 1_100_000_000, 300, "bf16", copy=True),
    ]


def draw(rng):
    """One more case: sizes log-uniform from a thousand elements to 12 GB of traffic, odd lengths and offsets among them."""
    op = rng.choice(["norm", "clip", "accumulate", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32", "f16", "mixed"])
    to = rng.choice(["f32", "f32", "bf16"]) if op in ("clip", "accumulate") else "f32"
    per = {"norm": 4, "clip": 8, "accumulate": 12, "adamw": 30}[op]
    n = int(math.exp(rng.uniform(math.log(1000), math.log(12e9 / per))))
    if rng.random() < 0.5:
        n = max(64, n // 64 * 64)
    return _case(None, op, n, rng.choice([1, 2, 12, 40, 75, 148, 300, 500]), dtype, to=to,
                 beta=rng.choice([0.0, 1.0, 1.0]) if op == "accumulate" else 1.0,
                 copy=op == "adamw" and rng.random() < 0.5, groups=rng.choice(["all", "all", "each", "kinds"]),
                 kind=rng.choice(["l2", "l2", "l2", "max"]) if op == "norm" else "l2",
                 layout=rng.choice(["padded", "packed", "strided"]))


# ---- inputs --------------------------------------------------------------------------------

def _shapes(case):
    """(rows, columns) of every tensor; one row for a vector.  The proportions are those of a decoder of width 768: embeddings, then
    per layer four matrices and eight vectors, then two vectors."""
    width = 768
    layer = [1, 1, 3 * width, 3, width, 1, 1, 1, 4 * width, 4, 4 * width, 1]
    base = [50257, 1024] + layer * 12 + [1, 1]
    n, count = case["n"], case["tensors"]
    weights = [base[i % len(base)] for i in range(count)]
    total, at, edges = sum(weights), 0, [0]
    for x in weights:
        at += x
        edges.append(round(n * at / total))
    shapes = []
    for x, size in zip(weights, (b - a for a, b in zip(edges, edges[1:]))):
        if x < width or size < 64:
            shapes.append((1, size))
        elif case["layout"] == "strided":
            cols = max(32, min(2048, round(math.sqrt(size / 8))))
            shapes.append((size // cols, cols))
        else:
            shapes.append((1, size))
    return shapes


def _types(case, shapes):
    biggest = max(r * c for r, c in shapes)
    return ["f32" if r * c * 100 < biggest else "bf16" for r, c in shapes] if case["dtype"] == "mixed" else [case["dtype"]] * len(shapes)


def _groups(case, shapes):
    if case["groups"] == "each":
        return list(range(len(shapes)))
    if case["groups"] == "kinds":
        biggest = max(r * c for r, c in shapes)
        return [1 if r * c * 100 < biggest else 0 for r, c in shapes]
    return [0] * len(shapes)


def _count(case):
    return {"all": 1, "kinds": 2, "each": case["tensors"]}[case["groups"]]


def _carve(shapes, types, layout, strided):
    """Tensors of these shapes in one buffer per type, which is filled with _GAP: (tensors, buffers)."""
    ends, places = {}, []
    for (r, c), t in zip(shapes, types):
        at = ends.get(t, 0)
        if layout != "packed":
            at = (at + 63) // 64 * 64
        ld = c + 40 if strided and r > 1 else c
        places.append((t, at, r, c, ld))
        ends[t] = at + r * ld
    buffers = {t: torch.full((max(1, end),), _GAP, dtype=_DTYPES[t], device=DEVICE) for t, end in sorted(ends.items())}
    tensors = [buffers[t].as_strided((r, c) if r > 1 else (c,), (ld, 1) if r > 1 else (1,), at) for t, at, r, c, ld in places]
    return tensors, buffers


def _fill(tensors, gen, spread, scale, square=False):
    """Normal values, tensor l on a scale of its own, log-uniform over 1e-3 to 1 where `spread`."""
    scales = torch.rand(len(tensors), device=DEVICE, generator=gen).mul_(-3 * math.log(10)).exp_().mul_(scale).tolist()
    for t, s in zip(tensors, scales):
        s = s if spread else scale
        rows = max(1, (1 << 26) // max(1, t.shape[-1])) if t.dim() == 2 else 1 << 26
        for part in t.split(rows):
            x = torch.randn(part.shape, device=DEVICE, generator=gen) * s
            part.copy_(x.square_() if square else x)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    shapes = _shapes(case)
    types, groups, layout = _types(case, shapes), _groups(case, shapes), case["layout"]
    s = {"case": case, "groups": groups, "count": _count(case), "group_ids": torch.tensor(groups, device=DEVICE),
         "grad_scale": 1.0 / LOSS_SCALE if case["dtype"] == "f16" else 1.0}
    s["grads"], s["grad_buffers"] = _carve(shapes, types, layout, layout == "strided")
    _fill(s["grads"], gen, True, 0.1 / s["grad_scale"])
    if case["op"] in ("clip", "accumulate"):
        # the list written is contiguous, whatever the gradients' layout
        s["to"], s["to_buffers"] = _carve(shapes, [case["to"]] * len(shapes), layout, False)
        _fill(s["to"], gen, True, 0.1)
    if case["op"] == "adamw":
        for name in ("w", "m", "v"):
            s[name], s[name + "_buffers"] = _carve(shapes, ["f32"] * len(shapes), layout, False)
            _fill(s[name], gen, False, 0.02, square=name == "v")
        if case["copy"]:
            s["copy"], s["copy_buffers"] = _carve(shapes, ["bf16"] * len(shapes), layout, False)
            for t in s["copy"]:
                t.zero_()
    if own:   # the handles that a training program keeps beside its tensors, and the records of its norms
        from paper_2412_21124_amd import binding as B
        s["lists"] = {"grads": B.make_tensor_list(s["grads"], groups=groups, num_groups=s["count"])}
        for name in ("to", "w", "m", "v", "copy"):
            if name in s:
                s["lists"][name] = B.make_tensor_list(s[name], like=s["lists"]["grads"])
        s["norms"] = B.make_norms(s["lists"]["grads"])
        s["views"] = B.norm_views(s["norms"])
        s["hyper"] = B.make_hyper(**HYPER)
    return s


def _outputs(s, norm, factor, flags):
    out = {"norm": norm, "factor": factor, "flags": flags}
    for name in ("to", "w", "m", "v", "copy"):
        if name + "_buffers" in s:
            out[name] = s[name + "_buffers"]
    return out


# ---- the framework's operators -------------------------------------------------------------

def _run_own(s):
    from paper_2412_21124_amd import binding as B
    case, lists, norms = s["case"], s["lists"], s["norms"]
    kind = B.NT_NORM_MAX if case["kind"] == "max" else B.NT_NORM_L2
    if case["op"] == "accumulate":
        B.normtest_accumulate(lists["to"], lists["grads"], beta=case["beta"], scale=s["grad_scale"], norms=norms, max_norm=MAX_NORM)
    else:
        B.normtest_grad_norm(lists["grads"], norms, max_norm=MAX_NORM, grad_scale=s["grad_scale"], kind=kind)
    if case["op"] == "clip":
        B.normtest_clip_grads(lists["grads"], norms, out=lists["to"])
    if case["op"] == "adamw":
        B.normtest_adamw_tensors(lists["grads"], lists["w"], lists["m"], lists["v"], s["hyper"], norms=norms, copy=lists.get("copy"))
    return _outputs(s, s["views"]["norm"], s["views"]["factor"], s["views"]["flags"])


# ---- their plain form ----------------------------------------------------------------------

def _flat(tensors):
    return torch.cat([t.reshape(-1) for t in tensors]).float()


def _store(flat, tensors):
    parts = flat.split([t.numel() for t in tensors])
    torch._foreach_copy_(tensors, [x.view(t.shape) for x, t in zip(parts, tensors)])


def _norms(s, flat, tensors, scale, kind):
    """(norm, coefficient, factor, flags) of every group of a list whose values are in `flat`."""
    if s["count"] == 1:
        raw = flat.abs().amax().reshape(1) if kind == "max" else flat.square().sum().reshape(1)
    else:
        parts = flat.split([t.numel() for t in tensors])
        raw = torch.zeros(s["count"], device=DEVICE)
        if kind == "max":
            raw.scatter_reduce_(0, s["group_ids"], torch.stack([x.abs().amax() if x.numel() else x.sum() for x in parts]), "amax")
        else:
            raw.index_add_(0, s["group_ids"], torch.stack([x.square().sum() for x in parts]))
    norm = (raw if kind == "max" else raw.sqrt()) * scale
    finite = torch.isfinite(norm)
    coef = torch.where(finite, (MAX_NORM / (norm + 1e-6)).clamp(max=1.0), 1.0)
    status = torch.where(finite, torch.where(norm == 0, 2, 0), 1)
    return norm, coef, coef * scale, torch.stack([status, (coef < 1).long()], 1).int()


def _spread(s, per_group, tensors):
    """A value per group, for every element of the list."""
    if s["count"] == 1:
        return per_group
    return torch.cat([x.expand(t.numel()) for x, t in zip(per_group[s["group_ids"]].split(1), tensors)])


def _run_plain(s):
    case, scale, grads = s["case"], s["grad_scale"], s["grads"]
    flat = _flat(grads)
    if case["op"] == "accumulate":
        flat = flat * scale
        _store(flat if case["beta"] == 0 else case["beta"] * _flat(s["to"]) + flat, s["to"])
        norm, _, factor, flags = _norms(s, _flat(s["to"]), s["to"], 1.0, "l2")
        return _outputs(s, norm, factor, flags)
    norm, _, factor, flags = _norms(s, flat, grads, scale, case["kind"])
    if case["op"] == "clip":
        _store(flat * _spread(s, factor, grads), s["to"])
    if case["op"] == "adamw":
        h = HYPER
        g = flat * _spread(s, factor, grads)
        m = h["beta1"] * _flat(s["m"]) + (1 - h["beta1"]) * g
        v = h["beta2"] * _flat(s["v"]) + (1 - h["beta2"]) * g * g
        _store(m, s["m"])
        _store(v, s["v"])
        root = (v / (1 - h["beta2"] ** h["step"])).sqrt() + h["eps"]
        w = (1 - h["lr"] * h["weight_decay"]) * _flat(s["w"]) - h["lr"] / (1 - h["beta1"] ** h["step"]) * m / root
        _store(w, s["w"])
        if case["copy"]:
            _store(w, s["copy"])
    return _outputs(s, norm, factor, flags)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    shapes = _shapes(case)
    size = {"bf16": 2, "f16": 2, "f32": 4}
    n = sum(r * c for r, c in shapes)
    read = sum(r * c * size[t] for (r, c), t in zip(shapes, _types(case, shapes)))
    out = n * size[case["to"]]
    if case["op"] == "norm":
        return {"bytes": read, "flops": 2 * n}
    if case["op"] == "clip":   # the gradients' second reading is not counted
        return {"bytes": read + out, "flops": 3 * n}
    if case["op"] == "accumulate":
        return {"bytes": read + (out if case["beta"] == 0 else 2 * out), "flops": 5 * n}
    return {"bytes": read + 24 * n + (2 * n if case["copy"] else 0), "flops": 18 * n}


# ---- 64 bits -------------------------------------------------------------------------------

def _wide(tensor):
    """The tensor's values in 64 bits, a piece at a time."""
    x = tensor.reshape(-1)
    for lo in range(0, x.numel(), _CHUNK):
        yield lo, x[lo:lo + _CHUNK].double()


def _exact_norms(s, tensors, scale, kind):
    total = [0.0] * s["count"]
    for t, g in zip(tensors, s["groups"]):
        for _, x in _wide(t):
            total[g] = max(total[g], float(x.abs().max())) if kind == "max" else total[g] + float(x.square().sum())
    norm = [scale * (x if kind == "max" else math.sqrt(x)) for x in total]
    coef = [min(1.0, MAX_NORM / (x + 1e-6)) for x in norm]
    return norm, [c * scale for c in coef]


def _blank(buffers):
    return {t: b.double() for t, b in buffers.items()}


def _placed(buffers, like, tensor, kind):
    """The part of the 64-bit buffer that stands for this tensor."""
    return buffers[kind].as_strided(tensor.shape, tensor.stride(), tensor.storage_offset()).view(-1)


def exact(case, seed):
    """The first pass on prepare(case, seed) in 64 bits."""
    s = prepare(case, seed)
    scale, groups = s["grad_scale"], s["groups"]
    out = {"flags": None}
    if case["op"] == "accumulate":
        buffers = _blank(s["to_buffers"])
        stored = []
        for x, y in zip(s["grads"], s["to"]):
            to = _placed(buffers, s["to_buffers"], y, case["to"])
            for lo, part in _wide(x):
                old = to[lo:lo + part.numel()]
                old.copy_(scale * part + (case["beta"] * old if case["beta"] else 0.0))
            stored.append(to.to(y.dtype))
        norm, factor = _exact_norms(s, stored, 1.0, "l2")
        out["to"] = buffers
    else:
        norm, factor = _exact_norms(s, s["grads"], scale, case["kind"])
    if case["op"] == "clip":
        buffers = _blank(s["to_buffers"])
        for x, y, g in zip(s["grads"], s["to"], groups):
            to = _placed(buffers, s["to_buffers"], y, case["to"])
            for lo, part in _wide(x):
                to[lo:lo + part.numel()] = factor[g] * part
        out["to"] = buffers
    if case["op"] == "adamw":
        h = HYPER
        wide = {name: _blank(s[name + "_buffers"]) for name in ("w", "m", "v")}
        for l, (x, g) in enumerate(zip(s["grads"], groups)):
            at = {name: _placed(wide[name], s[name + "_buffers"], s[name][l], "f32") for name in wide}
            for lo, part in _wide(x):
                here = slice(lo, lo + part.numel())
                grad = factor[g] * part
                m = at["m"][here].mul_(h["beta1"]).add_((1 - h["beta1"]) * grad)
                v = at["v"][here].mul_(h["beta2"]).add_((1 - h["beta2"]) * grad ** 2)
                step = (m / (1 - h["beta1"] ** h["step"])) / ((v / (1 - h["beta2"] ** h["step"])).sqrt() + h["eps"])
                w = at["w"][here]
                w.sub_(h["lr"] * (step + h["weight_decay"] * w))
        out.update(wide)
        if case["copy"]:
            copied = _blank(s["copy_buffers"])
            for l, t in enumerate(s["copy"]):
                _placed(copied, s["copy_buffers"], t, "bf16").copy_(_placed(wide["w"], None, s["w"][l], "f32"))
            out["copy"] = copied
    return dict(out, norm=torch.tensor(norm, dtype=torch.float64), factor=torch.tensor(factor, dtype=torch.float64))
