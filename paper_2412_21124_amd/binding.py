"""Binding of ``libnormtest.so`` (``include/normtest.h``): argument marshalling only, by ctypes and, for the calls of a training
loop, by ``csrc/callpath.cpp``.

Every step of the path runs in the library's HIP kernels.  torch supplies device memory and the
current stream, nothing else.  There is no CPU fallback: if the library cannot be loaded or a call
fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import importlib.util
import warnings
from dataclasses import dataclass
from typing import Optional

import torch

from . import build as _build

NT_F32, NT_BF16, NT_F16 = 0, 1, 2
NT_NORM_L2, NT_NORM_MAX = 0, 1
NT_SKIP_NONFINITE = 1
NT_DO_STATS, NT_DO_ADAMW, NT_PARTIAL, NT_WRITE_GBAR, NT_COORD_TEST, NT_ONE_PASS = 1, 2, 4, 8, 16, 32
NT_STATUS_NONFINITE = 1
NT_STATUS_ZERO_GRAD_NORM = 2
NT_STATUS_CLAMPED = 4
NT_STATUS_PARTIAL_ONLY = 8
NT_STATUS_T_SATURATED = 16
NT_STATUS_NO_STATS = 32
NT_STATUS_BAD_RANGE = 64
NT_OK, NT_ERR_BAD_ARG, NT_ERR_UNSUPPORTED, NT_ERR_WORKSPACE_TOO_SMALL, NT_ERR_TOO_LARGE, NT_ERR_HIP_BASE = 0, -1, -2, -3, -4, -1000
NT_ERR_SHARED_MEMORY = -6


class nt_hyper(ctypes.Structure):
    _fields_ = [
        ("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
        ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("eta", ctypes.c_double),
        ("step", ctypes.c_int64), ("b_k", ctypes.c_int64), ("b_max", ctypes.c_int64),
        ("round_to", ctypes.c_int64), ("ddof", ctypes.c_int32), ("flags", ctypes.c_uint32),
    ]


class nt_shard_info(ctypes.Structure):
    _fields_ = [
        ("shard_id", ctypes.c_int32), ("num_shards", ctypes.c_int32),
        ("shard_offset", ctypes.c_int64), ("d_global", ctypes.c_int64),
    ]


class nt_result(ctypes.Structure):
    _fields_ = [
        ("A", ctypes.c_double), ("B", ctypes.c_double), ("C", ctypes.c_double),
        ("A_lo", ctypes.c_double), ("B_lo", ctypes.c_double), ("C_lo", ctypes.c_double),
        ("gbar_sq", ctypes.c_double), ("var_l1", ctypes.c_double), ("T", ctypes.c_double),
        ("clip_coef", ctypes.c_double), ("next_b", ctypes.c_int64), ("coord_fail", ctypes.c_int64),
        ("pass_", ctypes.c_int32), ("status", ctypes.c_uint32), ("coord_max_ratio", ctypes.c_double),
    ]

    def as_dict(self) -> dict:
        d = {k: getattr(self, k) for k, _ in self._fields_}
        d["pass"] = d.pop("pass_")
        return d


RESULT_BYTES = ctypes.sizeof(nt_result)


class nt_layer_stats(ctypes.Structure):
    _fields_ = [
        ("A", ctypes.c_double), ("B", ctypes.c_double), ("C", ctypes.c_double),
        ("gbar_sq", ctypes.c_double), ("var_l1", ctypes.c_double), ("T", ctypes.c_double),
        ("n", ctypes.c_int64), ("coord_fail", ctypes.c_int64), ("pass_", ctypes.c_int32), ("status", ctypes.c_uint32),
        ("coord_max_ratio", ctypes.c_double),
    ]

    def as_dict(self) -> dict:
        d = {k: getattr(self, k) for k, _ in self._fields_}
        d["pass"] = d.pop("pass_")
        return d


LAYER_BYTES = ctypes.sizeof(nt_layer_stats)


class nt_tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("group", ctypes.c_int32)]


class nt_plan(ctypes.Structure):
    _fields_ = [("image", ctypes.c_void_p), ("bytes", ctypes.c_size_t), ("upload_bytes", ctypes.c_size_t), ("elements", ctypes.c_int64),
                ("tensors", ctypes.c_int32), ("groups", ctypes.c_int32), ("items", ctypes.c_uint32 * 2), ("slots", ctypes.c_uint32 * 2),
                ("slabs", ctypes.c_uint32 * 2),
                ("magic", ctypes.c_uint32), ("flags", ctypes.c_uint32)]


class nt_norm(ctypes.Structure):
    _fields_ = [("norm", ctypes.c_double), ("coef", ctypes.c_double), ("norm32", ctypes.c_float), ("factor", ctypes.c_float),
                ("status", ctypes.c_uint32), ("clipped", ctypes.c_int32), ("elements", ctypes.c_int64)]

    def as_dict(self) -> dict:
        return {k: getattr(self, k) for k, _ in self._fields_}


NORM_BYTES = ctypes.sizeof(nt_norm)


class NormtestError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed with code %d: %s" % (where, code, normtest_strerror(code)))


_lib = None
_fast = None   # the native call path (csrc/callpath.cpp), loaded with the library; None: every call is marshalled in Python


def _load_callpath():
    """The native call path, ready for calls, or None where it cannot be built or loaded: nothing but the time of a call depends on it."""
    try:
        spec = importlib.util.spec_from_file_location(__package__ + "._callpath", _build.ensure_callpath())
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.init(nt_hyper, nt_shard_info, torch.nn.Parameter, torch._C._cuda_getCurrentRawStream)
        return module
    except Exception as e:   # no compiler, no headers, a file that is no module of this Python and torch
        warnings.warn("normtest: calls are marshalled in Python, which a short step notices: %s: %s" % (type(e).__name__, e), RuntimeWarning)
        return None


def _done(rc: Optional[int], where: str) -> bool:
    """Whether the native call path took the call; raises if the library refused it."""
    if rc is not None and rc != NT_OK:
        raise NormtestError(rc, where)
    return rc is not None


def lib(path: Optional[str] = None):
    """The loaded C-ABI library (built on first use if missing).  `path` loads another build of it."""
    global _lib, _fast
    if _lib is None or path is not None:
        L = ctypes.CDLL(path if path is not None else _build.ensure_built())
        vp, i64 = ctypes.c_void_p, ctypes.c_int64
        L.normtest_tile_coords.argtypes = [i64]
        L.normtest_tile_coords.restype = i64
        L.normtest_workspace_bytes.argtypes = [i64, i64]
        L.normtest_workspace_bytes.restype = ctypes.c_size_t
        L.normtest_workspace_bytes_for.argtypes = [ctypes.c_int, i64, i64, ctypes.c_uint32]
        L.normtest_workspace_bytes_for.restype = ctypes.c_size_t
        L.normtest_step.argtypes = [vp, ctypes.c_int, i64, i64, i64, vp, vp, vp, vp,
                                    ctypes.POINTER(nt_hyper), ctypes.POINTER(nt_shard_info),
                                    vp, ctypes.c_size_t, vp, vp]
        L.normtest_step.restype = ctypes.c_int
        L.normtest_step_static.argtypes = [vp, ctypes.c_int, i64, i64, i64, vp, vp, vp, vp,
                                           ctypes.POINTER(nt_hyper), ctypes.POINTER(nt_shard_info), vp, vp]
        L.normtest_step_static.restype = ctypes.c_int
        L.normtest_static_max_coords.argtypes = [i64]
        L.normtest_static_max_coords.restype = i64
        L.normtest_step_rows.argtypes = [vp, ctypes.c_int, i64, i64, vp, vp, vp, vp,
                                         ctypes.POINTER(nt_hyper), ctypes.POINTER(nt_shard_info),
                                         vp, ctypes.c_size_t, vp, vp]
        L.normtest_step_rows.restype = ctypes.c_int
        L.normtest_combine.argtypes = [ctypes.POINTER(nt_result), ctypes.c_int32, i64,
                                       ctypes.POINTER(nt_hyper), ctypes.POINTER(nt_result)]
        L.normtest_combine.restype = ctypes.c_int
        L.normtest_step_clipped.argtypes = [vp, ctypes.c_int, i64, i64, i64, vp, vp, vp, vp, ctypes.c_double,
                                            ctypes.POINTER(nt_hyper), ctypes.POINTER(nt_shard_info),
                                            vp, ctypes.c_size_t, vp, vp]
        L.normtest_step_clipped.restype = ctypes.c_int
        L.normtest_layer_stats.argtypes = [vp, ctypes.c_int, ctypes.c_int, i64, i64, i64, vp, ctypes.c_int32, vp, vp, vp]
        L.normtest_layer_stats.restype = ctypes.c_int
        L.normtest_adamw_gbar.argtypes = [vp, i64, vp, vp, vp, ctypes.POINTER(nt_hyper), ctypes.c_double, vp, vp]
        L.normtest_adamw_gbar.restype = ctypes.c_int
        L.normtest_clip_coef.argtypes = [ctypes.c_double, ctypes.c_double]
        L.normtest_clip_coef.restype = ctypes.c_double
        L.normtest_resplit.argtypes = [i64, i64, i64, i64, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.normtest_resplit.restype = ctypes.c_int
        L.normtest_schedule_flags.argtypes = [i64, i64, i64, i64, ctypes.c_uint32]
        L.normtest_schedule_flags.restype = ctypes.c_uint32
        plan, dbl = ctypes.POINTER(nt_plan), ctypes.c_double
        L.normtest_plan_make.argtypes = [ctypes.POINTER(nt_tensor), ctypes.c_int32, ctypes.c_int32, plan, vp, ctypes.c_size_t]
        L.normtest_list_check.argtypes = [ctypes.POINTER(nt_tensor), ctypes.POINTER(nt_tensor), ctypes.c_int32, ctypes.c_uint32]
        L.normtest_grad_norm.argtypes = [plan, vp, ctypes.c_int32, dbl, dbl, vp, vp]
        L.normtest_clip_grads.argtypes = [plan, vp, vp, vp, vp]
        L.normtest_accumulate.argtypes = [plan, vp, vp, dbl, dbl, vp, ctypes.c_int32, dbl, dbl, vp, vp]
        L.normtest_adamw_tensors.argtypes = [plan, vp, vp, vp, vp, vp, ctypes.POINTER(nt_hyper), dbl, vp, ctypes.c_uint32, vp]
        for name in ("plan_make", "list_check", "grad_norm", "clip_grads", "accumulate", "adamw_tensors"):
            getattr(L, "normtest_" + name).restype = ctypes.c_int
        L.normtest_calib_copy.argtypes = [vp, vp, ctypes.c_size_t, vp]
        L.normtest_calib_copy.restype = ctypes.c_int
        L.normtest_calib_streams.argtypes = [vp, ctypes.c_size_t, i64, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                             ctypes.c_int, i64, vp]
        L.normtest_calib_streams.restype = ctypes.c_int
        L.normtest_strerror.argtypes = [ctypes.c_int]
        L.normtest_strerror.restype = ctypes.c_char_p
        for name in ("normtest_step", "normtest_step_rows", "normtest_step_clipped", "normtest_adamw_gbar", "normtest_layer_stats",
                     "normtest_workspace_bytes_for", "normtest_grad_norm", "normtest_clip_grads", "normtest_accumulate",
                     "normtest_adamw_tensors"):
            setattr(L, name + "_entry", ctypes.cast(getattr(L, name), ctypes.c_void_p).value)
        if _lib is None:
            _fast = _load_callpath()
        _lib = L
    return _lib


def normtest_strerror(code: int) -> str:
    return lib().normtest_strerror(code).decode()


def normtest_tile_coords(J: int) -> int:
    return int(lib().normtest_tile_coords(J))


def normtest_workspace_bytes(J: int, d: int) -> int:
    return int(lib().normtest_workspace_bytes(J, d))


def normtest_workspace_bytes_for(gdtype: int, J: int, d: int, flags: int) -> int:
    return int(lib().normtest_workspace_bytes_for(gdtype, J, d, flags))


def make_hyper(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, eta=0.1, step=1, b_k=1,
               b_max=0, round_to=1, ddof=1, flags=NT_DO_STATS | NT_DO_ADAMW) -> nt_hyper:
    return nt_hyper(lr, beta1, beta2, eps, weight_decay, eta, step, b_k, b_max, round_to, ddof, flags)


def _gdtype(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return NT_F32
    if t.dtype == torch.bfloat16:
        return NT_BF16
    raise TypeError("gradients must be float32 or bfloat16, got %s" % t.dtype)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _matrix_layout(grads: torch.Tensor, d: Optional[int], where: str):
    """(J, d, ld, device) of a (J, ld) gradient tensor whose rows are the gradient vectors."""
    if grads.dim() != 2 or (grads.shape[1] > 1 and grads.stride(1) != 1):
        raise ValueError("grads must be (J, ld) with a contiguous last axis")
    J = grads.shape[0]
    ld = grads.stride(0) if J > 1 else grads.shape[1]
    d = grads.shape[1] if d is None else d
    if grads.device.type != "cuda":
        raise ValueError("%s needs device tensors; there is no CPU path" % where)
    return J, d, ld, grads.device


def _check_vectors(dev, d: int, required: bool = False, **tensors):
    """w, m, v, gbar: contiguous float32 vectors of at least d elements on the gradients' device."""
    for name, t in tensors.items():
        if t is None and not required:
            continue
        if t is None or t.dtype != torch.float32 or t.device != dev or not t.is_contiguous() or t.numel() < d:
            raise ValueError("%s must be a contiguous float32 tensor of >= d elements on %s" % (name, dev))


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


# What the native call path does not take (an own stream, tensors of another device, buffers to be made here) goes through the checks
# below.  The stream's handle and the device are asked for directly: torch.cuda.current_stream builds a Stream object (1.9 us against
# 0.1) and torch.cuda.device is only entered when another device is current (1.3 us against 0.1).
def _stream_handle(stream: Optional[torch.cuda.Stream], dev: torch.device) -> int:
    return torch._C._cuda_getCurrentRawStream(dev.index) if stream is None else stream.cuda_stream


def _call(dev: torch.device, fn, *args) -> int:
    if torch._C._cuda_getDevice() == dev.index:
        return fn(*args)
    with torch.cuda.device(dev):
        return fn(*args)


def normtest_step(grads: torch.Tensor, w: Optional[torch.Tensor], m: Optional[torch.Tensor],
                  v: Optional[torch.Tensor], hyper: nt_hyper, *, d: Optional[int] = None,
                  shard: Optional[nt_shard_info] = None, gbar_out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, result: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Enqueue one step on `stream` (default: torch's current stream) and return the device tensor
    (uint8[sizeof(nt_result)]) that will hold the nt_result; read it with `read_result` after a sync.

    grads: (J, ld) device tensor whose rows are the gradient vectors (last axis contiguous); the first
    d columns are used (default: all).  w, m, v: float32 device vectors of length >= d, updated in place.
    """
    if stream is None and workspace is not None and result is not None:
        L = lib()
        if _fast and _done(_fast.step(L.normtest_step_entry, grads, w, m, v, hyper, d, shard, gbar_out, workspace, result), "normtest_step"):
            return result
    J, d, ld, dev = _matrix_layout(grads, d, "normtest_step")
    _check_vectors(dev, d, w=w, m=m, v=v, gbar_out=gbar_out)
    gdtype = _gdtype(grads)
    own_workspace = workspace is None
    if own_workspace:
        need = normtest_workspace_bytes_for(gdtype, J, d, hyper.flags)
        workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=dev)
    if result is None:
        result = torch.empty(RESULT_BYTES, dtype=torch.uint8, device=dev)
    rc = _call(dev, lib().normtest_step, _ptr(grads), gdtype, J, d, ld, _ptr(w), _ptr(m), _ptr(v), _ptr(gbar_out),
               ctypes.byref(hyper), ctypes.byref(shard) if shard is not None else None,
               _ptr(workspace), _nbytes(workspace), _ptr(result), _stream_handle(stream, dev))
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_step")
    if own_workspace:
        # keep the scratch alive until the stream has consumed it
        workspace.record_stream(torch.cuda.current_stream(dev) if stream is None else stream)
    return result


def normtest_static_max_coords(J: int) -> int:
    return int(lib().normtest_static_max_coords(J))


def normtest_step_static(grads: torch.Tensor, w: Optional[torch.Tensor], m: Optional[torch.Tensor],
                         v: Optional[torch.Tensor], hyper: nt_hyper, result: torch.Tensor, *, d: Optional[int] = None,
                         shard: Optional[nt_shard_info] = None, gbar_out: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """normtest_step without a workspace (the library's built-in scratch) and without any allocation here:
    the caller passes the device tensor for the nt_result."""
    J, d, ld, dev = _matrix_layout(grads, d, "normtest_step_static")
    _check_vectors(dev, d, w=w, m=m, v=v, gbar_out=gbar_out)
    if result is None or result.device != dev or _nbytes(result) < RESULT_BYTES:
        raise ValueError("result must be a device tensor of at least RESULT_BYTES bytes")
    rc = _call(dev, lib().normtest_step_static, _ptr(grads), _gdtype(grads), J, d, ld, _ptr(w), _ptr(m), _ptr(v),
               _ptr(gbar_out), ctypes.byref(hyper), ctypes.byref(shard) if shard is not None else None,
               _ptr(result), _stream_handle(stream, dev))
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_step_static")
    return result


def make_row_table(rows) -> torch.Tensor:
    """Device-resident table of the rows' addresses (int64[J]) for normtest_step_rows.  The caller keeps
    the rows and the table alive until the step has run."""
    dev = rows[0].device
    return torch.tensor([r.data_ptr() for r in rows], dtype=torch.int64, device=dev)


def normtest_step_rows(rows, w: Optional[torch.Tensor], m: Optional[torch.Tensor], v: Optional[torch.Tensor],
                       hyper: nt_hyper, *, d: Optional[int] = None, table: Optional[torch.Tensor] = None,
                       shard: Optional[nt_shard_info] = None, gbar_out: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, result: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """normtest_step for J separately allocated gradient rows (a sequence of 1-D device tensors of one dtype)."""
    if stream is None and table is not None and workspace is not None and result is not None:
        L = lib()
        if _fast and _done(_fast.step_rows(L.normtest_step_rows_entry, rows, w, m, v, hyper, d, table, shard, gbar_out, workspace, result),
                           "normtest_step_rows"):
            return result
    J = len(rows)
    dev = rows[0].device
    if dev.type != "cuda":
        raise ValueError("normtest_step_rows needs device tensors; there is no CPU path")
    d = min(r.numel() for r in rows) if d is None else d
    for r in rows:
        if r.dtype != rows[0].dtype or r.device != dev or r.dim() != 1 or not r.is_contiguous() or r.numel() < d:
            raise ValueError("rows must be contiguous 1-D tensors of one dtype and >= d elements on %s" % dev)
    _check_vectors(dev, d, w=w, m=m, v=v, gbar_out=gbar_out)
    if table is None:
        table = make_row_table(rows)
    own_workspace = workspace is None
    if own_workspace:
        need = normtest_workspace_bytes_for(_gdtype(rows[0]), J, d, hyper.flags)
        workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=dev)
    if result is None:
        result = torch.empty(RESULT_BYTES, dtype=torch.uint8, device=dev)
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    rc = _call(dev, lib().normtest_step_rows, _ptr(table), _gdtype(rows[0]), J, d, _ptr(w), _ptr(m), _ptr(v),
               _ptr(gbar_out), ctypes.byref(hyper), ctypes.byref(shard) if shard is not None else None,
               _ptr(workspace), _nbytes(workspace), _ptr(result), stream.cuda_stream)
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_step_rows")
    table.record_stream(stream)
    if own_workspace:
        workspace.record_stream(stream)
    return result


def normtest_step_clipped(grads: torch.Tensor, w: torch.Tensor, m: torch.Tensor, v: torch.Tensor,
                          gbar_buf: torch.Tensor, max_norm: float, hyper: nt_hyper, *, d: Optional[int] = None,
                          shard: Optional[nt_shard_info] = None, workspace: Optional[torch.Tensor] = None,
                          result: Optional[torch.Tensor] = None,
                          stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Two-phase gradient-clipped step (statistics + gbar, then AdamW on the clipped gbar); see normtest_step."""
    if stream is None and workspace is not None and result is not None:
        L = lib()
        if _fast and _done(_fast.step_clipped(L.normtest_step_clipped_entry, grads, w, m, v, gbar_buf, max_norm, hyper, d, shard, workspace,
                                              result), "normtest_step_clipped"):
            return result
    J, d, ld, dev = _matrix_layout(grads, d, "normtest_step_clipped")
    _check_vectors(dev, d, required=True, w=w, m=m, v=v, gbar_buf=gbar_buf)
    own_workspace = workspace is None
    if own_workspace:
        need = normtest_workspace_bytes_for(_gdtype(grads), J, d, hyper.flags | NT_WRITE_GBAR)
        workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=dev)
    if result is None:
        result = torch.empty(RESULT_BYTES, dtype=torch.uint8, device=dev)
    rc = _call(dev, lib().normtest_step_clipped, _ptr(grads), _gdtype(grads), J, d, ld, _ptr(w), _ptr(m), _ptr(v),
               _ptr(gbar_buf), float(max_norm), ctypes.byref(hyper), ctypes.byref(shard) if shard is not None else None,
               _ptr(workspace), _nbytes(workspace), _ptr(result), _stream_handle(stream, dev))
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_step_clipped")
    if own_workspace:
        workspace.record_stream(torch.cuda.current_stream(dev) if stream is None else stream)
    return result


def normtest_adamw_gbar(gbar: torch.Tensor, w: torch.Tensor, m: torch.Tensor, v: torch.Tensor, hyper: nt_hyper,
                        grad_scale: float = 1.0, *, d: Optional[int] = None, result: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> None:
    """AdamW on grad_scale (* result.clip_coef) * gbar for a mean gradient already in device memory."""
    if stream is None:
        L = lib()
        if _fast and _done(_fast.adamw_gbar(L.normtest_adamw_gbar_entry, gbar, w, m, v, hyper, grad_scale, d, result), "normtest_adamw_gbar"):
            return
    d = gbar.numel() if d is None else d
    dev = gbar.device
    if dev.type != "cuda":
        raise ValueError("normtest_adamw_gbar needs device tensors; there is no CPU path")
    _check_vectors(dev, d, required=True, gbar=gbar, w=w, m=m, v=v)
    rc = _call(dev, lib().normtest_adamw_gbar, _ptr(gbar), d, _ptr(w), _ptr(m), _ptr(v), ctypes.byref(hyper),
               float(grad_scale), _ptr(result), _stream_handle(stream, dev))
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_adamw_gbar")


def normtest_layer_stats(grads, layer_offsets: torch.Tensor, workspace: torch.Tensor, *, d: Optional[int] = None,
                         table: Optional[torch.Tensor] = None, layers: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Enqueue the per-layer table after a step that used `workspace` on the same stream.  grads: the (J, ld)
    tensor of that step, or the sequence of rows given to normtest_step_rows (then `table` may carry the
    address table already made).  layer_offsets: int64 device tensor of L+1 ascending offsets.  Returns the
    device tensor (uint8[L * sizeof(nt_layer_stats)]); read it with `read_layers` after a sync."""
    if stream is None and table is None and layers is not None and isinstance(grads, torch.Tensor):
        L = lib()
        if _fast and _done(_fast.layer_stats(L.normtest_layer_stats_entry, grads, layer_offsets, workspace,
                                             L.normtest_workspace_bytes_for_entry, d, layers), "normtest_layer_stats"):
            return layers
    rows = None if isinstance(grads, torch.Tensor) else list(grads)
    first = grads if rows is None else rows[0]
    dev = first.device
    if dev.type != "cuda":
        raise ValueError("normtest_layer_stats needs device tensors; there is no CPU path")
    if rows is None:
        J, d, ld, _ = _matrix_layout(grads, d, "normtest_layer_stats")
        gptr = _ptr(grads)
    else:
        J = len(rows)
        d = min(r.numel() for r in rows) if d is None else d
        ld = d
        if table is None:
            table = make_row_table(rows)
        gptr = _ptr(table)
    if (layer_offsets.dtype != torch.int64 or layer_offsets.device != dev or layer_offsets.dim() != 1
            or not layer_offsets.is_contiguous() or layer_offsets.numel() < 2):
        raise ValueError("layer_offsets must be a contiguous int64 device vector of L+1 >= 2 entries")
    L = layer_offsets.numel() - 1
    if workspace.device != dev or _nbytes(workspace) < normtest_workspace_bytes_for(_gdtype(first), J, d, NT_DO_STATS):
        raise ValueError("workspace must be the device workspace of the preceding step")
    if layers is None:
        layers = torch.empty(L * LAYER_BYTES, dtype=torch.uint8, device=dev)
    elif _nbytes(layers) < L * LAYER_BYTES:
        raise ValueError("layers must hold L * sizeof(nt_layer_stats) bytes")
    rc = _call(dev, lib().normtest_layer_stats, gptr, 0 if rows is None else 1, _gdtype(first), J, d, ld,
               _ptr(layer_offsets), L, _ptr(workspace), _ptr(layers), _stream_handle(stream, dev))
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_layer_stats")
    if table is not None:
        table.record_stream(torch.cuda.current_stream(dev) if stream is None else stream)
    return layers


def read_layers(layers: torch.Tensor, L: Optional[int] = None):
    """Synchronising read of a device nt_layer_stats array: a list of nt_layer_stats."""
    host = layers.cpu().numpy().tobytes()
    L = len(host) // LAYER_BYTES if L is None else L
    return [nt_layer_stats.from_buffer_copy(host, l * LAYER_BYTES) for l in range(L)]


# ---- lists of tensors ------------------------------------------------------------------------

_LIST_DTYPES = {torch.float32: NT_F32, torch.bfloat16: NT_BF16, torch.float16: NT_F16}
ANY_DTYPE = (1 << NT_F32) | (1 << NT_BF16) | (1 << NT_F16)


def _rows_of(t: torch.Tensor):
    """(rows, columns, row stride, order) of a tensor in memory: one row where its elements are dense.  order names its dimensions from
    the outermost in memory on, None where that is their own order: only then do elements of tensors of other shapes correspond."""
    n = t.numel()
    if t.is_contiguous():
        return 1, n, n, None
    dims = [i for i in range(t.dim()) if t.shape[i] != 1]
    by_stride = sorted(dims, key=lambda i: -t.stride(i))
    order = None if by_stride == dims else tuple(by_stride)
    merged = []   # (size, stride) from the innermost out
    for i in reversed(by_stride):
        if merged and t.stride(i) == merged[-1][0] * merged[-1][1]:
            merged[-1] = (merged[-1][0] * t.shape[i], merged[-1][1])
        else:
            merged.append((t.shape[i], t.stride(i)))
    if merged[0][1] != 1:
        merged.insert(0, (1, 1))   # a column of single elements
    if len(merged) == 1:
        return 1, n, n, order
    if len(merged) > 2 or merged[1][1] < merged[0][0]:
        raise ValueError("a tensor of a list must be dense or rows of one stride that do not overlap: got shape %s, strides %s"
                         % (tuple(t.shape), t.stride()))
    return merged[1][0], merged[0][0], merged[1][1], order


class TensorPlan:
    """How the tensors of a list are cut into pieces, on the device, with the scratch memory of its norms.  Made by make_tensor_list
    and shared by the lists made `like` it; one call at a time may use it."""

    def __init__(self, records, layouts, groups: int, device: torch.device):
        # layouts: (rows, columns, order, group, shape) of every tensor
        self.records, self.layouts, self.groups, self.device = records, layouts, groups, device
        self.record = nt_plan()
        rc = lib().normtest_plan_make(records, len(layouts), groups, ctypes.byref(self.record), None, 0)
        if rc == NT_OK:
            host = torch.empty(max(8, self.record.upload_bytes), dtype=torch.uint8)
            rc = lib().normtest_plan_make(records, len(layouts), groups, ctypes.byref(self.record), host.data_ptr(), host.numel())
        if rc != NT_OK:
            raise NormtestError(rc, "normtest_plan_make")
        self.image = torch.empty(max(16, self.record.bytes), dtype=torch.uint8, device=device)
        self.image[:host.numel()].copy_(host)
        self.record.image = self.image.data_ptr()
        self.stream = _stream_handle(None, device)


class TensorList:
    """Tensors of one device, as the calls on lists take them: their addresses in a table on the device, and a plan.  The tensors may
    change their values but not their memory, type or shape; `refresh` reads their addresses again.  A list holds its tensors: a gradient
    that a program drops and makes anew (zero_grad with set_to_none) is another tensor, which the list learns of from refresh only."""

    def __init__(self, tensors, plan: TensorPlan, records):
        self.plan = plan
        self.table = None
        self._check(records)
        self.tensors, self._records = tuple(tensors), records
        self._upload()

    def _check(self, records):
        rc = lib().normtest_list_check(records, self.plan.records, len(records), ANY_DTYPE)
        if rc == NT_ERR_SHARED_MEMORY:
            raise ValueError("two tensors of the list share memory (a tied weight is listed once)")
        if rc != NT_OK:
            raise NormtestError(rc, "normtest_list_check")

    def _upload(self):
        n = len(self.tensors)
        host = torch.frombuffer(bytearray(self._records), dtype=torch.uint8) if n else torch.zeros(8, dtype=torch.uint8)
        if self.table is None or self.table.numel() != host.numel():
            self.table = torch.empty(host.numel(), dtype=torch.uint8, device=self.plan.device)
            self.home = torch.cuda.current_stream(self.plan.device)   # whose memory it is
            self.stream = self.home.cuda_stream
            self.used = {}   # other streams that calls were made on since: {handle: stream}
        self.table.copy_(host)
        self.dtypes = {t.dtype for t in self.tensors}
        # the list as native code knows it, None: it does not; and for the native call path, which takes calls on the stream that table
        # and plan are memory of
        self.held = _fast and _fast.make_list(self.tensors, ctypes.addressof(self.plan.record), self.plan.record, self.table, self.stream) or None
        self.native = self.held if self.stream == self.plan.stream else None
        self._made_of = None if self.held else [_place(t) for t in self.tensors]
        self._held_by = _fast

    def refresh(self, tensors=None) -> "TensorList":
        """Reads the tensors' addresses again, or those of other tensors of the same shapes and layouts (gradients that were allocated
        anew).  Calls made before still take the old ones, on whatever stream they run, and calls made after it the new ones: the table is
        written in place, behind the calls that read it, and the host waits for that.  Replays of a graph that captured a call are not
        known here: refresh on the stream they are made on, or order them."""
        if tensors is not None:
            tensors = tuple(tensors)
            if len(tensors) != len(self.tensors):
                raise ValueError("the list has %d tensors, got %d" % (len(self.tensors), len(tensors)))
        else:
            tensors = self.tensors
        records = _like_records(tensors, self.plan)
        self._check(records)
        self.tensors, self._records = tensors, records
        here = torch.cuda.current_stream(self.plan.device)
        for handle, stream in {self.stream: self.home, **self.used}.items():
            if handle != here.cuda_stream:
                here.wait_stream(stream)
        self._upload()
        self.used.clear()
        return self

    def unchanged(self) -> bool:
        """Whether the tensors still are what the table on the device says: in a tensor of another type, shape or order at the same
        address, a call would read and write the old one."""
        if self.held:
            return bool(self._held_by.unchanged(self.held))
        return [_place(t) for t in self.tensors] == self._made_of

    def __len__(self):
        return len(self.tensors)


def _place(t: torch.Tensor):
    return t.data_ptr(), t.dtype, t.shape, t.stride()


def _check_tensor(t):
    if not isinstance(t, torch.Tensor) or t.layout != torch.strided:
        raise TypeError("a list holds dense torch tensors, got %s" % (t.layout if isinstance(t, torch.Tensor) else type(t).__name__))


def _check_listed(tensors, device):
    for t in tensors:
        _check_tensor(t)
        if t.dtype not in _LIST_DTYPES:
            raise TypeError("tensors of a list must be float32, bfloat16 or float16, got %s" % t.dtype)
        if t.device != device:
            raise ValueError("the tensors of a list must be on one device: got %s and %s" % (t.device, device))
    if device.type != "cuda":
        raise ValueError("lists need device tensors; there is no CPU path")


def _like_records(tensors, plan: TensorPlan):
    """Records of tensors that correspond, element by element in memory, to those the plan was made for."""
    _check_listed(tensors, plan.device)
    made = []
    for i, (t, (prows, pcols, order, group, shape)) in enumerate(zip(tensors, plan.layouts)):
        rows, cols, ld, own_order = _rows_of(t)
        same = (rows, cols) == (prows, pcols)
        if rows == 1 and cols == prows * pcols:   # dense: in the plan's rows
            rows, cols, ld, same = prows, pcols, pcols, True
        if not same or own_order != order or (order is not None and t.shape != shape):
            raise ValueError("tensor %d of the list does not lie in memory as the plan's: shape %s, strides %s against %s (make the plan "
                             "from the list that has row strides)" % (i, tuple(t.shape), t.stride(), tuple(shape)))
        made.append((t.data_ptr(), rows, cols, ld, _LIST_DTYPES[t.dtype], group))
    return (nt_tensor * len(made))(*made)


def make_tensor_list(tensors, groups=None, num_groups: Optional[int] = None, like: Optional[TensorList] = None, device=None) -> TensorList:
    """The tensors (parameters, gradients, moments: a sequence, on one device) as a list for the calls below.

    groups: a number from 0 on for every tensor, whose norms are then taken group by group (default: one group); num_groups: how many there
    are, where the last may have no tensor (default: up to the largest number).
    like: a list of corresponding tensors (same sizes; contiguous, or with the same dimensions in the same order in memory), whose plan and
    groups are shared: gradients, weights and moments of one model.  No two tensors share memory.  Tensors are dense, or rows of one stride (column slices); a plan
    made from dense tensors does not serve sliced ones.  device: of an empty sequence.
    Making a list copies its tables to the device and waits for that; make it once and keep it."""
    tensors = tuple(tensors)
    if like is not None:
        if groups is not None or num_groups is not None:
            raise ValueError("groups are those of the list given as like")
        if len(tensors) != len(like.tensors):
            raise ValueError("the lists differ in length: %d and %d tensors" % (len(tensors), len(like.tensors)))
        return TensorList(tensors, like.plan, _like_records(tensors, like.plan))
    if not tensors and device is None:
        raise ValueError("an empty list needs a device")
    if tensors:
        _check_tensor(tensors[0])
    device = tensors[0].device if tensors else torch.device(device)
    if device.type == "cuda" and device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    _check_listed(tensors, device)
    groups = [0] * len(tensors) if groups is None else [int(g) for g in groups]
    if len(groups) != len(tensors) or any(g < 0 for g in groups):
        raise ValueError("groups must hold a number from 0 on for every tensor")
    num_groups = max(groups, default=0) + 1 if num_groups is None else int(num_groups)
    if num_groups <= max(groups, default=0):
        raise ValueError("num_groups is %d, but a tensor is in group %d" % (num_groups, max(groups, default=0)))
    if num_groups >= 1 << 31:
        raise ValueError("a list has fewer than 2^31 groups, got %d" % num_groups)
    made, layouts = [], []
    for t, g in zip(tensors, groups):
        rows, cols, ld, order = _rows_of(t)
        made.append((t.data_ptr(), rows, cols, ld, _LIST_DTYPES[t.dtype], g))
        layouts.append((rows, cols, order, g, t.shape))
    records = (nt_tensor * len(made))(*made)
    return TensorList(tensors, TensorPlan(records, layouts, num_groups, device), records)


def make_norms(lst: TensorList) -> torch.Tensor:
    """Device memory for the norms of a list's groups (uint8[G * sizeof(nt_norm)])."""
    return torch.zeros(lst.plan.groups * NORM_BYTES, dtype=torch.uint8, device=lst.plan.device)


def _norms_for(lst: TensorList, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """make_norms for a call that writes every record.  On another stream than the current one they are that stream's memory: memory of the
    current stream could still be written by what runs there.  The caller may read them on either."""
    size, dev = lst.plan.groups * NORM_BYTES, lst.plan.device
    if _stream_handle(stream, dev) == _stream_handle(None, dev):
        return torch.empty(size, dtype=torch.uint8, device=dev)
    with torch.cuda.stream(stream):
        norms = torch.empty(size, dtype=torch.uint8, device=dev)
    norms.record_stream(torch.cuda.current_stream(dev))
    return norms


def norm_views(norms: torch.Tensor) -> dict:
    """Views of the records on the device, one entry per group: norm, factor (float32), flags (int32: status, clipped)."""
    words = NORM_BYTES // 4
    f, i = norms.view(torch.float32).view(-1, words), norms.view(torch.int32).view(-1, words)
    return {"norm": f[:, 4], "factor": f[:, 5], "flags": i[:, 6:8]}


def read_norms(norms: torch.Tensor):
    """Synchronising read of a device nt_norm array: a list of nt_norm."""
    host = norms.cpu().numpy().tobytes()
    return [nt_norm.from_buffer_copy(host, g * NORM_BYTES) for g in range(len(host) // NORM_BYTES)]


def _list_call(where: str, plan: TensorPlan, lists, norms, stream, fn, *args):
    """fn(plan, *args, stream) once the lists are known to be where their tables say, on their device."""
    for lst in lists:
        if not isinstance(lst, TensorList):
            raise TypeError("%s takes lists made by make_tensor_list, got %s" % (where, type(lst).__name__))
        if lst.plan is not plan:
            raise ValueError("%s: lists of different plans; make one `like` the other" % where)
        if not lst.unchanged():
            raise RuntimeError("%s: a tensor of a list has other memory, another type or shape than when the list was made; call its refresh()"
                               % where)
    for x in norms:
        if x is not None and (x.device != plan.device or not x.is_contiguous() or _nbytes(x) < plan.groups * NORM_BYTES):
            raise ValueError("norms must be the contiguous device memory of %d records on %s (make_norms)" % (plan.groups, plan.device))
    st = _stream_handle(stream, plan.device)
    rc = _call(plan.device, fn, ctypes.byref(plan.record), *args, st)
    if rc != NT_OK:
        raise NormtestError(rc, where)
    # memory of other streams stays until this one has used it
    others = [memory for memory, owner in [(plan.image, plan.stream), *[(lst.table, lst.stream) for lst in lists]] if owner != st]
    if others:
        stream = torch.cuda.current_stream(plan.device) if stream is None else stream
        for memory in others:
            memory.record_stream(stream)
        for lst in lists:
            if lst.stream != st:
                lst.used[st] = stream


def _native(lst):
    """What the native call path knows a list by: None for no list, False for what it does not take."""
    if lst is None:
        return None
    return (lst.native or False) if type(lst) is TensorList else False


def _first(where: str, lst) -> TensorPlan:
    if not isinstance(lst, TensorList):
        raise TypeError("%s takes lists made by make_tensor_list, got %s" % (where, type(lst).__name__))
    return lst.plan


def normtest_grad_norm(grads: TensorList, norms: Optional[torch.Tensor] = None, *, max_norm: float = 0.0, grad_scale: float = 1.0,
                       kind: int = NT_NORM_L2, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Enqueue the norms of the list's groups and their clipping factors for max_norm (0: none) on `stream` (default: torch's current
    stream).  Returns the device memory of the records (norms, or new): read_norms after a sync, norm_views without one."""
    if stream is None and norms is not None and type(grads) is TensorList:
        if _fast and _done(_fast.grad_norm(_lib.normtest_grad_norm_entry, grads.native, kind, max_norm, grad_scale, norms), "normtest_grad_norm"):
            return norms
    plan = _first("normtest_grad_norm", grads)
    if norms is None:
        norms = _norms_for(grads, stream)
    _list_call("normtest_grad_norm", plan, (grads,), (norms,), stream, lib().normtest_grad_norm, grads.table.data_ptr(), kind, float(max_norm),
               float(grad_scale), norms.data_ptr())
    return norms


def normtest_clip_grads(grads: TensorList, norms: torch.Tensor, *, out: Optional[TensorList] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> None:
    """Multiply the gradients by their groups' factors, in place or into the list `out` (of any types)."""
    if stream is None and type(grads) is TensorList:
        if _fast and _done(_fast.clip_grads(_lib.normtest_clip_grads_entry, grads.native, _native(out), norms), "normtest_clip_grads"):
            return
    plan = _first("normtest_clip_grads", grads)
    _list_call("normtest_clip_grads", plan, (grads,) if out is None else (grads, out), (norms,), stream, lib().normtest_clip_grads,
               grads.table.data_ptr(), None if out is None else out.table.data_ptr(), norms.data_ptr())


def normtest_clip_grad_norm(grads: TensorList, max_norm: float, norms: Optional[torch.Tensor] = None, *, grad_scale: float = 1.0,
                            kind: int = NT_NORM_L2, out: Optional[TensorList] = None,
                            stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Norms and clipping in one call: normtest_grad_norm, then normtest_clip_grads.  Returns the records."""
    norms = normtest_grad_norm(grads, norms, max_norm=max_norm, grad_scale=grad_scale, kind=kind, stream=stream)
    normtest_clip_grads(grads, norms, out=out, stream=stream)
    return norms


def normtest_accumulate(dst: TensorList, src: TensorList, *, beta: float = 1.0, scale: float = 1.0,
                        src_norms: Optional[torch.Tensor] = None, norms: Optional[torch.Tensor] = None, max_norm: float = 0.0,
                        grad_scale: float = 1.0, kind: int = NT_NORM_L2, stream: Optional[torch.cuda.Stream] = None) -> None:
    """dst <- beta dst + scale src, in fp32, rounded once to dst's types (beta 0: dst is not read).  src_norms: records whose factors
    multiply src too (every micro-batch clipped by itself).  norms: records that receive the norms of what is stored, as
    normtest_grad_norm(dst) with max_norm, grad_scale and kind would, from the same pass."""
    if stream is None and type(dst) is TensorList:
        if _fast and _done(_fast.accumulate(_lib.normtest_accumulate_entry, dst.native, _native(src), beta, scale, src_norms, kind, max_norm,
                                            grad_scale, norms), "normtest_accumulate"):
            return
    plan = _first("normtest_accumulate", dst)
    _list_call("normtest_accumulate", plan, (dst, src), (src_norms, norms), stream, lib().normtest_accumulate, dst.table.data_ptr(),
               src.table.data_ptr() if isinstance(src, TensorList) else None, float(beta), float(scale), _ptr(src_norms), kind, float(max_norm),
               float(grad_scale), _ptr(norms))


def normtest_adamw_tensors(grads: TensorList, w: TensorList, m: TensorList, v: TensorList, hyper: nt_hyper, *,
                           norms: Optional[torch.Tensor] = None, grad_scale: float = 1.0, copy: Optional[TensorList] = None,
                           skip_nonfinite: bool = False, stream: Optional[torch.cuda.Stream] = None) -> None:
    """AdamW on grad_scale * grads (* the factors of norms, which hold normtest_grad_norm's own grad_scale), in place on the float32
    lists w, m, v; copy: a list of any types that receives the new weights.  skip_nonfinite: tensors of a group whose norm is not finite
    are left alone."""
    where = "normtest_adamw_tensors"
    if stream is None and type(grads) is TensorList:
        if _fast and _done(_fast.adamw_tensors(_lib.normtest_adamw_tensors_entry, grads.native, _native(w), _native(m), _native(v), _native(copy),
                                               hyper, grad_scale, norms, NT_SKIP_NONFINITE if skip_nonfinite else 0), where):
            return
    plan = _first(where, grads)
    lists = (grads, w, m, v) if copy is None else (grads, w, m, v, copy)
    for lst in lists[1:4]:
        if isinstance(lst, TensorList) and not lst.dtypes <= {torch.float32}:
            raise ValueError("w, m, v must be lists of float32 tensors")
    tables = [lst.table.data_ptr() if isinstance(lst, TensorList) else None for lst in lists]
    _list_call(where, plan, lists, (norms,), stream, lib().normtest_adamw_tensors, *tables[:4], tables[4] if copy is not None else None,
               ctypes.byref(hyper), float(grad_scale), _ptr(norms), NT_SKIP_NONFINITE if skip_nonfinite else 0)


def normtest_clip_coef(gbar_sq: float, max_norm: float) -> float:
    return float(lib().normtest_clip_coef(gbar_sq, max_norm))


def normtest_resplit(b: int, J: int, accum_base: int, micro_max: int):
    """(micro_batch, accumulation_steps, global_batch) for a target global batch size b."""
    micro, accum, glob = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    rc = lib().normtest_resplit(b, J, accum_base, micro_max, ctypes.byref(micro), ctypes.byref(accum), ctypes.byref(glob))
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_resplit")
    return micro.value, accum.value, glob.value


def normtest_schedule_flags(step: int, test_interval: int, b_k: int, b_max: int, flags: int) -> int:
    return int(lib().normtest_schedule_flags(step, test_interval, b_k, b_max, flags))


def read_result(result: torch.Tensor) -> nt_result:
    """Synchronising read of the device nt_result."""
    host = result.cpu().numpy().tobytes()
    return nt_result.from_buffer_copy(host)


def normtest_combine(partials, J: int, hyper: nt_hyper) -> nt_result:
    arr = (nt_result * len(partials))(*partials)
    out = nt_result()
    rc = lib().normtest_combine(arr, len(partials), J, ctypes.byref(hyper), ctypes.byref(out))
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_combine")
    return out


def normtest_calib_copy(dst: torch.Tensor, src: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() < nbytes:
        raise ValueError("dst smaller than src")
    if stream is None:
        stream = torch.cuda.current_stream(src.device)
    with torch.cuda.device(src.device):
        rc = lib().normtest_calib_copy(_ptr(dst), _ptr(src), nbytes, ctypes.c_void_p(stream.cuda_stream))
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_calib_copy")


def calib_streams_bytes(coords: int, row_reads: int, reads: int, writes: int) -> int:
    """Scratch bytes normtest_calib_streams needs (the rule stated in the header)."""
    r2 = (coords * 2 + 255) // 256 * 256
    r4 = (coords * 4 + 255) // 256 * 256
    return row_reads * r2 + (reads + writes) * r4 + 16


def normtest_calib_streams(buf: torch.Tensor, coords: int, row_reads: int, reads: int, writes: int, rmw: bool = False,
                           launch_coords: int = 0, stream: Optional[torch.cuda.Stream] = None) -> None:
    if stream is None:
        stream = torch.cuda.current_stream(buf.device)
    with torch.cuda.device(buf.device):
        rc = lib().normtest_calib_streams(_ptr(buf), buf.numel() * buf.element_size(), coords, row_reads, reads, writes,
                                          1 if rmw else 0, launch_coords, ctypes.c_void_p(stream.cuda_stream))
    if rc != NT_OK:
        raise NormtestError(rc, "normtest_calib_streams")
