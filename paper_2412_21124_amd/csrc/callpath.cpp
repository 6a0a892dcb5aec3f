// Argument marshalling of the step entry points for the calls a training loop makes: plain tensors on the current device, with the
// workspace and the result handed over.  A short step is bound by the host, and of its time in Python most went into looking at the
// tensors.  Python / here, us a call, back to back: fused step of 4 fp32 rows, d = 1000 7.2 / 4.8 (the kernel's time), in buffers of their
// own 10.8 / 4.8, clipped 11.0 / 7.6; 32 rows in buffers of their own 21 / 7.8, 512 rows 190 / 55.
// Every function returns the library's code, or None for a call that it does not take, before anything is enqueued: the caller then goes
// through the checks in Python, which also word the exceptions.  Whatever is taken here passes those checks.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <memory>
#include <vector>

#include "normtest.h"

namespace {

struct Refused {};   // thrown where Python has to look

PyObject* raw_stream = nullptr;   // torch._C._cuda_getCurrentRawStream
PyObject* hyper_type = nullptr;
PyObject* shard_type = nullptr;
PyObject* parameter_type = nullptr;

// The tensor behind an argument: torch.Tensor itself or a Parameter, no other subclass, which may be anything.
const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o) && (PyObject*)Py_TYPE(o) != parameter_type) throw Refused();
  return THPVariable_Unpack(o);
}

struct Where {
  c10::Device device = c10::Device(c10::DeviceType::CPU);
  int64_t d = 0;
};

// The current device's tensors only: the library launches there.
void check_device(const at::Tensor& t) {
  if (!t.is_cuda() || c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice() != t.device()) throw Refused();
}

int dtype_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return NT_F32;
  if (t.scalar_type() == at::kBFloat16) return NT_BF16;
  throw Refused();
}

// w, m, v, the mean: contiguous float32 vectors of at least d elements beside the gradients, or None where that may be.
float* vector_of(PyObject* o, const Where& at_, bool required) {
  if (o == Py_None && !required) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != at::kFloat || t.device() != at_.device || !t.is_contiguous() || t.numel() < at_.d) throw Refused();
  return (float*)t.data_ptr();
}

int64_t integer(PyObject* o) {
  if (!PyLong_CheckExact(o)) throw Refused();
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw Refused();
  return x;
}

// Address of a ctypes structure; the argument holds it while the call runs.
template <class T>
const T* structure(PyObject* o, PyObject* type) {
  if ((PyObject*)Py_TYPE(o) != type) throw Refused();
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Refused();
  const T* p = view.len == (Py_ssize_t)sizeof(T) ? (const T*)view.buf : nullptr;
  PyBuffer_Release(&view);
  if (!p) throw Refused();
  return p;
}
const nt_shard_info* shard_of(PyObject* o) { return o == Py_None ? nullptr : structure<nt_shard_info>(o, shard_type); }

void* stream_of(const c10::Device& device) {
  PyObject* index = PyLong_FromLong(device.index());
  PyObject* handle = index ? PyObject_CallOneArg(raw_stream, index) : nullptr;
  Py_XDECREF(index);
  if (!handle) throw Refused();
  void* st = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  if (!st && PyErr_Occurred()) throw Refused();
  return st;
}

template <class F>
F* entry(PyObject* o) {
  void* p = PyLong_Check(o) ? PyLong_AsVoidPtr(o) : nullptr;
  if (!p) throw Refused();
  return (F*)p;
}

struct Bytes {
  void* data;
  size_t size;
};
Bytes bytes_of(PyObject* o) {
  const at::Tensor& t = tensor(o);
  return {t.data_ptr(), (size_t)(t.numel() * t.element_size())};
}

// (J, ld) tensor whose rows are the gradients; d: the argument, None for all columns.
struct Matrix {
  const void* data;
  int64_t J, ld;
  int dtype;
  Where at_;
};
Matrix matrix_of(PyObject* grads, PyObject* d) {
  const at::Tensor& g = tensor(grads);
  check_device(g);
  if (g.dim() != 2 || (g.size(1) > 1 && g.stride(1) != 1)) throw Refused();
  Matrix m;
  m.J = g.size(0);
  m.ld = m.J > 1 ? g.stride(0) : g.size(1);
  m.dtype = dtype_of(g);
  m.data = g.data_ptr();
  m.at_ = {g.device(), d == Py_None ? g.size(1) : integer(d)};
  return m;
}

// CALL with the interpreter released, as ctypes does.
template <class CALL>
PyObject* enqueue(CALL call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

template <class BODY>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, BODY body) {
  if (given != wanted) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return body();
  } catch (const Refused&) {
  } catch (const std::exception&) {
  }
  PyErr_Clear();
  Py_RETURN_NONE;
}

// step(entry, grads, w, m, v, hyper, d, shard, gbar_out, workspace, result)
PyObject* step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&] {
    auto* f = entry<decltype(normtest_step)>(a[0]);
    const Matrix g = matrix_of(a[1], a[6]);
    float *w = vector_of(a[2], g.at_, false), *m = vector_of(a[3], g.at_, false), *v = vector_of(a[4], g.at_, false);
    const nt_hyper* hyper = structure<nt_hyper>(a[5], hyper_type);
    const nt_shard_info* shard = shard_of(a[7]);
    float* gbar = vector_of(a[8], g.at_, false);
    const Bytes ws = bytes_of(a[9]);
    nt_result* res = (nt_result*)bytes_of(a[10]).data;
    void* st = stream_of(g.at_.device);
    return enqueue([&] { return f(g.data, (nt_dtype)g.dtype, g.J, g.at_.d, g.ld, w, m, v, gbar, hyper, shard, ws.data, ws.size, res, st); });
  });
}

// step_clipped(entry, grads, w, m, v, gbar_buf, max_norm, hyper, d, shard, workspace, result)
PyObject* step_clipped(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&] {
    auto* f = entry<decltype(normtest_step_clipped)>(a[0]);
    const Matrix g = matrix_of(a[1], a[8]);
    float *w = vector_of(a[2], g.at_, true), *m = vector_of(a[3], g.at_, true), *v = vector_of(a[4], g.at_, true);
    float* gbar = vector_of(a[5], g.at_, true);
    if (!PyFloat_CheckExact(a[6])) throw Refused();
    const double max_norm = PyFloat_AS_DOUBLE(a[6]);
    const nt_hyper* hyper = structure<nt_hyper>(a[7], hyper_type);
    const nt_shard_info* shard = shard_of(a[9]);
    const Bytes ws = bytes_of(a[10]);
    nt_result* res = (nt_result*)bytes_of(a[11]).data;
    void* st = stream_of(g.at_.device);
    return enqueue([&] {
      return f(g.data, (nt_dtype)g.dtype, g.J, g.at_.d, g.ld, w, m, v, gbar, max_norm, hyper, shard, ws.data, ws.size, res, st);
    });
  });
}

// step_rows(entry, rows, w, m, v, hyper, d, table, shard, gbar_out, workspace, result); rows: a list or tuple
PyObject* step_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&] {
    auto* f = entry<decltype(normtest_step_rows)>(a[0]);
    if (!PyList_CheckExact(a[1]) && !PyTuple_CheckExact(a[1])) throw Refused();
    const Py_ssize_t J = PySequence_Fast_GET_SIZE(a[1]);
    if (J < 1) throw Refused();
    PyObject** rows = PySequence_Fast_ITEMS(a[1]);
    const at::Tensor& first = tensor(rows[0]);
    check_device(first);
    const int dtype = dtype_of(first);
    int64_t shortest = INT64_MAX;
    for (Py_ssize_t j = 0; j < J; ++j) {
      const at::Tensor& r = tensor(rows[j]);
      if (r.scalar_type() != first.scalar_type() || r.device() != first.device() || r.dim() != 1 || !r.is_contiguous()) throw Refused();
      if (r.numel() < shortest) shortest = r.numel();
    }
    const Where at_ = {first.device(), a[6] == Py_None ? shortest : integer(a[6])};
    if (shortest < at_.d) throw Refused();
    float *w = vector_of(a[2], at_, false), *m = vector_of(a[3], at_, false), *v = vector_of(a[4], at_, false);
    const nt_hyper* hyper = structure<nt_hyper>(a[5], hyper_type);
    at::Tensor table = tensor(a[7]);
    if (!table.is_cuda()) throw Refused();
    const nt_shard_info* shard = shard_of(a[8]);
    float* gbar = vector_of(a[9], at_, false);
    const Bytes ws = bytes_of(a[10]);
    nt_result* res = (nt_result*)bytes_of(a[11]).data;
    void* st = stream_of(at_.device);
    const void* const* entries = (const void* const*)table.data_ptr();
    // the kernels read the table: its memory stays until they have
    table.record_stream(c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getStream(at_.device));
    return enqueue([&] { return f(entries, (nt_dtype)dtype, J, at_.d, w, m, v, gbar, hyper, shard, ws.data, ws.size, res, st); });
  });
}

// adamw_gbar(entry, gbar, w, m, v, hyper, grad_scale, d, result)
PyObject* adamw_gbar(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    auto* f = entry<decltype(normtest_adamw_gbar)>(a[0]);
    const at::Tensor& g = tensor(a[1]);
    check_device(g);
    const Where at_ = {g.device(), a[7] == Py_None ? g.numel() : integer(a[7])};
    float *gbar = vector_of(a[1], at_, true), *w = vector_of(a[2], at_, true), *m = vector_of(a[3], at_, true);
    float* v = vector_of(a[4], at_, true);
    const nt_hyper* hyper = structure<nt_hyper>(a[5], hyper_type);
    if (!PyFloat_CheckExact(a[6])) throw Refused();
    const double scale = PyFloat_AS_DOUBLE(a[6]);
    const nt_result* res = a[8] == Py_None ? nullptr : (const nt_result*)bytes_of(a[8]).data;
    void* st = stream_of(at_.device);
    return enqueue([&] { return f(gbar, at_.d, w, m, v, hyper, scale, res, st); });
  });
}

// layer_stats(entry, grads, layer_offsets, workspace, need, d, layers); grads: the (J, ld) tensor; need(gdtype, J, d, flags): bytes of the
// workspace the step needed, an entry of the library too
PyObject* layer_stats(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    auto* f = entry<decltype(normtest_layer_stats)>(a[0]);
    const Matrix g = matrix_of(a[1], a[5]);
    const at::Tensor& offsets = tensor(a[2]);
    if (offsets.scalar_type() != at::kLong || offsets.device() != g.at_.device || offsets.dim() != 1 || !offsets.is_contiguous() ||
        offsets.numel() < 2 || offsets.numel() > (1 << 24))
      throw Refused();
    const int32_t L = (int32_t)offsets.numel() - 1;
    if (tensor(a[3]).device() != g.at_.device) throw Refused();
    const Bytes ws = bytes_of(a[3]), layers = bytes_of(a[6]);
    if (ws.size < entry<decltype(normtest_workspace_bytes_for)>(a[4])((nt_dtype)g.dtype, g.J, g.at_.d, NT_DO_STATS)) throw Refused();
    if (layers.size < (size_t)L * sizeof(nt_layer_stats)) throw Refused();
    void* st = stream_of(g.at_.device);
    const int64_t* off = (const int64_t*)offsets.data_ptr();
    return enqueue([&] { return f(g.data, 0, (nt_dtype)g.dtype, g.J, g.at_.d, g.ld, off, L, ws.data, (nt_layer_stats*)layers.data, st); });
  });
}

// ---- lists of tensors ----
// A list as the binding made it: its tensors, what they were when its table on the device was written, and its plan.
// Of a tensor: address, type and number of dimensions, sizes, strides; in one array, as every call reads through it (5 lists of 300
// tensors: 6 us of a call's 10).
struct List {
  std::vector<at::Tensor> tensors;
  std::vector<int64_t> were;
  const nt_plan* plan;
  const nt_tensor* table;
  c10::Device device = c10::Device(c10::DeviceType::CPU);
  void* stream;      // that the tables were made on: another one has to hold their memory, which is left to Python
  bool all_f32;
  PyObject* owner;   // of the plan's record
};
int64_t kind_of(const at::Tensor& t) { return (int64_t)t.scalar_type() << 32 | t.dim(); }
const char list_name[] = "normtest.list";
void list_free(PyObject* capsule) {
  List* l = (List*)PyCapsule_GetPointer(capsule, list_name);
  if (!l) return;
  Py_XDECREF(l->owner);
  delete l;
}
// make_list(tensors, plan's address, its owner, table, stream's handle); tensors: a tuple
PyObject* make_list(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    if (!PyTuple_CheckExact(a[0])) throw Refused();
    std::unique_ptr<List> l(new List());
    l->all_f32 = true;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(a[0]); ++i) {
      l->tensors.push_back(tensor(PyTuple_GET_ITEM(a[0], i)));
      const at::Tensor& t = l->tensors.back();
      l->were.insert(l->were.end(), {(int64_t)(intptr_t)t.data_ptr(), kind_of(t)});
      l->were.insert(l->were.end(), t.sizes().begin(), t.sizes().end());
      l->were.insert(l->were.end(), t.strides().begin(), t.strides().end());
      l->all_f32 = l->all_f32 && l->tensors.back().scalar_type() == at::kFloat;
    }
    l->plan = entry<const nt_plan>(a[1]);
    const at::Tensor& table = tensor(a[3]);
    l->table = (const nt_tensor*)table.data_ptr();
    l->device = table.device();
    l->stream = PyLong_AsVoidPtr(a[4]);
    if (!l->stream && PyErr_Occurred()) throw Refused();
    PyObject* capsule = PyCapsule_New(l.get(), list_name, list_free);
    if (!capsule) throw Refused();
    Py_INCREF(a[2]);
    l->owner = a[2];
    l.release();
    return capsule;
  });
}
const List* held(PyObject* o) {
  if (!PyCapsule_IsValid(o, list_name)) throw Refused();
  return (const List*)PyCapsule_GetPointer(o, list_name);
}
bool same(const List& l) {
  const int64_t* was = l.were.data();
  for (const at::Tensor& t : l.tensors) {
    if ((int64_t)(intptr_t)t.data_ptr() != was[0] || kind_of(t) != was[1]) return false;
    was += 2;
    for (const auto& now : {t.sizes(), t.strides()})
      for (const int64_t x : now)
        if (x != *was++) return false;
  }
  return true;
}
// The list behind a capsule, its tensors what its table says; `first`: the list whose plan it has to share.
const List* list_of(PyObject* o, const List* first) {
  const List* l = held(o);
  if ((first && l->plan != first->plan) || !same(*l)) throw Refused();
  return l;
}
// unchanged(list): whether its tensors are what its table says
PyObject* unchanged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 1, [&] { return PyBool_FromLong(same(*held(a[0]))); });
}
const List* list_or_none(PyObject* o, const List* first) { return o == Py_None ? nullptr : list_of(o, first); }
nt_norm* norms_of(PyObject* o, const List& l, bool required) {
  if (o == Py_None && !required) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.device() != l.device || !t.is_contiguous() || (size_t)(t.numel() * t.element_size()) < (size_t)l.plan->groups * sizeof(nt_norm))
    throw Refused();
  return (nt_norm*)t.data_ptr();
}
// The current stream, if it is the one the tables were made on and its device the current one.
void* stream_of_list(const List& l) {
  if (c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice() != l.device) throw Refused();
  void* st = stream_of(l.device);
  if (st != l.stream) throw Refused();
  return st;
}
double number(PyObject* o) {
  if (!PyFloat_CheckExact(o)) throw Refused();
  return PyFloat_AS_DOUBLE(o);
}
int32_t small(PyObject* o) {
  const int64_t x = integer(o);
  if (x < 0 || x > 1 << 16) throw Refused();
  return (int32_t)x;
}

// grad_norm(entry, grads, kind, max_norm, grad_scale, norms)
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&] {
    auto* f = entry<decltype(normtest_grad_norm)>(a[0]);
    const List& g = *list_of(a[1], nullptr);
    const int32_t kind = small(a[2]);
    const double max_norm = number(a[3]), scale = number(a[4]);
    nt_norm* norms = norms_of(a[5], g, true);
    void* st = stream_of_list(g);
    return enqueue([&] { return f(g.plan, g.table, kind, max_norm, scale, norms, st); });
  });
}

// clip_grads(entry, grads, out, norms)
PyObject* clip_grads(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 4, [&] {
    auto* f = entry<decltype(normtest_clip_grads)>(a[0]);
    const List& g = *list_of(a[1], nullptr);
    const List* out = list_or_none(a[2], &g);
    const nt_norm* norms = norms_of(a[3], g, true);
    void* st = stream_of_list(g);
    return enqueue([&] { return f(g.plan, g.table, out ? out->table : nullptr, norms, st); });
  });
}

// accumulate(entry, dst, src, beta, scale, src_norms, kind, max_norm, grad_scale, norms)
PyObject* accumulate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    auto* f = entry<decltype(normtest_accumulate)>(a[0]);
    const List& dst = *list_of(a[1], nullptr);
    const List& src = *list_of(a[2], &dst);
    const double beta = number(a[3]), scale = number(a[4]), max_norm = number(a[7]), grad_scale = number(a[8]);
    const nt_norm* src_norms = norms_of(a[5], dst, false);
    const int32_t kind = small(a[6]);
    nt_norm* norms = norms_of(a[9], dst, false);
    void* st = stream_of_list(dst);
    return enqueue([&] { return f(dst.plan, dst.table, src.table, beta, scale, src_norms, kind, max_norm, grad_scale, norms, st); });
  });
}

// adamw_tensors(entry, grads, w, m, v, copy, hyper, grad_scale, norms, flags)
PyObject* adamw_tensors(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    auto* f = entry<decltype(normtest_adamw_tensors)>(a[0]);
    const List& g = *list_of(a[1], nullptr);
    const List &w = *list_of(a[2], &g), &m = *list_of(a[3], &g), &v = *list_of(a[4], &g);
    if (!w.all_f32 || !m.all_f32 || !v.all_f32) throw Refused();
    const List* copy = list_or_none(a[5], &g);
    const nt_hyper* hyper = structure<nt_hyper>(a[6], hyper_type);
    const double scale = number(a[7]);
    const nt_norm* norms = norms_of(a[8], g, false);
    const int32_t flags = small(a[9]);
    void* st = stream_of_list(g);
    return enqueue([&] { return f(g.plan, g.table, w.table, m.table, v.table, copy ? copy->table : nullptr, hyper, scale, norms, (uint32_t)flags, st); });
  });
}

// init(nt_hyper, nt_shard_info, torch.nn.Parameter, torch._C._cuda_getCurrentRawStream)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 4, [&]() -> PyObject* {
    PyObject** to[4] = {&hyper_type, &shard_type, &parameter_type, &raw_stream};
    for (int k = 0; k < 4; ++k) {
      Py_INCREF(a[k]);
      Py_XSETREF(*to[k], a[k]);
    }
    Py_RETURN_NONE;
  });
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(init),       FAST(step),        FAST(step_clipped), FAST(step_rows),
                         FAST(adamw_gbar), FAST(layer_stats), FAST(make_list), FAST(unchanged), FAST(grad_norm), FAST(clip_grads), FAST(accumulate),
                         FAST(adamw_tensors), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_callpath", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__callpath() { return PyModule_Create(&module); }
