// What the Python binding does on every call, in native code: checks and descriptors of torch tensors, the allocator callback, and
// the call itself.  On small frames a step is bound by the host: 19 us of the 43 that a frame of 2000 nodes takes passed
// in the interpreter between the GPU's work (tensors asked for type, shape, strides and address one attribute at a time).
//
// A fast path only: whatever is not a plain valid argument (other types, subclasses, wrong shapes, tensors without memory of their
// own, another current device) makes a function return None before anything has happened, and the binding goes the long way, which
// says what is wrong.  The library's functions come by address, so nothing here depends on which build of it is loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/Allocator.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <mutex>
#include <new>
#include <unordered_map>

#include "pipad.h"

namespace {

// ---- the memory of a frame ----------------------------------------------------------------------
// Pieces of torch's caching allocator by address; handed back all at once, or one by one.  Calls that use a frame at the same time
// may ask for memory at the same time, without the interpreter's lock.
struct Pieces {
  std::mutex mutex;
  std::unordered_map<void *, c10::DataPtr> by_address;
};
struct Buffers {
  PyObject_HEAD
  Pieces *pieces;
};

// pipad_alloc_fn; ctx: Pieces.  The current device's memory, in the order of its current stream (as torch.empty).
void *allocate(size_t bytes, void *ctx) noexcept {
  try {
    c10::DataPtr p = c10::GetAllocator(c10::DeviceType::CUDA)->allocate(std::max<size_t>(bytes, 256));
    void *const at = p.get();
    if (!at) return nullptr;
    Pieces &own = *static_cast<Pieces *>(ctx);
    std::lock_guard<std::mutex> lock(own.mutex);
    own.by_address.emplace(at, std::move(p));
    return at;
  } catch (...) {  // out of memory -> PIPAD_ERR_ALLOC
    return nullptr;
  }
}

PyObject *buffers_new(PyTypeObject *type, PyObject *, PyObject *) {
  Buffers *self = reinterpret_cast<Buffers *>(type->tp_alloc(type, 0));
  if (!self) return nullptr;
  self->pieces = new (std::nothrow) Pieces;
  if (!self->pieces) {
    Py_DECREF(self);
    return PyErr_NoMemory();
  }
  return reinterpret_cast<PyObject *>(self);
}
void buffers_dealloc(PyObject *o) {
  delete reinterpret_cast<Buffers *>(o)->pieces;
  Py_TYPE(o)->tp_free(o);
}
PyObject *buffers_clear(PyObject *o, PyObject *) {
  Pieces &own = *reinterpret_cast<Buffers *>(o)->pieces;
  decltype(own.by_address) gone;
  {
    std::lock_guard<std::mutex> lock(own.mutex);
    gone.swap(own.by_address);
  }
  Py_RETURN_NONE;
}
PyObject *buffers_pop(PyObject *o, PyObject *const *args, Py_ssize_t nargs) {  // as a dict's, with a default of None
  if (nargs < 1) return PyErr_Format(PyExc_TypeError, "pop(address, default)");
  void *const at = PyLong_AsVoidPtr(args[0]);
  if (!at && PyErr_Occurred()) return nullptr;
  Pieces &own = *reinterpret_cast<Buffers *>(o)->pieces;
  c10::DataPtr gone;
  {
    std::lock_guard<std::mutex> lock(own.mutex);
    auto it = own.by_address.find(at);
    if (it != own.by_address.end()) {
      gone = std::move(it->second);
      own.by_address.erase(it);
    }
  }
  Py_RETURN_NONE;
}
Py_ssize_t buffers_len(PyObject *o) {
  Pieces &own = *reinterpret_cast<Buffers *>(o)->pieces;
  std::lock_guard<std::mutex> lock(own.mutex);
  return (Py_ssize_t)own.by_address.size();
}
PyObject *buffers_context(PyObject *o, PyObject *) { return PyLong_FromVoidPtr(reinterpret_cast<Buffers *>(o)->pieces); }

PyMethodDef buffers_methods[] = {
    {"clear", buffers_clear, METH_NOARGS, "Hands everything back."},
    {"pop", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(buffers_pop)), METH_FASTCALL, "Hands back the piece at an address."},
    {"context", buffers_context, METH_NOARGS, "What the allocator callback is to be called with."},
    {nullptr, nullptr, 0, nullptr}};
PySequenceMethods buffers_sequence = [] {
  PySequenceMethods m{};
  m.sq_length = buffers_len;
  return m;
}();
PyTypeObject buffers_type = [] {
  PyTypeObject t{PyVarObject_HEAD_INIT(nullptr, 0)};
  t.tp_name = "paper_2301_00391_amd._host.Buffers";
  t.tp_basicsize = sizeof(Buffers);
  t.tp_flags = Py_TPFLAGS_DEFAULT;
  t.tp_doc = "Memory of a frame, from torch's allocator.";
  t.tp_new = buffers_new;
  t.tp_dealloc = buffers_dealloc;
  t.tp_methods = buffers_methods;
  t.tp_as_sequence = &buffers_sequence;
  return t;
}();

// ---- arguments ----------------------------------------------------------------------------------
// A torch.Tensor or Parameter as such (not a subclass, whose attributes may say something else) on a GPU, with strides.
inline const at::Tensor *plain_tensor(PyObject *o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(o);
  return t.defined() && t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}

struct Items {
  PyObject *const *at;
  Py_ssize_t count;
};
inline bool items(PyObject *o, Items *out) {  // of a list or tuple
  if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) return false;
  out->at = PySequence_Fast_ITEMS(o);
  out->count = PySequence_Fast_GET_SIZE(o);
  return true;
}

struct Matrices {
  float *ptr[PIPAD_MAX_K];
  int64_t ld, F;
};
// One [n, F] float32 matrix with contiguous columns: pointer, row stride.
inline bool matrix(PyObject *o, int64_t n, float **ptr, int64_t *ld, int64_t *F) {
  const at::Tensor *t = plain_tensor(o);
  if (!t || t->scalar_type() != at::kFloat || t->dim() != 2 || t->size(0) != n) return false;
  *F = t->size(1);
  if (*F > 1 && t->stride(1) != 1) return false;
  *ld = n > 1 ? t->stride(0) : std::max<int64_t>(t->stride(0), *F);
  *ptr = static_cast<float *>(t->data_ptr());
  return true;
}
// k [n, F] matrices that share their row stride, or one [n, k, F] tensor.
inline bool operand(PyObject *o, int64_t n, int64_t k, Matrices *m) {
  Items list;
  if (items(o, &list)) {
    if (list.count != k || k < 1) return false;
    for (Py_ssize_t t = 0; t < k; ++t) {
      int64_t ld, F;
      if (!matrix(list.at[t], n, &m->ptr[t], &ld, &F)) return false;
      if (t == 0) {
        m->ld = ld;
        m->F = F;
      } else if (F != m->F || (n > 1 && ld != m->ld)) {
        return false;
      }
    }
    return true;
  }
  const at::Tensor *x = plain_tensor(o);
  if (!x || x->scalar_type() != at::kFloat || x->dim() != 3 || x->size(0) != n || x->size(1) != k) return false;
  m->F = x->size(2);
  if (m->F > 1 && x->stride(2) != 1) return false;
  m->ld = n > 1 ? x->stride(0) : std::max<int64_t>(x->stride(0), m->F);
  float *const first = static_cast<float *>(x->data_ptr());
  for (int64_t t = 0; t < k; ++t) m->ptr[t] = first + x->stride(1) * t;
  return true;
}

// Every function: (address of the library's function, ...).  C++ exceptions (tensors without memory, sizes that are
// symbols) are a None as well: the long way meets them again.
template <class Body>
PyObject *guarded(Body body) {
  try {
    return body();
  } catch (...) {
    Py_RETURN_NONE;
  }
}
template <class Fn>
inline Fn address(PyObject *o) { return reinterpret_cast<Fn>(PyLong_AsVoidPtr(o)); }

// The library runs without the interpreter's lock, as under ctypes.
template <class Call>
inline int unlocked(Call call) {
  struct Unlock {
    PyThreadState *const state = PyEval_SaveThread();
    ~Unlock() { PyEval_RestoreThread(state); }
  } unlock;
  return call();
}

// build(address, snapshots, device index, flags, buffers, stream) -> (status, handle, n)
PyObject *build(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 6) return PyErr_Format(PyExc_TypeError, "build: six arguments");
  return guarded([&]() -> PyObject * {
    using Fn = decltype(&pipad_frame_build_overlap);
    Items snaps;
    const long index = PyLong_AsLong(args[2]);
    if (!items(args[1], &snaps) || snaps.count < 1 || snaps.count > PIPAD_MAX_K || Py_TYPE(args[4]) != &buffers_type) Py_RETURN_NONE;
    pipad_csr_t csr[PIPAD_MAX_K];
    for (Py_ssize_t t = 0; t < snaps.count; ++t) {
      Items pair;
      if (!items(snaps.at[t], &pair) || pair.count != 2) Py_RETURN_NONE;
      const at::Tensor *part[2];
      for (int q = 0; q < 2; ++q) {
        part[q] = plain_tensor(pair.at[q]);
        if (!part[q] || part[q]->scalar_type() != at::kInt || part[q]->get_device() != index || !part[q]->is_contiguous()) Py_RETURN_NONE;
      }
      const int64_t n = part[0]->numel() - 1, nnz = part[1]->numel();
      if (n < 0 || n > INT32_MAX || nnz > INT32_MAX) Py_RETURN_NONE;
      csr[t].n = (int32_t)n;
      csr[t].nnz = (int32_t)nnz;
      csr[t].rowptr = static_cast<const int32_t *>(part[0]->data_ptr());
      csr[t].colidx = nnz ? static_cast<const int32_t *>(part[1]->data_ptr()) : nullptr;
    }
    const Fn fn = address<Fn>(args[0]);
    const uint32_t flags = (uint32_t)PyLong_AsUnsignedLong(args[3]);
    Pieces *const own = reinterpret_cast<Buffers *>(args[4])->pieces;
    void *const stream = PyLong_AsVoidPtr(args[5]);
    if (PyErr_Occurred()) return nullptr;
    pipad_frame_t *frame = nullptr;
    const int32_t n = csr[0].n, k = (int32_t)snaps.count;
    const int status = unlocked([&] { return fn(n, k, csr, flags, allocate, own, stream, &frame); });
    return Py_BuildValue("iNi", status, PyLong_FromVoidPtr(frame), (int)n);
  });
}

// transpose(address, frame, buffers, stream) -> (status, handle)
PyObject *transpose(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 4) return PyErr_Format(PyExc_TypeError, "transpose: four arguments");
  return guarded([&]() -> PyObject * {
    using Fn = decltype(&pipad_frame_transpose);
    if (!PyLong_CheckExact(args[1]) || Py_TYPE(args[2]) != &buffers_type) Py_RETURN_NONE;
    const Fn fn = address<Fn>(args[0]);
    const pipad_frame_t *const frame = static_cast<const pipad_frame_t *>(PyLong_AsVoidPtr(args[1]));
    Pieces *const own = reinterpret_cast<Buffers *>(args[2])->pieces;
    void *const stream = PyLong_AsVoidPtr(args[3]);
    if (PyErr_Occurred()) return nullptr;
    pipad_frame_t *out = nullptr;
    const int status = unlocked([&] { return fn(frame, allocate, own, stream, &out); });
    return Py_BuildValue("iN", status, PyLong_FromVoidPtr(out));
  });
}

// aggregate(address, frame, n, k, X, Y, stream) -> status
PyObject *aggregate(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 7) return PyErr_Format(PyExc_TypeError, "aggregate: seven arguments");
  return guarded([&]() -> PyObject * {
    using Fn = decltype(&pipad_frame_aggregate);
    const int64_t n = PyLong_AsLongLong(args[2]), k = PyLong_AsLongLong(args[3]);
    const Fn fn = address<Fn>(args[0]);
    if (!PyLong_CheckExact(args[1])) Py_RETURN_NONE;  // (a frame that was closed)
    pipad_frame_t *const frame = static_cast<pipad_frame_t *>(PyLong_AsVoidPtr(args[1]));
    void *const stream = PyLong_AsVoidPtr(args[6]);
    if (PyErr_Occurred()) return nullptr;
    Matrices x, y;
    if (k < 1 || k > PIPAD_MAX_K || !operand(args[4], n, k, &x) || !operand(args[5], n, k, &y) || x.F != y.F || x.F > INT32_MAX) Py_RETURN_NONE;
    const int status = unlocked([&] { return fn(frame, (int32_t)x.F, x.ptr, x.ld, y.ptr, y.ld, stream); });
    return PyLong_FromLong(status);
  });
}

// subset(address, frame, n, k, snapshots, X, Y, stream) -> status
PyObject *subset(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 8) return PyErr_Format(PyExc_TypeError, "subset: eight arguments");
  return guarded([&]() -> PyObject * {
    using Fn = decltype(&pipad_frame_aggregate_subset);
    const int64_t n = PyLong_AsLongLong(args[2]), k = PyLong_AsLongLong(args[3]);
    const Fn fn = address<Fn>(args[0]);
    if (!PyLong_CheckExact(args[1])) Py_RETURN_NONE;  // (a frame that was closed)
    pipad_frame_t *const frame = static_cast<pipad_frame_t *>(PyLong_AsVoidPtr(args[1]));
    void *const stream = PyLong_AsVoidPtr(args[7]);
    if (PyErr_Occurred()) return nullptr;
    Items sel, xs, ys;
    if (k < 1 || k > PIPAD_MAX_K || !items(args[4], &sel) || !items(args[5], &xs) || !items(args[6], &ys) || sel.count < 1 ||
        sel.count > PIPAD_MAX_K || xs.count != k || ys.count != k)
      Py_RETURN_NONE;
    int32_t list[PIPAD_MAX_K];
    float *x[PIPAD_MAX_K] = {}, *y[PIPAD_MAX_K] = {};
    int64_t F = 0, ldx = 0, ldy = 0;
    for (Py_ssize_t q = 0; q < sel.count; ++q) {
      if (!PyLong_CheckExact(sel.at[q])) Py_RETURN_NONE;
      const long t = PyLong_AsLong(sel.at[q]);
      if (t < 0 || t >= k) {
        PyErr_Clear();
        Py_RETURN_NONE;
      }
      int64_t lx, ly, fx, fy;
      if (!matrix(xs.at[t], n, &x[t], &lx, &fx) || !matrix(ys.at[t], n, &y[t], &ly, &fy)) Py_RETURN_NONE;
      if (q == 0) {
        F = fx;
        ldx = lx;
        ldy = ly;
      }
      if (fx != F || fy != F || (n > 1 && (lx != ldx || ly != ldy)) || F > INT32_MAX) Py_RETURN_NONE;
      list[q] = (int32_t)t;
    }
    const int status =
        unlocked([&] { return fn(frame, (int32_t)sel.count, list, (int32_t)F, x, ldx, y, ldy, stream); });
    return PyLong_FromLong(status);
  });
}

// update(address, frame, n, k, X, W, bias or None, A or None, H, stream) -> status
PyObject *update(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 10) return PyErr_Format(PyExc_TypeError, "update: ten arguments");
  return guarded([&]() -> PyObject * {
    using Fn = decltype(&pipad_frame_aggregate_update);
    const int64_t n = PyLong_AsLongLong(args[2]), k = PyLong_AsLongLong(args[3]);
    const Fn fn = address<Fn>(args[0]);
    if (!PyLong_CheckExact(args[1])) Py_RETURN_NONE;  // (a frame that was closed)
    pipad_frame_t *const frame = static_cast<pipad_frame_t *>(PyLong_AsVoidPtr(args[1]));
    void *const stream = PyLong_AsVoidPtr(args[9]);
    if (PyErr_Occurred()) return nullptr;
    Matrices x, a, h;
    if (k < 1 || k > PIPAD_MAX_K || !operand(args[4], n, k, &x) || !operand(args[8], n, k, &h)) Py_RETURN_NONE;
    const bool keep = args[7] != Py_None;
    a.ld = x.F;
    if (keep && (!operand(args[7], n, k, &a) || a.F != x.F)) Py_RETURN_NONE;
    const at::Tensor *w = plain_tensor(args[5]);
    if (!w || w->scalar_type() != at::kFloat || w->dim() != 2 || w->size(0) != x.F || w->stride(1) != 1 || w->size(1) != h.F) Py_RETURN_NONE;
    const int64_t Fo = w->size(1);
    const float *bias = nullptr;
    if (args[6] != Py_None) {
      const at::Tensor *b = plain_tensor(args[6]);
      if (!b || b->scalar_type() != at::kFloat || b->dim() != 1 || b->size(0) != Fo || b->stride(0) != 1) Py_RETURN_NONE;
      bias = static_cast<const float *>(b->data_ptr());
    }
    if (x.F > INT32_MAX || Fo > INT32_MAX) Py_RETURN_NONE;
    const float *const weights = static_cast<const float *>(w->data_ptr());
    const int64_t ldw = x.F > 1 ? w->stride(0) : std::max(Fo, w->stride(0));
    const int status = unlocked([&] {
      return fn(frame, (int32_t)x.F, x.ptr, x.ld, weights, ldw, bias, (int32_t)Fo, keep ? a.ptr : nullptr, a.ld, h.ptr, h.ld, stream);
    });
    return PyLong_FromLong(status);
  });
}

// ---- operators on node rows ----------------------------------------------------------------------
// The operands of one call: the first says how many rows and matrices there are and where, all others go with it.
struct RowsCall {
  int64_t n = 0, k = 0;
  long device = -1;
  bool first(PyObject *o, long current, Matrices *m) {
    Items list;
    const at::Tensor *t = nullptr;
    if (items(o, &list)) {
      if (list.count < 1 || list.count > PIPAD_MAX_K || !(t = plain_tensor(list.at[0])) || t->dim() != 2) return false;
      n = t->size(0), k = list.count;
    } else {
      if (!(t = plain_tensor(o)) || t->dim() != 3 || t->size(1) < 1 || t->size(1) > PIPAD_MAX_K) return false;
      n = t->size(0), k = t->size(1);
    }
    device = t->get_device();
    return device == current && n <= INT32_MAX && rows(o, m) && m->F >= 1 && m->F <= INT32_MAX;
  }
  bool here(PyObject *o) const {  // (a plain tensor)
    return THPVariable_Unpack(o).get_device() == device;
  }
  bool rows(PyObject *o, Matrices *m) const {
    if (!operand(o, n, k, m)) return false;
    Items list;
    if (!items(o, &list)) return here(o);
    for (Py_ssize_t t = 0; t < list.count; ++t)
      if (!here(list.at[t])) return false;
    return true;
  }
  bool rows_or_none(PyObject *o, int64_t F, Matrices *m, bool *there) const {
    *there = o != Py_None;
    m->ld = 0;
    return !*there || (rows(o, m) && m->F == F);
  }
  bool vector(PyObject *o, int64_t F, const float **at) const {
    *at = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = plain_tensor(o);
    if (!t || t->scalar_type() != at::kFloat || t->dim() != 1 || t->size(0) != F || (F > 1 && t->stride(0) != 1) || !here(o)) return false;
    *at = static_cast<const float *>(t->data_ptr());
    return true;
  }
  bool weights(PyObject *o, int64_t rows, int64_t columns, const float **at, int64_t *ld) const {
    const at::Tensor *t = plain_tensor(o);
    if (!t || t->scalar_type() != at::kFloat || t->dim() != 2 || t->size(0) != rows || t->size(1) != columns || (columns > 1 && t->stride(1) != 1) || !here(o))
      return false;
    *at = static_cast<const float *>(t->data_ptr());
    *ld = rows > 1 ? t->stride(0) : std::max(columns, t->stride(0));
    return true;
  }
  // The memory that a call needs for itself, which goes back in the order of the current stream: that of the call.
  static c10::DataPtr memory(size_t bytes) {
    return bytes ? c10::GetAllocator(c10::DeviceType::CUDA)->allocate(bytes) : c10::DataPtr();
  }
  at::Tensor empty(at::IntArrayRef shape) const { return at::empty(shape, at::TensorOptions().dtype(at::kFloat).device(at::kCUDA, (c10::DeviceIndex)device)); }
};

// Wg, Wu, Wd, bg, bu, bd and the activation as a pipad_gated_ff_t
bool ff_block(const RowsCall &call, PyObject *const *args, int64_t F, long activation, pipad_gated_ff_t *b) {
  const at::Tensor *g = plain_tensor(args[0]), *d = plain_tensor(args[2]);
  if (!g || !d || g->dim() != 2 || d->dim() != 2) return false;
  const int64_t hidden = g->size(1), Fo = d->size(1);
  if (hidden < 1 || hidden > INT32_MAX || Fo < 1 || Fo > INT32_MAX) return false;
  b->F = (int32_t)F, b->hidden = (int32_t)hidden, b->Fo = (int32_t)Fo, b->activation = (int32_t)activation;
  return call.weights(args[0], F, hidden, &b->Wg, &b->ldwg) && call.weights(args[1], F, hidden, &b->Wu, &b->ldwu) &&
         call.weights(args[2], hidden, Fo, &b->Wd, &b->ldwd) && call.vector(args[3], hidden, &b->bg) && call.vector(args[4], hidden, &b->bu) &&
         call.vector(args[5], Fo, &b->bd);
}

// gated_ff(address, address of the size query, current device, stream, X, Wg, Wu, Wd, bg, bu, bd, activation, Y) -> status
PyObject *gated_ff(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 13) return PyErr_Format(PyExc_TypeError, "gated_ff: thirteen arguments");
  return guarded([&]() -> PyObject * {
    const auto fn = address<decltype(&pipad_gated_ff)>(args[0]);
    const auto size = address<decltype(&pipad_gated_ff_workspace)>(args[1]);
    const long current = PyLong_AsLong(args[2]), activation = PyLong_AsLong(args[11]);
    void *const stream = PyLong_AsVoidPtr(args[3]);
    if (PyErr_Occurred()) return nullptr;
    RowsCall call;
    Matrices x, y;
    pipad_gated_ff_t block;
    if (!call.first(args[4], current, &x) || !ff_block(call, args + 5, x.F, activation, &block) || !call.rows(args[12], &y) || y.F != block.Fo)
      Py_RETURN_NONE;
    size_t bytes = 0;
    int status = size(&block, (int32_t)call.n, (int32_t)call.k, 0, &bytes);
    if (status == PIPAD_OK) {
      const c10::DataPtr memory = RowsCall::memory(bytes);
      status = unlocked([&] { return fn(&block, (int32_t)call.n, (int32_t)call.k, x.ptr, x.ld, y.ptr, y.ld, memory.get(), bytes, stream); });
    }
    return PyLong_FromLong(status);
  });
}

// gated_ff_backward(address, address of the size query, current device, stream, X, Wg, Wu, Wd, bg, bu, None, activation, dY, dX or None, weights,
// biases) -> (status, dWg, dWu, dWd, dbg, dbu, dbd)
PyObject *gated_ff_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 16) return PyErr_Format(PyExc_TypeError, "gated_ff_backward: sixteen arguments");
  return guarded([&]() -> PyObject * {
    const auto fn = address<decltype(&pipad_gated_ff_backward)>(args[0]);
    const auto size = address<decltype(&pipad_gated_ff_workspace)>(args[1]);
    const long current = PyLong_AsLong(args[2]), activation = PyLong_AsLong(args[11]);
    void *const stream = PyLong_AsVoidPtr(args[3]);
    if (PyErr_Occurred()) return nullptr;
    const bool weights = args[14] == Py_True, biases = args[15] == Py_True;
    RowsCall call;
    Matrices x, dy, dx;
    pipad_gated_ff_t block;
    bool want_dx;
    if (!call.first(args[4], current, &x) || !ff_block(call, args + 5, x.F, activation, &block) || !call.rows(args[12], &dy) || dy.F != block.Fo ||
        !call.rows_or_none(args[13], x.F, &dx, &want_dx))
      Py_RETURN_NONE;
    at::Tensor made[6];
    pipad_gated_ff_grads_t grads{};
    if (weights) {
      made[0] = call.empty({block.F, block.hidden}), made[1] = call.empty({block.F, block.hidden}), made[2] = call.empty({block.hidden, block.Fo});
      grads.dWg = made[0].data_ptr<float>(), grads.dWu = made[1].data_ptr<float>(), grads.dWd = made[2].data_ptr<float>();
      grads.lddwg = grads.lddwu = block.hidden, grads.lddwd = block.Fo;
    }
    if (biases) {
      made[3] = call.empty({block.hidden}), made[4] = call.empty({block.hidden}), made[5] = call.empty({block.Fo});
      grads.dbg = made[3].data_ptr<float>(), grads.dbu = made[4].data_ptr<float>(), grads.dbd = made[5].data_ptr<float>();
    }
    size_t bytes = 0;
    int status = size(&block, (int32_t)call.n, (int32_t)call.k, 1, &bytes);
    if (status == PIPAD_OK) {
      const c10::DataPtr memory = RowsCall::memory(bytes);
      status = unlocked([&] {
        return fn(&block, (int32_t)call.n, (int32_t)call.k, x.ptr, x.ld, dy.ptr, dy.ld, want_dx ? dx.ptr : nullptr, dx.ld,
                  weights || biases ? &grads : nullptr, memory.get(), bytes, stream);
      });
    }
    PyObject *const out = PyTuple_New(7);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(status));
    for (int q = 0; q < 6; ++q) {
      if (!made[q].defined()) Py_INCREF(Py_None);
      PyTuple_SET_ITEM(out, 1 + q, made[q].defined() ? THPVariable_Wrap(std::move(made[q])) : Py_None);
    }
    return out;
  });
}

// post, pre, eps, scale, w_post, b_post, w_pre, b_pre as a pipad_residual_norm_t
bool norm_params(const RowsCall &call, PyObject *const *args, int64_t F, pipad_residual_norm_t *c) {
  c->F = (int32_t)F, c->post = (int32_t)PyLong_AsLong(args[0]), c->pre = (int32_t)PyLong_AsLong(args[1]), c->eps = (float)PyFloat_AsDouble(args[2]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return call.vector(args[3], F, &c->scale) && call.vector(args[4], F, &c->w_post) && call.vector(args[5], F, &c->b_post) &&
         call.vector(args[6], F, &c->w_pre) && call.vector(args[7], F, &c->b_pre);
}

// residual_norm(address, current device, stream, R, B, gate, post, pre, eps, scale, w_post, b_post, w_pre, b_pre, R_out, Z) -> status
PyObject *residual_norm(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 16) return PyErr_Format(PyExc_TypeError, "residual_norm: sixteen arguments");
  return guarded([&]() -> PyObject * {
    const auto fn = address<decltype(&pipad_residual_norm)>(args[0]);
    const long current = PyLong_AsLong(args[1]);
    void *const stream = PyLong_AsVoidPtr(args[2]);
    if (PyErr_Occurred()) return nullptr;
    RowsCall call;
    Matrices r, m[4];
    bool there[4];
    pipad_residual_norm_t norm;
    PyObject *const others[4] = {args[4], args[5], args[14], args[15]};
    if (!call.first(args[3], current, &r) || !norm_params(call, args + 6, r.F, &norm)) Py_RETURN_NONE;
    for (int q = 0; q < 4; ++q)
      if (!call.rows_or_none(others[q], r.F, &m[q], &there[q])) Py_RETURN_NONE;
    const auto at = [&](int q) { return there[q] ? m[q].ptr : nullptr; };
    const int status = unlocked([&] {
      return fn(&norm, (int32_t)call.n, (int32_t)call.k, r.ptr, r.ld, at(0), m[0].ld, at(1), m[1].ld, at(2), m[2].ld, at(3), m[3].ld, stream);
    });
    return PyLong_FromLong(status);
  });
}

// residual_norm_backward(address, address of the size query, current device, stream, R, dR_out, dZ, B, gate, post, pre, eps, scale, w_post, b_post,
// w_pre, None, dR, dB, dgate, vectors wanted: five truth values) -> (status, dscale, dw_post, db_post, dw_pre, db_pre)
PyObject *residual_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 25) return PyErr_Format(PyExc_TypeError, "residual_norm_backward: twenty-five arguments");
  return guarded([&]() -> PyObject * {
    const auto fn = address<decltype(&pipad_residual_norm_backward)>(args[0]);
    const auto size = address<decltype(&pipad_residual_norm_workspace)>(args[1]);
    const long current = PyLong_AsLong(args[2]);
    void *const stream = PyLong_AsVoidPtr(args[3]);
    if (PyErr_Occurred()) return nullptr;
    RowsCall call;
    Matrices r, m[7];
    bool there[7];
    pipad_residual_norm_t norm;
    PyObject *const others[7] = {args[7], args[8], args[5], args[6], args[17], args[18], args[19]};  // B, gate, dR_out, dZ, dR, dB, dgate
    if (!call.first(args[4], current, &r) || !norm_params(call, args + 9, r.F, &norm)) Py_RETURN_NONE;
    for (int q = 0; q < 7; ++q)
      if (!call.rows_or_none(others[q], r.F, &m[q], &there[q])) Py_RETURN_NONE;
    at::Tensor made[5];
    float *to[5] = {};
    bool any = false;
    for (int q = 0; q < 5; ++q)
      if (args[20 + q] == Py_True) {
        made[q] = call.empty({r.F});
        to[q] = made[q].data_ptr<float>();
        any = true;
      }
    const pipad_residual_norm_grads_t grads{to[0], to[1], to[2], to[3], to[4]};
    size_t bytes = 0;
    int status = any ? size(norm.F, (int32_t)call.n, (int32_t)call.k, &bytes) : PIPAD_OK;
    if (status == PIPAD_OK) {
      const c10::DataPtr memory = RowsCall::memory(bytes);
      const auto at = [&](int q) { return there[q] ? m[q].ptr : nullptr; };
      status = unlocked([&] {
        return fn(&norm, (int32_t)call.n, (int32_t)call.k, r.ptr, r.ld, at(0), m[0].ld, at(1), m[1].ld, at(2), m[2].ld, at(3), m[3].ld, at(4), m[4].ld,
                  at(5), m[5].ld, at(6), m[6].ld, any ? &grads : nullptr, memory.get(), bytes, stream);
      });
    }
    PyObject *const out = PyTuple_New(6);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(status));
    for (int q = 0; q < 5; ++q) {
      if (!made[q].defined()) Py_INCREF(Py_None);
      PyTuple_SET_ITEM(out, 1 + q, made[q].defined() ? THPVariable_Wrap(std::move(made[q])) : Py_None);
    }
    return out;
  });
}

PyMethodDef methods[] = {
    {"gated_ff", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(gated_ff)), METH_FASTCALL, "pipad_gated_ff"},
    {"gated_ff_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(gated_ff_backward)), METH_FASTCALL, "pipad_gated_ff_backward"},
    {"residual_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(residual_norm)), METH_FASTCALL, "pipad_residual_norm"},
    {"residual_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(residual_norm_backward)), METH_FASTCALL,
     "pipad_residual_norm_backward"},
    {"build", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(build)), METH_FASTCALL, "pipad_frame_build_overlap"},
    {"transpose", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(transpose)), METH_FASTCALL, "pipad_frame_transpose"},
    {"aggregate", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(aggregate)), METH_FASTCALL, "pipad_frame_aggregate or its static form"},
    {"subset", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(subset)), METH_FASTCALL, "pipad_frame_aggregate_subset"},
    {"update", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(update)), METH_FASTCALL, "pipad_frame_aggregate_update"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", "The binding's calls in native code.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() {
  if (PyType_Ready(&buffers_type) < 0) return nullptr;
  PyObject *m = PyModule_Create(&module);
  if (!m) return nullptr;
  Py_INCREF(&buffers_type);
  PyObject *const callback = PyLong_FromVoidPtr(reinterpret_cast<void *>(allocate));
  if (PyModule_AddObject(m, "Buffers", reinterpret_cast<PyObject *>(&buffers_type)) < 0 || !callback ||
      PyModule_AddObject(m, "ALLOCATE", callback) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
