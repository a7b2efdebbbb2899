// dc_bind.cpp -- argument marshalling of the paged cache's calls for dc.PagedCache.
//
// The same checks as the Python binding's, made on the tensors themselves: attributes read one by one from
// Python, the structure packed and the outputs made there take 8 to 12 us a call, a kernel's launch 2 (host time of
// a call, without and with this module: append of 8 tokens 16 and 4.2 us, attention of one sequence 13 and 4.6, a selection
// and attention over it 31 and 10). Whatever is not the ordinary case (an argument that some check refuses, given
// outputs, another device or stream) gets NotImplemented, and the Python binding handles it and says what is wrong.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "distillcache.h"

namespace {

struct Cache {
  dc_paged* h;
  int device;
  at::ScalarType dtype;
  long long kv_heads, q_heads, dim;
};

// The library that is loaded (release or debug).
struct {
  decltype(&dc_paged_append) append;
  decltype(&dc_paged_attend) attend;
  decltype(&dc_paged_attend_workspace) workspace;
  decltype(&dc_paged_select) select;
} g_lib;

const at::Tensor* tensor(PyObject* o, const Cache& c, at::ScalarType type) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != c.device || t.scalar_type() != type) return nullptr;
  return &t;
}

// A dense tensor of n elements, or null.
const void* vector(PyObject* o, const Cache& c, at::ScalarType type, long long n, bool& ok) {
  const at::Tensor* t = tensor(o, c, type);
  if (!t || t->numel() != n || !t->is_contiguous()) {
    ok = false;
    return nullptr;
  }
  return t->const_data_ptr();
}

struct Heads {
  const void* at = nullptr;
  long long rows = 0, step = 0, head = 0;
};

// A [rows][heads][dim] tensor, possibly a view, whose heads start on 16 bytes.
Heads heads(PyObject* o, const Cache& c, long long n, bool& ok) {
  Heads r;
  const at::Tensor* t = tensor(o, c, c.dtype);
  if (!t || t->dim() != 3 || t->size(1) != n || t->size(2) != c.dim || t->stride(2) != 1) {
    ok = false;
    return r;
  }
  r.at = t->const_data_ptr();
  r.rows = t->size(0);
  // (the stride of a dimension of one says nothing)
  r.step = r.rows > 1 ? t->stride(0) : n * c.dim;
  r.head = n > 1 ? t->stride(1) : c.dim;
  if ((r.step & 7) || (r.head & 7) || (reinterpret_cast<uintptr_t>(r.at) & 15)) ok = false;
  return r;
}

// tables and lens.
struct Batch {
  long long seqs = 0, width = 0;
  const int *tables = nullptr, *lens = nullptr;
};
Batch batch(PyObject* tables, PyObject* lens, const Cache& c, bool& ok) {
  Batch b;
  const at::Tensor* t = tensor(tables, c, at::kInt);
  if (!t || t->dim() != 2 || !t->is_contiguous() || t->size(0) > INT_MAX || t->size(1) > INT_MAX) {
    ok = false;
    return b;
  }
  b.seqs = t->size(0);
  b.width = t->size(1);
  b.tables = static_cast<const int*>(t->const_data_ptr());
  b.lens = static_cast<const int*>(vector(lens, c, at::kInt, b.seqs, ok));
  return b;
}

// A whole number that fits an int.
int whole(PyObject* o, bool& ok) {
  int over = 0;
  if (!PyLong_Check(o)) {
    ok = false;
    return 0;
  }
  const long x = PyLong_AsLongAndOverflow(o, &over);
  if (over || x < INT_MIN || x > INT_MAX) ok = false;
  return (int)x;
}
float number(PyObject* o, bool& ok) {
  if (!PyFloat_Check(o)) {
    ok = false;
    return 0.f;
  }
  return (float)PyFloat_AS_DOUBLE(o);
}

const Cache* cache_of(PyObject* o) {
  if (!PyCapsule_CheckExact(o)) return nullptr;
  const Cache* c = static_cast<Cache*>(PyCapsule_GetPointer(o, "dc_paged"));
  return c && c10::cuda::current_device() == c->device ? c : nullptr;
}

at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const Cache& c) {
  return at::Tensor(at::detail::empty_cuda(sizes, type, at::Device(at::kCUDA, (c10::DeviceIndex)c.device), c10::nullopt));
}

PyObject* elsewhere() { return Py_NewRef(Py_NotImplemented); }

// The result, or a refused call's status.
PyObject* result(dc_status st, const at::Tensor& t) { return st == DC_OK ? THPVariable_Wrap(t) : PyLong_FromLong(st); }

// Python exceptions instead of C++ ones (an allocation that failed).
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const c10::OutOfMemoryError&) {
    return elsewhere();  // (the Python binding meets it again, and raises what it always does)
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

template <class F>
dc_status call(F f) {
  dc_status st;
  Py_BEGIN_ALLOW_THREADS
  st = f();
  Py_END_ALLOW_THREADS
  return st;
}

// append(cache, q, k, v, tables, lens, inv_freq, layer, starts, q_weight, k_weight, eps, norm, interleaved)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const Cache* c = n == 14 ? cache_of(a[0]) : nullptr;
    if (!c) return elsewhere();
    bool ok = true;
    dc_paged_append_args x{};
    const Batch b = batch(a[4], a[5], *c, ok);
    const Heads k = heads(a[2], *c, c->kv_heads, ok), v = heads(a[3], *c, c->kv_heads, ok);
    Heads q;
    if (a[1] != Py_None) q = heads(a[1], *c, c->q_heads, ok);
    if (!ok || v.rows != k.rows || (a[1] != Py_None && q.rows != k.rows)) return elsewhere();
    if (a[6] != Py_None) {
      const at::Tensor* f = tensor(a[6], *c, at::kFloat);
      if (!f || !f->is_contiguous() || f->numel() > INT_MAX / 2) return elsewhere();
      x.rotary_dim = 2 * (int)f->numel();
      x.inv_freq = static_cast<const float*>(f->const_data_ptr());
    }
    if (a[8] != Py_None) x.starts = static_cast<const int*>(vector(a[8], *c, at::kInt, b.seqs + 1, ok));
    if (a[9] != Py_None) x.q_weight = static_cast<const float*>(vector(a[9], *c, at::kFloat, c->dim, ok));
    if (a[10] != Py_None) x.k_weight = static_cast<const float*>(vector(a[10], *c, at::kFloat, c->dim, ok));
    x.layer = whole(a[7], ok);
    x.eps = number(a[11], ok);
    if (!ok) return elsewhere();
    x.norm = a[12] == Py_True;
    x.interleaved = a[13] == Py_True;
    if ((!x.norm && a[12] != Py_False) || (!x.interleaved && a[13] != Py_False)) return elsewhere();
    x.seqs = (int)b.seqs;
    x.table_width = (int)b.width;
    x.tokens = k.rows;
    x.lens = b.lens;
    x.tables = b.tables;
    x.q = q.at;
    x.k = k.at;
    x.v = v.at;
    x.q_token_stride = q.step;
    x.q_head_stride = q.head;
    x.k_token_stride = k.step;
    x.k_head_stride = k.head;
    x.v_token_stride = v.step;
    x.v_head_stride = v.head;
    at::Tensor out;
    if (a[1] != Py_None) {
      out = empty({k.rows, c->q_heads, c->dim}, c->dtype, *c);
      x.q_out = out.data_ptr();
      x.q_out_token_stride = c->q_heads * c->dim;
      x.q_out_head_stride = c->dim;
    }
    const cudaStream_t s = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)c->device).stream();
    const dc_status st = call([&] { return g_lib.append(c->h, &x, s); });
    if (st == DC_OK && a[1] == Py_None) Py_RETURN_NONE;
    return result(st, out);
  });
}

// attend(cache, q, tables, lens, layer, selected, shared (address), with_lse, scale)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const Cache* c = n == 9 ? cache_of(a[0]) : nullptr;
    if (!c) return elsewhere();
    bool ok = true;
    dc_paged_attend_args x{};
    const Batch b = batch(a[2], a[3], *c, ok);
    const Heads q = heads(a[1], *c, c->q_heads, ok);
    if (!ok || q.rows != b.seqs) return elsewhere();
    if (a[5] != Py_None) {
      const at::Tensor* t = tensor(a[5], *c, at::kInt);
      if (!t || t->dim() != 3 || t->size(0) != b.seqs || t->size(1) != c->kv_heads || t->size(2) < 1 || t->size(2) > INT_MAX ||
          !t->is_contiguous())
        return elsewhere();
      x.selected = static_cast<const int*>(t->const_data_ptr());
      x.count = (int)t->size(2);
    }
    if (!PyLong_Check(a[6])) return elsewhere();
    x.shared = static_cast<const dc_paged_shared*>(PyLong_AsVoidPtr(a[6]));
    x.layer = whole(a[4], ok);
    x.scale = number(a[8], ok);
    const bool with_lse = a[7] == Py_True;
    if (!ok || PyErr_Occurred() || (!with_lse && a[7] != Py_False)) {
      PyErr_Clear();
      return elsewhere();
    }
    x.seqs = (int)b.seqs;
    x.table_width = (int)b.width;
    x.q = q.at;
    x.q_seq_stride = q.step;
    x.q_head_stride = q.head;
    x.lens = b.lens;
    x.tables = b.tables;
    size_t need = 0;
    if (const dc_status st = g_lib.workspace(c->h, x.seqs, x.table_width, x.count, x.shared, &need); st != DC_OK)
      return PyLong_FromLong(st);
    const at::Tensor out = empty({b.seqs, c->q_heads, c->dim}, c->dtype, *c);
    at::Tensor lse, work;
    if (with_lse) {
      lse = empty({b.seqs, c->q_heads}, at::kFloat, *c);
      x.lse = static_cast<float*>(lse.data_ptr());
    }
    if (need) {
      work = empty({(long long)need}, at::kByte, *c);
      x.workspace = work.data_ptr();
    }
    x.workspace_bytes = need;
    x.out = out.data_ptr();
    const cudaStream_t s = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)c->device).stream();
    const dc_status st = call([&] { return g_lib.attend(c->h, &x, s); });
    if (st != DC_OK || !with_lse) return result(st, out);
    PyObject *o = THPVariable_Wrap(out), *l = THPVariable_Wrap(lse), *both = o && l ? PyTuple_Pack(2, o, l) : nullptr;
    Py_XDECREF(o);
    Py_XDECREF(l);
    return both;
  });
}

// select(cache, q, tables, lens, count, layer, keep_first, keep_last)
PyObject* select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const Cache* c = n == 8 ? cache_of(a[0]) : nullptr;
    if (!c) return elsewhere();
    bool ok = true;
    dc_paged_select_args x{};
    const Batch b = batch(a[2], a[3], *c, ok);
    const Heads q = heads(a[1], *c, c->q_heads, ok);
    x.count = whole(a[4], ok);
    x.layer = whole(a[5], ok);
    x.keep_first = whole(a[6], ok);
    x.keep_last = whole(a[7], ok);
    if (!ok || q.rows != b.seqs || x.count < 1 || x.count > 65536) return elsewhere();
    x.seqs = (int)b.seqs;
    x.table_width = (int)b.width;
    x.q = q.at;
    x.q_seq_stride = q.step;
    x.q_head_stride = q.head;
    x.lens = b.lens;
    x.tables = b.tables;
    const at::Tensor out = empty({b.seqs, c->kv_heads, x.count}, at::kInt, *c);
    const long long need = 4 * b.seqs * c->kv_heads * b.width;
    at::Tensor work;
    if (need) {
      work = empty({need}, at::kByte, *c);
      x.workspace = work.data_ptr();
    }
    x.workspace_bytes = (size_t)need;
    x.out = static_cast<int*>(out.data_ptr());
    const cudaStream_t s = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)c->device).stream();
    return result(call([&] { return g_lib.select(c->h, &x, s); }), out);
  });
}

// cache(handle, device, fp16, kv_heads, q_heads, head_dim): what the calls' first argument is
PyObject* cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) return elsewhere();
  auto* c = new Cache{static_cast<dc_paged*>(PyLong_AsVoidPtr(a[0])), (int)PyLong_AsLong(a[1]),
                      a[2] == Py_True ? at::kHalf : at::kBFloat16, PyLong_AsLong(a[3]), PyLong_AsLong(a[4]), PyLong_AsLong(a[5])};
  if (PyErr_Occurred()) {
    delete c;
    return nullptr;
  }
  return PyCapsule_New(c, "dc_paged", [](PyObject* o) { delete static_cast<Cache*>(PyCapsule_GetPointer(o, "dc_paged")); });
}

// library(append, attend, attend_workspace, select): the functions' addresses
PyObject* library(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) return elsewhere();
  g_lib.append = reinterpret_cast<decltype(g_lib.append)>(PyLong_AsVoidPtr(a[0]));
  g_lib.attend = reinterpret_cast<decltype(g_lib.attend)>(PyLong_AsVoidPtr(a[1]));
  g_lib.workspace = reinterpret_cast<decltype(g_lib.workspace)>(PyLong_AsVoidPtr(a[2]));
  g_lib.select = reinterpret_cast<decltype(g_lib.select)>(PyLong_AsVoidPtr(a[3]));
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

PyCFunction function(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef g_methods[] = {{"append", function(append), METH_FASTCALL, nullptr},
                           {"attend", function(attend), METH_FASTCALL, nullptr},
                           {"select", function(select), METH_FASTCALL, nullptr},
                           {"cache", function(cache), METH_FASTCALL, nullptr},
                           {"library", function(library), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_dc_bind", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dc_bind() {
  PyObject* m = PyModule_Create(&g_module);
  // what it was built against
  if (m && (PyModule_AddStringConstant(m, "torch", DC_TORCH_VERSION) < 0 ||
            PyModule_AddObject(m, "python", PyUnicode_FromFormat("%d.%d", PY_MAJOR_VERSION, PY_MINOR_VERSION)) < 0))
    Py_CLEAR(m);
  return m;
}
