// Python side of the paged cache's calls: tensors to descriptors, outputs a caller left
// out, the C call.  A serving step's kernels take a few microseconds, and describing their
// ten tensors through ctypes takes longer than that (a decode call 21.7 us of host time,
// this way 10.6), so these calls are marshalled here.  Nothing is computed: every argument is checked, and every
// step done, behind the C ABI.
#include "moba.h"

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>

namespace {

// A tensor argument; raises where it is none, or not one of `device` (-1: sets it).
const at::Tensor* tensor(PyObject* o, int* device) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "expected a tensor, got %s", Py_TYPE(o)->tp_name);
    return nullptr;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) {
    PyErr_SetString(PyExc_ValueError, "the paged cache's tensors live on a GPU");
    return nullptr;
  }
  const int at = t.device().index();
  if (*device < 0) *device = at;
  if (at != *device) {
    PyErr_Format(PyExc_ValueError, "tensors on GPU %d and on GPU %d", *device, at);
    return nullptr;
  }
  return &t;
}

bool describe(const at::Tensor& t, moba_tensor* d) {
  switch (t.scalar_type()) {
    case at::kFloat: d->dtype = MOBA_F32; break;
    case at::kBFloat16: d->dtype = MOBA_BF16; break;
    case at::kInt: d->dtype = MOBA_I32; break;
    case at::kLong: d->dtype = MOBA_I64; break;
    case at::kFloat8_e4m3fn: d->dtype = MOBA_F8E4M3; break;
    default: PyErr_SetString(PyExc_TypeError, "unsupported dtype"); return false;
  }
  const auto shape = t.sizes(), stride = t.strides();
  const int n = (int)shape.size();
  if (n > 4) {
    PyErr_SetString(PyExc_ValueError, "at most 4 dimensions");
    return false;
  }
  d->data = t.data_ptr();
  d->ndim = n;
  for (int i = 0; i < 4; i++) {
    d->shape[i] = i < n ? shape[i] : 0;
    d->stride[i] = i < n ? stride[i] : 0;
  }
  return true;
}

bool describe(PyObject* o, int* device, moba_tensor* d) {
  const at::Tensor* t = tensor(o, device);
  return t && describe(*t, d);
}

// PagedCache: k, v, k_scale, v_scale, k_sum
struct Cache {
  moba_tensor t[5];
  moba_cache c{&t[0], &t[1], &t[2], &t[3], &t[4]};
};

bool describe_cache(PyObject* o, int* device, Cache* c) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 5) {
    PyErr_SetString(PyExc_TypeError, "expected a PagedCache");
    return false;
  }
  for (int i = 0; i < 5; i++) {
    if (i != 1) {
      if (!describe(PyTuple_GET_ITEM(o, i), device, &c->t[i])) return false;
      continue;
    }
    // V pages [N, Hkv, P / 64, 128, 64]: the rows of a page's tiles one after the other
    const at::Tensor* v = tensor(PyTuple_GET_ITEM(o, i), device);
    if (!v) return false;
    if (v->dim() != 5) {
      PyErr_SetString(PyExc_ValueError, "v has five dimensions");
      return false;
    }
    if (v->scalar_type() != at::kFloat8_e4m3fn) {
      PyErr_SetString(PyExc_TypeError, "unsupported dtype");
      return false;
    }
    if (v->size(2) > 1 && v->stride(2) != v->size(3) * v->stride(3)) {
      PyErr_SetString(PyExc_ValueError, "v's last three dims must be contiguous");
      return false;
    }
    c->t[1] = {v->data_ptr(), MOBA_F8E4M3, 4,
               {v->size(0), v->size(1), v->size(2) * v->size(3), v->size(4)},
               {v->stride(0), v->stride(1), v->stride(3), v->stride(4)}};
  }
  return true;
}

bool integer(PyObject* o, int64_t* x) {
  *x = PyLong_AsLongLong(o);
  return *x != -1 || !PyErr_Occurred();
}

// `given`, or a new tensor where it is None; a new reference.
PyObject* output(PyObject* given, at::IntArrayRef shape, const at::Tensor& like, at::ScalarType type) {
  if (given != Py_None) {
    Py_INCREF(given);
    return given;
  }
  return THPVariable_Wrap(at::empty(shape, like.options().dtype(type).requires_grad(false)));
}

bool arguments(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return false;
}

struct Refs {  // references given up on return, those handed out aside
  PyObject* o[5] = {};
  ~Refs() {
    for (PyObject* x : o) Py_XDECREF(x);
  }
};

// plan(add, lens, table, free_pages, num_free, page_size, num_tokens, lens_out, num_free_out,
//      cu_new, slots, refused, stream) -> (status, cu_new, slots, lens_out, num_free_out, refused)
PyObject* plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arguments(n, 13)) return nullptr;
  int device = -1;
  moba_tensor d[10];
  int64_t page, tokens, stream;
  for (int i = 0; i < 5; i++)
    if (!describe(a[i], &device, &d[i])) return nullptr;
  if (!integer(a[5], &page) || !integer(a[6], &tokens) || !integer(a[12], &stream)) return nullptr;
  const at::Tensor& like = THPVariable_Unpack(a[0]);
  const int64_t S = like.dim() > 0 ? like.size(0) : 0;
  if (tokens < 0) {
    PyErr_SetString(PyExc_ValueError, "num_tokens must not be negative");
    return nullptr;
  }
  Refs r;
  r.o[0] = output(a[9], {S + 1}, like, at::kInt);
  r.o[1] = output(a[10], {tokens}, like, at::kLong);
  r.o[2] = output(a[7], {S}, like, at::kInt);
  r.o[3] = output(a[8], {1}, like, at::kInt);
  r.o[4] = output(a[11], {1}, like, at::kInt);
  for (int i = 0; i < 5; i++)
    if (!r.o[i] || !describe(r.o[i], &device, &d[5 + i])) return nullptr;
  if (d[6].ndim != 1 || d[6].shape[0] != tokens) {
    PyErr_Format(PyExc_ValueError, "slots must have num_tokens (%lld) rows", (long long)tokens);
    return nullptr;
  }
  if (page != (int32_t)page) page = 0;  // (refused as such)
  const moba_status st =
      moba_cache_plan(&d[0], &d[1], &d[2], &d[3], &d[4], (int32_t)page, &d[7], &d[8], &d[5], &d[6],
                      &d[9], reinterpret_cast<hipStream_t>(stream));
  return Py_BuildValue("(iOOOOO)", (int)st, r.o[0], r.o[1], r.o[2], r.o[3], r.o[4]);
  END_HANDLE_TH_ERRORS
}

// write(k, v, slots, cache, stream) -> status
PyObject* write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arguments(n, 5)) return nullptr;
  int device = -1;
  moba_tensor d[3];
  Cache c;
  int64_t stream;
  for (int i = 0; i < 3; i++)
    if (!describe(a[i], &device, &d[i])) return nullptr;
  if (!describe_cache(a[3], &device, &c) || !integer(a[4], &stream)) return nullptr;
  return PyLong_FromLong(
      moba_cache_write(&d[0], &d[1], &d[2], &c.c, reinterpret_cast<hipStream_t>(stream)));
  END_HANDLE_TH_ERRORS
}

// decode(q, cache, table, lens, block_size, topk, out, lse, workspace, stream)
//   -> (status, out, lse)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arguments(n, 10)) return nullptr;
  int device = -1;
  moba_tensor q, table, lens, out, lse;
  Cache c;
  int64_t block, topk, stream;
  if (!describe(a[0], &device, &q) || !describe_cache(a[1], &device, &c) ||
      !describe(a[2], &device, &table) || !describe(a[3], &device, &lens) || !integer(a[4], &block) ||
      !integer(a[5], &topk) || !integer(a[9], &stream))
    return nullptr;
  if (q.ndim != 3 || table.ndim != 2) {
    PyErr_SetString(PyExc_ValueError, "q has three dimensions, table has two");
    return nullptr;
  }
  // (what does not fit 32 bits is refused for its value)
  block = std::min<int64_t>(std::max<int64_t>(block, -1), INT32_MAX);
  topk = std::min<int64_t>(std::max<int64_t>(topk, -1), INT32_MAX);
  const at::Tensor& like = THPVariable_Unpack(a[0]);
  Refs r;
  r.o[0] = output(a[6], like.sizes(), like, like.scalar_type());
  r.o[1] = output(a[7], {q.shape[1], q.shape[0]}, like, at::kFloat);
  if (!r.o[0] || !r.o[1] || !describe(r.o[0], &device, &out) || !describe(r.o[1], &device, &lse))
    return nullptr;
  at::Tensor ws;
  size_t bytes;
  if (a[8] != Py_None) {
    const at::Tensor* w = tensor(a[8], &device);
    if (!w) return nullptr;
    if (!w->is_contiguous()) {
      PyErr_SetString(PyExc_ValueError, "workspace must be contiguous");
      return nullptr;
    }
    ws = *w;
  } else {
    const int64_t heads = std::min<int64_t>(std::max(q.shape[1], c.t[0].shape[1]), INT32_MAX);
    bytes = heads < INT32_MAX && c.t[0].ndim == 4
                ? moba_cache_decode_workspace_bytes(
                      q.shape[0], table.shape[1], (int32_t)q.shape[1], (int32_t)c.t[0].shape[1],
                      (int32_t)std::min<int64_t>(c.t[0].shape[2], INT32_MAX), (int32_t)block, (int32_t)topk)
                : 0;
    ws = at::empty({(int64_t)std::max<size_t>(bytes, 16)},
                   like.options().dtype(at::kByte).requires_grad(false));
  }
  bytes = (size_t)ws.nbytes();
  const moba_status st = moba_cache_decode(&q, &c.c, &table, &lens, (int32_t)block, (int32_t)topk, &out,
                                           &lse, ws.data_ptr(), bytes,
                                           reinterpret_cast<hipStream_t>(stream));
  return Py_BuildValue("(iOO)", (int)st, r.o[0], r.o[1]);
  END_HANDLE_TH_ERRORS
}

PyMethodDef kMethods[] = {
    {"plan", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(plan)), METH_FASTCALL, nullptr},
    {"write", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(write)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(decode)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_cache_binding", nullptr, -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cache_binding(void) { return PyModule_Create(&kModule); }
