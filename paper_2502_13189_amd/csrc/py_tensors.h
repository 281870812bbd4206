// What the Python modules of the library share: tensors to descriptors, outputs that a caller left out.
// The includer defines kOwner first: whose tensors an error message speaks of.
#pragma once

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
    PyErr_Format(PyExc_ValueError, "%s tensors live on a GPU", kOwner);
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

}  // namespace
