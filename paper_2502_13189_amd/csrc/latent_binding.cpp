// Python side of rotary positions and latent attention: tensors to descriptors, outputs and workspaces
// that a caller left out, the C call.  Nothing is computed: every argument is checked, and every step
// done, behind the C ABI.
namespace {
constexpr const char* kOwner = "rotary positions' and latent attention's";
}

#include "py_tensors.h"

#include <cmath>

namespace {

// (freqs, amplitude, interleaved), pos, cu_seqlens, start (the last three: tensors or None)
struct Turn {
  moba_tensor t[4];
  moba_rotation r{};
};

bool describe_rotation(PyObject* o, PyObject* const* at, int* device, Turn* x) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3) {
    PyErr_SetString(PyExc_TypeError, "expected a Rotation");
    return false;
  }
  // (the only tensor of 64-bit floats)
  const at::Tensor* f = tensor(PyTuple_GET_ITEM(o, 0), device);
  if (!f) return false;
  if (f->scalar_type() != at::kDouble || f->dim() != 1) {
    PyErr_SetString(PyExc_TypeError, "a Rotation's freqs are a float64 tensor of one dimension");
    return false;
  }
  x->t[0] = {f->data_ptr(), MOBA_F64, 1, {f->size(0)}, {f->stride(0)}};
  const double amplitude = PyFloat_AsDouble(PyTuple_GET_ITEM(o, 1));
  if (amplitude == -1.0 && PyErr_Occurred()) return false;
  const int interleaved = PyObject_IsTrue(PyTuple_GET_ITEM(o, 2));
  if (interleaved < 0) return false;
  x->r.freqs = &x->t[0];
  x->r.amplitude = (float)amplitude;
  x->r.interleaved = interleaved;
  const moba_tensor** to[3] = {&x->r.pos, &x->r.cu_seqlens, &x->r.start};
  for (int i = 0; i < 3; i++) {
    if (at[i] == Py_None) continue;
    if (!describe(at[i], device, &x->t[1 + i])) return false;
    *to[i] = &x->t[1 + i];
  }
  return true;
}

bool real(PyObject* o, float* x) {
  const double y = PyFloat_AsDouble(o);
  if (y == -1.0 && PyErr_Occurred()) return false;
  *x = (float)y;
  return true;
}

bool dims(const moba_tensor& t, int n, const char* what) {
  if (t.ndim == n) return true;
  PyErr_Format(PyExc_ValueError, "%s must have %d dimensions", what, n);
  return false;
}

// `given` (uint8, contiguous), or new memory of at least `bytes`.
bool workspace(PyObject* given, size_t bytes, const at::Tensor& like, int* device, at::Tensor* ws) {
  if (given == Py_None) {
    *ws = at::empty({(int64_t)std::max<size_t>(bytes, 16)}, like.options().dtype(at::kByte).requires_grad(false));
    return true;
  }
  const at::Tensor* w = tensor(given, device);
  if (!w) return false;
  if (!w->is_contiguous()) {
    PyErr_SetString(PyExc_ValueError, "workspace must be contiguous");
    return false;
  }
  *ws = *w;
  return true;
}

int32_t narrow(int64_t x) { return (int32_t)std::min<int64_t>(std::max<int64_t>(x, -1), INT32_MAX); }

// rope(backward, q, k, rotation, pos, cu_seqlens, start, q_out, k_out, stream) -> (status, q_out, k_out)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arguments(n, 10)) return nullptr;
  int device = -1;
  const int backward = PyObject_IsTrue(a[0]);
  const bool two = a[2] != Py_None;
  moba_tensor q, k, qo, ko;
  Turn turn;
  int64_t stream;
  if (backward < 0 || !describe(a[1], &device, &q) || (two && !describe(a[2], &device, &k)) ||
      !describe_rotation(a[3], a + 4, &device, &turn) || !integer(a[9], &stream))
    return nullptr;
  if (!two && a[8] != Py_None) {
    PyErr_SetString(PyExc_ValueError, "an output of k without k");
    return nullptr;
  }
  Refs r;
  const at::Tensor& tq = THPVariable_Unpack(a[1]);
  r.o[0] = output(a[7], tq.sizes(), tq, tq.scalar_type());
  if (!r.o[0] || !describe(r.o[0], &device, &qo)) return nullptr;
  if (two) {
    const at::Tensor& tk = THPVariable_Unpack(a[2]);
    r.o[1] = output(a[8], tk.sizes(), tk, tk.scalar_type());
    if (!r.o[1] || !describe(r.o[1], &device, &ko)) return nullptr;
  }
  const moba_status st = (backward ? moba_rope_backward : moba_rope)(
      &q, two ? &k : nullptr, &turn.r, &qo, two ? &ko : nullptr, reinterpret_cast<hipStream_t>(stream));
  return Py_BuildValue("(iOO)", (int)st, r.o[0], two ? r.o[1] : Py_None);
  END_HANDLE_TH_ERRORS
}

// forward(q, k, k_rope, v, cu_seqlens, scale, out, lse, stream) -> (status, out, lse)
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arguments(n, 9)) return nullptr;
  int device = -1;
  moba_tensor d[5], out, lse;
  float scale;
  int64_t stream;
  for (int i = 0; i < 5; i++)
    if (!describe(a[i], &device, &d[i])) return nullptr;
  if (!real(a[5], &scale) || !integer(a[8], &stream) || !dims(d[0], 3, "q") || !dims(d[3], 3, "v")) return nullptr;
  const at::Tensor& like = THPVariable_Unpack(a[3]);
  Refs r;
  r.o[0] = output(a[6], like.sizes(), like, like.scalar_type());
  r.o[1] = output(a[7], {d[0].shape[1], d[0].shape[0]}, like, at::kFloat);
  if (!r.o[0] || !r.o[1] || !describe(r.o[0], &device, &out) || !describe(r.o[1], &device, &lse)) return nullptr;
  const moba_status st = moba_latent_forward(&d[0], &d[1], &d[2], &d[3], &d[4], scale, &out, &lse,
                                             reinterpret_cast<hipStream_t>(stream));
  return Py_BuildValue("(iOO)", (int)st, r.o[0], r.o[1]);
  END_HANDLE_TH_ERRORS
}

// backward(q, k, k_rope, v, cu_seqlens, out, lse, dout, scale, dq, dk, dk_rope, dv, workspace, stream)
//   -> (status, dq, dk, dk_rope, dv)
PyObject* backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arguments(n, 15)) return nullptr;
  int device = -1;
  moba_tensor d[8], g[4];
  float scale;
  int64_t stream;
  for (int i = 0; i < 8; i++)
    if (!describe(a[i], &device, &d[i])) return nullptr;
  if (!real(a[8], &scale) || !integer(a[14], &stream) || !dims(d[0], 3, "q")) return nullptr;
  Refs r;
  for (int i = 0; i < 4; i++) {
    const at::Tensor& like = THPVariable_Unpack(a[i]);
    r.o[i] = output(a[9 + i], like.sizes(), like, like.scalar_type());
    if (!r.o[i] || !describe(r.o[i], &device, &g[i])) return nullptr;
  }
  at::Tensor ws;
  if (!workspace(a[13], moba_latent_backward_workspace_bytes(d[0].shape[0], narrow(d[0].shape[1])),
                 THPVariable_Unpack(a[0]), &device, &ws))
    return nullptr;
  const moba_status st = moba_latent_backward(&d[0], &d[1], &d[2], &d[3], &d[4], scale, &d[5], &d[6], &d[7], &g[0],
                                              &g[1], &g[2], &g[3], ws.data_ptr(), (size_t)ws.nbytes(),
                                              reinterpret_cast<hipStream_t>(stream));
  return Py_BuildValue("(iOOOO)", (int)st, r.o[0], r.o[1], r.o[2], r.o[3]);
  END_HANDLE_TH_ERRORS
}

// write(c, k_rope, slots, pages, rotation, pos, cu_seqlens, start, stream) -> status
PyObject* write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arguments(n, 9)) return nullptr;
  int device = -1;
  moba_tensor d[4];
  Turn turn;
  int64_t stream;
  for (int i = 0; i < 4; i++)
    if (!describe(a[i], &device, &d[i])) return nullptr;
  const bool turned = a[4] != Py_None;
  if (turned && !describe_rotation(a[4], a + 5, &device, &turn)) return nullptr;
  if (!turned && (a[5] != Py_None || a[6] != Py_None || a[7] != Py_None)) {
    PyErr_SetString(PyExc_ValueError, "positions without a Rotation");
    return nullptr;
  }
  if (!integer(a[8], &stream)) return nullptr;
  return PyLong_FromLong(moba_latent_write(&d[0], &d[1], &d[2], turned ? &turn.r : nullptr, &d[3],
                                           reinterpret_cast<hipStream_t>(stream)));
  END_HANDLE_TH_ERRORS
}

// decode(q_c, q_rope, pages, table, lens, scale, out, lse, workspace, stream) -> (status, out, lse)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arguments(n, 10)) return nullptr;
  int device = -1;
  moba_tensor d[5], out, lse;
  float scale;
  int64_t stream;
  for (int i = 0; i < 5; i++)
    if (!describe(a[i], &device, &d[i])) return nullptr;
  if (!real(a[5], &scale) || !integer(a[9], &stream) || !dims(d[0], 3, "q_c") || !dims(d[2], 3, "pages") ||
      !dims(d[3], 2, "table"))
    return nullptr;
  const at::Tensor& like = THPVariable_Unpack(a[0]);
  Refs r;
  r.o[0] = output(a[6], like.sizes(), like, like.scalar_type());
  r.o[1] = output(a[7], {d[0].shape[1], d[0].shape[0]}, like, at::kFloat);
  if (!r.o[0] || !r.o[1] || !describe(r.o[0], &device, &out) || !describe(r.o[1], &device, &lse)) return nullptr;
  at::Tensor ws;
  if (!workspace(a[8],
                 moba_latent_decode_workspace_bytes(d[0].shape[0], d[3].shape[1], narrow(d[0].shape[1]),
                                                    narrow(d[2].shape[1])),
                 like, &device, &ws))
    return nullptr;
  const moba_status st = moba_latent_decode(&d[0], &d[1], &d[2], &d[3], &d[4], scale, &out, &lse, ws.data_ptr(),
                                            (size_t)ws.nbytes(), reinterpret_cast<hipStream_t>(stream));
  return Py_BuildValue("(iOO)", (int)st, r.o[0], r.o[1]);
  END_HANDLE_TH_ERRORS
}

#define METHOD(name) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {METHOD(rope),  METHOD(forward), METHOD(backward),
                          METHOD(write), METHOD(decode),  {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_latent_binding", nullptr, -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__latent_binding(void) { return PyModule_Create(&kModule); }
