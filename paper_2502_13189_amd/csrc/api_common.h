// What the host sides of the library share: per-phase timing, launch checks and the
// validation of tensor descriptors.
#pragma once

#include "moba.h"
#include "moba_internal.h"

#include <algorithm>
#include <cstdlib>
#include <mutex>
#include <vector>

namespace moba {

// ------------------------------------------------------------- profiling
struct PhaseRec {
  const char* name;
  hipEvent_t a, b;
};
inline bool g_prof = false;
inline std::vector<PhaseRec> g_recs;
inline std::mutex g_prof_mu;

struct Phase {
  hipStream_t st;
  PhaseRec rec{};
  bool on = false;
  Phase(const char* name, hipStream_t s) : st(s) {
    if (!g_prof || !name) return;
    // (an event recorded into a graph has no time; asking for it is an error, which the next
    // launch would be told of)
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (s && (hipStreamIsCapturing(s, &capture) != hipSuccess || capture != hipStreamCaptureStatusNone)) return;
    rec.name = name;
    if (hipEventCreate(&rec.a) != hipSuccess) return;
    if (hipEventCreate(&rec.b) != hipSuccess) { (void)hipEventDestroy(rec.a); return; }
    (void)hipEventRecord(rec.a, st);
    on = true;
  }
  ~Phase() {
    if (!on) return;
    (void)hipEventRecord(rec.b, st);
    std::lock_guard<std::mutex> lk(g_prof_mu);
    g_recs.push_back(rec);
  }
};

inline bool env_flag(const char* name) {
  const char* e = std::getenv(name);
  return e && e[0] && e[0] != '0';
}

// Read at every launch, so a process can switch it on and off.
inline bool debug_sync() { return env_flag("MOBA_DEBUG_SYNC"); }

#define MOBA_LAUNCH(expr)                                         \
  do {                                                            \
    hipError_t e_ = (expr);                                       \
    if (e_ != hipSuccess) return MOBA_ERR_HIP;                    \
    if (debug_sync() && hipStreamSynchronize(stream) != hipSuccess) \
      return MOBA_ERR_HIP;                                        \
  } while (0)
// ------------------------------------------------------------- validation
struct View {
  void* data;
  int64_t st, sh;  // token and head strides, elements
  int64_t H;
};

// Number of elements a descriptor spans (0 if any dimension is empty).
inline int64_t numel(const moba_tensor* t) {
  int64_t n = 1;
  for (int d = 0; d < t->ndim && d < 4; d++) n *= std::max<int64_t>(t->shape[d], 0);
  return n;
}

// A data pointer may be NULL only for an empty tensor.
inline bool missing(const moba_tensor* t) { return !t || (!t->data && (t->ndim < 1 || t->ndim > 4 || numel(t) > 0)); }

inline moba_status check_3d(const moba_tensor* t, int dtype, View* v) {
  if (missing(t)) return MOBA_ERR_NULL;
  if (t->dtype != dtype) return MOBA_ERR_DTYPE;
  if (t->ndim != 3) return MOBA_ERR_SHAPE;
  if (t->shape[0] < 0 || t->shape[1] < 1) return MOBA_ERR_SHAPE;
  if (t->shape[2] != kHeadDim) return MOBA_ERR_UNSUPPORTED;
  if (t->stride[2] != 1 || t->stride[0] < 0 || t->stride[1] < 0) return MOBA_ERR_LAYOUT;
  // 16-byte vector accesses: base and both strides must keep rows 16-byte aligned
  const int64_t per16 = dtype == MOBA_BF16 ? 8 : 4;
  if ((reinterpret_cast<uintptr_t>(t->data) & 15) != 0 || t->stride[0] % per16 != 0 ||
      t->stride[1] % per16 != 0)
    return MOBA_ERR_LAYOUT;
  v->data = t->data;
  v->st = t->stride[0];
  v->sh = t->stride[1];
  v->H = t->shape[1];
  return MOBA_OK;
}

inline moba_status check_contig(const moba_tensor* t, int dtype, int ndim, const int64_t* shape) {
  if (missing(t)) return MOBA_ERR_NULL;
  if (t->dtype != dtype) return MOBA_ERR_DTYPE;
  if (t->ndim != ndim) return MOBA_ERR_SHAPE;
  for (int d = 0; d < ndim; d++)
    if (t->shape[d] != shape[d]) return MOBA_ERR_SHAPE;
  if (numel(t) == 0) return MOBA_OK;  // strides of an empty tensor are irrelevant
  int64_t expect = 1;
  for (int d = ndim - 1; d >= 0; d--) {
    if (t->shape[d] > 1 && t->stride[d] != expect) return MOBA_ERR_LAYOUT;
    expect *= shape[d];
  }
  return MOBA_OK;
}

// Whether two [T, H, D] views of elements of `el` bytes may share memory.  Views of
// one wider buffer (equal token strides) share none if their heads lie apart in it.
inline bool share_memory(const View& a, const View& b, int64_t T, int64_t el) {
  const int64_t wa = (a.H - 1) * a.sh + kHeadDim, wb = (b.H - 1) * b.sh + kHeadDim;
  const int64_t ia = (int64_t)(reinterpret_cast<uintptr_t>(a.data) / el);
  const int64_t ib = (int64_t)(reinterpret_cast<uintptr_t>(b.data) / el);
  if (ia + (T - 1) * a.st + wa <= ib || ib + (T - 1) * b.st + wb <= ia) return false;
  if (a.st != b.st || wa > a.st || wb > a.st) return true;
  const int64_t d = ((ib - ia) % a.st + a.st) % a.st;  // b's heads from a's, within a token
  return d < wa || a.st - d < wb;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace moba
