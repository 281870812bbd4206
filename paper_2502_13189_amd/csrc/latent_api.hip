// Host side of rotary positions and latent attention: argument validation, the layout of the caller's
// workspaces and the launches.  Nothing here allocates, synchronizes or reads device memory.
#include "api_common.h"
#include "latent_internal.h"
#include "rope_internal.h"

#include <cmath>
#include <initializer_list>
#include <type_traits>

using namespace moba;

namespace {

constexpr int64_t kMost = int64_t(1) << 31;
// Tokens times heads of a backward call: 16 threads each (Delta), in whole work-groups, are below a launch's 2^32.
constexpr int64_t kMostBackward = (int64_t(1) << 28) - 16;

struct Rows3 {
  char* data;
  int64_t st, sh;  // elements
  int64_t T, H, D;
  int64_t el;      // bytes of an element
};

// A [T, H, D] tensor (H 0: [T, D]), last dim contiguous, rows at multiples of `align` bytes.
moba_status check_rows(const moba_tensor* t, int dtype, bool heads, int64_t D, int64_t align, Rows3* v) {
  if (missing(t)) return MOBA_ERR_NULL;
  if (t->dtype != dtype) return MOBA_ERR_DTYPE;
  const int nd = heads ? 3 : 2;
  if (t->ndim != nd || t->shape[0] < 0 || (heads && t->shape[1] < 1)) return MOBA_ERR_SHAPE;
  if (t->shape[nd - 1] != D) return MOBA_ERR_UNSUPPORTED;
  v->el = dtype == MOBA_F32 ? 4 : 2;
  v->T = t->shape[0];
  v->H = heads ? t->shape[1] : 1;
  v->D = D;
  // (a stride over one index, or of an empty tensor, is not used)
  v->st = v->T > 1 ? t->stride[0] : 0;
  v->sh = heads && v->H > 1 && v->T > 0 ? t->stride[1] : 0;
  v->data = static_cast<char*>(t->data);
  if (v->T == 0) return MOBA_OK;
  if ((D > 1 && t->stride[nd - 1] != 1) || v->st < 0 || v->sh < 0) return MOBA_ERR_LAYOUT;
  if (reinterpret_cast<uintptr_t>(t->data) % align != 0 || v->st * v->el % align != 0 || v->sh * v->el % align != 0)
    return MOBA_ERR_LAYOUT;
  return MOBA_OK;
}

// A tensor the call writes: rows do not lie on each other.
moba_status check_out(const moba_tensor* t, int dtype, bool heads, int64_t D, int64_t align, Rows3* v) {
  const moba_status st = check_rows(t, dtype, heads, D, align, v);
  if (st != MOBA_OK) return st;
  if (v->T == 0) return MOBA_OK;
  const bool by_token = (v->T == 1 || v->st >= (v->H - 1) * v->sh + D) && (v->H == 1 || v->sh >= D);
  const bool by_head = (v->H == 1 || v->sh >= (v->T - 1) * v->st + D) && (v->T == 1 || v->st >= D);
  return by_token || by_head ? MOBA_OK : MOBA_ERR_LAYOUT;
}

bool same_rows(const Rows3& a, const Rows3& b) {
  return a.data == b.data && a.st == b.st && a.sh == b.sh && a.T == b.T && a.H == b.H && a.D == b.D;
}

// n bytes as one row.
Rows3 bytes_at(const void* p, int64_t n) {
  return Rows3{static_cast<char*>(const_cast<void*>(p)), 0, 0, n > 0, 1, n, 1};
}

// A contiguous tensor as one row of bytes.
Rows3 flat(const moba_tensor* t) {
  return bytes_at(t->data, numel(t) * (t->dtype == MOBA_I64 || t->dtype == MOBA_F64 ? 8 : t->dtype == MOBA_BF16 ? 2 : 4));
}

// Whether two views may share memory.  Views of one wider buffer (equal strides) share none if no
// row of one lies on a row of the other.
bool may_share(const Rows3& a, const Rows3& b) {
  if (a.T == 0 || b.T == 0) return false;
  const auto bytes = [](const Rows3& v) { return ((v.T - 1) * v.st + (v.H - 1) * v.sh + v.D) * v.el; };
  if (a.data + bytes(a) <= b.data || b.data + bytes(b) <= a.data) return false;
  if (a.el != b.el) {
    const auto in_bytes = [](const Rows3& v) { return Rows3{v.data, v.st * v.el, v.sh * v.el, v.T, v.H, v.D * v.el, 1}; };
    return may_share(in_bytes(a), in_bytes(b));
  }
  if ((b.data - a.data) % a.el != 0) return true;
  const int64_t st = a.T > 1 ? a.st : b.st, sh = a.H > 1 ? a.sh : b.sh;
  if ((a.T > 1 && b.T > 1 && a.st != b.st) || (a.H > 1 && b.H > 1 && a.sh != b.sh)) return true;
  const int64_t d = (b.data - a.data) / a.el;  // row (i, j) of b minus row (k, l) of a: d + (i - k) st + (j - l) sh
  const bool token_outer = st >= sh;
  const int64_t so = token_outer ? st : sh, si = token_outer ? sh : st;
  const int64_t oa = token_outer ? a.T : a.H, ob = token_outer ? b.T : b.H;
  const int64_t ia = token_outer ? a.H : a.T, ib = token_outer ? b.H : b.T;
  if (so < (std::max(ia, ib) - 1) * si + std::max(a.D, b.D)) return true;  // (rows of different outer indices mix)
  const auto floor_div = [](int64_t x, int64_t y) { return x >= 0 ? x / y : -((-x + y - 1) / y); };
  for (int64_t o = -1; o <= 1; o++) {
    const int64_t x = so ? std::min(std::max(floor_div(d, so) + o, -(ob - 1)), oa - 1) : 0, rem = d - x * so;
    for (int64_t i = -1; i <= 1; i++) {
      const int64_t y = si ? std::min(std::max(floor_div(rem, si) + i, -(ib - 1)), ia - 1) : 0;
      const int64_t at = rem - y * si;  // b's row begins `at` elements behind a's
      if (at < a.D && -at < b.D) return true;
    }
  }
  return false;
}

// Whether one of the outputs may share memory with an input or another output.
moba_status check_apart(std::initializer_list<const Rows3*> outs, std::initializer_list<const Rows3*> ins) {
  for (auto o = outs.begin(); o != outs.end(); o++) {
    for (const Rows3* i : ins)
      if (may_share(**o, *i)) return MOBA_ERR_LAYOUT;
    for (auto p = o + 1; p != outs.end(); p++)
      if (may_share(**o, **p)) return MOBA_ERR_LAYOUT;
  }
  return MOBA_OK;
}

// Whether an output may share memory with what says where its rows stand and how fast they turn.
moba_status check_apart(const Rows3& out, const moba_rotation* r) {
  for (const moba_tensor* t : {r->freqs, r->pos, r->cu_seqlens, r->start})
    if (t && may_share(out, flat(t))) return MOBA_ERR_LAYOUT;
  return MOBA_OK;
}

// Rotation of T rows with heads of D dims.
moba_status check_rotation(const moba_rotation* r, int64_t T, int64_t D, Rotation* out) {
  if (!r || missing(r->freqs)) return MOBA_ERR_NULL;
  if (r->freqs->dtype != MOBA_F64) return MOBA_ERR_DTYPE;
  if (r->freqs->ndim != 1 || r->freqs->shape[0] < 1) return MOBA_ERR_SHAPE;
  if (r->freqs->shape[0] > D / 2) return MOBA_ERR_SHAPE;
  if (r->freqs->shape[0] > 1 && r->freqs->stride[0] != 1) return MOBA_ERR_LAYOUT;
  if (reinterpret_cast<uintptr_t>(r->freqs->data) % 8 != 0) return MOBA_ERR_LAYOUT;
  *out = Rotation{};
  out->freqs = static_cast<const double*>(r->freqs->data);
  out->half = (int)r->freqs->shape[0];
  out->amplitude = r->amplitude;
  out->sign = 1.0f;
  moba_status st;
  if (r->pos) {
    if (r->cu_seqlens || r->start) return MOBA_ERR_SHAPE;  // one of the two
    if (missing(r->pos)) return MOBA_ERR_NULL;
    if (r->pos->dtype != MOBA_I32 && r->pos->dtype != MOBA_I64) return MOBA_ERR_DTYPE;
    if ((st = check_contig(r->pos, r->pos->dtype, 1, &T)) != MOBA_OK) return st;
    out->pos = r->pos->data;
    out->pos64 = r->pos->dtype == MOBA_I64;
    return MOBA_OK;
  }
  if (missing(r->cu_seqlens)) return MOBA_ERR_NULL;
  if (r->cu_seqlens->ndim != 1 || r->cu_seqlens->shape[0] < 1) return MOBA_ERR_SHAPE;
  const int64_t n = r->cu_seqlens->shape[0], S = n - 1;
  if ((st = check_contig(r->cu_seqlens, MOBA_I32, 1, &n)) != MOBA_OK) return st;
  if (S >= kMost) return MOBA_ERR_UNSUPPORTED;
  if (r->start) {
    if (missing(r->start)) return MOBA_ERR_NULL;
    if ((st = check_contig(r->start, MOBA_I32, 1, &S)) != MOBA_OK) return st;
    out->start = S ? static_cast<const int32_t*>(r->start->data) : nullptr;
  }
  out->cu = static_cast<const int32_t*>(r->cu_seqlens->data);
  out->S = (int)S;
  return MOBA_OK;
}

moba_status rope_impl(const moba_tensor* q, const moba_tensor* k, const moba_rotation* rot,
                      moba_tensor* q_out, moba_tensor* k_out, bool backward, hipStream_t stream) {
  if (missing(q) || missing(q_out) || (k && missing(k))) return MOBA_ERR_NULL;
  if (!k != !k_out || (k_out && missing(k_out))) return MOBA_ERR_NULL;
  if (q->dtype != MOBA_BF16 && q->dtype != MOBA_F32) return MOBA_ERR_DTYPE;
  if (q->ndim != 3) return MOBA_ERR_SHAPE;
  const int64_t T = q->shape[0], D = q->shape[2], el = q->dtype == MOBA_F32 ? 4 : 2;
  if (D < 2 || D > 4096) return MOBA_ERR_UNSUPPORTED;
  RopeArgs a{};
  moba_status st;
  if ((st = check_rotation(rot, T, D, &a.r)) != MOBA_OK) return st;
  const moba_tensor* in[2] = {q, k};
  const moba_tensor* out[2] = {q_out, k_out};
  const int n = k ? 2 : 1;
  Rows3 vi[2], vo[2];
  for (int i = 0; i < n; i++) {
    if ((st = check_rows(in[i], q->dtype, true, D, el, &vi[i])) != MOBA_OK) return st;
    if ((st = check_out(out[i], q->dtype, true, D, el, &vo[i])) != MOBA_OK) return st;
    if (vi[i].T != T || vo[i].T != T || vo[i].H != vi[i].H) return MOBA_ERR_SHAPE;
    if (vi[i].H >= 65536) return MOBA_ERR_UNSUPPORTED;
  }
  for (int i = 0; i < n; i++)
    for (int j = 0; j < n; j++)
      if (may_share(vo[i], vi[j]) && !(i == j && same_rows(vo[i], vi[j]))) return MOBA_ERR_LAYOUT;
  if (n == 2 && may_share(vo[0], vo[1])) return MOBA_ERR_LAYOUT;
  for (int i = 0; i < n; i++)
    if ((st = check_apart(vo[i], rot)) != MOBA_OK) return st;
  if (T >= kMost) return MOBA_ERR_UNSUPPORTED;
  if (T == 0 || (a.r.cu && a.r.S == 0)) return MOBA_OK;
  // the widest piece that divides the pairs and the head and that every row is aligned to
  int vec = (int)(16 / el);
  const auto fits = [&](const Rows3& v) {
    return reinterpret_cast<uintptr_t>(v.data) % (vec * el) == 0 && v.st % vec == 0 && v.sh % vec == 0;
  };
  for (; vec > 1; vec /= 2) {
    bool ok = a.r.half % vec == 0 && D % vec == 0;
    for (int i = 0; i < n; i++) ok = ok && fits(vi[i]) && fits(vo[i]);
    if (ok) break;
  }
  a.q = vi[0].data; a.q_st = vi[0].st; a.q_sh = vi[0].sh;
  a.qo = vo[0].data; a.qo_st = vo[0].st; a.qo_sh = vo[0].sh;
  a.Hq = (int)vi[0].H;
  a.copy = 2 * a.r.half < D && !same_rows(vi[0], vo[0]);
  if (n == 2) {
    a.k = vi[1].data; a.k_st = vi[1].st; a.k_sh = vi[1].sh;
    a.ko = vo[1].data; a.ko_st = vo[1].st; a.ko_sh = vo[1].sh;
    a.Hk = (int)vi[1].H;
    a.copy = a.copy || (2 * a.r.half < D && !same_rows(vi[1], vo[1]));
  }
  a.T = T;
  a.D = (int)D;
  if (backward) a.r.sign = -1.0f;
  Phase ph(backward ? "rope_back" : "rope", stream);
  MOBA_LAUNCH(launch_rope(el == 2, rot->interleaved != 0, vec, a, stream));
  return MOBA_OK;
}

// pages [N, P, 576] bf16, a page's rows contiguous
moba_status check_latent_pages(const moba_tensor* t, __hip_bfloat16** data, int64_t* sp, int* N, int* P) {
  if (missing(t)) return MOBA_ERR_NULL;
  if (t->dtype != MOBA_BF16) return MOBA_ERR_DTYPE;
  if (t->ndim != 3 || t->shape[0] < 1) return MOBA_ERR_SHAPE;
  const int64_t p = t->shape[1];
  if (t->shape[2] != kRow || p < kLatStep || p > 256 || p % kLatStep != 0 || t->shape[0] >= kMost)
    return MOBA_ERR_UNSUPPORTED;
  if (t->stride[2] != 1 || t->stride[1] != kRow || (t->shape[0] > 1 && t->stride[0] < p * kRow) ||
      t->stride[0] % 8 != 0 || (reinterpret_cast<uintptr_t>(t->data) & 15) != 0)
    return MOBA_ERR_LAYOUT;
  *data = static_cast<__hip_bfloat16*>(t->data);
  *sp = t->stride[0];
  *N = (int)t->shape[0];
  *P = (int)p;
  return MOBA_OK;
}

// The pool's rows, as check_apart takes them.
Rows3 pool_rows(const __hip_bfloat16* data, int64_t sp, int N, int P) {
  return Rows3{reinterpret_cast<char*>(const_cast<__hip_bfloat16*>(data)), N > 1 ? sp : 0, kRow, N, P, kRow, 2};
}

// q, k, k_rope, v and cu_seqlens of the expanded form (in: those five)
moba_status check_latent(const moba_tensor* q, const moba_tensor* k, const moba_tensor* kr, const moba_tensor* v,
                         const moba_tensor* cu, float scale, LatentArgs* a, Rows3 (&in)[5]) {
  Rows3 &vq = in[0], &vk = in[1], &vr = in[2], &vv = in[3];
  moba_status st;
  if ((st = check_rows(q, MOBA_BF16, true, kQk, 16, &vq)) != MOBA_OK) return st;
  if ((st = check_rows(k, MOBA_BF16, true, kNope, 16, &vk)) != MOBA_OK) return st;
  if ((st = check_rows(kr, MOBA_BF16, false, kRopeDim, 16, &vr)) != MOBA_OK) return st;
  if ((st = check_rows(v, MOBA_BF16, true, kNope, 16, &vv)) != MOBA_OK) return st;
  if (missing(cu)) return MOBA_ERR_NULL;
  if (cu->dtype != MOBA_I32) return MOBA_ERR_DTYPE;
  if (cu->ndim != 1 || cu->shape[0] < 1) return MOBA_ERR_SHAPE;
  if (cu->shape[0] > 1 && cu->stride[0] != 1) return MOBA_ERR_LAYOUT;
  in[4] = flat(cu);
  const int64_t T = vq.T, H = vq.H, S = cu->shape[0] - 1;
  if (vk.T != T || vr.T != T || vv.T != T || vk.H != H || vv.H != H) return MOBA_ERR_SHAPE;
  // launches of less than 2^32 threads; rows within 32 bits of a tile's first
  if (T >= kMost || H >= 65536 || S >= kMost || T * H >= int64_t(1) << 28 ||
      (latent_places_bound(T, S) * H + 8) * 512 >= int64_t(1) << 32)
    return MOBA_ERR_UNSUPPORTED;
  for (const Rows3* x : {&vq, &vk, &vr, &vv})
    if (x->st >= int64_t(1) << 24) return MOBA_ERR_UNSUPPORTED;
  a->q = reinterpret_cast<const __hip_bfloat16*>(vq.data); a->q_st = vq.st; a->q_sh = vq.sh;
  a->k = reinterpret_cast<const __hip_bfloat16*>(vk.data); a->k_st = vk.st; a->k_sh = vk.sh;
  a->kr = reinterpret_cast<const __hip_bfloat16*>(vr.data); a->kr_st = vr.st;
  a->v = reinterpret_cast<const __hip_bfloat16*>(vv.data); a->v_st = vv.st; a->v_sh = vv.sh;
  a->cu = static_cast<const int32_t*>(cu->data);
  a->S = (int)S;
  a->H = (int)H;
  a->T = T;
  a->scale = scale;
  a->scale_log2 = (float)(1.4426950408889634 * (double)scale);
  return MOBA_OK;
}

moba_status check_scale(float scale) { return std::isfinite(scale) && scale > 0.0f ? MOBA_OK : MOBA_ERR_UNSUPPORTED; }

size_t backward_layout(int64_t T, int64_t H, char* base, LatentArgs* a) {
  size_t off = 0;
  const auto take = [&](auto** p, int64_t n) {
    *p = reinterpret_cast<std::remove_reference_t<decltype(*p)>>(base + off);
    off += ((size_t)n * sizeof(**p) + 15) / 16 * 16;
  };
  take(&a->ld, T * H);
  take(&a->dkr_part, T * H * kRopeDim);
  return off;
}

struct LatentShape {
  int heads, groups, shares;
};

moba_status decode_shape(int64_t S, int64_t W, int64_t H, int64_t P, LatentShape* d) {
  if (S < 0 || W < 1 || H < 1) return MOBA_ERR_SHAPE;
  if (P < kLatStep || P > 256 || P % kLatStep != 0) return MOBA_ERR_UNSUPPORTED;
  if (H > 4096 || S >= kMost || W >= kMost || S * W >= (int64_t(1) << 30) / (P / kLatStep) ||
      S * H >= int64_t(1) << 23)
    return MOBA_ERR_UNSUPPORTED;
  // heads of a group: 64, what a work-group's registers hold, read a row the fewest times; but fewer where the batch
  // (as far as the table says) has so little work that a step's length counts, and no more than there are.  16, 32 and
  // 64, us a call: 8000 tokens, 128 heads 20.0, 26.0, 37.3; 64000, 64 heads 35.7, 35.4, 46.5; 64 x 1000, 64 heads
  // 31, 33, 37; 64000, 128 heads 52.5, 42.5, 44.4; 192000, 64 heads 73, 59, 66; 128000, 128 heads 88, 65, 60; 64000,
  // 256 heads 87, 63, 57; 64 x 4000, 64 heads 98 (32), 90 (64).
  const int64_t work = S * W * P * H;  // (below 2^48)
  const int most = work <= 3 << 20 ? 16 : work <= 3 << 22 ? 32 : 64;
  d->heads = H <= 16 ? 16 : H <= 32 ? std::min(most, 32) : most;
  d->groups = (int)ceil_div(H, d->heads);
  const int64_t steps = std::max<int64_t>(1, S * W * (P / kLatStep));  // at most
  d->shares = (int)std::min<int64_t>(std::max(1, kLatGroups / d->groups), steps);
  return MOBA_OK;
}

size_t decode_layout(const LatentShape& d, int64_t S, char* base, LatentDecodeArgs* a) {
  size_t off = 0;
  const auto take = [&](auto** p, int64_t n) {
    *p = reinterpret_cast<std::remove_reference_t<decltype(*p)>>(base + off);
    off += ((size_t)n * sizeof(**p) + 15) / 16 * 16;
  };
  const int64_t rows = (int64_t)d.shares * 2 * d.groups * d.heads;
  take(&a->part_o, rows * kRank);
  take(&a->part_ml, rows);
  take(&a->first, S + 1);
  return off;
}

}  // namespace

extern "C" {

moba_status moba_rope(const moba_tensor* q, const moba_tensor* k, const moba_rotation* rot, moba_tensor* q_out,
                      moba_tensor* k_out, hipStream_t stream) {
  return rope_impl(q, k, rot, q_out, k_out, false, stream);
}

moba_status moba_rope_backward(const moba_tensor* dq_out, const moba_tensor* dk_out, const moba_rotation* rot,
                               moba_tensor* dq, moba_tensor* dk, hipStream_t stream) {
  return rope_impl(dq_out, dk_out, rot, dq, dk, true, stream);
}

moba_status moba_latent_forward(const moba_tensor* q, const moba_tensor* k, const moba_tensor* k_rope,
                                const moba_tensor* v, const moba_tensor* cu_seqlens, float scale, moba_tensor* out,
                                moba_tensor* lse, hipStream_t stream) {
  LatentArgs a{};
  Rows3 in[5], vo;
  moba_status st;
  if (missing(out) || missing(lse)) return MOBA_ERR_NULL;
  if ((st = check_latent(q, k, k_rope, v, cu_seqlens, scale, &a, in)) != MOBA_OK) return st;
  if ((st = check_out(out, MOBA_BF16, true, kNope, 16, &vo)) != MOBA_OK) return st;
  if (vo.T != a.T || vo.H != a.H) return MOBA_ERR_SHAPE;
  const int64_t ls[2] = {a.H, a.T};
  if ((st = check_contig(lse, MOBA_F32, 2, ls)) != MOBA_OK) return st;
  const Rows3 vl = flat(lse);
  if ((st = check_apart({&vo, &vl}, {&in[0], &in[1], &in[2], &in[3], &in[4]})) != MOBA_OK) return st;
  if ((st = check_scale(scale)) != MOBA_OK) return st;
  if (a.T == 0 || a.S == 0) return MOBA_OK;
  a.out = reinterpret_cast<__hip_bfloat16*>(vo.data); a.o_st = vo.st; a.o_sh = vo.sh;
  a.lse = static_cast<float*>(lse->data);
  Phase ph("latent_fwd", stream);
  MOBA_LAUNCH(launch_latent_forward(a, stream));
  return MOBA_OK;
}

size_t moba_latent_backward_workspace_bytes(int64_t T, int32_t H) {
  if (T < 1 || H < 1 || T >= kMost || T * H > kMostBackward) return 0;
  LatentArgs a{};
  return backward_layout(T, H, nullptr, &a);
}

moba_status moba_latent_backward(const moba_tensor* q, const moba_tensor* k, const moba_tensor* k_rope,
                                 const moba_tensor* v, const moba_tensor* cu_seqlens, float scale,
                                 const moba_tensor* out, const moba_tensor* lse, const moba_tensor* dout,
                                 moba_tensor* dq, moba_tensor* dk, moba_tensor* dk_rope, moba_tensor* dv,
                                 void* workspace, size_t workspace_bytes, hipStream_t stream) {
  LatentArgs a{};
  Rows3 in[5], vo, vd, gq, gk, gr, gv;
  moba_status st;
  if (missing(lse)) return MOBA_ERR_NULL;
  if ((st = check_latent(q, k, k_rope, v, cu_seqlens, scale, &a, in)) != MOBA_OK) return st;
  if ((st = check_rows(out, MOBA_BF16, true, kNope, 16, &vo)) != MOBA_OK) return st;
  if ((st = check_rows(dout, MOBA_BF16, true, kNope, 16, &vd)) != MOBA_OK) return st;
  if ((st = check_out(dq, MOBA_BF16, true, kQk, 16, &gq)) != MOBA_OK) return st;
  if ((st = check_out(dk, MOBA_BF16, true, kNope, 16, &gk)) != MOBA_OK) return st;
  if ((st = check_out(dk_rope, MOBA_BF16, false, kRopeDim, 16, &gr)) != MOBA_OK) return st;
  if ((st = check_out(dv, MOBA_BF16, true, kNope, 16, &gv)) != MOBA_OK) return st;
  for (const Rows3* x : {&vo, &vd, &gq, &gk, &gv})
    if (x->T != a.T || x->H != a.H) return MOBA_ERR_SHAPE;
  if (gr.T != a.T) return MOBA_ERR_SHAPE;
  if (vd.st >= int64_t(1) << 24 || a.T * a.H > kMostBackward) return MOBA_ERR_UNSUPPORTED;
  const int64_t ls[2] = {a.H, a.T};
  if ((st = check_contig(lse, MOBA_F32, 2, ls)) != MOBA_OK) return st;
  const Rows3 vl = flat(lse);
  if ((st = check_apart({&gq, &gk, &gr, &gv}, {&in[0], &in[1], &in[2], &in[3], &in[4], &vo, &vl, &vd})) != MOBA_OK)
    return st;
  if ((st = check_scale(scale)) != MOBA_OK) return st;
  if (a.T == 0 || a.S == 0) return MOBA_OK;
  if (!workspace) return MOBA_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 15) != 0) return MOBA_ERR_LAYOUT;
  const size_t need = backward_layout(a.T, a.H, static_cast<char*>(workspace), &a);
  if (workspace_bytes < need) return MOBA_ERR_NO_MEMORY;
  const Rows3 ws = bytes_at(workspace, (int64_t)need);
  if ((st = check_apart({&ws}, {&in[0], &in[1], &in[2], &in[3], &in[4], &vo, &vl, &vd, &gq, &gk, &gr, &gv})) != MOBA_OK)
    return st;
  a.out = reinterpret_cast<__hip_bfloat16*>(vo.data); a.o_st = vo.st; a.o_sh = vo.sh;
  a.lse = static_cast<float*>(lse->data);
  a.dout = reinterpret_cast<const __hip_bfloat16*>(vd.data); a.do_st = vd.st; a.do_sh = vd.sh;
  a.dq = reinterpret_cast<__hip_bfloat16*>(gq.data); a.dq_st = gq.st; a.dq_sh = gq.sh;
  a.dk = reinterpret_cast<__hip_bfloat16*>(gk.data); a.dk_st = gk.st; a.dk_sh = gk.sh;
  a.dkr = reinterpret_cast<__hip_bfloat16*>(gr.data); a.dkr_st = gr.st;
  a.dv = reinterpret_cast<__hip_bfloat16*>(gv.data); a.dv_st = gv.st; a.dv_sh = gv.sh;
  {
    Phase ph("latent_delta", stream);
    MOBA_LAUNCH(launch_latent_delta(a, stream));
  }
  // Few work-groups last as long as their longest chain of tiles, and both sides take about that in one launch.  One
  // after the other and together, us a call: 8192 tokens, 1 head 422, 251; 4096, 10 heads 387, 256; 2048, 32 heads 235,
  // 210; 256, 4 heads 36, 29; 5 sequences, 4583 tokens, 10 heads 192, 143, 32 heads (1280 work-groups) 402, 407; 8192,
  // 32 heads 2321, 2597 (the query side is the slower for the other's registers, heads are spread over the XCDs).
  // Sequences of a tile or so have no chains: 40 x 64 tokens, 4 heads 28, 34.
  if (a.S <= kLatRankedSeqs && a.T >= (int64_t)kLatKeys * a.S && latent_places_bound(a.T, a.S) * a.H <= kLatBoth) {
    {
      Phase ph("latent_first", stream);
      MOBA_LAUNCH(launch_latent_first(a, stream));
    }
    Phase ph("latent_both", stream);
    MOBA_LAUNCH(launch_latent_both(a, stream));
  } else {
    {
      Phase ph("latent_dq", stream);
      MOBA_LAUNCH(launch_latent_dq(a, stream));
    }
    Phase ph("latent_dkdv", stream);
    MOBA_LAUNCH(launch_latent_dkdv(a, stream));
  }
  Phase ph("latent_dkr", stream);
  MOBA_LAUNCH(launch_latent_dkr(a, stream));
  return MOBA_OK;
}

moba_status moba_latent_write(const moba_tensor* c, const moba_tensor* k_rope, const moba_tensor* slots,
                              const moba_rotation* rot, moba_tensor* pages, hipStream_t stream) {
  LatentWriteArgs a{};
  Rows3 vc, vr;
  moba_status st;
  if (missing(slots)) return MOBA_ERR_NULL;
  if ((st = check_latent_pages(pages, &a.pages, &a.p_sp, &a.N, &a.P)) != MOBA_OK) return st;
  if ((st = check_rows(c, MOBA_BF16, false, kRank, 16, &vc)) != MOBA_OK) return st;
  if ((st = check_rows(k_rope, MOBA_BF16, false, kRopeDim, 16, &vr)) != MOBA_OK) return st;
  const int64_t T = vc.T;
  if (vr.T != T) return MOBA_ERR_SHAPE;
  if ((st = check_contig(slots, MOBA_I64, 1, &T)) != MOBA_OK) return st;
  if (T > 0) {  // (tokens as the rows of one page: such a view may lie between the pages of a wider pool)
    const Rows3 pool = pool_rows(a.pages, a.p_sp, a.N, a.P);
    const Rows3 one_c{vc.data, 0, vc.st, 1, T, kRank, 2}, one_r{vr.data, 0, vr.st, 1, T, kRopeDim, 2};
    const Rows3 vs = flat(slots);
    if ((st = check_apart({&pool}, {&one_c, &one_r, &vs})) != MOBA_OK) return st;
  }
  if (rot) {
    if ((st = check_rotation(rot, T, kRopeDim, &a.r)) != MOBA_OK) return st;
    if (T > 0 && (st = check_apart(pool_rows(a.pages, a.p_sp, a.N, a.P), rot)) != MOBA_OK) return st;
    if (a.r.half != kRopeDim / 2) return MOBA_ERR_SHAPE;
  }
  if (T >= int64_t(1) << 28) return MOBA_ERR_UNSUPPORTED;  // (8 threads a token, 2^32 of a launch)
  if (T == 0 || (a.r.cu && a.r.S == 0)) return MOBA_OK;
  a.c = reinterpret_cast<const __hip_bfloat16*>(vc.data); a.c_st = vc.st;
  a.kr = reinterpret_cast<const __hip_bfloat16*>(vr.data); a.kr_st = vr.st;
  a.slots = static_cast<const int64_t*>(slots->data);
  a.T = T;
  a.rotate = rot != nullptr;
  Phase ph("latent_write", stream);
  MOBA_LAUNCH(launch_latent_write(rot && rot->interleaved != 0, a, stream));
  return MOBA_OK;
}

size_t moba_latent_decode_workspace_bytes(int64_t S, int64_t W, int32_t H, int32_t page_size) {
  LatentShape d{};
  if (decode_shape(S, W, H, page_size, &d) != MOBA_OK || S == 0) return 0;
  LatentDecodeArgs a{};
  return decode_layout(d, S, nullptr, &a);
}

moba_status moba_latent_decode(const moba_tensor* q_c, const moba_tensor* q_rope, const moba_tensor* pages,
                               const moba_tensor* table, const moba_tensor* lens, float scale, moba_tensor* out,
                               moba_tensor* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  LatentDecodeArgs a{};
  Rows3 vc, vr, vo;
  moba_status st;
  if (missing(table) || missing(lens) || missing(lse)) return MOBA_ERR_NULL;
  __hip_bfloat16* pool;
  if ((st = check_latent_pages(pages, &pool, &a.p_sp, &a.N, &a.P)) != MOBA_OK) return st;
  if ((st = check_rows(q_c, MOBA_BF16, true, kRank, 16, &vc)) != MOBA_OK) return st;
  if ((st = check_rows(q_rope, MOBA_BF16, true, kRopeDim, 16, &vr)) != MOBA_OK) return st;
  if ((st = check_out(out, MOBA_BF16, true, kRank, 16, &vo)) != MOBA_OK) return st;
  const int64_t S = vc.T, H = vc.H;
  if (vr.T != S || vr.H != H || vo.T != S || vo.H != H) return MOBA_ERR_SHAPE;
  const int64_t ls[2] = {H, S};
  if ((st = check_contig(lse, MOBA_F32, 2, ls)) != MOBA_OK) return st;
  if (table->dtype != MOBA_I32) return MOBA_ERR_DTYPE;
  if (table->ndim != 2 || table->shape[0] != S || table->shape[1] < 1) return MOBA_ERR_SHAPE;
  if (S > 0 && ((table->shape[1] > 1 && table->stride[1] != 1) || (S > 1 && table->stride[0] < table->shape[1])))
    return MOBA_ERR_LAYOUT;
  if ((st = check_contig(lens, MOBA_I32, 1, &S)) != MOBA_OK) return st;
  const Rows3 vp = pool_rows(pool, a.p_sp, a.N, a.P), vn = flat(lens), vl = flat(lse);
  const Rows3 vt{static_cast<char*>(table->data), S > 1 ? table->stride[0] : 0, 0, S, 1, table->shape[1], 4};
  if ((st = check_apart({&vo, &vl}, {&vc, &vr, &vp, &vt, &vn})) != MOBA_OK) return st;
  if ((st = check_scale(scale)) != MOBA_OK) return st;
  LatentShape d{};
  if ((st = decode_shape(S, table->shape[1], H, a.P, &d)) != MOBA_OK) return st;
  if (S == 0) return MOBA_OK;
  if (!workspace) return MOBA_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 15) != 0) return MOBA_ERR_LAYOUT;
  const size_t need = decode_layout(d, S, static_cast<char*>(workspace), &a);
  if (workspace_bytes < need) return MOBA_ERR_NO_MEMORY;
  const Rows3 ws = bytes_at(workspace, (int64_t)need);
  if ((st = check_apart({&ws}, {&vc, &vr, &vp, &vt, &vn, &vo, &vl})) != MOBA_OK) return st;
  a.qc = reinterpret_cast<const __hip_bfloat16*>(vc.data); a.qc_ss = vc.st; a.qc_sh = vc.sh;
  a.qr = reinterpret_cast<const __hip_bfloat16*>(vr.data); a.qr_ss = vr.st; a.qr_sh = vr.sh;
  a.pages = pool;
  a.table = static_cast<const int32_t*>(table->data);
  a.t_ss = S > 1 ? table->stride[0] : 0;
  a.lens = static_cast<const int32_t*>(lens->data);
  a.S = (int)S;
  a.W = (int)table->shape[1];
  a.H = (int)H;
  a.scale_log2 = (float)(1.4426950408889634 * (double)scale);
  a.out = reinterpret_cast<__hip_bfloat16*>(vo.data); a.o_ss = vo.st; a.o_sh = vo.sh;
  a.lse = static_cast<float*>(lse->data);
  a.shares = d.shares;
  a.groups = d.groups;
  {
    Phase ph("latent_decode", stream);
    MOBA_LAUNCH(launch_latent_decode(d.heads, a, stream));
  }
  Phase ph("latent_join", stream);
  MOBA_LAUNCH(launch_latent_join(d.heads, a, stream));
  return MOBA_OK;
}

}  // extern "C"
