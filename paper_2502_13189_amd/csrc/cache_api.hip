// Host side of the paged 8-bit cache: argument validation, the layout of the caller's
// workspace and the launches.  Nothing here allocates, synchronizes or reads device memory.
#include "api_common.h"
#include "cache_internal.h"
#include "decode_internal.h"

#include <cmath>
#include <type_traits>

using namespace moba;

namespace {

bool page_size_ok(int64_t P) {
  return P >= kCacheTile && P <= kCacheMaxPage && P % kCacheTile == 0;
}

// A [shape] tensor of the pool whose last two dims are contiguous, in 16-byte steps.
moba_status check_pages(const moba_tensor* t, int64_t N, int64_t Hkv, int64_t rows, int64_t cols,
                        uint8_t** data, int64_t* sp, int64_t* sh) {
  if (t->dtype != MOBA_F8E4M3) return MOBA_ERR_DTYPE;
  if (t->ndim != 4 || t->shape[0] != N || t->shape[1] != Hkv || t->shape[2] != rows ||
      t->shape[3] != cols)
    return MOBA_ERR_SHAPE;
  if (t->stride[3] != 1 || t->stride[2] != cols || t->stride[0] < 0 || t->stride[1] < 0 ||
      t->stride[0] % 16 != 0 || t->stride[1] % 16 != 0 ||
      (reinterpret_cast<uintptr_t>(t->data) & 15) != 0)
    return MOBA_ERR_LAYOUT;
  *data = static_cast<uint8_t*>(t->data);
  *sp = t->stride[0];
  *sh = t->stride[1];
  return MOBA_OK;
}

moba_status check_cache(const moba_cache* c, CachePool* p) {
  if (!c || missing(c->k) || missing(c->v) || missing(c->k_scale) || missing(c->v_scale) ||
      missing(c->k_sum))
    return MOBA_ERR_NULL;
  if (c->k->dtype != MOBA_F8E4M3) return MOBA_ERR_DTYPE;
  if (c->k->ndim != 4 || c->k->shape[0] < 1 || c->k->shape[1] < 1) return MOBA_ERR_SHAPE;
  const int64_t N = c->k->shape[0], Hkv = c->k->shape[1], P = c->k->shape[2];
  if (c->k->shape[3] != kHeadDim || !page_size_ok(P)) return MOBA_ERR_UNSUPPORTED;
  if (N >= (int64_t(1) << 31) || N * (P / kCacheTile) >= (int64_t(1) << 32) ||
      Hkv >= (int64_t(1) << 20))
    return MOBA_ERR_UNSUPPORTED;
  moba_status st;
  if ((st = check_pages(c->k, N, Hkv, P, kHeadDim, &p->k, &p->k_sp, &p->k_sh)) != MOBA_OK) return st;
  if ((st = check_pages(c->v, N, Hkv, P / kCacheTile * kHeadDim, kCacheTile, &p->v, &p->v_sp,
                        &p->v_sh)) != MOBA_OK)
    return st;
  const int64_t sums[3] = {N, Hkv, kHeadDim};
  if ((st = check_contig(c->k_scale, MOBA_F32, 2, sums)) != MOBA_OK) return st;
  if ((st = check_contig(c->v_scale, MOBA_F32, 2, sums)) != MOBA_OK) return st;
  if ((st = check_contig(c->k_sum, MOBA_F32, 3, sums)) != MOBA_OK) return st;
  if ((reinterpret_cast<uintptr_t>(c->k_sum->data) & 15) != 0) return MOBA_ERR_LAYOUT;
  p->k_scale = static_cast<float*>(c->k_scale->data);
  p->v_scale = static_cast<float*>(c->v_scale->data);
  p->k_sum = static_cast<float*>(c->k_sum->data);
  p->N = (int)N;
  p->Hkv = (int)Hkv;
  p->P = (int)P;
  return MOBA_OK;
}

// table [S, W] i32, rows contiguous
moba_status check_table(const moba_tensor* t, int64_t S) {
  if (t->dtype != MOBA_I32) return MOBA_ERR_DTYPE;
  if (t->ndim != 2 || t->shape[0] != S || t->shape[1] < 1) return MOBA_ERR_SHAPE;
  if (S * t->shape[1] >= (int64_t(1) << 31)) return MOBA_ERR_UNSUPPORTED;
  if (S == 0) return MOBA_OK;  // (strides of an empty tensor are irrelevant)
  if ((t->shape[1] > 1 && t->stride[1] != 1) || (S > 1 && t->stride[0] < t->shape[1]))
    return MOBA_ERR_LAYOUT;
  return MOBA_OK;
}

struct DecodeShape {
  int64_t S, W;
  int Hq, Hkv, P, B, topk;
  bool full, rows;          // rows: one launch, a work-group per (request, kv-head)
  int nblk, parts;          // MoBA
  int64_t most;             // 64-key steps of a row at most
  int shares, gate_shares;
};

// What a call of these sizes takes; fills the workspace's pointers from `base` (which may
// be null) and returns its bytes.
size_t decode_layout(const DecodeShape& d, char* base, CacheDecodeArgs* a) {
  if (d.rows) return 16;  // (unused, but the call's workspace is checked alike)
  size_t off = 0;
  const auto take = [&](auto** p, int64_t n) {
    *p = reinterpret_cast<std::remove_reference_t<decltype(*p)>>(base + off);
    off += ((size_t)n * sizeof(**p) + 15) / 16 * 16;
  };
  const int64_t G = d.Hq / d.Hkv;
  const int64_t partials = d.full ? (int64_t)d.shares * 2 * d.Hkv : d.parts > 1 ? d.S * d.Hkv * d.parts : 0;
  take(&a->part_o, partials * G * kHeadDim);
  take(&a->part_ml, partials * G);
  if (d.full) take(&a->join, std::min<int64_t>(d.S, d.shares) * d.Hkv);
  else take(&a->score, d.topk > 1 ? d.S * d.Hq * d.nblk : 0);
  return off;
}

// Whether a work-group takes each (request, kv-head) by itself.  It needs one launch instead
// of two (MoBA: three) and no joins, but a row is then one CU's, about 0.3 us per 64-key
// step, so a row's most (what its table row can hold, MoBA: select) is held against what
// the other way takes: its launches, while there is little to do, and the batch's share
// of the chip where there is much.  Whole calls, split and by rows, all rows full:
//   full  64 tokens .. 1024, up to 128 rows        11.1 .. 13.5 and 7.4 .. 11.3 us
//         2048: 16 rows 11.6, 16.0; 128 rows 18.6, 17.6 (ragged 12.5, 15.0); 2048 rows 187, 183
//         4096: 16 rows 13.0, 26.1; 512 rows 99, 94 (ragged 28, 35); 8192: 512 rows 185, 182
//   MoBA (256, top-4: up to 52 steps)  2048: 2 rows 16.4, 18.7 (ragged 13.4, 7.7), 64 rows 19.8,
//         20.8; 4096: 128 rows 30.1, 31.0, 2048 rows 272, 255; 8192: 128 rows 34.6, 36.2 (ragged
//         23.7, 28.9), 512 rows 95, 91
bool rows_in_one(const DecodeShape& d) {
  const int64_t rows = d.S * d.Hkv, held = d.W * (d.P / kCacheTile);
  if (d.full) return held <= std::min<int64_t>(std::max<int64_t>(rows / 4, 16), 64);
  if (d.nblk > kCacheRowBlocks) return false;
  // (a page's k_sum is 1/32 of a step's bytes)
  return d.most + d.W / 32 <= std::min<int64_t>(std::max<int64_t>(rows / 3, 34), 256);
}

// MoBA: work-groups for a (request, kv-head), whose waves have a step or more.  (Blocks of
// 1024, top-4; 256, 512, 768, 1024 work-groups: 8 ragged requests 42.4, 42.2, 42.7, 45.5 us, 32 x
// 65536 tokens 181, 186, 189, 185, ragged 103, 69, 71, 62; 1M tokens, blocks of 4096, top-12, 84.2,
// 84.9, 87.4, 90.9.  At most 64, 256, 1024 steps: 64 requests of 32768 tokens 310, 312, 312, ragged
// 107, 148, 148: a batch of this kind alone would be better off with 64.)
int parts_of(int64_t rows, int64_t most) {
  if (rows == 0 || rows >= int64_t(1) << 19) return 1;  // (as far as the grids go)
  const int64_t n = std::max(ceil_div(kCachePartGroups, rows), ceil_div(most, kCachePartSteps));
  return (int)std::max<int64_t>(1, std::min<int64_t>({n, ceil_div(most, 4), kCacheWaves}));
}

// Checks the sizes and settles how the call runs.
moba_status decode_shape(int64_t S, int64_t W, int64_t Hq, int64_t Hkv, int64_t P, int32_t block_size,
                         int32_t topk, DecodeShape* d) {
  if (S < 0 || W < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return MOBA_ERR_SHAPE;
  if (!page_size_ok(P) || Hq / Hkv > kDecodeMaxGroup) return MOBA_ERR_UNSUPPORTED;
  if (topk < 0) return MOBA_ERR_TOPK;
  if (topk > 0 && (block_size < 1 || block_size % P != 0)) return MOBA_ERR_BLOCK_SIZE;
  if (Hq >= (int64_t(1) << 20) || W >= (int64_t(1) << 31) || S >= (int64_t(1) << 31) ||
      S * W >= (int64_t(1) << 31) || S * Hq >= (int64_t(1) << 31) ||
      S * W * (P / kCacheTile) >= (int64_t(1) << 30) / Hkv || S * Hkv >= (int64_t(1) << 23))
    return MOBA_ERR_UNSUPPORTED;  // (the last: a launch's 2^32 work items)
  d->S = S;
  d->W = W;
  d->Hq = (int)Hq;
  d->Hkv = (int)Hkv;
  d->P = (int)P;
  const int64_t nblk = topk > 0 ? ceil_div(W * P, block_size) : 1;
  d->full = topk == 0 || topk >= nblk;
  d->B = d->full ? 0 : block_size;
  d->topk = d->full ? 0 : topk;
  if (!d->full && nblk > kMaxBlocksPerSeq) return MOBA_ERR_UNSUPPORTED;
  d->nblk = (int)nblk;
  d->most = W * (P / kCacheTile);
  if (!d->full)  // (a kv-head's heads may choose different blocks)
    d->most = std::min<int64_t>(d->most, std::min<int64_t>(nblk, Hq / Hkv * (topk - 1) + 1) * (block_size / kCacheTile));
  d->rows = rows_in_one(*d);
  const int64_t steps = S * W * (P / kCacheTile);  // at most, of a kv-head
  d->shares = (int)std::min<int64_t>(std::max<int64_t>(1, kCacheWaves / Hkv), std::max<int64_t>(steps, 1));
  d->parts = d->full ? 0 : parts_of(S * Hkv, d->most);
  d->gate_shares = (int)std::min<int64_t>(std::max<int64_t>(1, kCacheGateWaves / Hkv),
                                          std::max<int64_t>(S * nblk, 1));
  return MOBA_OK;
}

}  // namespace

extern "C" {

moba_status moba_cache_plan(const moba_tensor* add, const moba_tensor* lens, moba_tensor* table,
                            moba_tensor* free_pages, const moba_tensor* num_free,
                            int32_t page_size, moba_tensor* lens_out, moba_tensor* num_free_out,
                            moba_tensor* cu_new, moba_tensor* slots, moba_tensor* refused,
                            hipStream_t stream) {
  if (missing(add) || missing(lens) || missing(table) || missing(free_pages) || missing(num_free) ||
      missing(lens_out) || missing(num_free_out) || missing(cu_new) || missing(slots) ||
      missing(refused))
    return MOBA_ERR_NULL;
  if (add->dtype != MOBA_I32 || free_pages->dtype != MOBA_I32 || slots->dtype != MOBA_I64)
    return MOBA_ERR_DTYPE;
  if (add->ndim != 1 || free_pages->ndim != 1 || slots->ndim != 1 || add->shape[0] < 0 ||
      free_pages->shape[0] < 0 || slots->shape[0] < 0)
    return MOBA_ERR_SHAPE;
  const int64_t S = add->shape[0], N = free_pages->shape[0], T = slots->shape[0];
  const int64_t one = 1, s1 = S + 1;
  moba_status st;
  if ((st = check_contig(add, MOBA_I32, 1, &S)) != MOBA_OK) return st;
  if ((st = check_contig(lens, MOBA_I32, 1, &S)) != MOBA_OK) return st;
  if ((st = check_contig(lens_out, MOBA_I32, 1, &S)) != MOBA_OK) return st;
  if ((st = check_table(table, S)) != MOBA_OK) return st;
  if ((st = check_contig(free_pages, MOBA_I32, 1, &N)) != MOBA_OK) return st;
  if ((st = check_contig(num_free, MOBA_I32, 1, &one)) != MOBA_OK) return st;
  if ((st = check_contig(num_free_out, MOBA_I32, 1, &one)) != MOBA_OK) return st;
  if ((st = check_contig(cu_new, MOBA_I32, 1, &s1)) != MOBA_OK) return st;
  if ((st = check_contig(slots, MOBA_I64, 1, &T)) != MOBA_OK) return st;
  if ((st = check_contig(refused, MOBA_I32, 1, &one)) != MOBA_OK) return st;
  if (page_size < 1) return MOBA_ERR_BLOCK_SIZE;
  if (!page_size_ok(page_size) || S > kPlanMaxRequests || N >= (int64_t(1) << 31) ||
      T >= (int64_t(1) << 31))
    return MOBA_ERR_UNSUPPORTED;
  CachePlanArgs a{};
  a.add = static_cast<const int32_t*>(add->data);
  a.lens = static_cast<const int32_t*>(lens->data);
  a.table = static_cast<int32_t*>(table->data);
  a.t_ss = table->stride[0];
  a.free_pages = static_cast<int32_t*>(free_pages->data);
  a.num_free = static_cast<const int32_t*>(num_free->data);
  a.lens_out = static_cast<int32_t*>(lens_out->data);
  a.num_free_out = static_cast<int32_t*>(num_free_out->data);
  a.cu = static_cast<int32_t*>(cu_new->data);
  a.slots = static_cast<int64_t*>(slots->data);
  a.refused = static_cast<int32_t*>(refused->data);
  a.S = (int)S;
  a.W = (int)table->shape[1];
  a.N = (int)N;
  a.P = page_size;
  a.T = T;
  Phase ph("cache_plan", stream);
  MOBA_LAUNCH(launch_cache_plan(a, stream));
  return MOBA_OK;
}

moba_status moba_cache_write(const moba_tensor* k, const moba_tensor* v, const moba_tensor* slots,
                             const moba_cache* cache, hipStream_t stream) {
  if (missing(k) || missing(v) || missing(slots)) return MOBA_ERR_NULL;
  CacheWriteArgs a{};
  moba_status st;
  if ((st = check_cache(cache, &a.c)) != MOBA_OK) return st;
  if (k->dtype != MOBA_BF16 && k->dtype != MOBA_F32) return MOBA_ERR_DTYPE;
  View vk, vv;
  if ((st = check_3d(k, k->dtype, &vk)) != MOBA_OK) return st;
  if ((st = check_3d(v, k->dtype, &vv)) != MOBA_OK) return st;
  const int64_t T = k->shape[0];
  if (k->shape[1] != a.c.Hkv || v->shape[0] != T || v->shape[1] != a.c.Hkv) return MOBA_ERR_SHAPE;
  if ((st = check_contig(slots, MOBA_I64, 1, &T)) != MOBA_OK) return st;
  if (T >= (int64_t(1) << 31) || T * a.c.Hkv >= (int64_t(1) << 32)) return MOBA_ERR_UNSUPPORTED;
  if (T == 0) return MOBA_OK;
  a.k = vk.data; a.k_st = vk.st; a.k_sh = vk.sh;
  a.v = vv.data; a.v_st = vv.st; a.v_sh = vv.sh;
  a.slots = static_cast<const int64_t*>(slots->data);
  a.T = T;
  Phase ph("cache_write", stream);
  MOBA_LAUNCH(launch_cache_write(k->dtype == MOBA_BF16, a, stream));
  return MOBA_OK;
}

size_t moba_cache_decode_workspace_bytes(int64_t S, int64_t W, int32_t Hq, int32_t Hkv,
                                         int32_t page_size, int32_t block_size, int32_t topk) {
  DecodeShape d{};
  if (decode_shape(S, W, Hq, Hkv, page_size, block_size, topk, &d) != MOBA_OK || S == 0) return 0;
  CacheDecodeArgs a{};
  return decode_layout(d, nullptr, &a);
}

moba_status moba_cache_decode(const moba_tensor* q, const moba_cache* cache,
                              const moba_tensor* table, const moba_tensor* lens,
                              int32_t block_size, int32_t topk, moba_tensor* out, moba_tensor* lse,
                              void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (missing(q) || missing(table) || missing(lens) || missing(out) || missing(lse))
    return MOBA_ERR_NULL;
  CacheDecodeArgs a{};
  moba_status st;
  if ((st = check_cache(cache, &a.c)) != MOBA_OK) return st;
  View vq, vo;
  if ((st = check_3d(q, MOBA_BF16, &vq)) != MOBA_OK) return st;
  if ((st = check_3d(out, MOBA_BF16, &vo)) != MOBA_OK) return st;
  const int64_t S = q->shape[0], Hq = q->shape[1];
  if (out->shape[0] != S || out->shape[1] != Hq || Hq % a.c.Hkv != 0) return MOBA_ERR_SHAPE;
  // out may be q (a row of q is read before its result is written), not another view of its memory
  if (S > 0 && share_memory(vq, vo, S, 2) &&
      !(vq.data == vo.data && vq.sh == vo.sh && (S == 1 || vq.st == vo.st)))
    return MOBA_ERR_LAYOUT;
  const int64_t lshape[2] = {Hq, S};
  if ((st = check_contig(lse, MOBA_F32, 2, lshape)) != MOBA_OK) return st;
  if ((st = check_table(table, S)) != MOBA_OK) return st;
  if ((st = check_contig(lens, MOBA_I32, 1, &S)) != MOBA_OK) return st;
  DecodeShape d{};
  if ((st = decode_shape(S, table->shape[1], Hq, a.c.Hkv, a.c.P, block_size, topk, &d)) != MOBA_OK)
    return st;
  if (S == 0) return MOBA_OK;
  if (!workspace) return MOBA_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 15) != 0) return MOBA_ERR_LAYOUT;
  if (workspace_bytes < decode_layout(d, static_cast<char*>(workspace), &a))
    return MOBA_ERR_NO_MEMORY;
  a.q = static_cast<const __hip_bfloat16*>(vq.data); a.q_ss = vq.st; a.q_sh = vq.sh;
  a.out = static_cast<__hip_bfloat16*>(vo.data); a.o_ss = vo.st; a.o_sh = vo.sh;
  a.lse = static_cast<float*>(lse->data);
  a.table = static_cast<const int32_t*>(table->data);
  a.t_ss = table->stride[0];
  a.lens = static_cast<const int32_t*>(lens->data);
  a.S = (int)S;
  a.W = (int)d.W;
  a.Hq = d.Hq;
  a.G = d.Hq / d.Hkv;
  a.B = d.B;
  a.topk = d.topk;
  a.nblk = d.nblk;
  a.parts = d.parts;
  a.shares = d.shares;
  a.join_rows = d.S <= d.shares;
  a.gate_shares = d.gate_shares;
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)kHeadDim));
  if (d.rows) {
    Phase ph("cache_rows", stream);
    MOBA_LAUNCH(launch_cache_rows(d.full, a, stream));
    return MOBA_OK;
  }
  if (!d.full && d.topk > 1) {
    Phase ph("cache_gate", stream);
    MOBA_LAUNCH(launch_cache_gate(a, stream));
  }
  {
    Phase ph("cache_attend", stream);
    if (d.full) MOBA_LAUNCH(launch_cache_attend(a, stream));
    else MOBA_LAUNCH(launch_cache_parts(a, stream));
  }
  if (d.full || d.parts > 1) {
    Phase ph("cache_join", stream);
    MOBA_LAUNCH(launch_cache_join(d.full, a, stream));
  }
  return MOBA_OK;
}

}  // extern "C"
