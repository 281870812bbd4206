// Internal declarations of the paged 8-bit cache (plan, write, decode), shared by its host
// side and its kernels.
#pragma once

#include "cache_rules.h"
#include "moba_internal.h"

namespace moba {

constexpr int kCacheMaxPage = 256;   // largest page
constexpr int kPlanMaxRequests = 4096;
constexpr int kCacheMinExp = -100, kCacheMaxExp = 119;  // exponents of a page's scale

struct CachePool {
  uint8_t* k; int64_t k_sp, k_sh;  // [N, Hkv, P, 128], page and head strides in bytes
  uint8_t* v; int64_t v_sp, v_sh;  // [N, Hkv, P / 64, 128, 64]
  float* k_scale;                  // [N, Hkv]
  float* v_scale;
  float* k_sum;                    // [N, Hkv, 128]
  int N, Hkv, P;
};

// ------------------------------------------------------------------ plan
struct CachePlanArgs {
  const int32_t* add;
  const int32_t* lens;
  int32_t* table; int64_t t_ss;
  int32_t* free_pages;
  const int32_t* num_free;
  int32_t* lens_out;
  int32_t* num_free_out;
  int32_t* cu;
  int64_t* slots;
  int32_t* refused;
  int S, W, N, P;
  int64_t T;
};
hipError_t launch_cache_plan(const CachePlanArgs& a, hipStream_t st);

// ----------------------------------------------------------------- write
struct CacheWriteArgs {
  const void* k; int64_t k_st, k_sh;  // [T, Hkv, 128], elements
  const void* v; int64_t v_st, v_sh;
  const int64_t* slots;
  int64_t T;
  CachePool c;
};
hipError_t launch_cache_write(bool bf16, const CacheWriteArgs& a, hipStream_t st);

// ---------------------------------------------------------------- decode
constexpr int kCacheWaves = 2048;  // attention waves the chip holds: 8 on each of 256 CUs
constexpr int kCacheGateWaves = 8192;  // waves of the gate at most (one a block, if they suffice)
constexpr int64_t kCachePartGroups = 512;  // MoBA: work-groups that split rows fill, two on a CU
constexpr int64_t kCachePartSteps = 256;   // and the most steps of one, however many rows
constexpr int kCacheDecodeThreads = 256;
constexpr int kCacheRowBlocks = 128;   // MoBA blocks of a row that one work-group takes

// A row split over several shares.  Of a request's entry: the share it begins in, of a share's
// (where requests are more than shares): the request that begins in it; -1: none; and the shares
// it spans.
struct CacheJoin {
  int32_t at, count;
};

struct CacheDecodeArgs {
  const __hip_bfloat16* q; int64_t q_ss, q_sh;  // [S, Hq, D]
  CachePool c;
  const int32_t* table; int64_t t_ss;
  const int32_t* lens;
  int S, W, Hq, G;
  int B, topk;                                  // MoBA; nblk: blocks a table row holds
  int nblk;
  int parts;                                    // MoBA: work-groups for a (request, kv-head)
  __hip_bfloat16* out; int64_t o_ss, o_sh;
  float* lse;                                   // [Hq, S]
  float scale_log2;
  int shares;        // full: of the batch's 64-key steps, of each kv-head
  bool join_rows;    // full: an entry of join for every request, not for every share
  int gate_shares;   // of the batch's past blocks, of each kv-head
  // workspace
  double* score;     // [S, Hq, nblk] gate scores
  float* part_o;     // full [shares, 2, Hkv, G, D], MoBA [S, Hkv, parts, G, D]: unnormalised partials
  float2* part_ml;   // [..., G] their max (log2 domain) and sum
  CacheJoin* join;   // full [S (join_rows) or shares, Hkv]
};
// Gate, selection, attention and join in one launch, a work-group per (request, kv-head); for
// table rows of up to kCacheRowBlocks blocks (MoBA).  Needs no workspace.
hipError_t launch_cache_rows(bool full, const CacheDecodeArgs& a, hipStream_t st);
hipError_t launch_cache_gate(const CacheDecodeArgs& a, hipStream_t st);
hipError_t launch_cache_parts(const CacheDecodeArgs& a, hipStream_t st);
hipError_t launch_cache_attend(const CacheDecodeArgs& a, hipStream_t st);
hipError_t launch_cache_join(bool full, const CacheDecodeArgs& a, hipStream_t st);

}  // namespace moba
