// Latent attention: declarations shared by its host side and its kernels.
#pragma once

#include "moba_internal.h"

namespace moba {

constexpr int kNope = 128;              // dims of a head's queries and keys that hold no position
constexpr int kRopeDim = 64;            // and the rotary ones; the keys' are shared by all heads
constexpr int kQk = kNope + kRopeDim;   // dims a head scores, expanded
constexpr int kRank = 512;              // the latent vector
constexpr int kRow = kRank + kRopeDim;  // numbers a token has in the cache

// ------------------------------------------------------------- expanded form
constexpr int kLatRows = 256;   // query rows of a forward work-group (or half of it)
constexpr int kLatFew = 1024;   // half of it: up to so many work-groups,
constexpr int kLatLong = 4096;  // or for sequences shorter than this, on average
constexpr int kLatRowsDq = 128; // of a dQ work-group
constexpr int kLatKeys = 128;   // keys of a dK/dV work-group
constexpr int kLatTile = 64;    // tokens of a staged tile
// Few work-groups are ranked by the length of their chains, up to so many sequences (a lane each): the backward's two
// sides in one launch, up to so many work-groups a side; the forward's.
constexpr int kLatRankedSeqs = 64;
constexpr int kLatBoth = 1024;
constexpr int kLatRanked = 4096;

struct LatentArgs {
  const __hip_bfloat16* q; int64_t q_st, q_sh;    // [T, H, 192], elements
  const __hip_bfloat16* k; int64_t k_st, k_sh;    // [T, H, 128]
  const __hip_bfloat16* kr; int64_t kr_st;        // [T, 64]
  const __hip_bfloat16* v; int64_t v_st, v_sh;    // [T, H, 128]
  const int32_t* cu;                              // [S + 1], device
  int S, H;
  int64_t T;
  float scale, scale_log2;
  __hip_bfloat16* out; int64_t o_st, o_sh;        // [T, H, 128] (backward: read)
  float* lse;                                     // [H, T]
  // backward
  const __hip_bfloat16* dout; int64_t do_st, do_sh;
  __hip_bfloat16* dq; int64_t dq_st, dq_sh;
  __hip_bfloat16* dk; int64_t dk_st, dk_sh;
  __hip_bfloat16* dkr; int64_t dkr_st;
  __hip_bfloat16* dv; int64_t dv_st, dv_sh;
  float2* ld;      // [H, T]: lse * log2 e, <dout, out>
  float* dkr_part; // [H, T, 64]: a head's part of dkr
};
// Work-groups of a head at most, in any of the launches.
inline int64_t latent_places_bound(int64_t T, int64_t S) { return T / kLatKeys + S; }
hipError_t launch_latent_forward(const LatentArgs& a, hipStream_t st);
hipError_t launch_latent_delta(const LatentArgs& a, hipStream_t st);
hipError_t launch_latent_first(const LatentArgs& a, hipStream_t st);
hipError_t launch_latent_both(const LatentArgs& a, hipStream_t st);
hipError_t launch_latent_dq(const LatentArgs& a, hipStream_t st);
hipError_t launch_latent_dkdv(const LatentArgs& a, hipStream_t st);
hipError_t launch_latent_dkr(const LatentArgs& a, hipStream_t st);

// ------------------------------------------------------------- absorbed form
constexpr int kLatStep = 64;    // cached tokens of a decode step
constexpr int kLatGroups = 256; // work-groups of a decode call: one on each CU

struct LatentDecodeArgs {
  const __hip_bfloat16* qc; int64_t qc_ss, qc_sh;  // [S, H, 512]
  const __hip_bfloat16* qr; int64_t qr_ss, qr_sh;  // [S, H, 64]
  const __hip_bfloat16* pages; int64_t p_sp;       // [N, P, 576], page stride in elements
  int N, P;
  const int32_t* table; int64_t t_ss;              // [S, W]
  const int32_t* lens;
  int S, W, H;
  float scale_log2;
  __hip_bfloat16* out; int64_t o_ss, o_sh;         // [S, H, 512]
  float* lse;                                      // [H, S]
  int shares;                                      // of the batch's steps, for each group of heads
  int groups;                                      // groups of heads
  // workspace
  float* part_o;     // [shares, 2, groups, heads of a group * 512]: unnormalised partials, as the join reads them
  float2* part_ml;   // [shares, 2, groups, heads of a group]: their max (log2 domain) and sum
  uint32_t* first;   // [S + 1]: the batch's step at which a request begins; the batch's steps
};
// heads: of a group, 16, 32 or 64
hipError_t launch_latent_decode(int heads, const LatentDecodeArgs& a, hipStream_t st);
hipError_t launch_latent_join(int heads, const LatentDecodeArgs& a, hipStream_t st);

}  // namespace moba
