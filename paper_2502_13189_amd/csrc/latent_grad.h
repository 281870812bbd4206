// Backward of causal latent attention (expanded form): its two sides, for the kernels.  With the forward's lse and
// Delta_i = <dout_i, out_i>:
//   P = exp(z - lse),  dP = dout v^T,  dS = P (dP - Delta)
//   dq = scale dS [k; kr],  dk = scale dS^T q[0:128],  dkr = scale sum over heads of dS^T q[128:192],
//   dv = P^T dout
//
// Kernels, in launch order (small batches: delta, first, which forms Delta anew for the first rows (below), dq and
// dkdv in one launch, dkr):
//   delta  (lse log2 e, Delta) of every (head, token), 16 lanes a row.
//   dq     query side: a work-group of 4 waves owns 128 queries of a head, 32 a wave, and walks the keys
//          in tiles of 64 (k, v, kr staged as in the forward).  Per tile and wave S^T = K . Q^T (24
//          products), dP^T = V . dO^T (16), dQ^T += K^T . dS^T (24, transposed LDS reads).
//   dkdv   key side: a work-group of 4 waves owns 128 keys of a head, 32 a wave, and walks the
//          queries that see them, 64 at a time (q and dout staged).  Per 32 queries and wave
//          S = Q . K^T (12), dP = dO . V^T (8), dV^T += dO^T . P (8), dK^T += Q^T . dS (12).  A key
//          has one owner: no atomics.  The head's part of dkr leaves in fp32.
//   dkr    the heads' parts of dkr, summed in the order of the heads.
// Both loops are bound by the matrix cores and, about as much, by LDS reads (each operand of a product
// is read once a wave).  A wave's accumulators and its own rows (240 registers in dkdv) leave one
// wave a SIMD, so nothing but its own instructions fills a wait.  A tile's work is therefore laid out in
// slices of one product each: beside it go the operand reads of the product kSlicesAhead on, now and then a piece
// of the next tile's DMA (issued all at once it would hold the wave up for half a tile's products), and a share of
// the weights of the half tile before, whose exponentials so cost nothing of their own.
// P and dS enter their products as bf16, all sums are fp32.  On the diagonal's tiles dS enters as two bf16 terms:
// that costs 2% and takes its rounding from where a row's largest weights stand.  (Relative 2-norm errors of dq, 1946
// tokens: 0.0024 without, 0.0021 with the second term; 0.0017 is the rounding of dq alone.)  Delta is off by the
// rounding of out, the more the fewer keys a row has: where it can be had without, it is.
// 8192 tokens, 32 heads: delta 28 us, dq 0.97 to 0.99 ms (1.11 to 1.13 PFLOP/s), dkdv 1.25 to 1.28 ms (1.08 to 1.10),
// dkr 17 us.
#pragma once

#include "latent_tile.h"

#include <math.h>

#include <type_traits>

namespace moba {

// ================================================================ query side
constexpr int kBufDq = 2 * kWide + kSlim;  // k, v, kr
constexpr int kStageDq = kQk / 8 + 1;      // 16-byte chunks of a staged dq row (one pad)

// Rows of a sequence's first 64, whose Delta is formed anew (below).
enum class First { form, done, only };  // here; before; here, and nothing else

// dq of the place's rows of head h.  lds: 2 kBufDq.
template <First FIRST>
__device__ __forceinline__ void latent_dq_part(const LatentArgs& a, const Place& pl, int h, u32x4* lds) {
  constexpr int kWaves = kLatBwdWaves;
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qc = lane & 31, hh = lane >> 5;
  const int row = pl.t0 + 32 * wave + qc;
  const int64_t rt = pl.tok0 + min(row, pl.len - 1);
  const int kend = min(pl.t0 + kLatRowsDq, pl.len);

  bf16x8 qf[12], df[8];
  {
    const __hip_bfloat16* qrow = a.q + rt * a.q_st + (int64_t)h * a.q_sh + 8 * hh;
    const __hip_bfloat16* drow = a.dout + rt * a.do_st + (int64_t)h * a.do_sh + 8 * hh;
#pragma unroll
    for (int kk = 0; kk < 12; kk++) qf[kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(qrow + 16 * kk));
#pragma unroll
    for (int kk = 0; kk < 8; kk++) df[kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(drow + 16 * kk));
  }
  // into the accumulation registers, where the matrix cores read them as well as anywhere
#pragma unroll
  for (int kk = 0; kk < 12; kk++) asm volatile("" : "+a"(qf[kk]));
#pragma unroll
  for (int kk = 0; kk < 8; kk++) asm volatile("" : "+a"(df[kk]));
  float2 ld = a.ld[(int64_t)h * a.T + rt];
  const auto rows = [&](const __hip_bfloat16* p, int64_t st, int64_t sh) {
    return Rows{scalar_ptr(p + pl.tok0 * st + (int64_t)h * sh), (uint32_t)(st * 2), pl.len};
  };
  const Rows rk = rows(a.k, a.k_st, a.k_sh), rv = rows(a.v, a.v_st, a.v_sh), rr = rows(a.kr, a.kr_st, 0);
  const auto stage_piece = [&](int i, u32x4* buf, int x) {
    if (x < 4) stage_part<kWaves, true>(rk, i, buf, wave, lane, x);
    else if (x < 8) stage_part<kWaves, true>(rv, i, buf + kWide, wave, lane, x - 4);
    else stage_part<kWaves, false>(rr, i, buf + 2 * kWide, wave, lane, x - 8);
  };
  const auto stage = [&](int i, u32x4* buf) {
#pragma unroll
    for (int x = 0; x < kLatBwdDma; x++) stage_piece(i, buf, x);
  };
  uint32_t ow[8], os[4], tw[2][4], ts[2][2];
  const TrLane tl = tr_lane(qc, hh);
#pragma unroll
  for (int kk = 0; kk < 8; kk++) ow[kk] = at_wide(qc, 2 * kk + hh);
#pragma unroll
  for (int kk = 0; kk < 4; kk++) os[kk] = at_slim(qc, 2 * kk + hh);
#pragma unroll
  for (int x = 0; x < 2; x++) {
#pragma unroll
    for (int dt = 0; dt < 4; dt++) tw[x][dt] = tr_wide(tl, dt, x);
#pragma unroll
    for (int dt = 0; dt < 2; dt++) ts[x][dt] = tr_slim(tl, dt, x);
  }
  const float c2 = a.scale_log2;
  f32x16 acc[6];
#pragma unroll
  for (int dt = 0; dt < 6; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) acc[dt][r] = 0.0f;

  const int n = (kend + kLatTile - 1) / kLatTile;
  stage(0, lds);
  dma_wait();
  __syncthreads();
  // Rows of the sequence's first 64 have all their keys in tile 0: their Delta is formed anew, as the sum of P dP,
  // without the out's rounding to bf16, for dq and dkdv.
  if (FIRST != First::done && pl.t0 == 0 && wave < 2) {
    const char* b = reinterpret_cast<const char*>(lds);
    float delta = 0.0f;
#pragma unroll 1
    for (int th = 0; th <= wave; th++) {
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; r++) s[r] = dp[r] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < 12; kk++) {
        const char* at = kk < 8 ? b + 8192 * th + ow[kk & 7] : b + 2 * kWide * 16 + 4096 * th + os[(kk - 8) & 3];
        s = mfma(as_bf16x8(*reinterpret_cast<const u32x4*>(at)), qf[kk], s);
        if (kk < 8)
          dp = mfma(as_bf16x8(*reinterpret_cast<const u32x4*>(b + kWide * 16 + 8192 * th + ow[kk & 7])),
                    df[kk & 7], dp);
      }
#pragma unroll
      for (int j = 0; j < 16; j++) {
        const int key = 32 * th + 8 * (j >> 2) + 4 * hh + (j & 3);
        const float p = __builtin_amdgcn_exp2f(fmaf(s[j], c2, -ld.x)) * dp[j];
        delta += key <= row ? p : 0.0f;
      }
    }
    ld.y = delta + xor32(delta);
    if (hh == 0 && row < pl.len) a.ld[(int64_t)h * a.T + rt].y = ld.y;
  }
  if constexpr (FIRST == First::only) return;
  const auto step = [&](auto masked, int i) {
    constexpr bool edge = decltype(masked)::value;
    const char* bk = reinterpret_cast<const char*>(lds + (i & 1) * kBufDq);
    const char* bv = bk + kWide * 16;
    const char* br = bk + 2 * kWide * 16;
    u32x4* nbuf = lds + ((i + 1) & 1) * kBufDq;
    const int nt = min(i + 1, n - 1);  // (at the end the last tile once more: no branches between the slices)
    const int hi = row + 1 - i * kLatTile - 4 * hh;
    f32x16 s[2], dp[2];
#pragma unroll
    for (int th = 0; th < 2; th++)
#pragma unroll
      for (int r = 0; r < 16; r++) s[th][r] = dp[th][r] = 0.0f;
    // products 0 .. 39: S^T (12) and dP^T (8) of the two halves of the keys; 40 .. 63: dQ^T
    constexpr int kN = 64;
    u32x4 op[kN];
    uint32_t w[2][8], wl[2][8];  // dS of the halves, bf16 pairs; on the diagonal also what they leave out
    const auto fetch = [&](auto at) __attribute__((always_inline)) {
      constexpr int x = decltype(at)::value;
      if constexpr (x < 40) {
        constexpr int th = x / 20, y = x % 20, kk = y < 12 ? y : y - 12;
        if constexpr (y >= 12) op[x] = *reinterpret_cast<const u32x4*>(bv + 8192 * th + ow[kk]);
        else if constexpr (kk < 8) op[x] = *reinterpret_cast<const u32x4*>(bk + 8192 * th + ow[kk]);
        else op[x] = *reinterpret_cast<const u32x4*>(br + 4096 * th + os[kk - 8]);
      } else {
        constexpr int ks = (x - 40) / 6, dt = (x - 40) % 6;
        const char* b = dt < 4 ? bk + 16 * ks * 256 : br + 16 * ks * 128;
        op[x] = __builtin_bit_cast(u32x4, dt < 4 ? join16(tr16(b + tw[0][dt & 3]), tr16(b + tw[1][dt & 3]))
                                                 : join16(tr16(b + ts[0][dt & 1]), tr16(b + ts[1][dt & 1])));
      }
    };
    const auto use = [&](auto at) __attribute__((always_inline)) {
      constexpr int x = decltype(at)::value;
      if constexpr (x < 40) {
        constexpr int th = x / 20, y = x % 20, kk = y < 12 ? y : y - 12;
        if constexpr (y >= 12) dp[th] = mfma(as_bf16x8(op[x]), df[kk], dp[th]);
        else s[th] = mfma(as_bf16x8(op[x]), qf[kk], s[th]);
      } else {
        constexpr int ks = (x - 40) / 6, dt = (x - 40) % 6, th = ks / 2, e = 4 * (ks % 2);
        acc[dt] = mfma(as_bf16x8(op[x]), as_bf16x8(u32x4{w[th][e], w[th][e + 1], w[th][e + 2], w[th][e + 3]}), acc[dt]);
        if constexpr (edge)
          acc[dt] = mfma(as_bf16x8(op[x]), as_bf16x8(u32x4{wl[th][e], wl[th][e + 1], wl[th][e + 2], wl[th][e + 3]}), acc[dt]);
      }
    };
    // elements 2 e, 2 e + 1 of a half: P, then dS
    float p[2][16];
    const auto weigh = [&](int th, int j) __attribute__((always_inline)) {  // element j
      p[th][j] = __builtin_amdgcn_exp2f(fmaf(s[th][j], c2, -ld.x));
      if (edge) p[th][j] = 32 * th + 8 * (j >> 2) + (j & 3) < hi ? p[th][j] : 0.0f;
      asm volatile("" : "+v"(p[th][j]));  // (formed here, not where it is used)
    };
    const auto slope = [&](int th, int e) __attribute__((always_inline)) {
      const float d0 = p[th][2 * e] * (dp[th][2 * e] - ld.y), d1 = p[th][2 * e + 1] * (dp[th][2 * e + 1] - ld.y);
      w[th][e] = pack_bf16(d0, d1);
      if (edge) wl[th][e] = rest_bf16(w[th][e], d0, d1);
      asm volatile("" : "+v"(w[th][e]));
    };
    each<kSlicesAhead>(fetch);
    each<kN>([&](auto at) __attribute__((always_inline)) {
      constexpr int x = decltype(at)::value;
      use(at);
      if constexpr (x + kSlicesAhead < kN) fetch(Index<x + kSlicesAhead>());
      if constexpr (x % 5 == 3 && x / 5 < kLatBwdDma) stage_piece(nt, nbuf, x / 5);
      // one exponential to a slice, which with the operand reads is about what fits beside its product
      if constexpr (x >= 13 && x < 29) weigh(0, x - 13);
      if constexpr (x >= 25 && x < 33) slope(0, x - 25);
      if constexpr (x >= 33 && x < 49) weigh(1, x - 33);
      if constexpr (x >= 44 && x < 52) slope(1, x - 44);
      slice_end();
    });
    dma_wait();
    __syncthreads();
  };
  const int nfull = pl.t0 / kLatTile;
  for (int i = 0; i < nfull; i++) step(std::false_type(), i);
  for (int i = nfull; i < n; i++) step(std::true_type(), i);

  // each wave stages its 32 rows and writes them whole
  u32x4* stg = lds + wave * 32 * kStageDq;
  uint2* srow = reinterpret_cast<uint2*>(stg + qc * kStageDq);
  const float scl = a.scale;
#pragma unroll
  for (int dt = 0; dt < 6; dt++)
#pragma unroll
    for (int r4 = 0; r4 < 4; r4++)
      srow[(32 * dt + 8 * r4 + 4 * hh) >> 2] =
          make_uint2(pack_bf16(acc[dt][4 * r4] * scl, acc[dt][4 * r4 + 1] * scl),
                     pack_bf16(acc[dt][4 * r4 + 2] * scl, acc[dt][4 * r4 + 3] * scl));
  __builtin_amdgcn_s_waitcnt(0);  // (a wave's own LDS writes, read by its other lanes)
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < 12; j++) {
    const int y = 64 * j + lane, r = y / (kQk / 8), c = y % (kQk / 8), t = pl.t0 + 32 * wave + r;
    if (t < pl.len)
      reinterpret_cast<u32x4*>(a.dq + (pl.tok0 + t) * a.dq_st + (int64_t)h * a.dq_sh)[c] = stg[r * kStageDq + c];
  }
}

// ================================================================ key side
constexpr int kStage = 2 * kNope / 8 + 1;   // 16-byte chunks of a staged row of dk and dv (one pad)
constexpr int kBufKv = 2 * kWide + kSlim;  // q's first 128 dims, dout, q's rotary dims

// dk, dv and head h's part of dkr of the place's keys.
struct DkdvLds {
  u32x4 tiles[2 * kBufKv];
  __align__(16) float lse2[2][kLatTile], dlt[2][kLatTile];
};
static_assert(kLatBwdWaves * 32 * kStage <= 2 * kBufKv, "the staged rows fit");
static_assert(kBufKv == kBufDq, "either part's tiles");

__device__ __forceinline__ void latent_dkdv_part(const LatentArgs& a, const Place& pl, int h, DkdvLds& sh) {
  constexpr int kWaves = kLatBwdWaves;
  u32x4* const lds = sh.tiles;
  auto& lse2 = sh.lse2;
  auto& dlt = sh.dlt;
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qc = lane & 31, hh = lane >> 5;
  const int key = pl.t0 + 32 * wave + qc;  // this lane's key
  const int64_t kt = pl.tok0 + min(key, pl.len - 1);

  bf16x8 kf[12], vf[8];
  {
    const __hip_bfloat16* krow = a.k + kt * a.k_st + (int64_t)h * a.k_sh + 8 * hh;
    const __hip_bfloat16* rrow = a.kr + kt * a.kr_st + 8 * hh;
    const __hip_bfloat16* vrow = a.v + kt * a.v_st + (int64_t)h * a.v_sh + 8 * hh;
#pragma unroll
    for (int kk = 0; kk < 8; kk++) {
      kf[kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(krow + 16 * kk));
      vf[kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(vrow + 16 * kk));
    }
#pragma unroll
    for (int kk = 0; kk < 4; kk++) kf[8 + kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(rrow + 16 * kk));
  }
  const auto rows = [&](const __hip_bfloat16* p, int64_t st, int64_t sh) {
    return Rows{scalar_ptr(p + pl.tok0 * st + (int64_t)h * sh), (uint32_t)(st * 2), pl.len};
  };
  const Rows rq = rows(a.q, a.q_st, a.q_sh), rr = rows(a.q + kNope, a.q_st, a.q_sh), rd = rows(a.dout, a.do_st, a.do_sh);
  const auto stage_piece = [&](int i, u32x4* buf, int x) {
    if (x < 4) stage_part<kWaves, true>(rq, i, buf, wave, lane, x);
    else if (x < 8) stage_part<kWaves, true>(rd, i, buf + kWide, wave, lane, x - 4);
    else stage_part<kWaves, false>(rr, i, buf + 2 * kWide, wave, lane, x - 8);
  };
  const auto stage = [&](int i, u32x4* buf) {
#pragma unroll
    for (int x = 0; x < kLatBwdDma; x++) stage_piece(i, buf, x);
  };
  // a row's lse and Delta; a row past the sequence's end gets no weight
  const float2* ldh = a.ld + (int64_t)h * a.T + pl.tok0;
  const auto row_ld = [&](int i) {
    const int t = i * kLatTile + lane;
    return t < pl.len ? ldh[t] : make_float2(INFINITY, 0.0f);
  };
  uint32_t ow[8], os[4], tw[2][4], ts[2][2];
  const TrLane tl = tr_lane(qc, hh);
#pragma unroll
  for (int kk = 0; kk < 8; kk++) ow[kk] = at_wide(qc, 2 * kk + hh);
#pragma unroll
  for (int kk = 0; kk < 4; kk++) os[kk] = at_slim(qc, 2 * kk + hh);
#pragma unroll
  for (int x = 0; x < 2; x++) {
#pragma unroll
    for (int dt = 0; dt < 4; dt++) tw[x][dt] = tr_wide(tl, dt, x);
#pragma unroll
    for (int dt = 0; dt < 2; dt++) ts[x][dt] = tr_slim(tl, dt, x);
  }
  const float c2 = a.scale_log2;
  f32x16 dk[6], dv[4];
#pragma unroll
  for (int r = 0; r < 16; r++) {
#pragma unroll
    for (int dt = 0; dt < 6; dt++) dk[dt][r] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < 4; dt++) dv[dt][r] = 0.0f;
  }

  const int i0 = pl.t0 / kLatTile, n = (pl.len + kLatTile - 1) / kLatTile;
  stage(i0, lds + (i0 & 1) * kBufKv);
  if (wave == 0) {
    const float2 x = row_ld(i0);
    lse2[i0 & 1][lane] = x.x;
    dlt[i0 & 1][lane] = x.y;
  }
  dma_wait();
  __syncthreads();
  const auto step = [&](auto masked, int i) {
    constexpr bool edge = decltype(masked)::value;
    const int cur = i & 1;
    const char* bq = reinterpret_cast<const char*>(lds + cur * kBufKv);
    const char* bd = bq + kWide * 16;
    const char* br = bq + 2 * kWide * 16;
    u32x4* nbuf = lds + (cur ^ 1) * kBufKv;
    float2 nx;
    const int nt = min(i + 1, n - 1);  // (at the end the last tile once more: no branches between the slices)
    if (wave == 0) nx = row_ld(nt);
    f32x16 s[2], dp[2];
#pragma unroll
    for (int st = 0; st < 2; st++)
#pragma unroll
      for (int r = 0; r < 16; r++) s[st][r] = dp[st][r] = 0.0f;
    // products 0 .. 39: S (12) and dP (8) of the two halves of the rows; 40 .. 79: dV^T and dK^T
    constexpr int kN = 80;
    u32x4 op[kN];
    uint32_t wp[2][8], wd[2][8], wl[2][8];  // P and dS of the halves, bf16 pairs; and what dS's leave out
    float2 lv[16], dl[16];
    const auto fetch = [&](auto n_) __attribute__((always_inline)) {
      constexpr int x = decltype(n_)::value;
      if constexpr (x < 40) {
        constexpr int st = x / 20, y = x % 20, kk = y < 12 ? y : y - 12;
        if constexpr (y >= 12) op[x] = *reinterpret_cast<const u32x4*>(bd + 8192 * st + ow[kk]);
        else if constexpr (kk < 8) op[x] = *reinterpret_cast<const u32x4*>(bq + 8192 * st + ow[kk]);
        else op[x] = *reinterpret_cast<const u32x4*>(br + 4096 * st + os[kk - 8]);
      } else {
        constexpr int y = x - 40, r0 = 16 * (y / 10), z = y % 10, dt = z < 4 ? z : z - 4;  // dV's four tiles, dK's six
        const char* b = z < 4 ? bd + r0 * 256 : dt < 4 ? bq + r0 * 256 : br + r0 * 128;
        op[x] = __builtin_bit_cast(u32x4, dt < 4 ? join16(tr16(b + tw[0][dt & 3]), tr16(b + tw[1][dt & 3]))
                                                 : join16(tr16(b + ts[0][dt & 1]), tr16(b + ts[1][dt & 1])));
      }
    };
    const auto use = [&](auto n_) __attribute__((always_inline)) {
      constexpr int x = decltype(n_)::value;
      if constexpr (x < 40) {
        constexpr int st = x / 20, y = x % 20, kk = y < 12 ? y : y - 12;
        if constexpr (y >= 12) dp[st] = mfma(as_bf16x8(op[x]), vf[kk], dp[st]);
        else s[st] = mfma(as_bf16x8(op[x]), kf[kk], s[st]);
      } else {
        constexpr int y = x - 40, st = y / 20, e = 4 * (y / 10 % 2), z = y % 10;
        const uint32_t(&w)[8] = z < 4 ? wp[st] : wd[st];
        const bf16x8 b = as_bf16x8(u32x4{w[e], w[e + 1], w[e + 2], w[e + 3]});
        if constexpr (z < 4) dv[z] = mfma(as_bf16x8(op[x]), b, dv[z]);
        else dk[z - 4] = mfma(as_bf16x8(op[x]), b, dk[z - 4]);
        if constexpr (edge && z >= 4)
          dk[z - 4] = mfma(as_bf16x8(op[x]), as_bf16x8(u32x4{wl[st][e], wl[st][e + 1], wl[st][e + 2], wl[st][e + 3]}), dk[z - 4]);
      }
    };
    // elements 2 e, 2 e + 1 of a half, rows r and r + 1: P, then dS
    float p[2][16];
    const auto row_at = [&](int st, int e) { return 32 * st + 8 * (e >> 1) + 4 * hh + 2 * (e & 1); };
    const auto fetch_lse = [&](int st, int e) __attribute__((always_inline)) {
      lv[8 * st + e] = *reinterpret_cast<const float2*>(&lse2[cur][row_at(st, e)]);
    };
    const auto fetch_delta = [&](int st, int e) __attribute__((always_inline)) {
      dl[8 * st + e] = *reinterpret_cast<const float2*>(&dlt[cur][row_at(st, e)]);
    };
    const auto weigh = [&](int st, int j) __attribute__((always_inline)) {  // element j
      const float2 l = lv[8 * st + j / 2];
      float x = __builtin_amdgcn_exp2f(fmaf(s[st][j], c2, j % 2 ? -l.y : -l.x));
      if (edge) x = i * kLatTile + row_at(st, j / 2) + j % 2 >= key ? x : 0.0f;
      p[st][j] = x;
      if (j % 2) wp[st][j / 2] = pack_bf16(p[st][j - 1], x);
      asm volatile("" : "+v"(p[st][j]));  // (formed here, not where it is used)
      if (j % 2) asm volatile("" : "+v"(wp[st][j / 2]));
    };
    const auto slope = [&](int st, int e) __attribute__((always_inline)) {
      const float2 d = dl[8 * st + e];
      const float d0 = p[st][2 * e] * (dp[st][2 * e] - d.x), d1 = p[st][2 * e + 1] * (dp[st][2 * e + 1] - d.y);
      wd[st][e] = pack_bf16(d0, d1);
      if (edge) wl[st][e] = rest_bf16(wd[st][e], d0, d1);
      asm volatile("" : "+v"(wd[st][e]));
    };
    each<kSlicesAhead>(fetch);
    each<kN>([&](auto n_) __attribute__((always_inline)) {
      constexpr int x = decltype(n_)::value;
      use(n_);
      if constexpr (x + kSlicesAhead < kN) fetch(Index<x + kSlicesAhead>());
      if constexpr (x % 6 == 4 && x / 6 < kLatBwdDma) stage_piece(nt, nbuf, x / 6);
      // one exponential or one pair of dS to a slice, which is about what fits beside its product
      if constexpr (x >= 9 && x < 25 && x % 2 == 1) fetch_lse(0, (x - 9) / 2);
      if constexpr (x >= 13 && x < 29) weigh(0, x - 13);
      if constexpr (x >= 25 && x < 33) fetch_delta(0, x - 25);
      if constexpr (x >= 29 && x < 37) slope(0, x - 29);
      if constexpr (x >= 33 && x < 49 && x % 2 == 1) fetch_lse(1, (x - 33) / 2);
      if constexpr (x >= 37 && x < 53) weigh(1, x - 37);
      if constexpr (x >= 49 && x < 57) fetch_delta(1, x - 49);
      if constexpr (x >= 53 && x < 61) slope(1, x - 53);
      slice_end();
    });
    dma_wait();
    if (wave == 0) {
      lse2[cur ^ 1][lane] = nx.x;
      dlt[cur ^ 1][lane] = nx.y;
    }
    __syncthreads();
  };
  // (the diagonal's rows, and those of the last tile, which may end past the sequence: their lse is inf)
  const int iedge = min(n, i0 + kLatKeys / kLatTile);
  for (int i = i0; i < iedge; i++) step(std::true_type(), i);
  for (int i = iedge; i < n; i++) step(std::false_type(), i);

  // each wave stages its 32 rows, dk beside dv and then the part of dkr, and writes them whole
  const float scl = a.scale;
  u32x4* stg = lds + wave * 32 * kStage;
  uint2* srow = reinterpret_cast<uint2*>(stg + qc * kStage);
#pragma unroll
  for (int dt = 0; dt < 4; dt++)
#pragma unroll
    for (int r4 = 0; r4 < 4; r4++) {
      const int d = (32 * dt + 8 * r4 + 4 * hh) >> 2;
      srow[d] = make_uint2(pack_bf16(dk[dt][4 * r4] * scl, dk[dt][4 * r4 + 1] * scl),
                           pack_bf16(dk[dt][4 * r4 + 2] * scl, dk[dt][4 * r4 + 3] * scl));
      srow[d + kNope / 4] = make_uint2(pack_bf16(dv[dt][4 * r4], dv[dt][4 * r4 + 1]),
                                       pack_bf16(dv[dt][4 * r4 + 2], dv[dt][4 * r4 + 3]));
    }
  const auto settle = [] {  // a wave's own LDS writes, read by its other lanes
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_wave_barrier();
  };
  settle();
#pragma unroll
  for (int j = 0; j < 16; j++) {
    const int y = 64 * j + lane, r = y / 32, c = y % 32, t = pl.t0 + 32 * wave + r;
    __hip_bfloat16* row = c < 16 ? a.dk + (pl.tok0 + t) * a.dk_st + (int64_t)h * a.dk_sh
                                 : a.dv + (pl.tok0 + t) * a.dv_st + (int64_t)h * a.dv_sh;
    if (t < pl.len) reinterpret_cast<u32x4*>(row)[c % 16] = stg[r * kStage + c];
  }
  settle();
  float4* sr = reinterpret_cast<float4*>(stg + qc * kStage);
#pragma unroll
  for (int dt = 0; dt < 2; dt++)
#pragma unroll
    for (int r4 = 0; r4 < 4; r4++)
      sr[(32 * dt + 8 * r4 + 4 * hh) >> 2] = make_float4(dk[4 + dt][4 * r4] * scl, dk[4 + dt][4 * r4 + 1] * scl,
                                                         dk[4 + dt][4 * r4 + 2] * scl, dk[4 + dt][4 * r4 + 3] * scl);
  settle();
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const int y = 64 * j + lane, r = y / 16, c = y % 16, t = pl.t0 + 32 * wave + r;
    if (t < pl.len) reinterpret_cast<u32x4*>(a.dkr_part + ((int64_t)h * a.T + pl.tok0 + t) * kRopeDim)[c] = stg[r * kStage + c];
  }
}

}  // namespace moba
