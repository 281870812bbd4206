// Key side of the backward of causal latent attention: dk, dv and a head's part of dkr (see latent_bwd.hip).
#include "latent_tile.h"

#include <math.h>

namespace moba {
namespace {

constexpr int kWaves = kLatBwdWaves;

constexpr int kStage = 2 * kNope / 8 + 1;   // 16-byte chunks of a staged row of dk and dv (one pad)
constexpr int kBufKv = 2 * kWide + kSlim;  // q's first 128 dims, dout, q's rotary dims

__global__ __launch_bounds__(64 * kWaves, 1) void latent_dkdv_kernel(LatentArgs a) {
  static_assert(kWaves * 32 * kStage <= 2 * kBufKv, "the staged rows fit");
  __shared__ u32x4 lds[2 * kBufKv];
  __shared__ __align__(16) float lse2[2][kLatTile], dlt[2][kLatTile];
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qc = lane & 31, hh = lane >> 5;
  Work wk;
  if (!latent_work<false>(a, latent_places(a.T, a.S, kLatKeys), &wk)) return;
  Place pl;
  if (!latent_place(a, wk.place, kLatKeys, &pl)) return;
  const int h = __builtin_amdgcn_readfirstlane(wk.h);
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

}  // namespace

hipError_t launch_latent_dkdv(const LatentArgs& a, hipStream_t st) {
  latent_dkdv_kernel<<<latent_grid(a, kLatKeys), 64 * kWaves, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace moba
