// Backward of causal latent attention (expanded form).  With the forward's lse and Delta_i =
// <dout_i, out_i>:
//   P = exp(z - lse),  dP = dout v^T,  dS = P (dP - Delta)
//   dq = scale dS [k; kr],  dk = scale dS^T q[0:128],  dkr = scale sum over heads of dS^T q[128:192],
//   dv = P^T dout
//
// Kernels, in launch order:
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
// wave a SIMD.  P and dS enter their products as bf16, all sums are fp32.
#include "latent_tile.h"

#include <math.h>

#include <type_traits>

namespace moba {
namespace {

constexpr int kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;

__global__ __launch_bounds__(256) void latent_delta_kernel(LatentArgs a) {
  const int64_t r = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;  // t * H + h
  const int l16 = threadIdx.x % 16;
  if (r >= a.T * a.H) return;  // the 16 lanes of a row leave together
  const int64_t t = r / a.H;
  const int h = (int)(r - t * a.H);
  const u32x4 ow = *reinterpret_cast<const u32x4*>(a.out + t * a.o_st + (int64_t)h * a.o_sh + 8 * l16);
  const u32x4 dw = *reinterpret_cast<const u32x4*>(a.dout + t * a.do_st + (int64_t)h * a.do_sh + 8 * l16);
  float acc = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    acc = fmaf(__uint_as_float(ow[i] << 16), __uint_as_float(dw[i] << 16), acc);
    acc = fmaf(__uint_as_float(ow[i] & 0xffff0000u), __uint_as_float(dw[i] & 0xffff0000u), acc);
  }
#pragma unroll
  for (int m = 8; m >= 1; m >>= 1) acc += __shfl_xor(acc, m, 64);
  if (l16 == 0) {
    const int64_t i = (int64_t)h * a.T + t;
    a.ld[i] = make_float2(a.lse[i] * kLog2e, acc);
  }
}

// ================================================================ dQ
constexpr int kBufDq = 2 * kWide + kSlim;  // k, v, kr
constexpr int kStageDq = kQk / 8 + 1;      // 16-byte chunks of a staged dq row (one pad)

__global__ __launch_bounds__(64 * kWaves, 1) void latent_dq_kernel(LatentArgs a) {
  __shared__ u32x4 lds[2 * kBufDq];
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qc = lane & 31, hh = lane >> 5;
  Work wk;
  if (!latent_work<true>(a, latent_places(a.T, a.S, kLatRowsDq), &wk)) return;
  Place pl;
  if (!latent_place(a, wk.place, kLatRowsDq, &pl)) return;
  const int h = __builtin_amdgcn_readfirstlane(wk.h);
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
  const float2 ld = a.ld[(int64_t)h * a.T + rt];
  const auto rows = [&](const __hip_bfloat16* p, int64_t st, int64_t sh) {
    return Rows{scalar_ptr(p + pl.tok0 * st + (int64_t)h * sh), (uint32_t)(st * 2), pl.len};
  };
  const Rows rk = rows(a.k, a.k_st, a.k_sh), rv = rows(a.v, a.v_st, a.v_sh), rr = rows(a.kr, a.kr_st, 0);
  const auto stage = [&](int i, u32x4* buf) {
    stage_tile<kWaves, true>(rk, i, buf, wave, lane);
    stage_tile<kWaves, true>(rv, i, buf + kWide, wave, lane);
    stage_tile<kWaves, false>(rr, i, buf + 2 * kWide, wave, lane);
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
  const auto step = [&](auto masked, int i) {
    constexpr bool edge = decltype(masked)::value;
    const char* bk = reinterpret_cast<const char*>(lds + (i & 1) * kBufDq);
    const char* bv = bk + kWide * 16;
    const char* br = bk + 2 * kWide * 16;
    if (i + 1 < n) stage(i + 1, lds + ((i + 1) & 1) * kBufDq);
    f32x16 s[2], dp[2];
#pragma unroll
    for (int th = 0; th < 2; th++)
#pragma unroll
      for (int r = 0; r < 16; r++) s[th][r] = dp[th][r] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < 12; kk++)
#pragma unroll
      for (int th = 0; th < 2; th++) {
        const u32x4 op = kk < 8 ? *reinterpret_cast<const u32x4*>(bk + 8192 * th + ow[kk & 7])
                                : *reinterpret_cast<const u32x4*>(br + 4096 * th + os[(kk - 8) & 3]);
        s[th] = mfma(as_bf16x8(op), qf[kk], s[th]);
        if (kk < 8)
          dp[th] = mfma(as_bf16x8(*reinterpret_cast<const u32x4*>(bv + 8192 * th + ow[kk & 7])), df[kk & 7], dp[th]);
      }
    const int hi = row + 1 - i * kLatTile - 4 * hh;
    bf16x8 db[4];
#pragma unroll
    for (int th = 0; th < 2; th++)
#pragma unroll
      for (int s2 = 0; s2 < 2; s2++) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          float d[2];
#pragma unroll
          for (int u = 0; u < 2; u++) {
            const int j = 8 * s2 + 2 * e + u, key = 32 * th + 8 * (j >> 2) + (j & 3);
            const float p = __builtin_amdgcn_exp2f(fmaf(s[th][j], c2, -ld.x));
            d[u] = p * (dp[th][j] - ld.y);
            if (edge) d[u] = key < hi ? d[u] : 0.0f;
          }
          w[e] = pack_bf16(d[0], d[1]);
        }
        db[2 * th + s2] = as_bf16x8(u32x4{w[0], w[1], w[2], w[3]});
      }
#pragma unroll
    for (int ks = 0; ks < 4; ks++)
#pragma unroll
      for (int dt = 0; dt < 6; dt++) {
        const char* b = dt < 4 ? bk + 16 * ks * 256 : br + 16 * ks * 128;
        const bf16x8 kt = dt < 4 ? join16(tr16(b + tw[0][dt & 3]), tr16(b + tw[1][dt & 3]))
                                 : join16(tr16(b + ts[0][dt & 1]), tr16(b + ts[1][dt & 1]));
        acc[dt] = mfma(kt, db[ks], acc[dt]);
      }
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

// ============================================================== dK, dV
constexpr int kBufKv = 2 * kWide + kSlim;  // q's first 128 dims, dout, q's rotary dims

__global__ __launch_bounds__(64 * kWaves, 1) void latent_dkdv_kernel(LatentArgs a) {
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
  const auto stage = [&](int i, u32x4* buf) {
    stage_tile<kWaves, true>(rq, i, buf, wave, lane);
    stage_tile<kWaves, true>(rd, i, buf + kWide, wave, lane);
    stage_tile<kWaves, false>(rr, i, buf + 2 * kWide, wave, lane);
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
    float2 nx;
    const bool more = i + 1 < n;
    if (more) {
      if (wave == 0) nx = row_ld(i + 1);
      stage(i + 1, lds + (cur ^ 1) * kBufKv);
    }
#pragma unroll
    for (int st = 0; st < 2; st++) {
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; r++) s[r] = dp[r] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < 12; kk++) {
        const u32x4 op = kk < 8 ? *reinterpret_cast<const u32x4*>(bq + 8192 * st + ow[kk & 7])
                                : *reinterpret_cast<const u32x4*>(br + 4096 * st + os[(kk - 8) & 3]);
        s = mfma(as_bf16x8(op), kf[kk], s);
        if (kk < 8)
          dp = mfma(as_bf16x8(*reinterpret_cast<const u32x4*>(bd + 8192 * st + ow[kk & 7])), vf[kk & 7], dp);
      }
      bf16x8 pb[2], sb[2];
#pragma unroll
      for (int s2 = 0; s2 < 2; s2++) {
        uint32_t wp[4], wd[4];
#pragma unroll
        for (int x = 0; x < 2; x++) {  // rows 32 st + 16 s2 + 8 x + 4 hh + (0 .. 3)
          const int r0 = 32 * st + 16 * s2 + 8 * x + 4 * hh;
          const float4 l4 = *reinterpret_cast<const float4*>(&lse2[cur][r0]);
          const float4 d4 = *reinterpret_cast<const float4*>(&dlt[cur][r0]);
          const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
          float p[4], d[4];
#pragma unroll
          for (int c = 0; c < 4; c++) {
            const int j = 8 * s2 + 4 * x + c;
            p[c] = __builtin_amdgcn_exp2f(fmaf(s[j], c2, -lv[c]));
            d[c] = p[c] * (dp[j] - dl[c]);
            if (edge) {
              const bool sees = i * kLatTile + r0 + c >= key;
              p[c] = sees ? p[c] : 0.0f;
              d[c] = sees ? d[c] : 0.0f;
            }
          }
          wp[2 * x] = pack_bf16(p[0], p[1]);
          wp[2 * x + 1] = pack_bf16(p[2], p[3]);
          wd[2 * x] = pack_bf16(d[0], d[1]);
          wd[2 * x + 1] = pack_bf16(d[2], d[3]);
        }
        pb[s2] = as_bf16x8(u32x4{wp[0], wp[1], wp[2], wp[3]});
        sb[s2] = as_bf16x8(u32x4{wd[0], wd[1], wd[2], wd[3]});
      }
#pragma unroll
      for (int s2 = 0; s2 < 2; s2++) {
        const int r0 = 32 * st + 16 * s2;
#pragma unroll
        for (int dt = 0; dt < 4; dt++)
          dv[dt] = mfma(join16(tr16(bd + r0 * 256 + tw[0][dt]), tr16(bd + r0 * 256 + tw[1][dt])), pb[s2], dv[dt]);
#pragma unroll
        for (int dt = 0; dt < 4; dt++)
          dk[dt] = mfma(join16(tr16(bq + r0 * 256 + tw[0][dt]), tr16(bq + r0 * 256 + tw[1][dt])), sb[s2], dk[dt]);
#pragma unroll
        for (int dt = 0; dt < 2; dt++)
          dk[4 + dt] =
              mfma(join16(tr16(br + r0 * 128 + ts[0][dt]), tr16(br + r0 * 128 + ts[1][dt])), sb[s2], dk[4 + dt]);
      }
    }
    dma_wait();
    if (more && wave == 0) {
      lse2[cur ^ 1][lane] = nx.x;
      dlt[cur ^ 1][lane] = nx.y;
    }
    __syncthreads();
  };
  // (the diagonal's rows, and those of the last tile, which may end past the sequence: their lse is inf)
  const int iedge = min(n, i0 + kLatKeys / kLatTile);
  for (int i = i0; i < iedge; i++) step(std::true_type(), i);
  for (int i = iedge; i < n; i++) step(std::false_type(), i);

  if (key >= pl.len) return;
  const float scl = a.scale;
  __hip_bfloat16* krow = a.dk + kt * a.dk_st + (int64_t)h * a.dk_sh;
  __hip_bfloat16* vrow = a.dv + kt * a.dv_st + (int64_t)h * a.dv_sh;
  float* rrow = a.dkr_part + ((int64_t)h * a.T + kt) * kRopeDim;
#pragma unroll
  for (int dt = 0; dt < 4; dt++)
#pragma unroll
    for (int r4 = 0; r4 < 4; r4++) {
      const int d = 32 * dt + 8 * r4 + 4 * hh;
      *reinterpret_cast<uint2*>(krow + d) = make_uint2(pack_bf16(dk[dt][4 * r4] * scl, dk[dt][4 * r4 + 1] * scl),
                                                       pack_bf16(dk[dt][4 * r4 + 2] * scl, dk[dt][4 * r4 + 3] * scl));
      *reinterpret_cast<uint2*>(vrow + d) = make_uint2(pack_bf16(dv[dt][4 * r4], dv[dt][4 * r4 + 1]),
                                                       pack_bf16(dv[dt][4 * r4 + 2], dv[dt][4 * r4 + 3]));
    }
#pragma unroll
  for (int dt = 0; dt < 2; dt++)
#pragma unroll
    for (int r4 = 0; r4 < 4; r4++)
      *reinterpret_cast<float4*>(rrow + 32 * dt + 8 * r4 + 4 * hh) =
          make_float4(dk[4 + dt][4 * r4] * scl, dk[4 + dt][4 * r4 + 1] * scl, dk[4 + dt][4 * r4 + 2] * scl,
                      dk[4 + dt][4 * r4 + 3] * scl);
}

// dkr: a thread sums four dims of a token over the heads, in their order.
__global__ __launch_bounds__(256) void latent_dkr_kernel(LatentArgs a) {
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t t = x / (kRopeDim / 4);
  if (t >= a.T) return;
  if (t < a.cu[0] || t >= a.cu[a.S]) return;  // (a row of no sequence: left as it is)
  const int c = (int)(x % (kRopeDim / 4));
  const float4* p = reinterpret_cast<const float4*>(a.dkr_part) + t * (kRopeDim / 4) + c;
  float4 s = p[0];
  for (int h = 1; h < a.H; h++) {
    const float4 y = p[(int64_t)h * a.T * (kRopeDim / 4)];
    s.x += y.x;
    s.y += y.y;
    s.z += y.z;
    s.w += y.w;
  }
  reinterpret_cast<uint2*>(a.dkr + t * a.dkr_st)[c] = make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
}

}  // namespace

hipError_t launch_latent_delta(const LatentArgs& a, hipStream_t st) {
  latent_delta_kernel<<<(unsigned)((a.T * a.H + 15) / 16), 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_latent_dq(const LatentArgs& a, hipStream_t st) {
  latent_dq_kernel<<<latent_grid(a, kLatRowsDq), 64 * kWaves, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_latent_dkdv(const LatentArgs& a, hipStream_t st) {
  latent_dkdv_kernel<<<latent_grid(a, kLatKeys), 64 * kWaves, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_latent_dkr(const LatentArgs& a, hipStream_t st) {
  latent_dkr_kernel<<<(unsigned)((a.T * (kRopeDim / 4) + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace moba
