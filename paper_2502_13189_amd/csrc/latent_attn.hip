// Causal latent attention, expanded form: z_ij = scale (<q_i[0:128], k_j> + <q_i[128:192], kr_j>),
// out_i = sum_j softmax(z_i)_j v_j, where kr is one rotary key for all heads.
//
// Bound by the matrix cores: 640 operations a scored pair and 640 bytes a (head, token).  Work-group = NW
// waves (8, or 4 for small batches) = 32 NW queries of one head; wave w owns queries 32w .. 32w + 31, one per
// lane column.  Keys come in tiles of 64: k and v (128 dims each) and kr (64) are staged row-major in LDS by
// DMA, two buffers each (80 KiB), tile i + 1 in flight while tile i is used, one barrier a tile.  On
// v_mfma_f32_32x32x16_bf16, per tile and wave:
//   S^T (keys x queries) = K . Q^T    2 halves x 12 k-steps, Q in registers
//   online softmax in 32 bits: a lane holds one query and 32 of the 64 keys.  Weights are formed
//     under the running max, which is raised only when a lane's weights sum to more than 2^8
//   O^T (dims x queries) += V^T . P^T  4 dim tiles x 4 k-steps, V^T by transposed LDS reads
// Queries and keys are cut at the same multiples of 32, so of a wave's halves of tiles one is masked, the
// diagonal one; those before it are whole, those behind it are left out.
// The weights enter the second product as bf16 (at most 2^-8 of each, independent of each other: it adds
// to the result about what its own rounding to bf16 does, 0.0020 of its 2-norm against 0.0015); all sums are fp32.
// 16384 tokens, 32 heads: 2.26 to 2.36 ms, 1.16 to 1.22 PFLOP/s of the 1.23 to 1.39 that large matrix products reach here
// (the chip's clock falls under either).
#include "latent_tile.h"

#include <math.h>

namespace moba {
namespace {

constexpr int kBufChunks = 2 * kWide + kSlim;  // k, v, kr
constexpr float kSumLimit = 256.0f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kStageRow = kNope / 8 + 1;  // 16-byte chunks of a staged result row (one pad)

// P^T operands of NH halves of a tile under the running max m; returns the lane's sum of weights.
template <int NH>
__device__ __forceinline__ float weights(const f32x16 (&s)[NH], float m, bf16x8 (&pb)[2 * NH], float c2) {
  float ts = 0.0f;
#pragma unroll
  for (int th = 0; th < NH; th++)
#pragma unroll
    for (int s2 = 0; s2 < 2; s2++) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[th][8 * s2 + 2 * e], c2, -m));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[th][8 * s2 + 2 * e + 1], c2, -m));
        w[e] = pack_bf16(p0, p1);
        ts += p0 + p1;
      }
      pb[2 * th + s2] = as_bf16x8(u32x4{w[0], w[1], w[2], w[3]});
    }
  return ts;
}

template <int NH>
__device__ __forceinline__ void softmax(const f32x16 (&s)[NH], float& m, float& l, f32x16 (&o)[4],
                                        bf16x8 (&pb)[2 * NH], float c2) {
  float ts = 0.0f;
  bool redo = __builtin_amdgcn_ballot_w64(m == -INFINITY) != 0;
  if (!redo) {
    ts = weights(s, m, pb, c2);
    redo = __builtin_amdgcn_ballot_w64(!(ts <= kSumLimit)) != 0;
  }
  if (redo) {
    float mx = -INFINITY;
#pragma unroll
    for (int th = 0; th < NH; th++)
#pragma unroll
      for (int r = 0; r < 16; r++) mx = fmaxf(mx, s[th][r]);
    mx = fmaxf(mx, xor32(mx)) * c2;
    const float m_new = fmaxf(m, mx);
    const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < 4; dt++)
#pragma unroll
      for (int r = 0; r < 16; r++) o[dt][r] *= alpha;
    m = m_new;
    ts = weights(s, m == -INFINITY ? 0.0f : m, pb, c2);
  }
  l += ts;
}

// Whether 32 rows of a wide tile hold a value that is not finite (all lanes alike).
__device__ __forceinline__ bool holds_odd(const char* vb, int lane) {
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
  u16x8 most = 0;
#pragma unroll
  for (int j = 0; j < kWide / 128; j++) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(vb + (64 * j + lane) * 16) & 0x7f807f80u;
    most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x8, w));
  }
  int odd = 0;
#pragma unroll
  for (int e = 0; e < 8; e++) odd |= most[e] == 0x7f80;
  return __builtin_amdgcn_ballot_w64(odd != 0) != 0;
}

// O^T += V^T . P^T of a diagonal half that holds values that are not finite: a weight of 0 must not
// meet them, since a row may not see what it does not attend.  One key at a time, and a row takes
// the product of those that it attends.  hi: keys of the half that the lane's row attends.
__device__ __forceinline__ void pv_by_key(f32x16 (&o)[4], const char* vb, const uint32_t (&ov)[2][4],
                                          const bf16x8 (&pb)[2], int hi, int hh) {
#pragma unroll
  for (int ks = 0; ks < 2; ks++)
#pragma unroll 1
    for (int kk = 0; kk < 16; kk++) {
      u32x4 only;  // element e of an operand: key 16 ks + 8 (e / 4) + 4 hh + e % 4
#pragma unroll
      for (int w = 0; w < 4; w++) {
        const int k0 = 8 * (w >> 1) + 4 * hh + 2 * (w & 1);
        only[w] = k0 == kk ? 0xffffu : k0 + 1 == kk ? 0xffff0000u : 0;
      }
      const bool attends = 16 * ks + kk < hi;
#pragma unroll
      for (int dt = 0; dt < 4; dt++) {
        const char* b = vb + 16 * ks * 256;
        const u32x4 v = __builtin_bit_cast(u32x4, join16(tr16(b + ov[0][dt]), tr16(b + ov[1][dt])));
        f32x16 t;
#pragma unroll
        for (int r = 0; r < 16; r++) t[r] = 0.0f;
        t = mfma(as_bf16x8(v & only), pb[ks], t);
#pragma unroll
        for (int r = 0; r < 16; r++) o[dt][r] += attends ? t[r] : 0.0f;
      }
    }
}

// Whether work-groups are ranked by the length of their chains, so that a chip that is filled a few times over ends
// with short ones (but a head's work-groups then lie on all XCDs).  As latent_work has them and ranked, us: 8192
// tokens, 10 heads 335, 217; 4 x 2000, 16 heads 117, 97; 1000 and 40 x 100, 16 heads 46, 32; 4096, 32 heads 188, 176; 8 x
// 300, 128 heads 108, 104; 8 x 1000, 4 heads 33, 30.  Below a work-group a CU there is no order (2048, 4 heads 45, 46), and
// sequences of a tile have no chains (40 x 64, 32 heads 26, 28).
__device__ __forceinline__ bool by_rank(const LatentArgs& a, int64_t groups) {
  return a.S <= kLatRankedSeqs && groups > 256 && groups <= kLatRanked && a.T > (int64_t)kLatTile * a.S;
}

template <int NW>
__global__ __launch_bounds__(64 * NW, 8 / NW) void latent_forward_kernel(LatentArgs a) {
  constexpr int kRows = 32 * NW;
  __shared__ u32x4 lds[2 * kBufChunks];
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qc = lane & 31, hh = lane >> 5;

  Place pl;
  int h;
  const int64_t places = latent_places(a.T, a.S, kRows);
  if (kRows == kLatKeys && by_rank(a, places * a.H)) {
    int more;
    if (!latent_ranked(a, blockIdx.x, &pl, &h, &more)) return;
  } else {
    Work wk;
    if (!latent_work<true>(a, places, &wk)) return;
    if (!latent_place(a, wk.place, kRows, &pl)) return;
    h = __builtin_amdgcn_readfirstlane(wk.h);
  }
  const int row = pl.t0 + 32 * wave + qc;         // this lane's query, within the sequence
  const int rc = min(row, pl.len - 1);
  const int kend = min(pl.t0 + kRows, pl.len);
  const int base = pl.t0 + 32 * wave;             // the wave's first query

  bf16x8 qf[12];
  {
    const __hip_bfloat16* qrow = a.q + (pl.tok0 + rc) * a.q_st + (int64_t)h * a.q_sh + 8 * hh;
#pragma unroll
    for (int kk = 0; kk < 12; kk++) qf[kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(qrow + 16 * kk));
  }
  const auto rows = [&](const __hip_bfloat16* p, int64_t st, int64_t sh) {
    return Rows{scalar_ptr(p + pl.tok0 * st + (int64_t)h * sh), (uint32_t)(st * 2), pl.len};
  };
  const Rows rk = rows(a.k, a.k_st, a.k_sh), rv = rows(a.v, a.v_st, a.v_sh), rr = rows(a.kr, a.kr_st, 0);
  const auto stage = [&](int i, u32x4* buf) {
    stage_tile<NW, true>(rk, i, buf, wave, lane);
    stage_tile<NW, true>(rv, i, buf + kWide, wave, lane);
    stage_tile<NW, false>(rr, i, buf + 2 * kWide, wave, lane);
  };

  // operand offsets: rows qc (+ 32: the same swizzle, 32 rows on), chunk 2 kk + hh
  uint32_t ok[8], orr[4], ov[2][4];
#pragma unroll
  for (int kk = 0; kk < 8; kk++) ok[kk] = at_wide(qc, 2 * kk + hh);
#pragma unroll
  for (int kk = 0; kk < 4; kk++) orr[kk] = at_slim(qc, 2 * kk + hh);
  const TrLane tl = tr_lane(qc, hh);
#pragma unroll
  for (int x = 0; x < 2; x++)
#pragma unroll
    for (int dt = 0; dt < 4; dt++) ov[x][dt] = tr_wide(tl, dt, x);

  const float c2 = a.scale_log2;
  f32x16 o[4];
  float m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int dt = 0; dt < 4; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) o[dt][r] = 0.0f;

  const int n = (kend + kLatTile - 1) / kLatTile;
  stage(0, lds);
  dma_wait();
  __syncthreads();
  const int nfull = pl.t0 / kLatTile;  // tiles before the diagonal's
  for (int i = 0; i < nfull; i++) {
    const char* buf = reinterpret_cast<const char*>(lds + (i & 1) * kBufChunks);
    if (i + 1 < n) stage(i + 1, lds + ((i + 1) & 1) * kBufChunks);
    f32x16 s[2];
    {
      const char* bk = buf;
      const char* br = buf + 2 * kWide * 16;
#pragma unroll
      for (int th = 0; th < 2; th++)
#pragma unroll
        for (int r = 0; r < 16; r++) s[th][r] = 0.0f;
      u32x4 op[24];
#pragma unroll
      for (int j = 0; j < 24; j++) {
        const int th = j & 1, kk = j >> 1;
        op[j] = kk < 8 ? *reinterpret_cast<const u32x4*>(bk + 8192 * th + ok[kk & 7])
                       : *reinterpret_cast<const u32x4*>(br + 4096 * th + orr[(kk - 8) & 3]);
      }
#pragma unroll
      for (int j = 0; j < 24; j++) s[j & 1] = mfma(as_bf16x8(op[j]), qf[j >> 1], s[j & 1]);
      __builtin_amdgcn_sched_group_barrier(0x100, kPre, 0);
#pragma unroll
      for (int j = 0; j < 24 - kPre; j++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, kPre, 0);
    }
    bf16x8 pb[4];
    softmax(s, m, l, o, pb, c2);
    {
      const char* bv = buf + kWide * 16;
      s16x4 t0[16], t1[16];
#pragma unroll
      for (int j = 0; j < 16; j++) {
        const char* b = bv + 16 * (j >> 2) * 256;
        t0[j] = tr16(b + ov[0][j & 3]);
        t1[j] = tr16(b + ov[1][j & 3]);
      }
#pragma unroll
      for (int j = 0; j < 16; j++) o[j & 3] = mfma(join16(t0[j], t1[j]), pb[j >> 2], o[j & 3]);
      __builtin_amdgcn_sched_group_barrier(0x100, 2 * kPre, 0);
#pragma unroll
      for (int j = 0; j < 16 - kPre; j++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, kPre, 0);
    }
    dma_wait();
    __syncthreads();
  }
  // the diagonal's tiles, by halves: each wave those up to its own rows' (and none if it has no rows)
  const int stop = base < pl.len ? base : -1;
  for (int i = nfull; i < n; i++) {
    if (i + 1 < n) stage(i + 1, lds + ((i + 1) & 1) * kBufChunks);
#pragma unroll 1
    for (int th = 0; th < 2; th++) {
      const int u0 = i * kLatTile + 32 * th;
      if (u0 > stop) break;
      const char* bk = reinterpret_cast<const char*>(lds + (i & 1) * kBufChunks) + 8192 * th;
      const char* bv = bk + kWide * 16;
      const char* br = reinterpret_cast<const char*>(lds + (i & 1) * kBufChunks) + 2 * kWide * 16 + 4096 * th;
      f32x16 s[1];
#pragma unroll
      for (int r = 0; r < 16; r++) s[0][r] = 0.0f;
      u32x4 op[12];
#pragma unroll
      for (int j = 0; j < 12; j++)
        op[j] = j < 8 ? *reinterpret_cast<const u32x4*>(bk + ok[j & 7]) : *reinterpret_cast<const u32x4*>(br + orr[(j - 8) & 3]);
#pragma unroll
      for (int j = 0; j < 12; j++) s[0] = mfma(as_bf16x8(op[j]), qf[j], s[0]);
      const bool diagonal = u0 == stop;
      if (diagonal) {
#pragma unroll
        for (int r = 0; r < 16; r++)
          if (8 * (r >> 2) + 4 * hh + (r & 3) > qc) s[0][r] = -INFINITY;
      }
      bf16x8 pb[2];
      softmax(s, m, l, o, pb, c2);
      if (diagonal && holds_odd(bv, lane)) {
        pv_by_key(o, bv, ov, pb, qc + 1, hh);
      } else {
        s16x4 t0[8], t1[8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const char* b = bv + 16 * (j >> 2) * 256;
          t0[j] = tr16(b + ov[0][j & 3]);
          t1[j] = tr16(b + ov[1][j & 3]);
        }
#pragma unroll
        for (int j = 0; j < 8; j++) o[j & 3] = mfma(join16(t0[j], t1[j]), pb[j >> 2], o[j & 3]);
      }
    }
    dma_wait();
    __syncthreads();
  }

  // the buffers are free: each wave stages its 32 rows and writes them whole
  const float lt = l + xor32(l);
  const float inv = 1.0f / lt;
  if (hh == 0 && row < pl.len)
    a.lse[(int64_t)h * a.T + pl.tok0 + row] = (m + __builtin_amdgcn_logf(lt)) * kLn2;
  u32x4* stg = lds + wave * 32 * kStageRow;
  uint2* srow = reinterpret_cast<uint2*>(stg + qc * kStageRow);
#pragma unroll
  for (int dt = 0; dt < 4; dt++)
#pragma unroll
    for (int r4 = 0; r4 < 4; r4++)
      srow[(32 * dt + 8 * r4 + 4 * hh) >> 2] =
          make_uint2(pack_bf16(o[dt][4 * r4] * inv, o[dt][4 * r4 + 1] * inv),
                     pack_bf16(o[dt][4 * r4 + 2] * inv, o[dt][4 * r4 + 3] * inv));
  __builtin_amdgcn_s_waitcnt(0);  // (a wave's own LDS writes, read by its other lanes)
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const int rr2 = 4 * j + (lane >> 4), t = base + rr2;
    if (t < pl.len)
      reinterpret_cast<u32x4*>(a.out + (pl.tok0 + t) * a.o_st + (int64_t)h * a.o_sh)[lane & 15] =
          stg[rr2 * kStageRow + (lane & 15)];
  }
}

}  // namespace

// Queries of a work-group: 256, which reads k and v half as often, where many long sequences' work fills the chip; else
// 128, two work-groups on a CU, which leaves fewer waves without rows and the last ones alone for less long.  256 and
// 128 (ranked where by_rank says so), us: 1 x 256 tokens, 32 heads 16.5, 12.9; 8 x 1000, 4 heads 37.2, 30.0; 4096, 8
// heads 111, 87; 100 x 100, 32 heads 140, 103; 4096, 32 heads 204, 176; 2048, 128 heads 208, 196; 8192, 32 heads 604, 609;
// 16384, 32 heads 2278, 2358.
hipError_t launch_latent_forward(const LatentArgs& a, hipStream_t st) {
  if (latent_places(a.T, a.S, kLatRows) * a.H <= kLatFew || a.T < kLatLong * (int64_t)a.S)
    latent_forward_kernel<4><<<latent_grid(a, 128), 256, 0, st>>>(a);
  else
    latent_forward_kernel<8><<<latent_grid(a, 256), 512, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace moba
