// Decode over the paged 8-bit cache: one new query per request, full attention or MoBA.
//
// Every attended key and value is one byte per dim, read once per kv-head for all query
// heads of its group: 256 bytes for at most 4 x 128 x 16 FLOP, so HBM bounds it.
//
// Lengths are known on the device alone.  For full attention the batch's keys are cut into
// 64-key steps and the steps, request after request, into equal shares, one wave each; every wave
// finds its own share from a prefix sum over the lengths.  So a ragged batch, one long
// request and many short ones all keep the chip evenly busy, and the workspace does not depend on
// lengths: a share leaves at most two partial rows (the one it enters with and the one it leaves
// with), which a second launch joins; a row inside one share is finished there.  A MoBA row
// has no more steps than its heads choose blocks, so rows differ little and each gets as
// many work-groups as the other (parts).  Where rows are short, a work-group per row does all
// in one launch instead (rows).
//
//   attend  a step's K and V go from memory to the matrix cores through registers alone.
//           S^T = K q^T on 16x16x32 MFMAs: a lane has 16 bytes of a key for two operands.
//           The keys of a step are dealt to the four 16-key operands so that a lane's 16
//           scores of a head are 16 consecutive tokens, which is what it then needs as the
//           operand of O^T = V^T P^T, with V's 16 tokens of a dim being one 16-byte load of the
//           page's token-minor tile.  e4m3 is exact in bf16; the weights enter as three
//           bf16 terms, which hold their 24 bits (in two, 17 bits, whole calls over 1M tokens take
//           355.4 us, so 355.8; a ragged batch 46.0 and 47.2), the scales through the logits and the
//           weights.  1M tokens, 32/8 heads: 2.15 GB, 354 us a call in
//           a row with the join (6.1 TB/s, bare loads reach 6.2), 349 us the launch at
//           best; more loads in flight (next keys or whole steps ahead) or more waves gain
//           nothing.
//   gate    MoBA: a wave adds a block's k_sum rows and takes its scores with the group's
//           heads, in 64 bits
//   parts   MoBA: a wave finds the (k-1)-th highest score of a head bit by bit; the group's
//           heads' blocks become one ascending list with a mask of heads for each, and the
//           work-group attends its part of their steps
//   join    log-sum-exp merge of split rows
//   rows    all of it for one (request, kv-head)
#include "cache_internal.h"
#include "decode_internal.h"

#include <math.h>

#include <type_traits>

namespace moba {
namespace {

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kRescale = 8.0f;  // a running max may lag by 2^8 before sums are rescaled

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// Eight e4m3 codes to eight bf16, exactly.
__device__ __forceinline__ bf16x8_t to_bf16(uint32_t a, uint32_t b) {
  union {
    bf16x2_t h[4];
    bf16x8_t v;
  } r;
  r.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
  r.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  r.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
  r.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  return r.v;
}

// Tokens request s attends.
__device__ __forceinline__ int held(const CacheDecodeArgs& a, int s) {
  return (int)min((int64_t)max(a.lens[s], 0), (int64_t)a.W * a.c.P);
}

// ------------------------------------------------------------------ shares
// The rows' units in a sum over all rows: pre[i] units lie before the i-th of the 256
// groups of `per` rows.  (The host sees to it that the sum stays below 2^31.)
struct Sums {
  int pre[kCacheDecodeThreads];
  int part[kCacheDecodeThreads / 64];
  int total;
};

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from 1 lane below in a row of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row 0's last to row 1, 2's to 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31's to rows 2 and 3
  return x;
}

template <typename F>
__device__ __forceinline__ void sum_rows(Sums& sm, int rows, F units) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (rows + kCacheDecodeThreads - 1) / kCacheDecodeThreads;
  int mine = 0;
  for (int i = 0, r = tid * per; i < per && r < rows; i++, r++) mine += units(r);
  int x = wave_scan(mine);
  if (lane == 63) sm.part[wave] = x;
  __syncthreads();
  for (int w = 0; w < wave; w++) x += sm.part[w];
  sm.pre[tid] = x - mine;
  if (tid == kCacheDecodeThreads - 1) sm.total = x;
  __syncthreads();
}

// The row that unit u (< total) belongs to, for a whole wave; base: units before the row.
template <typename F>
__device__ __forceinline__ int find_row(const Sums& sm, int rows, int u, F units, int* base) {
  const int lane = threadIdx.x & 63;
  const int per = (rows + kCacheDecodeThreads - 1) / kCacheDecodeThreads;
  int below = 0;  // groups that begin at or before u (the last of them is not empty)
#pragma unroll
  for (int i = 0; i < kCacheDecodeThreads / 64; i++)
    below += __popcll(__ballot(sm.pre[64 * i + lane] <= u));
  const int r0 = (below - 1) * per, r1 = min(r0 + per, rows);
  int acc = sm.pre[below - 1];
  if (per == 1) {
    *base = __builtin_amdgcn_readfirstlane(acc);
    return r0;
  }
  for (int r = r0; r < r1; r += 64) {
    const int n = r + lane < r1 ? units(r + lane) : 0;
    const int x = wave_scan(n);
    const unsigned long long past = __ballot(acc + x > u);
    if (past) {
      const int at = __ffsll((long long)past) - 1;
      *base = __builtin_amdgcn_readlane(acc + x - n, at);
      return r + at;
    }
    acc += __builtin_amdgcn_readlane(x, 63);
  }
  *base = 0;  // (not reached: u < total)
  return rows;
}

// ------------------------------------------------------------------ attend
// A step: 64 keys of one page.
struct Step {
  int64_t page;   // 0 where the table's entry is none of the pool
  int tile;       // 64-token tile of the page
  int nk;         // keys attended: the step's first nk
  uint32_t heads; // of the group, that attend it
};

struct Tile {
  u32x4_t k[4][2];  // operand t, dims 64 j + 16 (lane / 16)
  u32x4_t v[8];     // dim 16 i + lane % 16, tokens 16 (lane / 16) ..
  float ks, vs;
};

// Sums of a row's steps: head lane % 16 of the group, dims 16 i + 4 (lane / 16) + e.
struct Row {
  f32x4_t acc[8];
  float m, l;  // running maximum (log2 domain) and sum of weights
};

// Attends steps first .. last - 1 of request s (length len) for kv-head g, by one wave.
// MOBA: steps of the listed blocks, otherwise of all keys.
template <bool MOBA>
__device__ __forceinline__ void attend_steps(const CacheDecodeArgs& a, int s, int g, int len,
                                             const uint32_t* list, int first, int last, Row& r) {
  const CachePool& c = a.c;
  const int Hkv = c.Hkv, G = a.G, P = c.P;
  const int lane = threadIdx.x & 63, hc = lane & 15, quad = lane >> 4;
  const int spb = MOBA ? a.B / kCacheTile : 0;  // steps per block
  const int koff = (16 * (hc >> 2) + (hc & 3)) * kHeadDim + 16 * quad;
  const int voff = hc * kCacheTile + 16 * quad;
  const int32_t* row = a.table + s * a.t_ss;
  // B operands: q of head hc, the dims of the K operands
  bf16x8_t qb[4];
  {
    const __hip_bfloat16* qp = a.q + s * a.q_ss + (int64_t)(g * G + min(hc, G - 1)) * a.q_sh;
#pragma unroll
    for (int f = 0; f < 4; f++)
      qb[f] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(
                                               qp + 64 * (f >> 1) + 16 * quad + 8 * (f & 1)));
  }
  const auto step_at = [&](int x) {
    Step st;
    int tok = kCacheTile * x;
    st.heads = 0xffffu;
    if constexpr (MOBA) {
      const int bi = x / spb;
      const uint32_t e = __builtin_amdgcn_readfirstlane(list[bi]);
      tok = (int)(e & 0xffffu) * a.B + kCacheTile * (x - bi * spb);
      st.heads = e >> 16;
    }
    const int pn = tok / P;
    const int id = row[pn];
    const bool ok = (uint32_t)id < (uint32_t)c.N;
    st.page = ok ? id : 0;
    st.tile = (tok - pn * P) / kCacheTile;
    st.nk = ok ? min(kCacheTile, len - tok) : 0;
    return st;
  };
  const auto load = [&](Tile& t, const Step& st) {
    const uint8_t* kp = c.k + st.page * c.k_sp + g * c.k_sh + st.tile * (kCacheTile * kHeadDim);
    const uint8_t* vp = c.v + st.page * c.v_sp + g * c.v_sh + st.tile * (kCacheTile * kHeadDim);
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int j = 0; j < 2; j++)
        t.k[i][j] = *reinterpret_cast<const u32x4_t*>(kp + koff + 4 * kHeadDim * i + 64 * j);
#pragma unroll
    for (int i = 0; i < 8; i++)
      t.v[i] = *reinterpret_cast<const u32x4_t*>(vp + voff + 16 * kCacheTile * i);
    t.ks = c.k_scale[st.page * Hkv + g];
    t.vs = c.v_scale[st.page * Hkv + g];
  };
  f32x4_t(&acc)[8] = r.acc;
#pragma unroll
  for (int i = 0; i < 8; i++) acc[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -INFINITY, l = 0.0f;
  const auto fold = [&](Tile& t, const Step& st) {
    // a lane's scores: head hc, tokens 16 quad + 4 i + e
    float z[16];
    const float zs = t.ks * a.scale_log2;
    const bool mine = !MOBA || ((st.heads >> hc) & 1);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int f = 0; f < 4; f++) {
        const u32x4_t kw = t.k[i][f >> 1];
        x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            f & 1 ? to_bf16(kw[2], kw[3]) : to_bf16(kw[0], kw[1]), qb[f], x, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 4; e++) z[4 * i + e] = x[e] * zs;
    }
    if (st.nk < kCacheTile) {
      const int left = st.nk - 16 * quad;  // of this lane's tokens
      if (st.nk <= 0) t.vs = 0.0f;  // (no page: its scale may be anything, too)
#pragma unroll
      for (int i = 0; i < 16; i++) z[i] = i < left ? z[i] : -INFINITY;
      // their values may hold anything
#pragma unroll
      for (int i = 0; i < 8; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const int n = min(max(left - 4 * e, 0), 4);
          t.v[i][e] &= n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1;
        }
    }
    if constexpr (MOBA) {
#pragma unroll
      for (int i = 0; i < 16; i++) z[i] = mine ? z[i] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < 16; i++) top = fmaxf(top, z[i]);
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    if (__ballot(top > m + kRescale || (m == -INFINITY && top > -INFINITY))) {
      const float mn = fmaxf(m, top);
      const float sc = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= sc;
#pragma unroll
      for (int i = 0; i < 8; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) acc[i][e] *= sc;
    }
    const float mr = m == -INFINITY ? 0.0f : m;
    // weights times the page's scale, as three bf16 terms: all 24 bits
    u32x4_t w[3][2];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float p0 = __builtin_amdgcn_exp2f(z[2 * i] - mr);
      const float p1 = __builtin_amdgcn_exp2f(z[2 * i + 1] - mr);
      l += p0 + p1;
      float v0 = p0 * t.vs, v1 = p1 * t.vs;
#pragma unroll
      for (int n = 0; n < 3; n++) {
        const uint32_t x = pack_bf16(v0, v1);
        w[n][i >> 2][i & 3] = x;
        v0 -= bf16_lo(x);
        v1 -= bf16_hi(x);
      }
    }
    const auto product = [&](const bf16x8_t& vb, int n, int f, const f32x4_t& o) {
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, __builtin_bit_cast(bf16x8_t, w[n][f]), o, 0, 0, 0);
    };
    if constexpr (MOBA) {
      // A head that does not attend the block has weights of 0 there, but 0 times a NaN among
      // its values is NaN: such a sum stays as it was.  (One sum at a time, in few registers: 50
      // requests of 4096 tokens 57.7 us, two at a time 61.4.)
#pragma unroll
      for (int i = 0; i < 8; i++) {
        f32x4_t o = acc[i];
#pragma unroll
        for (int f = 0; f < 2; f++) {
          const bf16x8_t vb = to_bf16(t.v[i][2 * f], t.v[i][2 * f + 1]);
#pragma unroll
          for (int n = 0; n < 3; n++) o = product(vb, n, f, o);
        }
#pragma unroll
        for (int e = 0; e < 4; e++) acc[i][e] = mine ? o[e] : acc[i][e];
      }
      return;
    }
    // Two sums side by side: a product waits for the one before it in its own sum.  (Ragged batch
    // 48.9 us one after the other, 47.2 so.)
#pragma unroll
    for (int i0 = 0; i0 < 8; i0 += 2) {
#pragma unroll
      for (int f = 0; f < 2; f++) {
        bf16x8_t vb[2];
#pragma unroll
        for (int i = 0; i < 2; i++) vb[i] = to_bf16(t.v[i0 + i][2 * f], t.v[i0 + i][2 * f + 1]);
#pragma unroll
        for (int n = 0; n < 3; n++)
#pragma unroll
          for (int i = 0; i < 2; i++) acc[i0 + i] = product(vb[i], n, f, acc[i0 + i]);
      }
    }
  };
  Step st = step_at(min(first, max(last - 1, 0)));
  for (int x = first; x < last; x++) {
    Tile t;
    load(t, st);
    const Step next = step_at(min(x + 1, last - 1));  // (its page is known by the time it is needed)
    fold(t, st);
    st = next;
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  r.m = m;
  r.l = l;
}

// The row's result, from its sums; for lanes of the group's heads.
__device__ __forceinline__ void write_row(const CacheDecodeArgs& a, int s, int h, int quad, const Row& r) {
  const float inv = r.l > 0.0f || r.l != r.l ? 1.0f / r.l : 0.0f;
  __hip_bfloat16* o = a.out + s * a.o_ss + h * a.o_sh + 4 * quad;
#pragma unroll
  for (int i = 0; i < 8; i++)
    *reinterpret_cast<uint2*>(o + 16 * i) =
        make_uint2(pack_bf16(r.acc[i][0] * inv, r.acc[i][1] * inv),
                   pack_bf16(r.acc[i][2] * inv, r.acc[i][3] * inv));
  if (quad == 0)
    a.lse[(int64_t)h * a.S + s] = r.m == -INFINITY && r.l == 0.0f
                                      ? -INFINITY : (r.m + __builtin_amdgcn_logf(r.l)) * kLn2;
}

// A request that attends nothing.
__device__ __forceinline__ void write_nothing(const CacheDecodeArgs& a, int s, int h, int lane) {
  *reinterpret_cast<uint32_t*>(a.out + s * a.o_ss + h * a.o_sh + 2 * lane) = 0;
  if (lane == 0) a.lse[(int64_t)h * a.S + s] = -INFINITY;
}

__global__ __launch_bounds__(kCacheDecodeThreads, 2) void cache_attend_kernel(CacheDecodeArgs a) {
  __shared__ Sums sums;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = a.c.Hkv, G = a.G;
  const auto units = [&](int s) { return cache_steps(held(a, s)); };
  sum_rows(sums, a.S, units);
  const int w = blockIdx.x * (kCacheDecodeThreads / 64) + wave;
  // rows that attend nothing
  for (int r = w; r < a.S * Hkv; r += gridDim.x * (kCacheDecodeThreads / 64)) {
    const int s = r / Hkv, h0 = r % Hkv * G;
    if (a.lens[s] > 0) continue;
    for (int h = h0; h < h0 + G; h++) write_nothing(a, s, h, lane);
    if (lane == 0 && a.join_rows) a.join[r] = {-1, 0};
  }
  const int share = w / Hkv, g = w % Hkv;
  if (share >= a.shares) return;
  const int total = __builtin_amdgcn_readfirstlane(sums.total);
  // Two waves per SIMD hide a few steps' latency; where each would have many, one does as
  // well, with half the partials (1024 and 2048 waves: 1M tokens 354 and 367 us, ragged
  // batch, 8 steps a wave, 55.8 and 57.8)
  // Nor need they all have one step rather than half of them two (a partial of 16 heads is as many
  // bytes as a step): one request of 131072 tokens, 16/1 heads, 39.2 us with one, 27.8 with two.
  const bool half = total / 6 >= a.shares || (total <= a.shares && 2 * total > a.shares);
  const int used = half ? (a.shares + 1) / 2 : a.shares;
  const int per_share = (total + used - 1) / used;
  int u = (int)min((int64_t)share * per_share, (int64_t)total);
  const int u_end = (int)min((int64_t)u + per_share, (int64_t)total);
  CacheJoin join = {-1, 0};
  if (u < u_end) {
    int base;
    int s = __builtin_amdgcn_readfirstlane(find_row(sums, a.S, u, units, &base));
    const int hc = lane & 15, quad = lane >> 4;
    while (u < u_end) {
      const int n = __builtin_amdgcn_readfirstlane(units(s));
      if (n == 0) {
        s++;
        continue;
      }
      const int first = u - base, last = min(n, u_end - base);
      Row x;
      attend_steps<false>(a, s, g, held(a, s), nullptr, first, last, x);
      // a lane's sums: head hc, dims 16 i + 4 quad + e
      const bool whole = first == 0 && last == n;
      if (hc < G) {
        if (whole) {
          write_row(a, s, g * G + hc, quad, x);
        } else {
          const int64_t at = (((int64_t)share * 2 + (first == 0)) * Hkv + g) * G + hc;
          float* o = a.part_o + at * kHeadDim + 4 * quad;
#pragma unroll
          for (int i = 0; i < 8; i++)
            *reinterpret_cast<f32x4_t*>(o + 16 * i) = x.acc[i];
          if (quad == 0) a.part_ml[at] = make_float2(x.m, x.l);
        }
      }
      if (first == 0) {
        join = {-1, 0};
        if (last < n) join = {a.join_rows ? share : s, (base + n - 1) / per_share - share + 1};
        if (lane == 0 && a.join_rows) a.join[(int64_t)s * Hkv + g] = join;
      }
      u = base + last;
      base += n;
      s++;
    }
  }
  if (lane == 0 && !a.join_rows) a.join[(int64_t)share * Hkv + g] = join;
}

// -------------------------------------------------------------------- join
// One work-group per head of a request, or of a share where requests are more (join_rows: with
// those of every share always, 2048 times 16 heads, 18 requests of 10496 tokens, 16/1 heads,
// took 33.8 us instead of 21.2); it may find that nothing is split.  Full: the partials are
// slot 1 of the row's first share and slot 0 of those after it.  Bound by latency: the
// entry, then partials, maxima and sums together.
// (As 512-thread work-groups, or with half a wave per short row and a work-group for a long
// one's heads, a ragged batch of 8 took 9 us, this way 6.)
constexpr int kJoinThreads = 256;
constexpr int kJoinGroups = kJoinThreads / (kHeadDim / 4);

__global__ __launch_bounds__(kJoinThreads) void cache_join_kernel(CacheDecodeArgs a, bool full) {
  __shared__ float wt[kCacheWaves];
  __shared__ float red[2][kJoinThreads / 64];
  __shared__ f32x4_t part[kJoinGroups][kHeadDim / 4];
  const int G = a.G, tid = threadIdx.x;
  const int Hkv = a.c.Hkv, hl = blockIdx.x % G;
  const int64_t at = blockIdx.x / G;
  const int i = (int)(at / Hkv), g = (int)(at % Hkv);  // request or share
  CacheJoin jn = {i, a.parts};
  if (full) jn = a.join[at];
  else if (a.lens[i] <= 0) return;
  if (jn.at < 0) return;
  const bool of_row = !full || a.join_rows;
  const int s = of_row ? i : jn.at, first = of_row ? jn.at : i;
  const auto slot = [&](int i) {
    return (full ? ((int64_t)(first + i) * 2 + (i == 0)) * Hkv + g : at * a.parts + i) * G + hl;
  };
  const int d4 = tid & 31, grp = tid >> 5;  // the thread's partials are grp + 8 i
  f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
  float top = -INFINITY, l = 0.0f;
  const auto run = [&](auto ahead) {
    constexpr int kAhead = decltype(ahead)::value;
    f32x4_t x[kAhead];
    const auto fetch = [&](int i0) {
#pragma unroll
      for (int e = 0; e < kAhead; e++)
        x[e] = reinterpret_cast<const f32x4_t*>(
            a.part_o + slot(min(i0 + kJoinGroups * e, jn.count - 1)) * kHeadDim)[d4];
    };
    fetch(grp);  // (in flight while the weights are found)
    for (int i = tid; i < jn.count; i += kJoinThreads) {
      wt[i] = a.part_ml[slot(i)].x;
      top = fmaxf(top, wt[i]);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    if ((tid & 63) == 0) red[0][tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    for (int i = tid; i < jn.count; i += kJoinThreads) {
      wt[i] = __builtin_amdgcn_exp2f(wt[i] - (top == -INFINITY ? 0.0f : top));
      l = fmaf(wt[i], a.part_ml[slot(i)].y, l);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) l += __shfl_xor(l, d, 64);
    if ((tid & 63) == 0) red[1][tid >> 6] = l;
    __syncthreads();
    l = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    for (int i0 = grp; i0 < jn.count; i0 += kJoinGroups * kAhead) {
      if (i0 != grp) fetch(i0);
#pragma unroll
      for (int e = 0; e < kAhead; e++) {
        const int i = i0 + kJoinGroups * e;
        const float y = wt[min(i, jn.count - 1)];
#pragma unroll
        for (int k = 0; k < 4; k++) o[k] = i < jn.count ? fmaf(y, x[e][k], o[k]) : o[k];
      }
    }
  };
  if (jn.count <= 2 * kJoinGroups) run(std::integral_constant<int, 2>{});
  else run(std::integral_constant<int, 16>{});
  part[grp][d4] = o;
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int i = 1; i < kJoinGroups; i++)
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] += part[i][d4][e];
  const int h = g * G + hl;
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  *reinterpret_cast<uint2*>(a.out + s * a.o_ss + h * a.o_sh + 4 * d4) =
      make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
  if (d4 == 0)
    a.lse[(int64_t)h * a.S + s] =
        top == -INFINITY && l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

// -------------------------------------------------------------------- gate
// Past blocks of request s.
__device__ __forceinline__ int past_blocks(const CacheDecodeArgs& a, int s) {
  const int len = held(a, s);
  return len > 0 ? (len - 1) / a.B : 0;
}

// x of another lane: of its quad, its 8 or its 16 (CTRL), for two-word values.
template <int CTRL>
__device__ __forceinline__ double lane_of(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, false);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}

// put(head of the group, score) for past block j of request s and kv-head g, by a wave.
template <typename Put>
__device__ __forceinline__ void block_scores(const CacheDecodeArgs& a, int s, int g, int j, Put put) {
  const CachePool& c = a.c;
  const int Hkv = c.Hkv, G = a.G, lane = threadIdx.x & 63;
  const int per = a.B / c.P;  // pages per block
  const int half = lane >> 5, d4 = 4 * (lane & 31);  // half a wave per page row, 4 dims a lane
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  for (int p0 = 0; p0 < per; p0 += 64) {
    const int np = min(64, per - p0);
    const int id = a.table[s * a.t_ss + (int64_t)j * per + p0 + min(lane, np - 1)];
    for (int p = 0; p < np; p += 16) {
      float4 x[8];
      bool ok[8];
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const int at = p + 2 * e;
        const int page0 = __builtin_amdgcn_readlane(id, min(at, np - 1));
        const int page1 = __builtin_amdgcn_readlane(id, min(at + 1, np - 1));
        const int page = half ? page1 : page0;
        ok[e] = at + half < np && (uint32_t)page < (uint32_t)c.N;
        x[e] = *reinterpret_cast<const float4*>(
            c.k_sum + ((int64_t)(ok[e] ? page : 0) * Hkv + g) * kHeadDim + d4);
      }
#pragma unroll
      for (int e = 0; e < 8; e++) {
        sum[0] += ok[e] ? (double)x[e].x : 0.0;
        sum[1] += ok[e] ? (double)x[e].y : 0.0;
        sum[2] += ok[e] ? (double)x[e].z : 0.0;
        sum[3] += ok[e] ? (double)x[e].w : 0.0;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; i++) sum[i] += __shfl_xor(sum[i], 32, 64);
  // half a wave per head, two heads at a time
  for (int h0 = 0; h0 < G; h0 += 4) {
    double x[2];
#pragma unroll
    for (int e = 0; e < 2; e++) {
      const int h = g * G + min(h0 + 2 * e + half, G - 1);
      const uint2 qw = *reinterpret_cast<const uint2*>(a.q + s * a.q_ss + h * a.q_sh + d4);
      x[e] = (double)bf16_lo(qw.x) * sum[0] + (double)bf16_hi(qw.x) * sum[1] +
             (double)bf16_lo(qw.y) * sum[2] + (double)bf16_hi(qw.y) * sum[3];
    }
#pragma unroll
    for (int e = 0; e < 2; e++) {
      x[e] += lane_of<0xb1>(x[e]);  // the neighbour, the other pair, four and eight lanes
      x[e] += lane_of<0x4e>(x[e]);
      x[e] += lane_of<0x141>(x[e]);
      x[e] += lane_of<0x140>(x[e]);
      x[e] += __shfl_xor(x[e], 16, 64);
      const int hl = h0 + 2 * e + half;
      if ((lane & 31) == 0 && hl < G) put(hl, x[e]);
    }
  }
}

__global__ __launch_bounds__(kCacheDecodeThreads) void cache_gate_kernel(CacheDecodeArgs a) {
  __shared__ Sums sums;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = a.c.Hkv, G = a.G;
  const auto units = [&](int s) { return past_blocks(a, s); };
  sum_rows(sums, a.S, units);
  const int w = blockIdx.x * (kCacheDecodeThreads / 64) + wave;
  const int share = w / Hkv, g = w % Hkv;
  const int total = __builtin_amdgcn_readfirstlane(sums.total);
  const int per_share = (total + a.gate_shares - 1) / a.gate_shares;
  int u = (int)min((int64_t)share * per_share, (int64_t)total);
  const int u_end = (int)min((int64_t)u + per_share, (int64_t)total);
  if (share >= a.gate_shares || u >= u_end) return;
  int base;
  int s = __builtin_amdgcn_readfirstlane(find_row(sums, a.S, u, units, &base));
  while (u < u_end) {
    const int n = __builtin_amdgcn_readfirstlane(units(s));
    const int last = min(n, u_end - base);
    for (int j = u - base; j < last; j++) {
      block_scores(a, s, g, j, [&](int hl, double x) {
        a.score[((int64_t)s * a.Hq + g * G + hl) * a.nblk + j] = x;
      });
    }
    u = base + last;
    base += n;
    s++;
  }
}

// ------------------------------------------------------------------ select
// A total order of doubles as unsigned integers, NaN with the lowest; never 0.
__device__ __forceinline__ uint64_t order_of(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x == x ? x + 0.0 : -INFINITY);  // (-0 is 0)
  return b >> 63 ? ~b : b | (uint64_t(1) << 63);
}

// put(x, mask of the kept blocks 64 x ..) for the nh highest scores among `past` blocks (of
// equal ones the first), by a wave.  NW: words of 64 blocks.  (Searching 64 bits at once, from the
// first bit on, whole calls: 1049 blocks, top-8, 3 heads to a kv-head 55.0 us, this way 32.9; 2048
// blocks, 16 heads 186, 105; up to 256 blocks the same.)
template <int NW, typename Score, typename Put>
__device__ __forceinline__ void keep_blocks(int past, int nh, Score score, Put put) {
  const int lane = threadIdx.x & 63;
  uint64_t key[NW];
#pragma unroll
  for (int x = 0; x < NW; x++) {
    const int j = 64 * x + lane;
    key[x] = j >= past ? 0 : nh == 0 || nh == past ? 1 : order_of(score(j));  // (else there are none)
  }
  // the largest bound that at least nh keys reach, its upper word first
  const auto upper = [&](int x) { return (uint32_t)(key[x] >> 32); };
  const auto reaching = [&](uint32_t c) {  // keys whose upper word reaches c
    int n = 0;
#pragma unroll
    for (int x = 0; x < NW; x++) {
      if constexpr (NW < 16) n += __popcll(__ballot(upper(x) >= c));
      else n += upper(x) >= c;
    }
    return NW < 16 ? n : __builtin_amdgcn_readlane(wave_scan(n), 63);
  };
  uint32_t high = 0;
  uint64_t bound = nh == past ? 1 : 0;
  int reach = nh == past ? nh : 0;  // keys that reach it, where that was counted
  const bool search = nh > 0 && nh < past;
  int bit = 31;
  if (NW >= 16 && search && nh <= 64) {
    // the lanes' highest: nh of them reach the nh-th, so it bounds from below; what it has in
    // common with the highest of all needs no search
    uint32_t most = 0, least = 0, top = 0;
#pragma unroll
    for (int x = 0; x < NW; x++) most = max(most, upper(x));
#pragma unroll 1
    for (int b = 31; b >= 0; b--) {
      const uint32_t m = 1u << b;
      if (__popcll(__ballot(most >= (least | m))) >= nh) least |= m;
      if (__ballot(most >= (top | m))) top |= m;
    }
    const uint32_t differ = least ^ top;
    bit = differ ? 31 - __clz(differ) : -1;
    high = bit < 31 ? least >> (bit + 1) << (bit + 1) : 0;
  }
#pragma unroll 1
  for (; bit >= 0 && search && reach != nh; bit--) {
    const uint32_t cand = high | 1u << bit;
    const int n = reaching(cand);
    if (n >= nh) {
      high = cand;
      reach = n;
    }
  }
  if (search) bound = (uint64_t)high << 32;
#pragma unroll 1
  for (bit = 31; bit >= 0 && search && reach != nh; bit--) {
    const uint64_t cand = bound | (uint64_t)1 << bit;
    int n = 0;
#pragma unroll
    for (int x = 0; x < NW; x++) n += __popcll(__ballot(key[x] >= cand));
    if (n >= nh) {
      bound = cand;
      reach = n;
    }
  }
  // all keys above the bound, and of those that equal it the first ones
  int above = 0;
#pragma unroll
  for (int x = 0; x < NW; x++) above += __popcll(__ballot(key[x] > bound));
  int ties = nh - above;
#pragma unroll
  for (int x = 0; x < NW; x++) {
    const unsigned long long eq = __ballot(key[x] == bound && key[x] != 0);
    const bool take = key[x] > bound || (key[x] == bound && key[x] != 0 &&
                                         __popcll(eq & ((1ull << lane) - 1)) < ties);
    const unsigned long long m = __ballot(take && nh > 0);
    ties -= min(ties, (int)__popcll(eq));
    if (lane == 0) put(x, m);
  }
}

// The group's kept blocks as one ascending list, and the current block for all heads; returns
// the steps.  For all threads of a work-group, kept being complete.
template <int NW>
struct Kept {
  unsigned long long of[kDecodeMaxGroup][NW];
  int before[NW + 1];
};
template <int NW>
__device__ __forceinline__ int block_list(const CacheDecodeArgs& a, Kept<NW>& k, int past, int len, uint32_t* list) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, G = a.G;
  if (tid < NW) {
    unsigned long long any = 0;
    for (int hl = 0; hl < G; hl++) any |= k.of[hl][tid];
    const int n = __popcll(any);
    int incl = n;
#pragma unroll
    for (int d = 1; d < NW; d <<= 1) {
      const int o = __shfl_up(incl, d, 64);
      if (lane >= d) incl += o;
    }
    k.before[tid] = incl - n;
    if (tid == NW - 1) k.before[NW] = incl;
  }
  __syncthreads();
  const int nu = k.before[NW];
  for (int x = wave; x < NW; x += (int)blockDim.x / 64) {
    uint32_t heads = 0;
    for (int hl = 0; hl < G; hl++) heads |= (uint32_t)((k.of[hl][x] >> lane) & 1) << hl;
    const unsigned long long any = __ballot(heads != 0);
    if (heads) list[k.before[x] + __popcll(any & ((1ull << lane) - 1))] = (uint32_t)(64 * x + lane) | heads << 16;
  }
  if (tid == 0) list[nu] = (uint32_t)past | 0xffff0000u;
  return nu * (a.B / kCacheTile) + cache_steps(len - past * a.B);
}

// -------------------------------------------------------------------- rows
// Short rows, a work-group for each (request, kv-head): gate, selection, attention and the
// join of its waves in one launch.  A CU alone takes about 0.3 us per step (52 GB/s) with 4, 8
// or 16 waves (kRowWaves).
template <int WAVES>
struct WaveSums {
  f32x4_t of[4][8][64];
  float m[WAVES][16], l[WAVES][16];
};

// The work-group's sums of a row in its first wave, from its waves'.
template <int WAVES>
__device__ __forceinline__ void add_waves(WaveSums<WAVES>& sm, Row& r) {
  const int lane = threadIdx.x & 63, hc = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (quad == 0) sm.m[wave][hc] = r.m;
  __syncthreads();
  float m = sm.m[0][hc];
#pragma unroll
  for (int w = 1; w < WAVES; w++) m = fmaxf(m, sm.m[w][hc]);
  const float sc = __builtin_amdgcn_exp2f(r.m - (m == -INFINITY ? 0.0f : m));
  if (quad == 0) sm.l[wave][hc] = r.l * sc;
#pragma unroll
  for (int i = 0; i < 8; i++)
#pragma unroll
    for (int e = 0; e < 4; e++) r.acc[i][e] *= sc;
  // four waves' sums at a time to the first four, then to two and one
  const auto hand = [&](int from, int n) {
    if (wave >= from && wave < from + n) {
#pragma unroll
      for (int i = 0; i < 8; i++) sm.of[wave - from][i][lane] = r.acc[i];
    }
    __syncthreads();
    if (wave < n) {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const f32x4_t x = sm.of[wave][i][lane];
#pragma unroll
        for (int e = 0; e < 4; e++) r.acc[i][e] += x[e];
      }
    }
    __syncthreads();
  };
#pragma unroll
  for (int from = 4; from < WAVES; from += 4) hand(from, 4);
  hand(2, 2);
  hand(1, 1);
  r.m = m;
  r.l = 0.0f;
#pragma unroll
  for (int w = 0; w < WAVES; w++) r.l += sm.l[w][hc];
}

// (Waves per SIMD: two work-groups of eight waves on a CU take the 128 registers that they
// would go past; 192 ragged rows of 32 kv-heads 226 us so, 232 with one.)
template <bool MOBA, int kRowWaves>
__global__ __launch_bounds__(64 * kRowWaves, kRowWaves / 2) void cache_rows_kernel(CacheDecodeArgs a) {
  constexpr int kBlocks = kCacheRowBlocks;
  static_assert(kBlocks % 64 == 0 && kDecodeMaxGroup * kBlocks * 8 <= 4 * 8 * 64 * 16,
                "the scores fit where the sums are joined");
  __shared__ WaveSums<kRowWaves> sums;
  __shared__ Kept<kBlocks / 64> kept;
  __shared__ uint32_t list[kBlocks];
  const int lane = threadIdx.x & 63, hc = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.G, Hkv = a.c.Hkv;
  const int s = blockIdx.x / Hkv, g = blockIdx.x % Hkv;
  const int len = __builtin_amdgcn_readfirstlane(held(a, s));
  if (len == 0) {
    for (int hl = wave; hl < G; hl += kRowWaves) write_nothing(a, s, g * G + hl, lane);
    return;
  }
  int steps = cache_steps(len);
  if constexpr (MOBA) {
    const int past = past_blocks(a, s), nh = min(a.topk - 1, past);
    double* score = reinterpret_cast<double*>(sums.of);  // [G, kBlocks]
    if (nh > 0 && nh < past) {
      for (int j = wave; j < past; j += kRowWaves)
        block_scores(a, s, g, j, [&](int hl, double x) { score[hl * kBlocks + j] = x; });
      __syncthreads();
    }
    for (int hl = wave; hl < G; hl += kRowWaves)
      keep_blocks<kBlocks / 64>(past, nh, [&](int j) { return score[hl * kBlocks + j]; },
                                [&](int x, unsigned long long m) { kept.of[hl][x] = m; });
    __syncthreads();
    steps = block_list(a, kept, past, len, list);
    __syncthreads();
  }
  // equal parts of the steps to the waves
  const int part = (steps + kRowWaves - 1) / kRowWaves;
  const int first = min(wave * part, steps), last = min(first + part, steps);
  Row r;
  attend_steps<MOBA>(a, s, g, len, list, first, last, r);
  add_waves(sums, r);
  if (wave == 0 && hc < G) write_row(a, s, g * G + hc, quad, r);
}

// ------------------------------------------------------------------- parts
// MoBA, past a gate launch: a.parts work-groups for each (request, kv-head), each of which
// selects the row's blocks (the same for all of them) and attends its part of their steps.
// Selection in a launch of its own before shares of equal steps, and this: 8 ragged requests
// (130K tokens, blocks of 1024, top-4) 54.5 and 44.1 us, 4 x 4096 tokens 26.5 and 18.8, 1M
// tokens 90.6 and 88.6, 4096 blocks of 64, top-40, 113 and 106.  NW: words of 64 blocks.
constexpr int kPartWaves = 4;

template <int NW>
__global__ __launch_bounds__(64 * kPartWaves, 2) void cache_parts_kernel(CacheDecodeArgs a) {
  __shared__ WaveSums<kPartWaves> sums;
  __shared__ Kept<NW> kept;
  __shared__ uint32_t list[64 * NW];
  const int lane = threadIdx.x & 63, hc = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.G, Hkv = a.c.Hkv;
  const int r = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int s = r / Hkv, g = r % Hkv;
  const int len = __builtin_amdgcn_readfirstlane(held(a, s));
  if (len == 0) {  // (the join leaves such a row)
    for (int hl = wave; hl < G && part == 0; hl += kPartWaves) write_nothing(a, s, g * G + hl, lane);
    return;
  }
  const int past = past_blocks(a, s), nh = min(a.topk - 1, past), spb = a.B / kCacheTile;
  // the steps are no more than if no two heads chose the same block
  const int64_t most = (int64_t)min((int64_t)G * nh, (int64_t)past) * spb + spb;
  Row x;
  int first = 0, last = 0;
  if (part * kPartWaves < most) {
    for (int hl = wave; hl < G; hl += kPartWaves) {
      const double* sc = a.score + ((int64_t)s * a.Hq + g * G + hl) * a.nblk;
      keep_blocks<NW>(past, nh, [&](int j) { return sc[j]; },
                      [&](int w, unsigned long long m) { kept.of[hl][w] = m; });
    }
    __syncthreads();
    const int steps = block_list(a, kept, past, len, list);
    __syncthreads();
    const int each = (steps + a.parts * kPartWaves - 1) / (a.parts * kPartWaves);
    first = (int)min((int64_t)(part * kPartWaves + wave) * each, (int64_t)steps);
    last = min(first + each, steps);
  } else {
    if (threadIdx.x == 0) list[0] = (uint32_t)past;  // (an empty part looks at it, too)
    __syncthreads();
  }
  attend_steps<true>(a, s, g, len, list, first, last, x);
  add_waves(sums, x);
  if (wave != 0 || hc >= G) return;
  if (a.parts == 1) {
    write_row(a, s, g * G + hc, quad, x);
    return;
  }
  const int64_t at = (int64_t)blockIdx.x * G + hc;
  float* o = a.part_o + at * kHeadDim + 4 * quad;
#pragma unroll
  for (int i = 0; i < 8; i++) *reinterpret_cast<f32x4_t*>(o + 16 * i) = x.acc[i];
  if (quad == 0) a.part_ml[at] = make_float2(x.m, x.l);
}

}  // namespace

hipError_t launch_cache_gate(const CacheDecodeArgs& a, hipStream_t st) {
  const int64_t waves = (int64_t)a.gate_shares * a.c.Hkv;
  cache_gate_kernel<<<(unsigned)((waves + 3) / 4), kCacheDecodeThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_parts(const CacheDecodeArgs& a, hipStream_t st) {
  const unsigned groups = (unsigned)(a.S * a.c.Hkv * a.parts);
  if (a.nblk <= 256) cache_parts_kernel<4><<<groups, 64 * kPartWaves, 0, st>>>(a);
  else if (a.nblk <= 1024) cache_parts_kernel<16><<<groups, 64 * kPartWaves, 0, st>>>(a);
  else if (a.nblk <= 2048) cache_parts_kernel<32><<<groups, 64 * kPartWaves, 0, st>>>(a);
  else cache_parts_kernel<kMaxBlocksPerSeq / 64><<<groups, 64 * kPartWaves, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_rows(bool full, const CacheDecodeArgs& a, hipStream_t st) {
  const unsigned groups = (unsigned)(a.S * a.c.Hkv);
  // Eight waves finish a row sooner (its gate and selection above all); where there are rows
  // for four work-groups of four waves on every CU, the shorter ones run on past the longer:
  // 6144 rows of 16 .. 512 tokens 73 -> 54 us, 2048 rows of 16 .. 1024 39 -> 32, MoBA 16 .. 4096 88
  // -> 82; all rows equal, or up to 4096 tokens with full attention: 2 to 4% slower.
  const bool four = groups >= 512 && (!full || a.W * a.c.P <= 2048);
  if (full && four) cache_rows_kernel<false, 4><<<groups, 64 * 4, 0, st>>>(a);
  else if (full) cache_rows_kernel<false, 8><<<groups, 64 * 8, 0, st>>>(a);
  else if (four) cache_rows_kernel<true, 4><<<groups, 64 * 4, 0, st>>>(a);
  else cache_rows_kernel<true, 8><<<groups, 64 * 8, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_attend(const CacheDecodeArgs& a, hipStream_t st) {
  const int64_t waves = (int64_t)a.shares * a.c.Hkv;
  cache_attend_kernel<<<(unsigned)((waves + 3) / 4), kCacheDecodeThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_join(bool full, const CacheDecodeArgs& a, hipStream_t st) {
  const int64_t groups = (int64_t)(full && !a.join_rows ? a.shares : a.S) * a.Hq;
  cache_join_kernel<<<(unsigned)groups, kJoinThreads, 0, st>>>(a, full);
  return hipGetLastError();
}

}  // namespace moba
