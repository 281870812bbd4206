// Decode over a paged latent cache (absorbed form): a request's cached token j is one row u_j of 576
// numbers, 512 of the latent vector and 64 of the rotary key, for all heads.  For a head's query
// (qc, qr): z_j = scale <(qc, qr), u_j>, out = sum_j softmax(z)_j u_j[0:512].
//
// A row is 1152 bytes and 2176 operations a head: at 128 heads the matrix cores take about as long as
// memory does, with fewer heads memory is the bound.  A row is read once for scores and values: it is staged in
// LDS and serves as the row operand of the first product and, by transposed reads, of the second.
//
// Work-group = 4 waves, a group of M = 16, 32 or 64 heads, one on each CU.  The batch's steps (64 tokens of a
// request) stand in one line, cut into equal runs, one for each share: a work-group for each group of heads.  A
// request that lies in one run is finished there, the others leave partials that a second kernel joins.
// Two buffers of 64 rows (72 KiB each), step i + 1 in flight while step i is used.  On
// v_mfma_f32_32x32x16_bf16 (M = 64) or v_mfma_f32_16x16x32_bf16, per step:
//   S^T (tokens x heads) = U . Q^T   wave w scores tokens 16 w .. of all heads, Q in registers
//   P^T under the running max, through LDS as bf16, for all waves
//   O^T (dims x heads) += U^T . P^T  wave w owns dims 128 w .. 128 w + 127
// The running max is raised only when some weight of the step passes 2^8; the step's weights are then formed
// again.  The weights enter the second product as bf16 (at most 2^-8 of each, independent of each other: results are
// off by up to 0.0021 of their 2-norm, by 0.0017 from their own rounding alone; all 24 bits of a weight would take the
// second product three times over), all sums are fp32.
//
// 2^20 tokens, 128 heads: 333 us (in a row of such calls 370, the clock falls) and the join 13, 3.6 TB/s and 880
// TFLOP/s; 48 requests of 100 to 30000 tokens (261732 in all), 128 heads: 124 (136) and 12.  A step of M = 64 takes some 5000 cycles at the 2.0 GHz that the chip keeps
// under this load: scores 2400 (1152 of products; the DMA's 18 instructions a wave go out beside them, and the path
// from L2 to LDS, 33 bytes a cycle of a CU, needs 2200 for a step's rows), weights 650, values 1500 (1024), flag and
// barriers 300.  A run's start takes 11 us: lengths, table, rows, queries, next lengths and table one after the other (loads
// return in order, so a length asked for behind the rows waits for them, and so on), then the queries' way into registers.
//
// Tried, whole calls: groups of 128 heads, a row read once for all, 7700 cycles a step of twice the work, but twice
// the partials to write and join: 2^20 tokens 326 us against 345, the 48 requests 155 against 132, 128 of 1000 tokens
// 86 against 64, so it pays from some 10^6 tokens a call on alone.  Two waves a SIMD, half the dims each: 354 against
// 345, since their registers spill.
#include "latent_internal.h"
#include "latent_tile.h"

#include <math.h>

namespace moba {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRowChunks = kRow / 8;                   // 72
constexpr int kStepChunks = kLatStep * kRowChunks;     // 4608
constexpr int kDma = kStepChunks / (64 * kWaves);      // DMA instructions a wave (18)
constexpr int kPRow = kLatStep + 8;                    // bf16 of a head's row of P (padded)
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kMaxWeight = 256.0f;
constexpr int kInAcc = 62;                             // 16-byte operands of the queries in accumulation registers
constexpr int kDmaFirst = 13;                          // DMA instructions beside the first product
constexpr int kAhead = 6;                              // operand reads ahead of their products

// The 72 chunks of a row: two rows to the bank period, as swz_slim in latent_tile.h has it, in
// groups of 8 chunks.
__device__ __forceinline__ uint32_t at_row(int r, int c) {
  return (uint32_t)(r * (kRowChunks * 16) + ((c ^ swz_slim(r)) * 16));
}

__device__ __forceinline__ f32x4 product(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 product(bf16x8 a, bf16x8 b, f32x16 c) { return mfma(a, b, c); }

// A product's tile: kT x kT results of kK terms.  Lane c + kT g holds column c, rows row(i); as an
// operand, 16-byte chunk g of the row or column c.
template <int T>
struct Tile;
template <>
struct Tile<16> {
  typedef f32x4 Acc;
  static constexpr int kN = 4, kK = 32;
  static __device__ __forceinline__ int row(int i, int g) { return 4 * g + i; }
  static __device__ __forceinline__ Acc zero() { return Acc{0.0f, 0.0f, 0.0f, 0.0f}; }
};
template <>
struct Tile<32> {
  typedef f32x16 Acc;
  static constexpr int kN = 16, kK = 16;
  static __device__ __forceinline__ int row(int i, int g) { return 8 * (i >> 2) + 4 * g + (i & 3); }
  static __device__ __forceinline__ Acc zero() {
    Acc a;
#pragma unroll
    for (int i = 0; i < 16; i++) a[i] = 0.0f;
    return a;
  }
};

// Tokens of a request, and its steps.
__device__ __forceinline__ int tokens_of(const LatentDecodeArgs& a, int s) {
  const int64_t n = a.lens[s], most = (int64_t)a.W * a.P;
  return (int)(n < 0 ? 0 : n > most ? most : n);
}
__device__ __forceinline__ int steps_in(int tokens) { return (int)(((uint32_t)tokens + kLatStep - 1) / kLatStep); }
__device__ __forceinline__ int steps_of(const LatentDecodeArgs& a, int s) { return steps_in(tokens_of(a, s)); }

// The line of n steps (below 2^30) in runs, one a share: the first n % shares of them are a step longer.
struct Runs {
  uint32_t q, r;
  __device__ __forceinline__ Runs(uint32_t n, uint32_t shares) : q(n / shares), r(n - n / shares * shares) {}
  __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * q + min(w, r); }
  // the share that holds step y
  __device__ __forceinline__ uint32_t share(uint32_t y) const {
    const uint32_t x = r * (q + 1);
    return y < x ? y / (q + 1) : r + (y - x) / max(q, 1u);
  }
};

// dma16_at with the LDS address in a scalar register (the s_nop: see there).
__device__ __forceinline__ void dma16_to(const char* base, uint32_t off, uint32_t to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "{m0}"(to) : "memory");
}

template <int M>
__global__ __launch_bounds__(kThreads, 1) void latent_decode_kernel(LatentDecodeArgs a) {
  // first product: a wave scores 16 tokens for all heads, tiles of 16 x 16
  using S = Tile<16>;
  constexpr int kHs = M / 16;                    // head tiles
  constexpr int kNk = kRow / S::kK;              // products of a score
  static_assert(kNk == kDma, "a DMA instruction goes out beside each product");
  // second product: a wave sums 128 dims of all heads, tiles of T x T
  constexpr int T = M == 64 ? 32 : 16;
  using V = Tile<T>;
  using Acc = typename V::Acc;
  constexpr int kHt = M / T;                     // head tiles
  constexpr int kDt = 128 / T, kPd = 64 / T;     // dim tiles of a wave; those of 8 chunks (4 or 2)
  constexpr int kKs = kLatStep / V::kK;          // products over a step's tokens
  __shared__ u32x4 lds[2 * kStepChunks];
  __shared__ __align__(16) __hip_bfloat16 pl[M * kPRow];
  __shared__ float red[kWaves][M];
  __shared__ int flag[2];
  __shared__ uint32_t scan[kWaves + 1];
  __shared__ int begin_s;
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cs = lane % 16, gs = lane / 16;  // lane's place in a tile of the first product
  const int c = lane % T, g = lane / T;      // and of the second

  // work-groups go round-robin to the 8 XCDs: those of one run sit on one of them
  const int per = 8 * a.groups;
  const int hg = (int)(blockIdx.x % per) / 8;
  const int w = (int)(blockIdx.x / per) * 8 + (int)(blockIdx.x % 8);
  const int h0 = hg * M;

  // ---- where the run begins: every thread sums the steps of a range of requests
  const int span = (a.S + kThreads - 1) / kThreads;
  const int sb = min(a.S, tid * span), se = min(a.S, sb + span);
  uint32_t mine = 0;
  for (int s = sb; s < se; s++) mine += steps_of(a, s);
  uint32_t upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = __shfl_up(upto, d, 64);
    if (lane >= d) upto += x;
  }
  if (lane == 63) scan[wave] = upto;
  __syncthreads();
  uint32_t base = 0, total = 0;
#pragma unroll
  for (int i = 0; i < kWaves; i++) {
    if (i < wave) base += scan[i];
    total += scan[i];
  }
  upto += base;
  const Runs runs(total, a.shares);
  const uint32_t x0 = w < a.shares ? runs.begin(w) : 0, x1 = w < a.shares ? runs.begin(w + 1) : 0;
  if (tid == 0) {
    flag[0] = flag[1] = 0;
    if (blockIdx.x == 0) a.first[a.S] = total;
  }
  if (x0 < x1 && upto - mine <= x0 && x0 < upto) {  // one thread
    uint32_t y = upto - mine;
    int s = sb;
    while (span > 1) {
      const uint32_t n = steps_of(a, s);
      if (x0 < y + n) break;
      y += n;
      s++;
    }
    begin_s = s;
    scan[kWaves] = y;
  }
  // requests that begin in the share's run leave where (for the join)
  if (hg == 0) {
    uint32_t y = upto - mine;
    for (int s = sb; s < se && y < x1; s++) {
      if (y >= x0) a.first[s] = y;
      if (span > 1) y += steps_of(a, s);
    }
  }
  __syncthreads();
  if (x0 >= x1) return;
  int s = __builtin_amdgcn_readfirstlane(begin_s);
  uint32_t sx = __builtin_amdgcn_readfirstlane(scan[kWaves]);  // the step at which request s begins

  // ---- lanes' parts of the DMA and the operands
  // DMA instruction wave + 4 x: nine of a wave's fill 32 rows, the other nine the same chunks 32 rows on
  uint32_t doff[kDma / 2];
#pragma unroll
  for (int x = 0; x < kDma / 2; x++) {
    const int j = 64 * (wave + kWaves * x) + lane;
    doff[x] = at_row(j / kRowChunks, j % kRowChunks);  // (the swizzle is its own inverse)
  }
  const uint32_t tp = (uint32_t)a.P / kLatStep;  // steps of a page
  struct Src {
    int id, at;  // a step's page and its place there
  };
  // Lane l holds entry p0 + l of the request's table row: a load of its own at every step would be waited for
  // together with the DMA in flight.
  uint32_t p0 = 0;
  int ids = 0;
  const auto entries = [&](int s_, uint32_t from) {
    return a.table[(int64_t)s_ * a.t_ss + min(from + lane, (uint32_t)a.W - 1)];
  };
  const auto source = [&](int s_, int step_) {
    const uint32_t pg = (uint32_t)step_ / tp;
    if (pg - p0 >= 64) {
      p0 = pg;
      ids = entries(s_, pg);
      asm volatile("" : "+v"(ids));  // (used here: so waited for here, not after the branch)
    }
    return Src{__builtin_amdgcn_readlane(ids, pg - p0), (int)((uint32_t)step_ - pg * tp)};
  };
  const auto held = [&](int id) { return id >= 0 && id < a.N; };
  const auto origin = [&](const Src& x_) {  // (where there is no page its rows are cleared before they are used)
    return scalar_ptr(a.pages + (held(x_.id) ? (int64_t)x_.id : 0) * a.p_sp + x_.at * (kLatStep * kRow));
  };
  // DMA instruction x of a step whose rows begin at src; where mask is 0, of one 16-byte piece for all lanes
  const auto stage = [&](int x, const char* src, uint32_t to, uint32_t mask) {
    dma16_to(src + (x / (kDma / 2)) * (kLatStep / 2 * kRow * 2), doff[x % (kDma / 2)] & mask, to + kWaves * 1024 * x);
  };
  // where this wave's DMA begins in each buffer
  const uint32_t to0 = lds_addr(lds) + 1024 * wave, to1 = to0 + kStepChunks * 16;
  // row operand: row 16 wave + cs, chunk 4 k + gs at orow[k % 2] + 128 (k / 2)
  uint32_t orow[2];
#pragma unroll
  for (int k = 0; k < 2; k++) orow[k] = at_row(16 * wave + cs, 4 * k + gs);
  // transposed: lane's group g holds tokens kK ks + 8 g + 4 x + (0 .. 3) of dim T dt + c of the
  // wave's: otr[x][dt % kPd] + 128 (dt / kPd)
  uint32_t otr[2][kPd];
#pragma unroll
  for (int x = 0; x < 2; x++)
#pragma unroll
    for (int dt = 0; dt < kPd; dt++) {
      const int i = lane & 15;
      otr[x][dt] = at_row(8 * g + 4 * x + (i >> 2), 16 * wave + (T / 8) * dt + 2 * (c >> 4) + ((i & 3) >> 1)) + 8 * (i & 1);
    }

  const float c2 = a.scale_log2;
  int step = (int)(x0 - sx), par = 0;
  p0 = (uint32_t)step / tp;
  ids = entries(s, p0);
  Src at = source(s, step);  // where the staged step stands
  {
    const char* src = origin(at);
#pragma unroll
    for (int x = 0; x < kDma; x++) stage(x, src, to0, ~0u);
  }
  int len = __builtin_amdgcn_readfirstlane(tokens_of(a, s));
  for (uint32_t x = x0; x < x1;) {
    // ---------------------------------------------------------- one request
    const int ns = steps_in(len);
    const int last = (int)min((uint32_t)ns, x1 - sx);  // steps step .. last - 1 are the run's
    const bool whole = step == 0 && last == ns;
    const int64_t pslot = ((int64_t)w * 2 + (x == x0 ? 0 : 1)) * a.groups + hg;
    // the queries of the group's heads, through the buffer that no step is staged in, as 64 rows
    u32x4* lq = lds + (par ^ 1) * kStepChunks;
    {
      const __hip_bfloat16* qc = a.qc + (int64_t)s * a.qc_ss;
      const __hip_bfloat16* qr = a.qr + (int64_t)s * a.qr_ss;
      int ln = lane;
      asm volatile("" : "+v"(ln));  // (else the places below are held in registers for the whole run)
#pragma unroll
      for (int x0_ = 0; x0_ < (M * kRowChunks / 64 + kWaves - 1) / kWaves; x0_++) {
        const int j = wave + kWaves * x0_;
        if (j >= M * kRowChunks / 64) break;
        const int y = 64 * j + ln, r = y / kRowChunks, ch = (y % kRowChunks) ^ swz_slim(r);
        const int64_t h = min(h0 + r, a.H - 1);
        dma16(ch < kRank / 8 ? qc + h * a.qc_sh + 8 * ch : qr + h * a.qr_sh + 8 * (ch - kRank / 8), lq + 64 * j);
      }
    }
    // the request after this one, if the run goes on
    int s2 = s, len2 = 0;
    uint32_t sx2 = sx;
    if (sx + ns < x1) {
      sx2 = sx + ns;
      do len2 = __builtin_amdgcn_readfirstlane(tokens_of(a, ++s2));
      while (len2 == 0);
    }
    int ids2 = s2 != s ? entries(s2, 0) : 0;
    asm volatile("" : "+v"(ids2));
    const Src first2 = Src{__builtin_amdgcn_readfirstlane(ids2), 0};
    dma_wait();
    __syncthreads();
    // Into the accumulation registers, where the matrix cores read them as well as anywhere, as many as
    // those hold (the others are full).  One at a time: the pin behind a read waits for it, which for 64 heads
    // takes about as long as a step, once a request and run.
    u32x4 qf[kHs][kNk];
#pragma unroll
    for (int y = 0; y < kHs * kNk; y++) {
      const int t = y / kNk, k = y % kNk;
      qf[t][k] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(lq) + at_row(16 * t + cs, 4 * (k % 2) + gs) +
                                                 128 * (k / 2));
      if (y < kInAcc) asm volatile("" : "+a"(qf[t][k]));
      if (y % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();  // (the next step is staged there)
    Acc o[kDt][kHt];
    float m[kHs], l[kHs];
#pragma unroll
    for (int t = 0; t < kHs; t++) {
      m[t] = -INFINITY;
      l[t] = 0.0f;
    }
#pragma unroll
    for (int dt = 0; dt < kDt; dt++)
#pragma unroll
      for (int t = 0; t < kHt; t++) o[dt][t] = V::zero();

    // where the step after stands
    Src next = step + 1 < last ? source(s, step + 1) : first2;
    const char* src = origin(next);

    for (; step < last; step++, x++, par ^= 1) {
      u32x4* lb = lds + par * kStepChunks;
      const char* buf = reinterpret_cast<const char*>(lb);
      dma_wait();
      // ---- rows that are not to be seen: past the request's end, or of no page
      const int live = held(at.id) ? min(kLatStep, len - step * kLatStep) : 0;
      __syncthreads();
      if (live < kLatStep) {
        for (int j = live * kRowChunks + tid; j < kStepChunks; j += kThreads) lb[j] = u32x4{0, 0, 0, 0};
        __syncthreads();
      }
      at = next;
      // the next step's DMA goes out piece by piece, between the products: 18 at once would hold the wave up for
      // as long as all products take
      const uint32_t to = par ? to0 : to1;
      // (with no step to come they fetch next to nothing, into a buffer that nothing reads)
      const uint32_t on = step + 1 < last || s2 != s ? ~0u : 0;
      next = step + 2 < last ? source(s, step + 2) : first2;

      // ---- scores
      f32x4 z[kHs];
      {
#pragma unroll
        for (int u = 0; u < kHs; u++) z[u] = S::zero();
        u32x4 op[kNk];
        const auto fetch = [&](int k) { op[k] = *reinterpret_cast<const u32x4*>(buf + orow[k % 2] + 128 * (k / 2)); };
#pragma unroll
        for (int k = 0; k < kAhead; k++) fetch(k);
#pragma unroll
        for (int k = 0; k < kNk; k++) {
#pragma unroll
          for (int u = 0; u < kHs; u++) z[u] = product(as_bf16x8(op[k]), as_bf16x8(qf[u][k]), z[u]);
          if (k + kAhead < kNk) fetch(k + kAhead);
          if (k < kDmaFirst) stage(k, src, to, on);
        }
      }
      if (live < kLatStep) {
#pragma unroll
        for (int u = 0; u < kHs; u++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            if (16 * wave + S::row(i, gs) >= live) z[u][i] = -INFINITY;
      }
      // ---- weights under the running max, as bf16 into LDS; the lane's sums
      float ts[kHs];
      const auto weigh = [&]() {
#pragma unroll
        for (int u = 0; u < kHs; u++) {
          const float mu = m[u] == -INFINITY ? 0.0f : m[u];
          float p[4];
          ts[u] = 0.0f;
#pragma unroll
          for (int j = 0; j < 4; j++) {
            p[j] = __builtin_amdgcn_exp2f(fmaf(z[u][j], c2, -mu));
            ts[u] += p[j];
          }
          *reinterpret_cast<uint2*>(&pl[(16 * u + cs) * kPRow + 16 * wave + 4 * gs]) =
              make_uint2(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]));
        }
      };
      weigh();
      bool high = false;  // (a sum past the limit: a weight may be; a first step has no max yet)
#pragma unroll
      for (int u = 0; u < kHs; u++) high |= ts[u] > kMaxWeight || m[u] == -INFINITY;
      if (high) flag[par] = 1;
      __syncthreads();
      // (the first operands of the values are on their way while the flag is looked at)
      const int raise = flag[par];
      constexpr int kY = kKs * kDt;
      s16x4 t0[kY], t1[kY];
      bf16x8 pb[kKs * kHt];
      const auto value = [&](int y) {
        const int ks = y / kDt, dt = y % kDt;
        if (dt == 0) {
#pragma unroll
          for (int t = 0; t < kHt; t++)
            pb[ks * kHt + t] = as_bf16x8(*reinterpret_cast<const u32x4*>(&pl[(T * t + c) * kPRow + V::kK * ks + 8 * g]));
        }
        const char* b = buf + V::kK * ks * (kRowChunks * 16) + 128 * (dt / kPd);
        t0[y] = tr16(b + otr[0][dt % kPd]);
        t1[y] = tr16(b + otr[1][dt % kPd]);
      };
#pragma unroll
      for (int y = 0; y < kAhead / 2; y++) value(y);
      if (raise != 0) {
        // the step's max of every head, over the waves
#pragma unroll
        for (int u = 0; u < kHs; u++) {
          float mx = fmaxf(fmaxf(z[u][0], z[u][1]), fmaxf(z[u][2], z[u][3])) * c2;
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          if (gs == 0) red[wave][16 * u + cs] = fmaxf(mx, m[u]);
        }
        __syncthreads();
        float al[kHs];
#pragma unroll
        for (int u = 0; u < kHs; u++) {
          float mx = red[0][16 * u + cs];
#pragma unroll
          for (int i = 1; i < kWaves; i++) mx = fmaxf(mx, red[i][16 * u + cs]);
          al[u] = mx == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[u] - mx);
          l[u] *= al[u];
          m[u] = mx;
        }
        __syncthreads();
        // (the sums' tiles hold other heads a lane: the ratios go through LDS)
#pragma unroll
        for (int u = 0; u < kHs; u++)
          if (wave == 0 && gs == 0) red[0][16 * u + cs] = al[u];
        weigh();
        __syncthreads();
        if (tid == 0) flag[par] = 0;  // (read again two steps on, behind that step's barriers)
#pragma unroll
        for (int t = 0; t < kHt; t++) {
          const float f = red[0][T * t + c];
#pragma unroll
          for (int dt = 0; dt < kDt; dt++)
#pragma unroll
            for (int i = 0; i < V::kN; i++) o[dt][t][i] *= f;
        }
#pragma unroll
        for (int y = 0; y < kAhead / 2; y++) value(y);  // (the weights are others now)
      }
#pragma unroll
      for (int u = 0; u < kHs; u++) l[u] += ts[u];
      // ---- values
      {
        const char* src2 = origin(next);
#pragma unroll
        for (int y = 0; y < kY; y++) {
#pragma unroll
          for (int t = 0; t < kHt; t++) o[y % kDt][t] = product(join16(t0[y], t1[y]), pb[y / kDt * kHt + t], o[y % kDt][t]);
          if (y + kAhead / 2 < kY) value(y + kAhead / 2);
          if (y < kDma - kDmaFirst) stage(kDmaFirst + y, src, to, on);
        }
        src = src2;
      }
    }

    // ------------------------------------------------- the request's result
    // sums of the weights, over the lanes and waves that hold a head's tokens; and its max
    __syncthreads();
    float* mrow = reinterpret_cast<float*>(pl);
#pragma unroll
    for (int u = 0; u < kHs; u++) {
      float y = l[u];
      y += __shfl_xor(y, 16, 64);
      y += __shfl_xor(y, 32, 64);
      if (gs == 0) red[wave][16 * u + cs] = y;
      if (gs == 0 && wave == 0) mrow[16 * u + cs] = m[u];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kHt; t++) {
      const int hl = T * t + c, h = h0 + hl;
      float lt = red[0][hl];
#pragma unroll
      for (int i = 1; i < kWaves; i++) lt += red[i][hl];
      const float mt = mrow[hl];
      if (h < a.H) {
        const int d0 = 128 * wave;
        if (whole) {
          const float inv = lt > 0.0f || lt != lt ? 1.0f / lt : 0.0f;  // (nothing attended: 0; NaN stays)
          __hip_bfloat16* dst = a.out + (int64_t)s * a.o_ss + (int64_t)h * a.o_sh + d0;
#pragma unroll
          for (int dt = 0; dt < kDt; dt++)
#pragma unroll
            for (int i = 0; i < V::kN; i += 4)
              *reinterpret_cast<uint2*>(dst + T * dt + V::row(i, g)) =
                  make_uint2(pack_bf16(o[dt][t][i] * inv, o[dt][t][i + 1] * inv),
                             pack_bf16(o[dt][t][i + 2] * inv, o[dt][t][i + 3] * inv));
          if (wave == 0 && g == 0) a.lse[(int64_t)h * a.S + s] = (mt + __builtin_amdgcn_logf(lt)) * kLn2;
        } else {
          // as the lanes hold it
          f32x4* dst = reinterpret_cast<f32x4*>(a.part_o) + pslot * (M * kRank / 4) + lane;
#pragma unroll
          for (int dt = 0; dt < kDt; dt++)
#pragma unroll
            for (int i = 0; i < V::kN; i += 4)
              dst[(((wave * kDt + dt) * kHt + t) * (V::kN / 4) + i / 4) * 64] =
                  f32x4{o[dt][t][i], o[dt][t][i + 1], o[dt][t][i + 2], o[dt][t][i + 3]};
          if (wave == 0 && g == 0) a.part_ml[pslot * M + hl] = make_float2(mt, lt);
        }
      }
    }
    __syncthreads();
    s = s2;
    sx = sx2;
    step = 0;
    len = len2;
    p0 = 0;
    ids = ids2;
  }
  dma_wait();  // (LDS is another work-group's after the end)
}

// Joins a request's partials, in the order of its steps.  A work-group takes 256 pieces of four dims of a head, as
// the decode kernel's lanes held them, of one request; PARTS threads share a piece's partials, in runs whose sums
// are added up in order.  Requests of one run are finished already; empty ones get 0 and -inf here.
template <int M, int PARTS>
__global__ __launch_bounds__(256 * PARTS) void latent_join_kernel(LatentDecodeArgs a, uint32_t wg0) {
  constexpr int T = M == 64 ? 32 : 16;
  using V = Tile<T>;
  constexpr int kHt = M / T, kDt = 128 / T, kI = V::kN / 4, kBlocks = M * kRank / 4 / 256;
  constexpr int kHeads = M == 16 ? 16 : 32;  // of a work-group's pieces
  constexpr int kRowsAt = 256 * PARTS / kHeads;  // threads that share a head's partials below
  __shared__ float fac[kLatGroups + 1][kHeads];
  __shared__ float2 red[kRowsAt][kHeads];
  __shared__ f32x4 part[PARTS][256];
  const uint32_t wg = wg0 + blockIdx.x;
  const int blk = (int)(wg % kBlocks);
  const int hg = (int)(wg / kBlocks % (uint32_t)a.groups), s = (int)(wg / kBlocks / (uint32_t)a.groups);
  const int tid = threadIdx.x, piece = tid % 256, p = tid / 256;
  // the piece: tile t of the heads and dt of a wave's dims, rows 4 i ..
  const int lane = piece % 64;
  const int y = (blk * 256 + piece) / 64, i4 = y % kI, t = y / kI % kHt, dt = y / kI / kHt % kDt, wv = y / kI / kHt / kDt;
  const int hl = T * t + lane % T, h = hg * M + hl;
  const int d = 128 * wv + T * dt + V::row(4 * i4, lane / T);
  uint2* dst = reinterpret_cast<uint2*>(a.out + (int64_t)s * a.o_ss + (int64_t)min(h, a.H - 1) * a.o_sh + d);
  // (the pieces of dims 0 .. 3 write the head's lse)
  const bool lead = p == 0 && d == 0 && h < a.H;
  const int ns = steps_of(a, s);
  const uint32_t y0 = a.first[s], total = a.first[a.S];  // (y0 of an empty request: anything)
  if (ns == 0) {
    if (p == 0 && h < a.H) *dst = make_uint2(0, 0);
    if (lead) a.lse[(int64_t)h * a.S + s] = -INFINITY;
    return;
  }
  const Runs runs(total, a.shares);
  const int w0 = (int)runs.share(y0), w1 = (int)runs.share(y0 + ns - 1);
  if (w0 == w1) return;  // finished by its work-group
  const int n = w1 - w0 + 1;
  // the first partial may be a run's second one: the run began with another request
  const int64_t slot0 = (int64_t)w0 * 2 * a.groups + hg;
  const auto slot = [&](int i) { return slot0 + (i == 0 ? (runs.begin(w0) < y0 ? a.groups : 0) : (int64_t)i * 2 * a.groups); };
  // the heads' maxima, and each partial's factor
  const int hb = M == 64 ? 32 * (blk % 2) : 0, eh = tid % kHeads, er = tid / kHeads;
  float m = -INFINITY;
  for (int i = er; i < n; i += kRowsAt) m = fmaxf(m, a.part_ml[slot(i) * M + hb + eh].x);
  red[er][eh].x = m;
  __syncthreads();
  for (int i = 0; i < kRowsAt; i++) m = fmaxf(m, red[i][eh].x);
  const float mu = m == -INFINITY ? 0.0f : m;
  float l = 0.0f;
  for (int i = er; i < n; i += kRowsAt) {
    const float2 v = a.part_ml[slot(i) * M + hb + eh];
    const float f = __builtin_amdgcn_exp2f(v.x - mu);
    fac[i][eh] = f;
    l = fmaf(v.y, f, l);
  }
  __syncthreads();
  red[er][eh] = make_float2(m, l);
  __syncthreads();
  const int me = hl - hb;
  m = red[0][me].x;
  l = 0.0f;
  for (int i = 0; i < kRowsAt; i++) l += red[i][me].y;
  const int per = (n + PARTS - 1) / PARTS, i0 = p * per, i1 = min(n, i0 + per);
  const f32x4* src = reinterpret_cast<const f32x4*>(a.part_o) + blk * 256 + piece;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = i0; i < i1; i += 8) {
    f32x4 x[8];
#pragma unroll
    for (int j = 0; j < 8; j++) x[j] = src[slot(min(i + j, i1 - 1)) * (M * kRank / 4)];
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float f = fac[min(i + j, i1 - 1)][me];
#pragma unroll
      for (int e = 0; e < 4; e++) acc[e] = i + j < i1 ? fmaf(x[j][e], f, acc[e]) : acc[e];
    }
  }
  if constexpr (PARTS > 1) {
    part[p][piece] = acc;
    __syncthreads();
    if (p != 0) return;
#pragma unroll
    for (int i = 1; i < PARTS; i++) acc += part[i][piece];
  }
  if (h >= a.H) return;
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  *dst = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
  if (lead) a.lse[(int64_t)h * a.S + s] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int M>
hipError_t decode(const LatentDecodeArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)((a.shares + 7) / 8 * 8 * a.groups);
  latent_decode_kernel<M><<<grid, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

template <int M, int PARTS>
hipError_t join_pieces(const LatentDecodeArgs& a, hipStream_t st) {
  // (up to three heads still take 16 heads' work-groups: 2^21 requests pass one launch's work items)
  return launch_pieces((int64_t)a.S * a.groups * (M * kRank / 4 / 256), 256 * PARTS, [&](uint32_t first, unsigned n) {
    latent_join_kernel<M, PARTS><<<n, 256 * PARTS, 0, st>>>(a, first);
  });
}

template <int M>
hipError_t join(const LatentDecodeArgs& a, hipStream_t st) {
  // few requests: many partials each.  One thread a piece and four, us a call: 131072 tokens, 16 heads 57, 45, 128
  // heads 71, 61; 8 x 16000 35.6, 35.4 and 63, 66; 16 x 8000 34.7, 35.0 and 63, 72; 64 x 4000 62, 67 and 120, 164.
  return a.S <= 8 ? join_pieces<M, 4>(a, st) : join_pieces<M, 1>(a, st);
}

}  // namespace

hipError_t launch_latent_decode(int heads, const LatentDecodeArgs& a, hipStream_t st) {
  return heads == 16 ? decode<16>(a, st) : heads == 32 ? decode<32>(a, st) : decode<64>(a, st);
}

hipError_t launch_latent_join(int heads, const LatentDecodeArgs& a, hipStream_t st) {
  return heads == 16 ? join<16>(a, st) : heads == 32 ? join<32>(a, st) : join<64>(a, st);
}

}  // namespace moba
