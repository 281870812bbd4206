// Decode over a paged latent cache (absorbed form): a request's cached token j is one row u_j of 576
// numbers, 512 of the latent vector and 64 of the rotary key, for all heads.  For a head's query
// (qc, qr): z_j = scale <(qc, qr), u_j>, out = sum_j softmax(z)_j u_j[0:512].
//
// A row is 1152 bytes and 2176 operations a head: 64 heads and more are bound by the matrix cores about as
// much as by memory, few heads by memory alone.  A row is read once for scores and values: it is staged in
// LDS and serves as the row operand of the first product and, by transposed reads, of the second.
//
// Work-group = 4 waves, a group of M = 16, 32 or 64 heads, one on each CU.  The batch's steps (64 tokens of a
// request) stand in one line, and every share of heads-groups work-groups takes an equal run of it; a
// request that lies in one run is finished there, the others leave partials that a second kernel joins.
// Two buffers of 64 rows (72 KiB each), step i + 1 in flight while step i is used.  On
// v_mfma_f32_16x16x32_bf16, per step:
//   S^T (tokens x heads) = U . Q^T   the waves share out tokens and heads (M = 64: 2 x 2, else 4 x 1),
//                                    Q in registers
//   P^T under the running max, through LDS as bf16, for all waves
//   O^T (dims x heads) += U^T . P^T  wave w owns dims 128 w .. 128 w + 127
// The running max is raised only when some weight of the step would pass 2^8.
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
constexpr float kMaxLog2 = 8.0f;                       // weights stay at most 2^8

// The 72 chunks of a row: two rows to the bank period, as swz_slim in latent_tile.h has it, in
// groups of 8 chunks.
__device__ __forceinline__ uint32_t at_row(int r, int c) {
  return (uint32_t)(r * (kRowChunks * 16) + ((c ^ swz_slim(r)) * 16));
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ int steps_of(const LatentDecodeArgs& a, int s) {
  const int64_t n = a.lens[s], most = (int64_t)a.W * a.P;
  return (int)(((n < 0 ? 0 : n > most ? most : n) + kLatStep - 1) / kLatStep);
}

// Of the line of steps, share w's run: [n w / shares, n (w + 1) / shares)
__device__ __forceinline__ int64_t run_begin(int64_t n, int64_t w, int shares) { return n * w / shares; }

template <int M>
__global__ __launch_bounds__(kThreads, 1) void latent_decode_kernel(LatentDecodeArgs a) {
  constexpr int kHt = M / 16;                  // head tiles of the group
  constexpr int kWh = M == 64 ? 2 : 1;         // waves over heads in the first product
  constexpr int kWt = kWaves / kWh;            // and over tokens
  constexpr int kTt = 4 / kWt, kHw = kHt / kWh;  // token and head tiles of a wave
  __shared__ u32x4 lds[2 * kStepChunks];
  __shared__ __align__(16) __hip_bfloat16 pl[M * kPRow];
  __shared__ float red[kWt][M];
  __shared__ int flag[2];
  __shared__ int64_t scan[kWaves + 2];
  __shared__ int begin_s;
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, g4 = lane >> 4;
  const int wt = wave % kWt, wh = wave / kWt;

  // work-groups go round-robin to the 8 XCDs: those of one run sit on one of them
  const int per = 8 * a.groups;
  const int hg = (int)(blockIdx.x % per) / 8;
  const int w = (int)(blockIdx.x / per) * 8 + (int)(blockIdx.x % 8);
  const int h0 = hg * M;

  // ---- where the run begins: every thread sums the steps of a range of requests
  const int span = (a.S + kThreads - 1) / kThreads;
  const int sb = min(a.S, tid * span), se = min(a.S, sb + span);
  int64_t mine = 0;
  for (int s = sb; s < se; s++) mine += steps_of(a, s);
  int64_t upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t x = __shfl_up(upto, d, 64);
    if (lane >= d) upto += x;
  }
  if (lane == 63) scan[wave] = upto;
  __syncthreads();
  int64_t base = 0, total = 0;
#pragma unroll
  for (int i = 0; i < kWaves; i++) {
    if (i < wave) base += scan[i];
    total += scan[i];
  }
  upto += base;
  const int64_t x0 = w < a.shares ? run_begin(total, w, a.shares) : 0;
  const int64_t x1 = w < a.shares ? run_begin(total, w + 1, a.shares) : 0;
  if (tid == 0) {
    flag[0] = flag[1] = 0;
    if (blockIdx.x == 0) a.first[a.S] = total;
  }
  if (x0 < x1 && upto - mine <= x0 && x0 < upto) {  // one thread
    int64_t y = upto - mine;
    int s = sb;
    for (;; s++) {
      const int n = steps_of(a, s);
      if (x0 < y + n) break;
      y += n;
    }
    begin_s = s;
    scan[kWaves] = y;
  }
  // requests that begin in the share's run leave where (for the join)
  if (hg == 0) {
    int64_t y = upto - mine;
    for (int s = sb; s < se && y < x1; s++) {
      if (y >= x0) a.first[s] = y;
      y += steps_of(a, s);
    }
  }
  __syncthreads();
  if (x0 >= x1) return;
  int s = __builtin_amdgcn_readfirstlane(begin_s);
  int64_t sx = uniform64(scan[kWaves]);  // the step at which request s begins

  // ---- lanes' parts of the DMA and the operands
  // DMA instruction wave + 4 x: nine of a wave's fill 32 rows, the other nine the same chunks 32 rows on
  uint32_t doff[kDma / 2];
#pragma unroll
  for (int x = 0; x < kDma / 2; x++) {
    const int j = 64 * (wave + kWaves * x) + lane;
    doff[x] = at_row(j / kRowChunks, j % kRowChunks);  // (the swizzle is its own inverse)
  }
  const auto entry = [&](int s_, int step_) {
    return a.table[(int64_t)s_ * a.t_ss + (int)((int64_t)step_ * kLatStep / a.P)];
  };
  const auto held = [&](int id) { return id >= 0 && id < a.N; };
  const auto stage = [&](int id, int step_, u32x4* buf) {
    // (where there is no page its rows are cleared before they are used)
    const int at = (int)((int64_t)step_ * kLatStep % a.P);
    const char* src = scalar_ptr(a.pages + (held(id) ? (int64_t)id : 0) * a.p_sp + at * kRow);
#pragma unroll
    for (int x = 0; x < kDma; x++)
      dma16_at(src + (x / (kDma / 2)) * (kLatStep / 2 * kRow * 2), doff[x % (kDma / 2)],
               buf + 64 * (wave + kWaves * x));
  };
  // row operand: row 16 t + c16, chunk 4 k + g4 at orow[t][k % 2] + 128 (k / 2)
  uint32_t orow[kTt][2];
#pragma unroll
  for (int t = 0; t < kTt; t++)
#pragma unroll
    for (int k = 0; k < 2; k++) orow[t][k] = at_row(16 * (kTt * wt + t) + c16, 4 * k + g4);
  // transposed: lane's group g4 holds tokens 32 ks + 8 g4 + 4 x + (0 .. 3) of dim 16 dt + c16 of the
  // wave's: otr[x][dt % 4] + 128 (dt / 4)
  uint32_t otr[2][4];
#pragma unroll
  for (int x = 0; x < 2; x++)
#pragma unroll
    for (int dt = 0; dt < 4; dt++)
      otr[x][dt] = at_row(8 * g4 + 4 * x + (c16 >> 2), 16 * wave + 2 * dt + ((c16 & 3) >> 1)) + 8 * (c16 & 1);

  const float c2 = a.scale_log2;
  int step = (int)(x0 - sx), par = 0;
  int id = entry(s, step);  // the page of the step that is staged
  stage(id, step, lds);
  for (int64_t x = x0; x < x1;) {
    // ---------------------------------------------------------- one request
    const int64_t len = min((int64_t)a.lens[s], (int64_t)a.W * a.P);
    const int ns = steps_of(a, s);
    const int last = (int)min((int64_t)ns, x1 - sx);  // steps step .. last - 1 are the run's
    const bool whole = step == 0 && last == ns;
    const int64_t pslot = ((int64_t)w * 2 + (x == x0 ? 0 : 1)) * a.groups + hg;
    bf16x8 qf[kHw][kRow / 32];
#pragma unroll
    for (int t = 0; t < kHw; t++) {
      const int h = min(h0 + 16 * (kHw * wh + t) + c16, a.H - 1);
      const __hip_bfloat16* qc = a.qc + (int64_t)s * a.qc_ss + (int64_t)h * a.qc_sh + 8 * g4;
      const __hip_bfloat16* qr = a.qr + (int64_t)s * a.qr_ss + (int64_t)h * a.qr_sh + 8 * g4;
#pragma unroll
      for (int k = 0; k < kRow / 32; k++)
        qf[t][k] = as_bf16x8(*reinterpret_cast<const u32x4*>(k < kRank / 32 ? qc + 32 * k : qr + 32 * (k - kRank / 32)));
    }
    f32x4 o[8][kHt];
    float m[kHw], l[kHw];
#pragma unroll
    for (int t = 0; t < kHw; t++) {
      m[t] = -INFINITY;
      l[t] = 0.0f;
    }
#pragma unroll
    for (int dt = 0; dt < 8; dt++)
#pragma unroll
      for (int t = 0; t < kHt; t++) o[dt][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // the request after this one, if the run goes on
    int s2 = s;
    int64_t sx2 = sx;
    if (sx + ns < x1) {
      sx2 = sx + ns;
      do s2++;
      while (steps_of(a, s2) == 0);
    }
    // the page of the step after, loaded a step ahead of its use
    int next = step + 1 < last ? entry(s, step + 1) : s2 != s ? entry(s2, 0) : 0;

    for (; step < last; step++, x++, par ^= 1) {
      u32x4* lb = lds + par * kStepChunks;
      const char* buf = reinterpret_cast<const char*>(lb);
      dma_wait();
      // ---- rows that are not to be seen: past the request's end, or of no page
      const int live = held(id) ? (int)min((int64_t)kLatStep, len - (int64_t)step * kLatStep) : 0;
      __syncthreads();
      if (live < kLatStep) {
        for (int j = live * kRowChunks + tid; j < kStepChunks; j += kThreads) lb[j] = u32x4{0, 0, 0, 0};
        __syncthreads();
      }
      id = next;
      if (step + 1 < last) stage(id, step + 1, lds + (par ^ 1) * kStepChunks);
      else if (s2 != s) stage(id, 0, lds + (par ^ 1) * kStepChunks);
      if (step + 2 < last) next = entry(s, step + 2);
      else if (step + 2 == last && s2 != s) next = entry(s2, 0);

      // ---- scores
      f32x4 z[kTt][kHw];
#pragma unroll
      for (int t = 0; t < kTt; t++)
#pragma unroll
        for (int u = 0; u < kHw; u++) z[t][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < kRow / 32; k++)
#pragma unroll
        for (int t = 0; t < kTt; t++) {
          const bf16x8 op = as_bf16x8(*reinterpret_cast<const u32x4*>(buf + orow[t][k & 1] + 128 * (k >> 1)));
#pragma unroll
          for (int u = 0; u < kHw; u++) z[t][u] = mfma16(op, qf[u][k], z[t][u]);
        }
      if (live < kLatStep) {
#pragma unroll
        for (int t = 0; t < kTt; t++)
#pragma unroll
          for (int u = 0; u < kHw; u++)
#pragma unroll
            for (int i = 0; i < 4; i++)
              if (16 * (kTt * wt + t) + 4 * g4 + i >= live) z[t][u][i] = -INFINITY;
      }
      // ---- weights under the running max
      bool high = false;
#pragma unroll
      for (int u = 0; u < kHw; u++) {
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < kTt; t++)
#pragma unroll
          for (int i = 0; i < 4; i++) {
            z[t][u][i] *= c2;
            mx = fmaxf(mx, z[t][u][i]);
          }
        high |= mx > m[u] + kMaxLog2;
      }
      if (high) flag[par] = 1;
      __syncthreads();
      const bool raise = flag[par] != 0;
      if (raise) {
        // the step's max of every head, over the waves that hold its tokens
#pragma unroll
        for (int u = 0; u < kHw; u++) {
          float mx = -INFINITY;
#pragma unroll
          for (int t = 0; t < kTt; t++)
#pragma unroll
            for (int i = 0; i < 4; i++) mx = fmaxf(mx, z[t][u][i]);
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          if (g4 == 0) red[wt][16 * (kHw * wh + u) + c16] = fmaxf(mx, m[u]);
        }
        __syncthreads();
        // (every wave rescales its dims of all heads: the old max of a head is what all waves that
        // score it hold; those of the other heads come through LDS as their ratio)
        float mo[kHw];
#pragma unroll
        for (int u = 0; u < kHw; u++) {
          float mx = red[0][16 * (kHw * wh + u) + c16];
#pragma unroll
          for (int i = 1; i < kWt; i++) mx = fmaxf(mx, red[i][16 * (kHw * wh + u) + c16]);
          mo[u] = m[u];
          m[u] = mx;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kHw; u++) {
          const float al = m[u] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mo[u] - m[u]);
          l[u] *= al;
          if (wt == 0 && g4 == 0) red[0][16 * (kHw * wh + u) + c16] = al;
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kHt; t++) {
          const float al = red[0][16 * t + c16];
#pragma unroll
          for (int dt = 0; dt < 8; dt++) o[dt][t] *= al;
        }
      }
#pragma unroll
      for (int u = 0; u < kHw; u++) {
        const float mu = m[u] == -INFINITY ? 0.0f : m[u];
#pragma unroll
        for (int t = 0; t < kTt; t++) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; i++) {
            p[i] = __builtin_amdgcn_exp2f(z[t][u][i] - mu);
            l[u] += p[i];
          }
          *reinterpret_cast<uint2*>(&pl[(16 * (kHw * wh + u) + c16) * kPRow + 16 * (kTt * wt + t) + 4 * g4]) =
              make_uint2(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]));
        }
      }
      __syncthreads();
      if (tid == 0) flag[par] = 0;  // (read again two steps on, behind that step's barriers)
      // ---- values
#pragma unroll
      for (int ks = 0; ks < 2; ks++) {
        bf16x8 pb[kHt];
#pragma unroll
        for (int t = 0; t < kHt; t++)
          pb[t] = as_bf16x8(*reinterpret_cast<const u32x4*>(&pl[(16 * t + c16) * kPRow + 32 * ks + 8 * g4]));
#pragma unroll
        for (int dt = 0; dt < 8; dt++) {
          const char* b = buf + 32 * ks * (kRowChunks * 16) + 128 * (dt >> 2);
          const bf16x8 v = join16(tr16(b + otr[0][dt & 3]), tr16(b + otr[1][dt & 3]));
#pragma unroll
          for (int t = 0; t < kHt; t++) o[dt][t] = mfma16(v, pb[t], o[dt][t]);
        }
      }
    }

    // ------------------------------------------------- the request's result
    // sums of the weights, over the lanes and waves that hold a head's tokens; and its max
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kHw; u++) {
      float y = l[u];
      y += __shfl_xor(y, 16, 64);
      y += __shfl_xor(y, 32, 64);
      if (g4 == 0) red[wt][16 * (kHw * wh + u) + c16] = y;
    }
    float* mrow = reinterpret_cast<float*>(pl);
#pragma unroll
    for (int u = 0; u < kHw; u++)
      if (wt == 0 && g4 == 0) mrow[16 * (kHw * wh + u) + c16] = m[u];
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kHt; t++) {
      const int hl = 16 * t + c16, h = h0 + hl;
      float lt = red[0][hl];
#pragma unroll
      for (int i = 1; i < kWt; i++) lt += red[i][hl];
      const float mt = mrow[hl];
      if (h < a.H) {
        if (whole) {
          const float inv = lt > 0.0f || lt != lt ? 1.0f / lt : 0.0f;  // (nothing attended: 0; NaN stays)
          __hip_bfloat16* dst = a.out + (int64_t)s * a.o_ss + (int64_t)h * a.o_sh + 128 * wave + 4 * g4;
#pragma unroll
          for (int dt = 0; dt < 8; dt++)
            *reinterpret_cast<uint2*>(dst + 16 * dt) =
                make_uint2(pack_bf16(o[dt][t][0] * inv, o[dt][t][1] * inv), pack_bf16(o[dt][t][2] * inv, o[dt][t][3] * inv));
          if (wave == 0 && g4 == 0) a.lse[(int64_t)h * a.S + s] = (mt + __builtin_amdgcn_logf(lt)) * kLn2;
        } else {
          float* dst = a.part_o + (pslot * M + hl) * kRank + 128 * wave + 4 * g4;
#pragma unroll
          for (int dt = 0; dt < 8; dt++) *reinterpret_cast<f32x4*>(dst + 16 * dt) = o[dt][t];
          if (wave == 0 && g4 == 0) a.part_ml[pslot * M + hl] = make_float2(mt, lt);
        }
      }
    }
    __syncthreads();
    s = s2;
    sx = sx2;
    step = 0;
  }
}

// Joins a request's partials, in the order of its steps: a work-group per (request, head), two dims a
// thread.  Requests of one run are finished already; empty ones get 0 and -inf here.
template <int M>
__global__ __launch_bounds__(256) void latent_join_kernel(LatentDecodeArgs a) {
  const int s = (int)(blockIdx.x / (uint32_t)a.H), h = (int)(blockIdx.x % (uint32_t)a.H);
  const int d = 2 * threadIdx.x;
  uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + (int64_t)s * a.o_ss + (int64_t)h * a.o_sh + d);
  const int ns = steps_of(a, s);
  if (ns == 0) {
    *dst = 0;
    if (threadIdx.x == 0) a.lse[(int64_t)h * a.S + s] = -INFINITY;
    return;
  }
  const int64_t total = a.first[a.S], y0 = a.first[s], y1 = y0 + ns;
  // share w holds steps [total w / shares, ...): the one of step y is the last whose run begins at or before
  // y and is not empty
  const auto share_of = [&](int64_t y) {
    int64_t w = y * a.shares / total;
    while (run_begin(total, w + 1, a.shares) <= y) w++;
    while (run_begin(total, w, a.shares) > y) w--;
    return (int)w;
  };
  const int w0 = share_of(y0), w1 = share_of(y1 - 1);
  if (w0 == w1) return;  // finished by its work-group
  const int hg = h / M, hl = h % M;
  const auto slot = [&](int w) {
    const int second = run_begin(total, w, a.shares) < y0;  // the run began with another request
    return (((int64_t)w * 2 + second) * a.groups + hg) * M + hl;
  };
  float m = -INFINITY;
  for (int w = w0; w <= w1; w++)
    if (run_begin(total, w, a.shares) < run_begin(total, w + 1, a.shares)) m = fmaxf(m, a.part_ml[slot(w)].x);
  const float mu = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, o0 = 0.0f, o1 = 0.0f;
  for (int w = w0; w <= w1; w++) {
    if (run_begin(total, w, a.shares) >= run_begin(total, w + 1, a.shares)) continue;
    const int64_t at = slot(w);
    const float2 ml = a.part_ml[at];
    const float f = __builtin_amdgcn_exp2f(ml.x - mu);
    const float2 x = *reinterpret_cast<const float2*>(a.part_o + at * kRank + d);
    l = fmaf(ml.y, f, l);
    o0 = fmaf(x.x, f, o0);
    o1 = fmaf(x.y, f, o1);
  }
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  *dst = pack_bf16(o0 * inv, o1 * inv);
  if (threadIdx.x == 0) a.lse[(int64_t)h * a.S + s] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int M>
hipError_t decode(const LatentDecodeArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)((a.shares + 7) / 8 * 8 * a.groups);
  latent_decode_kernel<M><<<grid, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

template <int M>
hipError_t join(const LatentDecodeArgs& a, hipStream_t st) {
  latent_join_kernel<M><<<(unsigned)((int64_t)a.S * a.H), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_latent_decode(int heads, const LatentDecodeArgs& a, hipStream_t st) {
  return heads == 16 ? decode<16>(a, st) : heads == 32 ? decode<32>(a, st) : decode<64>(a, st);
}

hipError_t launch_latent_join(int heads, const LatentDecodeArgs& a, hipStream_t st) {
  return heads == 16 ? join<16>(a, st) : heads == 32 ? join<32>(a, st) : join<64>(a, st);
}

}  // namespace moba
