// Rotary positions.  A pair (x, y) of a head's dims at position p becomes
//   (x cos(p f) - y sin(p f), x sin(p f) + y cos(p f)) * amplitude
// with the pair's frequency f; the gradient is the same with -p.  Pairs are dims (i, i + half) or
// (2i, 2i + 1) of the first 2 half dims of a head.
//
// Bound by memory: every element is read and written once.  A thread takes one group of `vec` pairs of
// a token, forms its cosines and sines once (about 30 instructions a pair, most of it the 64-bit
// turns) and applies them to HEADS heads, whose two 16-byte pieces each are loaded before the first is
// used.  65012 tokens, 32 + 8 heads of 128 dims, bf16 (1.33 GB): 233 us, 5.7 TB/s (torch's copies of as much 5.0 to 5.5).
#include "rope_internal.h"

namespace moba {
namespace {

constexpr int kThreads = 256;

template <typename E, int V, bool INTERLEAVED, int HEADS>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, int64_t t0, uint32_t total, uint32_t items,
                                                       uint32_t groups) {
  const uint32_t x = blockIdx.x * kThreads + threadIdx.x;
  if (x >= total) return;
  const uint32_t row = x / items, item = x - row * items;
  const int64_t t = t0 + row / groups;
  const int h0 = (int)(row % groups) * HEADS, heads = a.Hq + a.Hk;
  int64_t p;
  if (!row_position(a.r, t, &p)) return;
  const int nturn = a.r.half / V;
  const bool turns = (int)item < nturn;
  // the thread's two pieces of a head
  int d0, d1;
  bool both = true;
  if (turns) {
    d0 = INTERLEAVED ? 2 * V * (int)item : V * (int)item;
    d1 = INTERLEAVED ? d0 + V : d0 + a.r.half;
  } else {
    d0 = 2 * a.r.half + 2 * V * ((int)item - nturn);
    both = d0 + V < a.D;
    d1 = both ? d0 + V : d0;
  }
  using P = Piece<E, V>;
  P u[HEADS], w[HEADS];
#pragma unroll
  for (int i = 0; i < HEADS; i++) {
    const int h = min(h0 + i, heads - 1);
    const E* src = h < a.Hq ? static_cast<const E*>(a.q) + t * a.q_st + h * a.q_sh
                            : static_cast<const E*>(a.k) + t * a.k_st + (h - a.Hq) * a.k_sh;
    u[i] = *reinterpret_cast<const P*>(src + d0);
    w[i] = *reinterpret_cast<const P*>(src + d1);
  }
  if (turns) {
    float c[V], s[V];
#pragma unroll
    for (int j = 0; j < V; j++) cos_sin_at(a.r, V * (int)item + j, p, &c[j], &s[j]);
#pragma unroll
    for (int i = 0; i < HEADS; i++)
#pragma unroll
      for (int j = 0; j < V; j++) {
        // (interleaved, the 2V elements of u and w are V pairs)
        E& e0 = INTERLEAVED ? (2 * j < V ? u[i].e[(2 * j) % V] : w[i].e[(2 * j) % V]) : u[i].e[j];
        E& e1 = INTERLEAVED ? (2 * j + 1 < V ? u[i].e[(2 * j + 1) % V] : w[i].e[(2 * j + 1) % V]) : w[i].e[j];
        float f0 = to_f32(e0), f1 = to_f32(e1);
        turn_pair(f0, f1, c[j], s[j]);
        e0 = from_f32<E>(f0);
        e1 = from_f32<E>(f1);
      }
  }
#pragma unroll
  for (int i = 0; i < HEADS; i++) {
    const int h = h0 + i;
    if (h >= heads) break;
    E* dst = h < a.Hq ? static_cast<E*>(a.qo) + t * a.qo_st + h * a.qo_sh
                      : static_cast<E*>(a.ko) + t * a.ko_st + (h - a.Hq) * a.ko_sh;
    *reinterpret_cast<P*>(dst + d0) = u[i];
    if (both) *reinterpret_cast<P*>(dst + d1) = w[i];
  }
}

template <typename E, int V, bool INTERLEAVED, int HEADS>
hipError_t rope_launches(const RopeArgs& a, hipStream_t st) {
  const uint32_t rest = a.copy ? (uint32_t)((a.D - 2 * a.r.half + 2 * V - 1) / (2 * V)) : 0;
  const uint32_t items = (uint32_t)(a.r.half / V) + rest;
  const uint32_t groups = (uint32_t)((a.Hq + a.Hk + HEADS - 1) / HEADS);
  const int64_t per = (int64_t)items * groups;        // threads of a token (host: below 2^31)
  const int64_t most = ((int64_t(1) << 31) - 1) / per;  // tokens of a launch
  for (int64_t t = 0; t < a.T; t += most) {
    const int64_t n = a.T - t < most ? a.T - t : most;
    const uint32_t total = (uint32_t)(n * per);
    rope_kernel<E, V, INTERLEAVED, HEADS>
        <<<(total + kThreads - 1) / kThreads, kThreads, 0, st>>>(a, t, total, items, groups);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Heads a thread takes: four, which form a pair's cosine and sine once and have eight loads in flight, unless that
// leaves most SIMDs without a wave.  One and four heads, us a call (32 + 8 heads of 128 dims, bf16): 256 tokens (82K
// threads of one head) 4.5, 4.7; 1024 7.7, 6.9; 2048 13.2, 9.6; 8192 37, 30; 65536 307, 244.
template <typename E, int V, bool INTERLEAVED>
hipError_t rope_heads(const RopeArgs& a, hipStream_t st) {
  const int64_t threads = a.T * (a.Hq + a.Hk) * (a.D / (2 * V));
  if (threads >= int64_t(1) << 17) return rope_launches<E, V, INTERLEAVED, 4>(a, st);
  return rope_launches<E, V, INTERLEAVED, 1>(a, st);
}

template <typename E, int V>
hipError_t rope_layout(bool interleaved, const RopeArgs& a, hipStream_t st) {
  return interleaved ? rope_heads<E, V, true>(a, st) : rope_heads<E, V, false>(a, st);
}

// ================================================================ latent write
// A token's row of the cache: 512 numbers as they are, then the 64 of the rotary key, turned.  A copy, bound by
// memory.  A wave takes 8 tokens: their 512 numbers a lane's 16 bytes of each, their rotary keys 8 lanes each
// with 4 pairs; all loads go out before the first is used.  117017 tokens: 44 us a launch, 6.1 TB/s (its rows
// lie in the last-level cache in part); one token of 62 requests: 3 us, latency.
constexpr int kRank = 512, kRot = 64, kRowLen = kRank + kRot, kTokens = 8;

template <bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void latent_write_kernel(LatentWriteArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t t0 = ((int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64) * kTokens;
  if (t0 >= a.T) return;
  // what a token has is loaded before it is known whether it has a slot
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 c[kTokens];
#pragma unroll
  for (int j = 0; j < kTokens; j++) {
    const int64_t at = t0 + j < a.T ? t0 + j : a.T - 1;
    c[j] = reinterpret_cast<const u32x4*>(a.c + at * a.c_st)[lane];
  }
  // lane 8 j + i: 4 pairs of token j's rotary key
  const int i = lane & 7;
  const bool real = t0 + (lane >> 3) < a.T;
  const int64_t t = real ? t0 + (lane >> 3) : a.T - 1;
  using P = Piece<__hip_bfloat16, 4>;
  const int d0 = INTERLEAVED ? 8 * i : 4 * i, d1 = INTERLEAVED ? d0 + 4 : d0 + kRot / 2;
  P u = *reinterpret_cast<const P*>(a.kr + t * a.kr_st + d0), w = *reinterpret_cast<const P*>(a.kr + t * a.kr_st + d1);
  const int64_t slot = a.slots[t];
  // its row in the pool; null: none
  __hip_bfloat16* dst = nullptr;
  int64_t p = 0;
  const bool placed = !a.rotate || row_position(a.r, t, &p);  // (a row of no sequence is left out)
  if (real && placed && slot >= 0 && slot < (int64_t)a.N * a.P) {
    const uint64_t page = (uint64_t)slot / (uint32_t)a.P;
    dst = a.pages + (int64_t)page * a.p_sp + (slot - (int64_t)page * a.P) * kRowLen;
  }
  if (dst) {
    if (a.rotate) {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        float cs, sn;
        cos_sin_at(a.r, 4 * i + j, p, &cs, &sn);
        __hip_bfloat16& e0 = INTERLEAVED ? (j < 2 ? u.e[(2 * j) % 4] : w.e[(2 * j) % 4]) : u.e[j];
        __hip_bfloat16& e1 = INTERLEAVED ? (j < 2 ? u.e[(2 * j + 1) % 4] : w.e[(2 * j + 1) % 4]) : w.e[j];
        float f0 = to_f32(e0), f1 = to_f32(e1);
        turn_pair(f0, f1, cs, sn);
        e0 = from_f32<__hip_bfloat16>(f0);
        e1 = from_f32<__hip_bfloat16>(f1);
      }
    }
    *reinterpret_cast<P*>(dst + kRank + d0) = u;
    *reinterpret_cast<P*>(dst + kRank + d1) = w;
  }
#pragma unroll
  for (int j = 0; j < kTokens; j++) {
    const uint64_t x = reinterpret_cast<uint64_t>(dst);
    __hip_bfloat16* to = reinterpret_cast<__hip_bfloat16*>(
        ((uint64_t)__builtin_amdgcn_readlane((uint32_t)(x >> 32), 8 * j) << 32) |
        (uint32_t)__builtin_amdgcn_readlane((uint32_t)x, 8 * j));
    if (to) reinterpret_cast<u32x4*>(to)[lane] = c[j];
  }
}

}  // namespace

hipError_t launch_rope(bool bf16, bool interleaved, int vec, const RopeArgs& a, hipStream_t st) {
  if (a.T == 0 || a.Hq + a.Hk == 0) return hipSuccess;
  if (bf16) {
    using E = __hip_bfloat16;
    switch (vec) {
      case 8: return rope_layout<E, 8>(interleaved, a, st);
      case 4: return rope_layout<E, 4>(interleaved, a, st);
      case 2: return rope_layout<E, 2>(interleaved, a, st);
      default: return rope_layout<E, 1>(interleaved, a, st);
    }
  }
  switch (vec) {
    case 4: return rope_layout<float, 4>(interleaved, a, st);
    case 2: return rope_layout<float, 2>(interleaved, a, st);
    default: return rope_layout<float, 1>(interleaved, a, st);
  }
}

hipError_t launch_latent_write(bool interleaved, const LatentWriteArgs& a, hipStream_t st) {
  constexpr int kPer = kThreads / 64 * kTokens;
  const unsigned grid = (unsigned)((a.T + kPer - 1) / kPer);
  if (interleaved) latent_write_kernel<true><<<grid, kThreads, 0, st>>>(a);
  else latent_write_kernel<false><<<grid, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace moba
