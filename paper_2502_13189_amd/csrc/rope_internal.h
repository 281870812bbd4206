// Rotary positions: what the host sides and the kernels that rotate share.
#pragma once

#include "moba_internal.h"

namespace moba {

// Where a call's rows stand and how fast their pairs turn.  Positions come either from pos,
// or from the packed sequences (row t of sequence s stands at start[s] + t - cu[s]).
struct Rotation {
  const double* freqs;  // [half], radians a position
  const void* pos;      // [T] i32, or i64 (pos64); null: from cu and start
  const int32_t* cu;    // [S + 1]
  const int32_t* start; // [S], null: all 0
  int S;
  int half;             // pairs of a head
  bool pos64;
  float amplitude;
  float sign;           // 1, or -1: the transpose (backward)
};

struct RopeArgs {
  const void* q; int64_t q_st, q_sh;  // [T, Hq, D], elements
  const void* k; int64_t k_st, k_sh;  // [T, Hk, D]
  void* qo; int64_t qo_st, qo_sh;
  void* ko; int64_t ko_st, ko_sh;
  int64_t T;
  int Hq, Hk, D;
  bool copy;                          // the dims that do not turn are copied
  Rotation r;
};
// vec: elements of a piece (16 bytes at most); it divides half and D, and all rows begin at multiples
// of it.
hipError_t launch_rope(bool bf16, bool interleaved, int vec, const RopeArgs& a, hipStream_t st);

struct LatentWriteArgs {
  const __hip_bfloat16* c; int64_t c_st;    // [T, 512]
  const __hip_bfloat16* kr; int64_t kr_st;  // [T, 64]
  const int64_t* slots;
  int64_t T;
  __hip_bfloat16* pages; int64_t p_sp;      // [N, P, 576], page stride in elements
  int N, P;
  bool rotate;
  Rotation r;
};
hipError_t launch_latent_write(bool interleaved, const LatentWriteArgs& a, hipStream_t st);

// ------------------------------------------------------------ device helpers
// A row's position; false: the row is of no sequence.
__device__ __forceinline__ bool row_position(const Rotation& r, int64_t t, int64_t* p) {
  if (r.pos) {
    *p = r.pos64 ? static_cast<const int64_t*>(r.pos)[t] : static_cast<const int32_t*>(r.pos)[t];
    return true;
  }
  int lo = 0, hi = r.S - 1;  // the last sequence that begins at or before t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (r.cu[mid] <= t) lo = mid; else hi = mid - 1;
  }
  const int64_t at = t - r.cu[lo];
  if (at < 0 || t >= r.cu[lo + 1]) return false;
  *p = at + (r.start ? r.start[lo] : 0);
  return true;
}

// A frequency as turns a position, a 64-bit fraction: whole turns do not count, so the angle of
// any position is that fraction times the position modulo 2^64, exact but for the fraction's own
// rounding (below 2^-52 of a turn: 2^-30 radians at position 2^20, frequencies up to 1).
__device__ __forceinline__ uint64_t turns_of(double freq) {
  const double turns = freq * 0.15915494309189533577;  // 1 / (2 pi)
  // (a little below 0 rounds to a whole turn, which 64 bits do not hold)
  return (uint64_t)(fmin(turns - floor(turns), 0x1.fffffffffffffp-1) * 18446744073709551616.0);
}

// cos and sin of a 64-bit fraction of a turn.  The nearest quarter turn is taken off exactly; the rest, x
// in [-pi/4, pi/4], goes into the Taylor series, whose first terms left out (x^11 / 11!, x^12 / 12!)
// stay below 2^-29 and 2^-33.
__device__ __forceinline__ void cos_sin(uint64_t turns, float* c, float* s) {
  const uint32_t t = (uint32_t)(turns >> 32);
  const uint32_t quarter = (t + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(t - (quarter << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float u = x * x;
  float sn = fmaf(u, 2.7557319e-6f, -1.9841270e-4f);
  sn = fmaf(u, sn, 8.3333333e-3f);
  sn = fmaf(u, sn, -1.6666667e-1f);
  sn = fmaf(x * u, sn, x);
  float cs = fmaf(u, -2.7557319e-7f, 2.4801587e-5f);
  cs = fmaf(u, cs, -1.3888889e-3f);
  cs = fmaf(u, cs, 4.1666667e-2f);
  cs = fmaf(u, cs, -0.5f);
  cs = fmaf(u, cs, 1.0f);
  const bool swap = quarter & 1;
  const float a = swap ? sn : cs, b = swap ? cs : sn;
  *c = (quarter + 1) & 2 ? -a : a;
  *s = quarter & 2 ? -b : b;
}

__device__ __forceinline__ void cos_sin_at(const Rotation& r, int i, int64_t p, float* c, float* s) {
  cos_sin(turns_of(r.freqs[i]) * (uint64_t)p, c, s);
  *c *= r.amplitude;
  *s *= r.amplitude * r.sign;
}

// N elements as they are held, 16 bytes at most, in one access.
template <typename E, int N>
struct __align__(sizeof(E) * N) Piece {
  E e[N];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__hip_bfloat16 x) { return __bfloat162float(x); }
template <typename E>
__device__ __forceinline__ E from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __hip_bfloat16 from_f32<__hip_bfloat16>(float x) { return __float2bfloat16(x); }

// (x, y) = (x c - y s, x s + y c)
__device__ __forceinline__ void turn_pair(float& x, float& y, float c, float s) {
  const float a = fmaf(x, c, -(y * s));
  y = fmaf(x, s, y * c);
  x = a;
}

}  // namespace moba
