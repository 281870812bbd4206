// New keys and values into their slots of the paged 8-bit cache.
//
// A page's tokens of one kv-head share a scale 2^e, so its run of new tokens is one
// work-group's: the largest finite |x| gives e (not less than the page's own where older
// tokens stay), x 2^-e is rounded to e4m3 once, older tokens are rounded again where e
// grew, and k_sum is the integer sum of the page's codes in units of 2^(e - 9), which no
// order of adding changes.
//
// The work is bound by HBM: 2 x 128 elements read and as many bytes written per token and
// kv-head, and the older keys of a page that is appended to (for k_sum).  Each of the
// page's 64-token tiles has 256 threads, each 4 tokens x 8 dims of K and of V held in
// registers from the one read through maximum, rounding and store.  V turns over in LDS
// (a thread's 4 tokens of a dim are one dword of the tile) and leaves in rows of 64 tokens.
#include "cache_internal.h"

#include <math.h>

#include <type_traits>

namespace moba {
namespace {

constexpr int kTileThreads = 256;
constexpr int kMaxTiles = kCacheMaxPage / kCacheTile;
constexpr int kVRow = 17;  // dwords per V row in LDS (16 and one to spread the banks)

typedef float f32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Four floats to four e4m3 codes (ties to even; NaN stays NaN).
__device__ __forceinline__ uint32_t pack_f8(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
__device__ __forceinline__ void unpack_f8(uint32_t w, float* f) {
  const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
}

// 2^e, e in [-126, 127]
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The least e with amax <= 448 * 2^e = 0.875 * 2^(e + 9), within the limits.
__device__ __forceinline__ int scale_exp(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int x = (int)(u >> 23) - 126;                // amax = m * 2^x, m in [0.5, 1)
  const int e = (u & 0x7fffffu) <= 0x600000u ? x - 9 : x - 8;  // m <= 0.875
  return min(max(e, kCacheMinExp), kCacheMaxExp);    // (0 and subnormals: x <= -126)
}

// The exponent of a scale this cache wrote; of any other value, one that is not below it.
__device__ __forceinline__ int held_exp(float scale) {
  const uint32_t u = __float_as_uint(scale);
  if ((int32_t)u <= 0 || u >= 0x7f800000u) return kCacheMinExp;
  const int e = (int)(u >> 23) - 127 + ((u & 0x7fffffu) ? 1 : 0);
  return min(max(e, kCacheMinExp), kCacheMaxExp);
}

struct Eight {
  float x[8];
};
__device__ __forceinline__ Eight load8(const __hip_bfloat16* p) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  return {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y),
          bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w)};
}
__device__ __forceinline__ Eight load8(const float* p) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  return {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

// x * 2^-e saturated to the largest code; NaN where x is not finite.
__device__ __forceinline__ float scaled(float x, float inv) {
  const float y = fminf(fmaxf(x * inv, -448.0f), 448.0f);
  return fabsf(x) < INFINITY ? y : NAN;
}

// One work-group per window of `window` tokens and kv-head: the runs that begin in it, one
// after the other.  blockDim.x = 256 * (P / 64).
template <typename T>
__global__ __launch_bounds__(kTileThreads* kMaxTiles) void cache_write_kernel(CacheWriteArgs a,
                                                                              int window,
                                                                              uint32_t first) {
  __shared__ uint32_t vt[kMaxTiles][kHeadDim * kVRow];
  __shared__ int ksum[kHeadDim];
  __shared__ int knan[kHeadDim];
  __shared__ uint32_t amax[2];
  __shared__ int run_len;
  __shared__ unsigned long long begins[kTileThreads / 64];
  const CachePool& c = a.c;
  const int tid = threadIdx.x, tile = tid / kTileThreads, tt = tid % kTileThreads;
  const uint32_t group = first + blockIdx.x;
  const int h = group % c.Hkv;
  const int64_t w0 = (int64_t)(group / c.Hkv) * window;
  const int64_t pool = (int64_t)c.N * c.P;
  const int x4 = 4 * (tt / 16), c8 = 8 * (tt % 16);  // this thread's tokens and dims of its tile
  // the rows of the window (at most 256) where a run begins
  if (tid < kTileThreads) {
    const int64_t t = w0 + tid;
    bool begin = false;
    if (tid < window && t < a.T) {
      const int64_t slot = a.slots[t];
      begin = slot >= 0 && slot < pool &&
              (t == 0 || slot % c.P == 0 || a.slots[t - 1] != slot - 1);
    }
    const unsigned long long m = __ballot(begin);
    if ((tid & 63) == 0) begins[tid >> 6] = m;
  }
  __syncthreads();
  unsigned long long left = begins[0];
  for (int word = 0;;) {
    while (left == 0 && ++word < kTileThreads / 64) left = begins[word];
    if (left == 0) break;
    const int64_t t0 = w0 + 64 * word + __ffsll((long long)left) - 1;
    left &= left - 1;
    const int64_t slot = a.slots[t0];
    const int64_t page = slot / c.P;
    const int o = (int)(slot - page * c.P);
    // the run's length: the first row that does not follow, or the page's end
    __syncthreads();  // (the last run's reads of shared memory are done)
    if (tid == 0) run_len = (int)min((int64_t)(c.P - o), a.T - t0);
    if (tid < kHeadDim) ksum[tid] = knan[tid] = 0;
    if (tid < 2) amax[tid] = 0;
    __syncthreads();
    if (tid > 0 && tid < c.P - o && t0 + tid < a.T && a.slots[t0 + tid] != slot + tid)
      atomicMin(&run_len, tid);
    __syncthreads();
    const int n = run_len;
    // this thread's tokens: new ones of the run, earlier ones of the page
    const int p0 = kCacheTile * tile + x4;  // place of the first in the page
    Eight kx[4], vx[4];
    float km = 0.0f, vm = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = p0 + i - o;
      if (r >= 0 && r < n) {
        kx[i] = load8(static_cast<const T*>(a.k) + (t0 + r) * a.k_st + h * a.k_sh + c8);
        vx[i] = load8(static_cast<const T*>(a.v) + (t0 + r) * a.v_st + h * a.v_sh + c8);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = p0 + i - o;
      if (r >= 0 && r < n) {
#pragma unroll
        for (int d = 0; d < 8; d++) {
          const float ka = fabsf(kx[i].x[d]), va = fabsf(vx[i].x[d]);
          km = fmaxf(km, ka < INFINITY ? ka : 0.0f);
          vm = fmaxf(vm, va < INFINITY ? va : 0.0f);
        }
      }
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
      km = fmaxf(km, __shfl_xor(km, m, 64));
      vm = fmaxf(vm, __shfl_xor(vm, m, 64));
    }
    if ((tid & 63) == 0) {  // (non-negative floats order as their bits)
      atomicMax(&amax[0], __float_as_uint(km));
      atomicMax(&amax[1], __float_as_uint(vm));
    }
    const int64_t ph = page * c.Hkv + h;
    const int ke0 = o > 0 ? held_exp(c.k_scale[ph]) : kCacheMinExp;
    const int ve0 = o > 0 ? held_exp(c.v_scale[ph]) : kCacheMinExp;
    const float ks0 = o > 0 ? c.k_scale[ph] : 0.0f, vs0 = o > 0 ? c.v_scale[ph] : 0.0f;
    __syncthreads();
    const int ke = max(ke0, scale_exp(__uint_as_float(amax[0])));
    const int ve = max(ve0, scale_exp(__uint_as_float(amax[1])));
    const float kinv = exp2_int(-ke), vinv = exp2_int(-ve);
    // what the older tokens are multiplied by; 1: they keep their bits
    const float kre = ks0 * kinv, vre = vs0 * vinv;
    const bool kold = o > 0 && ks0 != exp2_int(ke), vold = o > 0 && vs0 != exp2_int(ve);
    uint8_t* kp = c.k + page * c.k_sp + h * c.k_sh;
    uint8_t* vp = c.v + page * c.v_sp + h * c.v_sh;
    // K: codes, their sum
    int sum[8];
    uint32_t bad = 0;
#pragma unroll
    for (int d = 0; d < 8; d++) sum[d] = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int p = p0 + i, r = p - o;
      if (r >= n) continue;
      uint2 w;
      uint2* at = reinterpret_cast<uint2*>(kp + p * kHeadDim + c8);
      float f[8];
      if (r >= 0) {
#pragma unroll
        for (int d = 0; d < 8; d++) f[d] = scaled(kx[i].x[d], kinv);
      } else {
        w = *at;
        if (kold) {
          unpack_f8(w.x, f);
          unpack_f8(w.y, f + 4);
#pragma unroll
          for (int d = 0; d < 8; d++) f[d] *= kre;
        }
      }
      if (r >= 0 || kold) {
        w.x = pack_f8(f[0], f[1], f[2], f[3]);
        w.y = pack_f8(f[4], f[5], f[6], f[7]);
        *at = w;
      }
      unpack_f8(w.x, f);
      unpack_f8(w.y, f + 4);
#pragma unroll
      for (int d = 0; d < 8; d++) {
        const bool is_nan = f[d] != f[d];
        bad |= is_nan ? 1u << d : 0u;
        sum[d] += is_nan ? 0 : (int)(f[d] * 512.0f);
      }
    }
#pragma unroll
    for (int d = 0; d < 8; d++) {
      int s = sum[d];
      s += __shfl_xor(s, 16, 64);
      s += __shfl_xor(s, 32, 64);
      if ((tid & 63) < 16 && s) atomicAdd(&ksum[c8 + d], s);
      if ((bad >> d) & 1) knan[c8 + d] = 1;
    }
    // V: the tile in LDS, token innermost
#pragma unroll
    for (int d = 0; d < 8; d++) {
      float f[4];
      uint32_t w = 0;
      if (vold && p0 < o) {
        w = *reinterpret_cast<const uint32_t*>(vp + tile * kCacheTile * kHeadDim +
                                               (c8 + d) * kCacheTile + x4);
        unpack_f8(w, f);
#pragma unroll
        for (int i = 0; i < 4; i++) f[i] *= vre;
      }
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int r = p0 + i - o;
        if (r >= 0) f[i] = r < n ? scaled(vx[i].x[d], vinv) : 0.0f;
        else if (!vold) f[i] = 0.0f;
      }
      vt[tile][(c8 + d) * kVRow + x4 / 4] = pack_f8(f[0], f[1], f[2], f[3]);
    }
    __syncthreads();
    // rows out: a thread has half a row, 32 tokens; those that changed are [from, o + n)
    {
      const int from = vold ? 0 : o;
      const int d = tt / 2, half = tt % 2;
      const int q0 = kCacheTile * tile + 32 * half;  // place of its first token in the page
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; i++) w[i] = vt[tile][d * kVRow + 8 * half + i];
      uint8_t* at = vp + tile * kCacheTile * kHeadDim + d * kCacheTile + 32 * half;
      if (q0 >= from && q0 + 32 <= o + n) {
        reinterpret_cast<uint4*>(at)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(at)[1] = make_uint4(w[4], w[5], w[6], w[7]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const int q = q0 + 4 * i;
          if (q >= from && q + 4 <= o + n) {
            reinterpret_cast<uint32_t*>(at)[i] = w[i];
          } else {
#pragma unroll
            for (int j = 0; j < 4; j++)
              if (q + j >= from && q + j < o + n) at[4 * i + j] = (uint8_t)(w[i] >> (8 * j));
          }
        }
      }
    }
    if (tid < kHeadDim)
      c.k_sum[ph * kHeadDim + tid] = knan[tid] ? NAN : (float)ksum[tid] * exp2_int(ke - 9);
    if (tid == 0) {
      c.k_scale[ph] = exp2_int(ke);
      c.v_scale[ph] = exp2_int(ve);
    }
  }
}

}  // namespace

hipError_t launch_cache_write(bool bf16, const CacheWriteArgs& a, hipStream_t st) {
  if (a.T <= 0) return hipSuccess;
  // A work-group takes the runs that begin in its window one after the other: a window of
  // one token where every row may be a run of its own (a decode step), up to a page's
  // tokens where there are rows enough to fill the chip either way.
  int window = 1;
  while (window < a.c.P && a.T * a.c.Hkv / (2 * window) >= 4096) window *= 2;
  const int64_t groups = (a.T + window - 1) / window * a.c.Hkv;
  const int threads = kTileThreads * (a.c.P / kCacheTile);
  return launch_pieces(groups, threads, [&](uint32_t first, unsigned n) {
    if (bf16) cache_write_kernel<__hip_bfloat16><<<n, threads, 0, st>>>(a, window, first);
    else cache_write_kernel<float><<<n, threads, 0, st>>>(a, window, first);
  });
}

}  // namespace moba
