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
// page's 64-token tiles has 256 threads, each 4 tokens x 8 dims of K and of V, held in
// registers as they were read through maximum, rounding and store.  V turns over in
// registers (4 tokens x 4 dims of codes) and LDS and leaves in rows of 64 tokens.  The
// maximum is that of the bit patterns and the rounding the hardware's scaled conversion; the
// maximum tells where a run has an infinity, a NaN or a value past the largest scale, and
// such a run is read again and rounded value by value.  A run of one token, a request's in a
// decode step, is one wave's, several in a work-group side by side.
//
// Measured: 117017 tokens of ragged prompts, 8 kv-heads, bf16, pages of 128 (724 MB): 149
// us a call in a row, 4.8 TB/s, the rate of a large copy (with the elements held, measured and rounded as
// floats, one by one, 347).  One token for each of 62 requests: 7 us; of 1024: 28 (as whole
// work-groups' runs 40), with pages of 256 28 too (196).  A wave per tile, V turned over in
// registers alone, was slower but for pages of 256.
#include "cache_internal.h"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace moba {
namespace {

constexpr int kTileThreads = 256;
constexpr int kVRow = 17;  // dwords per V row in LDS (16 and one to spread the banks)

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef short s16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

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
__device__ __forceinline__ int scale_exp(uint32_t amax_bits) {
  const int x = (int)(amax_bits >> 23) - 126;        // amax = m * 2^x, m in [0.5, 1)
  const int e = (amax_bits & 0x7fffffu) <= 0x600000u ? x - 9 : x - 8;  // m <= 0.875
  return min(max(e, kCacheMinExp), kCacheMaxExp);    // (0 and subnormals: x <= -126)
}
constexpr uint32_t kMostBits = 0x7f600000u;  // 448 * 2^kCacheMaxExp, past which values saturate

// The exponent of a scale this cache wrote; of any other value, one that is not below it.
__device__ __forceinline__ int held_exp(float scale) {
  const uint32_t u = __float_as_uint(scale);
  if ((int32_t)u <= 0 || u >= 0x7f800000u) return kCacheMinExp;
  const int e = (int)(u >> 23) - 127 + ((u & 0x7fffffu) ? 1 : 0);
  return min(max(e, kCacheMinExp), kCacheMaxExp);
}

// Eight elements of a row as they are in memory.
template <typename T>
struct Eight;

template <>
struct Eight<__hip_bfloat16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const __hip_bfloat16* p) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  }
  __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0; }
  __device__ __forceinline__ float at(int d) const { return d & 1 ? bf16_hi(w[d >> 1]) : bf16_lo(w[d >> 1]); }
  // the largest |x| so far, as two 16-bit patterns
  __device__ __forceinline__ uint32_t top(uint32_t m) const {
#pragma unroll
    for (int i = 0; i < 4; i++)
      m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(
              __builtin_bit_cast(u16x2_t, m), __builtin_bit_cast(u16x2_t, w[i] & 0x7fff7fffu)));
    return m;
  }
  // the pattern of that value as a float
  static __device__ __forceinline__ uint32_t bits(uint32_t m) { return max(m & 0xffff0000u, m << 16); }
  // four codes from element 4 i on, scaled by 1 / scale
  __device__ __forceinline__ uint32_t codes(int i, float scale) const {
    s16x2_t r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, w[2 * i]), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, w[2 * i + 1]), scale, true);
    return __builtin_bit_cast(uint32_t, r);
  }
};

template <>
struct Eight<float> {
  float f[8];
  __device__ __forceinline__ void load(const float* p) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = 0.0f;
  }
  __device__ __forceinline__ float at(int d) const { return f[d]; }
  __device__ __forceinline__ uint32_t top(uint32_t m) const {
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
    return m;
  }
  static __device__ __forceinline__ uint32_t bits(uint32_t m) { return m; }
  __device__ __forceinline__ uint32_t codes(int i, float scale) const {
    s16x2_t r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f[4 * i], f[4 * i + 1], scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f[4 * i + 2], f[4 * i + 3], scale, true);
    return __builtin_bit_cast(uint32_t, r);
  }
};

// The largest finite |x| among eight, as a float's pattern.
template <typename T>
__device__ __forceinline__ uint32_t fine_top(const Eight<T>& x, uint32_t m) {
#pragma unroll
  for (int d = 0; d < 8; d++) {
    const uint32_t u = __float_as_uint(x.at(d)) & 0x7fffffffu;
    m = max(m, u < 0x7f800000u ? u : 0u);
  }
  return m;
}
// Four codes of x / 2^e (inv = 2^-e) from element 4 i on: saturated, NaN for what is not finite.
template <typename T>
__device__ __forceinline__ uint32_t odd_codes(const Eight<T>& x, int i, float inv) {
  float y[4];
#pragma unroll
  for (int d = 0; d < 4; d++) {
    const float z = x.at(4 * i + d);
    y[d] = fabsf(z) < INFINITY ? fminf(fmaxf(z * inv, -448.0f), 448.0f) : NAN;
  }
  return pack_f8(y[0], y[1], y[2], y[3]);
}

__device__ __forceinline__ uint32_t rescaled(uint32_t w, float by) {
  float f[4];
  unpack_f8(w, f);
  return pack_f8(f[0] * by, f[1] * by, f[2] * by, f[3] * by);
}

// Four words of four bytes, turned over.
__device__ __forceinline__ void turn(const uint32_t* c, uint32_t* r) {
  const uint32_t t0 = __builtin_amdgcn_perm(c[1], c[0], 0x05010400u);
  const uint32_t t1 = __builtin_amdgcn_perm(c[1], c[0], 0x07030602u);
  const uint32_t u0 = __builtin_amdgcn_perm(c[3], c[2], 0x05010400u);
  const uint32_t u1 = __builtin_amdgcn_perm(c[3], c[2], 0x07030602u);
  r[0] = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
  r[1] = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
  r[2] = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
  r[3] = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
}

// A run of one token (a request's in a decode step), by one wave: lanes 0 .. 7 have its key's
// 16 dims each, lanes 8 .. 15 its value's; eight lanes each read an older key for the sum.
template <typename T, int TILES>
__device__ __forceinline__ void write_single(const CacheWriteArgs& a, int64_t t, int64_t slot, int h) {
  const CachePool& c = a.c;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));  // (opaque, as in the kernel below)
  const uint32_t page = (uint32_t)(slot >> 6) / TILES;
  const int o = (int)(slot - (int64_t)page * (TILES * kCacheTile));
  const int64_t ph = (int64_t)page * c.Hkv + h;
  uint8_t* kp = c.k + page * c.k_sp + h * c.k_sh;
  uint8_t* vp = c.v + page * c.v_sp + h * c.v_sh;
  const int d16 = 16 * (lane & 7), row = lane >> 3;
  const bool value = lane & 8;  // (for lanes below 16)
  Eight<T> x[2];
  x[0].clear();
  x[1].clear();
  if (lane < 16) {
    const T* at = value ? static_cast<const T*>(a.v) + t * a.v_st + h * a.v_sh
                        : static_cast<const T*>(a.k) + t * a.k_st + h * a.k_sh;
    x[0].load(at + d16);
    x[1].load(at + d16 + 8);
  }
  const float ks0 = o > 0 ? c.k_scale[ph] : 0.0f, vs0 = o > 0 ? c.v_scale[ph] : 0.0f;
  // older keys, eight rows a load, half a tile in flight
  uint4 old[4];
  const auto older = [&](int p0) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int p = p0 + 8 * i + row;
      old[i] = make_uint4(0, 0, 0, 0);
      if (p < o) old[i] = *reinterpret_cast<const uint4*>(kp + p * kHeadDim + d16);
    }
  };
  older(0);
  uint32_t m = fine_top(x[1], fine_top(x[0], 0));
#pragma unroll
  for (int i = 1; i < 8; i *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, i, 64));
  const uint32_t km = __builtin_amdgcn_readlane(m, 0), vm = __builtin_amdgcn_readlane(m, 8);
  const int ke = max(o > 0 ? held_exp(ks0) : kCacheMinExp, scale_exp(km));
  const int ve = max(o > 0 ? held_exp(vs0) : kCacheMinExp, scale_exp(vm));
  const bool kold = o > 0 && ks0 != exp2_int(ke), vold = o > 0 && vs0 != exp2_int(ve);
  const float kre = ks0 * exp2_int(-ke), vre = vs0 * exp2_int(-ve);
  const float inv = exp2_int(value ? -ve : -ke);
  const uint32_t code[4] = {odd_codes(x[0], 0, inv), odd_codes(x[0], 1, inv), odd_codes(x[1], 0, inv),
                            odd_codes(x[1], 1, inv)};
  // Sums of codes, multiples of 2^-9: exact in fp32 over up to 64 tokens, and a lane has at
  // most 33; over the lanes as integers.  NaN where one is NaN.
  static_assert(kCacheMaxPage / 8 + 1 <= 64, "a lane's sums are exact");
  float f[16];
#pragma unroll
  for (int d = 0; d < 16; d++) f[d] = 0.0f;
  const auto add = [&](uint32_t w, int e) {
    float g[4];
    unpack_f8(w, g);
#pragma unroll
    for (int d = 0; d < 4; d++) f[4 * e + d] += g[d];
  };
#pragma unroll 1
  for (int p0 = 0; p0 < o; p0 += kCacheTile / 2) {
    if (p0 > 0) older(p0);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int p = p0 + 8 * i + row;
      uint32_t w[4] = {old[i].x, old[i].y, old[i].z, old[i].w};
      if (kold) {
#pragma unroll
        for (int e = 0; e < 4; e++) w[e] = rescaled(w[e], kre);
        if (p < o) *reinterpret_cast<uint4*>(kp + p * kHeadDim + d16) = make_uint4(w[0], w[1], w[2], w[3]);
      }
#pragma unroll
      for (int e = 0; e < 4; e++) add(w[e], e);
      __builtin_amdgcn_sched_barrier(0);  // (rows side by side would need all registers)
    }
  }
  if (lane < 8) {
#pragma unroll
    for (int e = 0; e < 4; e++) add(code[e], e);
    *reinterpret_cast<uint4*>(kp + o * kHeadDim + d16) = make_uint4(code[0], code[1], code[2], code[3]);
  }
#pragma unroll
  for (int d = 0; d < 16; d++) {
    int sum = f[d] == f[d] ? (int)(f[d] * 512.0f) : 1 << 27;  // (a page's sums stay within 2^26)
#pragma unroll
    for (int i = 8; i < 64; i *= 2) sum += __shfl_xor(sum, i, 64);
    f[d] = sum > 1 << 26 ? NAN : (float)sum * exp2_int(ke - 9);
  }
  if (lane < 8) {
    float4* out = reinterpret_cast<float4*>(c.k_sum + ph * kHeadDim + d16);
#pragma unroll
    for (int e = 0; e < 4; e++) out[e] = make_float4(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3]);
  }
  if (vold) {  // the older values, 16 tokens of a dim at a time
#pragma unroll 1
    for (int i = lane; i < (o + kCacheTile - 1) / kCacheTile * (kHeadDim * 4); i += 64) {
      const int p = i / (kHeadDim * 4) * kCacheTile + 16 * (i & 3);  // place of its first token
      uint4* at = reinterpret_cast<uint4*>(vp + 16 * i);
      const uint4 was = *at;
      uint32_t w[4] = {was.x, was.y, was.z, was.w};
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int n = o - p - 4 * e;  // older tokens from this word on
        const uint32_t keep = n >= 4 ? 0u : n <= 0 ? ~0u : ~0u << (8 * n);
        w[e] = (w[e] & keep) | (rescaled(w[e], vre) & ~keep);
      }
      *at = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __threadfence_block();  // (the new value's bytes, written next, lie in the same words)
  }
  if (lane >= 8 && lane < 16) {
    uint8_t* at = vp + (o / kCacheTile) * (kCacheTile * kHeadDim) + d16 * kCacheTile + o % kCacheTile;
#pragma unroll
    for (int d = 0; d < 16; d++) at[d * kCacheTile] = (uint8_t)(code[d / 4] >> (8 * (d & 3)));
  }
  if (lane == 0) {
    c.k_scale[ph] = exp2_int(ke);
    c.v_scale[ph] = exp2_int(ve);
  }
}

// One work-group per window of `window` tokens (at most a page's) and kv-head: the runs
// that begin in it, with SINGLES those of one token a wave each first, then one after the
// other.  TILES: the page's 64-token tiles.
// (Waves per SIMD: where the next more would spill much; three tiles need six for two
// work-groups.)
template <typename T, int TILES, bool SINGLES>
__global__ __launch_bounds__(kTileThreads* TILES, sizeof(T) != 2 ? 4 : SINGLES && TILES != 3 ? 5 : 6) void
cache_write_kernel(CacheWriteArgs a, int window, uint32_t first) {
  constexpr int P = TILES * kCacheTile;
  __shared__ uint32_t vt[TILES][kHeadDim * kVRow];
  __shared__ int ksum[kHeadDim];
  __shared__ int knan[kHeadDim];
  __shared__ uint32_t amax[2], fine_max[2];
  __shared__ unsigned long long begins[TILES];     // rows of the window where a run begins
  __shared__ unsigned long long follows[2 * TILES];  // rows that continue the one before
  __shared__ int64_t slot_at[P];
  const CachePool& c = a.c;
  int tid = threadIdx.x;
  const uint32_t group = first + blockIdx.x;
  const int h = group % c.Hkv;
  const int64_t w0 = (int64_t)(group / c.Hkv) * window;
  const int64_t pool = (int64_t)c.N * P;
  if (tid < 2 * P) {  // (runs that begin in the window end within a page of it)
    const int64_t t = w0 + tid;
    bool follow = false, begin = false;
    if (t < a.T && tid < window + P) {
      const int64_t slot = a.slots[t];
      const bool in_pool = slot >= 0 && slot < pool;
      const uint32_t off = (uint32_t)(slot >> 6) % TILES * kCacheTile + ((uint32_t)slot & 63);
      follow = in_pool && off != 0 && t > 0 && a.slots[t - 1] == slot - 1;
      begin = in_pool && !follow && tid < window;
      if (tid < window) slot_at[tid] = slot;
    }
    const unsigned long long f = __ballot(follow), b = __ballot(begin);
    if ((tid & 63) == 0) {
      follows[tid >> 6] = f;
      if (tid < P) begins[tid >> 6] = b;
    }
  }
  __syncthreads();
  // rows that begin a run and that none follows
  const auto singles = [&](int word) {
    return SINGLES ? begins[word] & ~(follows[word] >> 1 | follows[word + 1] << 63) : 0;
  };
  if constexpr (SINGLES) {
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int nth = 0;
    for (int word = 0; word < TILES; word++) {
      for (unsigned long long w = singles(word); w; w &= w - 1, nth++) {
        if (nth % (kTileThreads / 64 * TILES) != wave) continue;
        const int i = 64 * word + __ffsll((long long)w) - 1;
        write_single<T, TILES>(a, w0 + i, slot_at[i], h);
      }
    }
  }
  unsigned long long left = begins[0] & ~singles(0);
  for (int word = 0;;) {
    while (left == 0 && ++word < TILES) left = begins[word] & ~singles(word);
    if (left == 0) break;
    // (opaque, so that what follows from it is computed here: kept across the loop it takes
    // half of the registers)
    asm volatile("" : "+v"(tid));
    const int tile = tid / kTileThreads, tt = tid % kTileThreads;
    const int x4 = 4 * (tt / 16), c8 = 8 * (tt % 16);  // this thread's tokens and dims of its tile
    const int i0 = 64 * word + __ffsll((long long)left) - 1;
    left &= left - 1;
    const int64_t t0 = w0 + i0;
    const int64_t slot = slot_at[i0];
    const uint32_t page = (uint32_t)(slot >> 6) / TILES;
    const int o = (int)(slot - (int64_t)page * P);
    int n = 1;
    for (int i = i0 + 1; i < 2 * P;) {
      const unsigned long long rest = ~(follows[i >> 6] >> (i & 63));
      const int ones = min(rest ? __ffsll((long long)rest) - 1 : 64, 64 - (i & 63));
      n += ones;
      i += ones;
      if ((i & 63) != 0 || ones == 0) break;
    }
    // this thread's tokens: new ones of the run, earlier ones of the page
    const int p0 = kCacheTile * tile + x4;  // place of the first in the page
    const int64_t ph = (int64_t)page * c.Hkv + h;
    uint8_t* kp = c.k + page * c.k_sp + h * c.k_sh;
    uint8_t* vp = c.v + page * c.v_sp + h * c.v_sh;
    const auto row_at = [&](const void* x, int64_t st, int64_t sh, int r) {
      return static_cast<const T*>(x) + (t0 + r) * st + h * sh + c8;
    };
    Eight<T> kx[4], vx[4];
    uint2 kc[4], vc[4];  // their codes, and the older keys'
    uint32_t km = 0, vm = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = p0 + i - o;
      kx[i].clear();
      vx[i].clear();
      kc[i] = make_uint2(0, 0);
      if (r >= 0 && r < n) {
        kx[i].load(row_at(a.k, a.k_st, a.k_sh, r));
        vx[i].load(row_at(a.v, a.v_st, a.v_sh, r));
      } else if (r < 0) {
        kc[i] = *reinterpret_cast<const uint2*>(kp + (p0 + i) * kHeadDim + c8);
      }
    }
    const float ks0 = o > 0 ? c.k_scale[ph] : 0.0f, vs0 = o > 0 ? c.v_scale[ph] : 0.0f;
    __syncthreads();  // (the last run's reads of shared memory are done)
    if (tid < kHeadDim) ksum[tid] = knan[tid] = 0;
    if (tid < 2) amax[tid] = fine_max[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; i++) {
      km = kx[i].top(km);
      vm = vx[i].top(vm);
    }
    km = Eight<T>::bits(km);
    vm = Eight<T>::bits(vm);
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
      km = max(km, (uint32_t)__shfl_xor((int)km, m, 64));
      vm = max(vm, (uint32_t)__shfl_xor((int)vm, m, 64));
    }
    if ((tid & 63) == 0) {  // (patterns of non-negative floats order as the floats)
      atomicMax(&amax[0], km);
      atomicMax(&amax[1], vm);
    }
    __syncthreads();
    const bool odd = max(amax[0], amax[1]) > kMostBits;
    // (odd is the same for all threads; the rows are read again, to need few registers)
    if (odd) {
      km = vm = 0;
#pragma unroll 1
      for (int r = max(p0 - o, 0); r < min(p0 + 4 - o, n); r++) {
        Eight<T> x;
        x.load(row_at(a.k, a.k_st, a.k_sh, r));
        km = fine_top(x, km);
        x.load(row_at(a.v, a.v_st, a.v_sh, r));
        vm = fine_top(x, vm);
      }
      atomicMax(&fine_max[0], km);
      atomicMax(&fine_max[1], vm);
      __syncthreads();
    }
    const int ke = max(o > 0 ? held_exp(ks0) : kCacheMinExp, scale_exp(odd ? fine_max[0] : amax[0]));
    const int ve = max(o > 0 ? held_exp(vs0) : kCacheMinExp, scale_exp(odd ? fine_max[1] : amax[1]));
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if (p0 + i >= o) kc[i] = make_uint2(kx[i].codes(0, exp2_int(ke)), kx[i].codes(1, exp2_int(ke)));
      vc[i] = make_uint2(vx[i].codes(0, exp2_int(ve)), vx[i].codes(1, exp2_int(ve)));
    }
    if (odd) {
#pragma unroll 1
      for (int r = max(p0 - o, 0); r < min(p0 + 4 - o, n); r++) {
        Eight<T> x;
        x.load(row_at(a.k, a.k_st, a.k_sh, r));
        const uint2 kw = make_uint2(odd_codes(x, 0, exp2_int(-ke)), odd_codes(x, 1, exp2_int(-ke)));
        x.load(row_at(a.v, a.v_st, a.v_sh, r));
        const uint2 vw = make_uint2(odd_codes(x, 0, exp2_int(-ve)), odd_codes(x, 1, exp2_int(-ve)));
#pragma unroll
        for (int i = 0; i < 4; i++) {
          if (p0 + i - o != r) continue;
          kc[i] = kw;
          vc[i] = vw;
        }
      }
    }
    // older tokens keep their bits where the scale stays
    const bool kold = o > 0 && ks0 != exp2_int(ke), vold = o > 0 && vs0 != exp2_int(ve);
    const float kre = ks0 * exp2_int(-ke), vre = vs0 * exp2_int(-ve);
    // K: codes, and their sums (multiples of 2^-9, exact in fp32 over a tile's 64 tokens)
    float sum[8];
#pragma unroll
    for (int d = 0; d < 8; d++) sum[d] = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = p0 + i - o;
      float f[8];
      if (r < 0 && kold) {
        kc[i].x = rescaled(kc[i].x, kre);
        kc[i].y = rescaled(kc[i].y, kre);
      }
      if (r < n && (r >= 0 || kold))
        *reinterpret_cast<uint2*>(kp + (p0 + i) * kHeadDim + c8) = kc[i];
      unpack_f8(kc[i].x, f);  // (rows past the run hold zeros)
      unpack_f8(kc[i].y, f + 4);
#pragma unroll
      for (int d = 0; d < 8; d++) sum[d] += f[d];
    }
#pragma unroll
    for (int d = 0; d < 8; d++) {
      float s = sum[d];
      s += __shfl_xor(s, 16, 64);
      s += __shfl_xor(s, 32, 64);
      if ((tid & 63) < 16) {
        if (s != s) knan[c8 + d] = 1;
        else if (s != 0.0f) atomicAdd(&ksum[c8 + d], (int)(s * 512.0f));
      }
    }
    // V: the tile in LDS, token innermost
    uint32_t vw[8];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      uint32_t code[4];
#pragma unroll
      for (int j = 0; j < 4; j++) code[j] = i ? vc[j].y : vc[j].x;
      turn(code, vw + 4 * i);
    }
    if (vold && p0 < o) {
      const uint32_t keep = o - p0 >= 4 ? 0u : 0xffffffffu << (8 * (o - p0));  // new tokens' bytes
#pragma unroll
      for (int d = 0; d < 8; d++) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(vp + tile * kCacheTile * kHeadDim +
                                                              (c8 + d) * kCacheTile + x4);
        vw[d] = (vw[d] & keep) | (rescaled(w, vre) & ~keep);
      }
    }
#pragma unroll
    for (int d = 0; d < 8; d++) vt[tile][(c8 + d) * kVRow + x4 / 4] = vw[d];
    __syncthreads();
    // rows out, 16 tokens at a time: those that changed are [from, o + n) of the page
    const int from = vold ? 0 : o;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int piece = i * kTileThreads + tt, d = piece / 4, q = piece % 4;
      const int q0 = kCacheTile * tile + 16 * q;  // place of its first token in the page
      if (q0 + 16 <= from || q0 >= o + n) continue;
      const uint32_t* w = &vt[tile][d * kVRow + 4 * q];
      uint8_t* at = vp + tile * kCacheTile * kHeadDim + 16 * piece;
      if (q0 >= from && q0 + 16 <= o + n) {
        *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        for (int j = max(from - q0, 0); j < min(o + n - q0, 16); j++)
          at[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
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

template <typename T, int TILES>
hipError_t launch(const CacheWriteArgs& a, hipStream_t st) {
  // A work-group takes the runs that begin in its window: of four tokens for each of the
  // page's tiles (its waves) where every row may be a run of its own (a decode step), and of as
  // many times that, up to a page, as lets the chip hold all work-groups at once (about
  // 1024 tiles' worth; with four times as many, and half of them): 10000 tokens of one prompt,
  // pages of 128, 2 kv-heads 10.3 us (37.3, 10.6), 8 kv-heads 19.1 (38.2, 19.0), 64 x 16 tokens 11.2
  // (18.1, 14.8), one token each of 1024 requests, pages of 256, 27.5 (28.2, 34.2); 1024 x 40
  // tokens, pages of 128, 2 kv-heads 58.0 (43.5, 57.4).
  // Where rows are many they are prompts', and the kernel without the path of single tokens
  // needs fewer registers: 117017 tokens of prompts take 149 us with it and 157 with the other.
  constexpr int P = TILES * kCacheTile, threads = kTileThreads * TILES;
  const int64_t rows = a.T * a.c.Hkv;
  const int window = (int)std::min<int64_t>(4 * TILES * ((rows + 4095) / 4096), P);
  const int64_t groups = (a.T + window - 1) / window * a.c.Hkv;
  return launch_pieces(groups, threads, [&](uint32_t first, unsigned n) {
    if (rows < 64 * 4096) cache_write_kernel<T, TILES, true><<<n, threads, 0, st>>>(a, window, first);
    else cache_write_kernel<T, TILES, false><<<n, threads, 0, st>>>(a, window, first);
  });
}

template <typename T>
hipError_t launch(const CacheWriteArgs& a, hipStream_t st) {
  const int tiles = a.c.P / kCacheTile;
  return tiles == 1   ? launch<T, 1>(a, st)
         : tiles == 2 ? launch<T, 2>(a, st)
         : tiles == 3 ? launch<T, 3>(a, st)
                      : launch<T, 4>(a, st);
}

}  // namespace

hipError_t launch_cache_write(bool bf16, const CacheWriteArgs& a, hipStream_t st) {
  if (a.T <= 0) return hipSuccess;
  return bf16 ? launch<__hip_bfloat16>(a, st) : launch<float>(a, st);
}

}  // namespace moba
