// Backward of causal latent attention (see latent_grad.h): Delta, the query side, dkr.
#include "latent_grad.h"

namespace moba {
namespace {

constexpr int kWaves = kLatBwdWaves;
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

__global__ __launch_bounds__(64 * kWaves, 1) void latent_dq_kernel(LatentArgs a) {
  __shared__ u32x4 lds[2 * kBufDq];
  Work wk;
  if (!latent_work<true>(a, latent_places(a.T, a.S, kLatRowsDq), &wk)) return;
  Place pl;
  if (!latent_place(a, wk.place, kLatRowsDq, &pl)) return;
  latent_dq_part<First::form>(a, pl, __builtin_amdgcn_readfirstlane(wk.h), lds);
}

// Delta of each sequence's first 64 rows, where both sides run at once.
__global__ __launch_bounds__(64 * kWaves, 1) void latent_first_kernel(LatentArgs a) {
  __shared__ u32x4 lds[2 * kBufDq];
  Place pl;
  const int s = (int)(blockIdx.x / (uint32_t)a.H);
  if (!latent_first(a, s, &pl)) return;
  latent_dq_part<First::only>(a, pl, (int)(blockIdx.x % (uint32_t)a.H), lds);
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

hipError_t launch_latent_first(const LatentArgs& a, hipStream_t st) {
  latent_first_kernel<<<(unsigned)((int64_t)a.S * a.H), 64 * kWaves, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_latent_dkr(const LatentArgs& a, hipStream_t st) {
  latent_dkr_kernel<<<(unsigned)((a.T * (kRopeDim / 4) + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace moba
