// Key side of the backward of causal latent attention, and both sides in one launch (see latent_grad.h).
#include "latent_grad.h"

namespace moba {
namespace {

constexpr int kWaves = kLatBwdWaves;
static_assert(kLatKeys == kLatRowsDq, "latent_both_kernel's tiles are either side's");

__global__ __launch_bounds__(64 * kWaves, 1) void latent_dkdv_kernel(LatentArgs a) {
  __shared__ DkdvLds sh;
  Work wk;
  if (!latent_work<false>(a, latent_places(a.T, a.S, kLatKeys), &wk)) return;
  Place pl;
  if (!latent_place(a, wk.place, kLatKeys, &pl)) return;
  latent_dkdv_part(a, pl, __builtin_amdgcn_readfirstlane(wk.h), sh);
}

// Both sides of a small batch: work-groups of either side, those with the longest chains of tiles first, whatever
// their sequence and head.  Runs of 8 ranks of the key side alternate with 8 of the query side.
__global__ __launch_bounds__(64 * kWaves, 1) void latent_both_kernel(LatentArgs a) {
  __shared__ DkdvLds sh;
  const bool keys = blockIdx.x / 8 % 2 == 0;
  Place pl;
  int h, more;
  if (!latent_ranked(a, blockIdx.x / 16 * 8 + blockIdx.x % 8, &pl, &h, &more)) return;
  if (keys) {
    pl.t0 = more * kLatKeys;
    latent_dkdv_part(a, pl, h, sh);
  } else {
    latent_dq_part<First::done>(a, pl, h, sh.tiles);
  }
}

}  // namespace

hipError_t launch_latent_dkdv(const LatentArgs& a, hipStream_t st) {
  latent_dkdv_kernel<<<latent_grid(a, kLatKeys), 64 * kWaves, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_latent_both(const LatentArgs& a, hipStream_t st) {
  latent_both_kernel<<<2 * latent_grid(a, kLatKeys), 64 * kWaves, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace moba
