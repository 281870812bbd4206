// Block tables and slot maps of a serving step, from the requests' lengths.
//
// With h = ceil(len / P) pages held, a request that grows to len' takes ceil(len' / P) - h
// pages off the free list and one that ends gives its h back, so everything follows
// from three prefix sums over the requests (new tokens, pages given back, pages needed), done by
// one work-group: the whole step of a decode batch is a few hundred integers, bound by the
// latency of one launch and its chain of dependent loads (add and lens, the free list, the
// table).  The slots of a long prompt are the only bytes in quantity (8 per token): past
// kPlanOwnTokens of them a second launch writes them over the whole chip.
#include "cache_internal.h"

namespace moba {
namespace {

constexpr int kPlanOwnTokens = 8192;
constexpr int kPlanPer = 4;         // requests per thread at most, of kPlanThreads
constexpr int kPlanThreads = kPlanMaxRequests / kPlanPer;
constexpr int kSlotThreads = 256;
constexpr int kSlotPer = 8;         // tokens per thread of the second launch

// Inclusive sum over the work-group's threads.  part: one word per wave.
__device__ __forceinline__ int64_t group_scan(int64_t x, int64_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up((long long)x, d, 64);
    if (lane >= d) x += o;
  }
  if (blockDim.x == 64) return x;
  if (lane == 63) part[wave] = x;
  __syncthreads();
  for (int w = 0; w < wave; w++) x += part[w];
  __syncthreads();
  return x;
}

// Last index i of [0, n) with pre[i] <= x (pre ascending, pre[0] <= x).
__device__ __forceinline__ int find_last(const int32_t* pre, int n, int64_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int64_t slot_of(const int32_t* row, int64_t pos, int P) {
  const uint32_t j = (uint32_t)pos / (uint32_t)P;
  return (int64_t)row[j] * P + ((uint32_t)pos - j * P);
}

// own_slots: this launch writes slots; otherwise only the one of each request's first
// token (where cache_slots_kernel finds whether the request was refused).
__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(CachePlanArgs a, bool own_slots) {
  extern __shared__ int32_t lds[];
  __shared__ int64_t part[kPlanThreads / 64];
  __shared__ int64_t totals[3];  // pages given back, pages taken, new tokens
  __shared__ int nrefused;
  int32_t* pre = lds;             // [S] exclusive sums: pages given back, then pages taken
  int32_t* cu = lds + a.S;        // [S]
  int32_t* old = lds + 2 * a.S;   // [S] length before the step, ~length where nothing is granted
  const int tid = threadIdx.x, nt = blockDim.x, S = a.S, P = a.P;
  const int64_t cap = min((int64_t)a.W * P, (int64_t)INT32_MAX);  // (lengths are 32-bit)
  const int per = (S + nt - 1) / nt;  // <= kPlanPer
  const int s0 = tid * per;
  int64_t len[kPlanPer], tok[kPlanPer], need[kPlanPer];
  bool ended[kPlanPer];
  int64_t sum_tok = 0, sum_back = 0, sum_need = 0;
#pragma unroll
  for (int i = 0; i < kPlanPer; i++) {
    len[i] = tok[i] = need[i] = 0;
    ended[i] = false;
    if (i >= per || s0 + i >= S) continue;
    const int ad = a.add[s0 + i];
    len[i] = min((int64_t)max(a.lens[s0 + i], 0), cap);
    ended[i] = ad < 0;
    tok[i] = max(ad, 0);
    sum_tok += tok[i];
    if (ended[i]) sum_back += ((uint32_t)len[i] + P - 1) / P;
  }
  const int64_t nfree = min(max((int64_t)*a.num_free, (int64_t)0), (int64_t)a.N);
  if (tid == 0) nrefused = 0;
  const int64_t in_tok = group_scan(sum_tok, part);
  const int64_t in_back = group_scan(sum_back, part);
  int64_t upto = in_tok - sum_tok;
#pragma unroll
  for (int i = 0; i < kPlanPer; i++) {
    upto += tok[i];
    if (ended[i] || len[i] + tok[i] > cap || upto > a.T) need[i] = -1;  // not to be granted
    else need[i] = ((uint32_t)(len[i] + tok[i]) + P - 1) / P - ((uint32_t)len[i] + P - 1) / P;
    sum_need += max(need[i], (int64_t)0);
  }
  const int64_t in_need = group_scan(sum_need, part);
  if (tid == nt - 1) totals[0] = in_back;
  if (tid == nt - 1) totals[2] = in_tok;
  if (tid == 0) totals[1] = 0;
  __syncthreads();
  const int64_t back = min(totals[0], (int64_t)a.N - nfree);
  const int64_t avail = nfree + back;
  // prefixes and results of this thread's requests
  int64_t t = in_tok - sum_tok, b = in_back - sum_back, w = in_need - sum_need;
  int gone = 0;
  int64_t taken = 0;  // of the last request granted
  int32_t first_taken[kPlanPer];
#pragma unroll
  for (int i = 0; i < kPlanPer; i++) {
    first_taken[i] = (int32_t)min(w, avail);
    if (i >= per || s0 + i >= S) continue;
    const int s = s0 + i;
    pre[s] = (int32_t)min(b, back);
    cu[s] = (int32_t)min(t, a.T);
    a.cu[s] = cu[s];
    t += tok[i];
    if (ended[i]) b += ((uint32_t)len[i] + P - 1) / P;
    w += max(need[i], (int64_t)0);
    const bool granted = need[i] >= 0 && (need[i] == 0 || w <= avail);
    if (granted) taken = w;
    old[s] = granted ? (int32_t)len[i] : ~(int32_t)len[i];
    a.lens_out[s] = ended[i] ? 0 : (int32_t)(len[i] + (granted ? tok[i] : 0));
    gone += !granted && !ended[i];
  }
  if (gone) atomicAdd(&nrefused, gone);
  // w grows with s, so the pages taken are the largest granted sum within avail
  if (taken > 0 && taken <= avail) atomicMax((long long*)&totals[1], (long long)taken);
  __syncthreads();
  const int64_t take = totals[1];
  if (tid == 0) {
    a.cu[S] = (int32_t)min(totals[2], a.T);
    *a.refused = nrefused;
    *a.num_free_out = (int32_t)(avail - take);
  }
  // pages of ended requests to the end of the free list
  for (int64_t i = tid; i < back; i += nt) {
    const int s = find_last(pre, S, i);
    a.free_pages[nfree + i] = a.table[s * a.t_ss + (i - pre[s])];
  }
  __threadfence_block();
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPlanPer; i++)
    if (i < per && s0 + i < S) pre[s0 + i] = first_taken[i];
  __syncthreads();
  for (int64_t i = tid; i < take; i += nt) {
    const int s = find_last(pre, S, i);
    const uint32_t held = ((uint32_t)old[s] + P - 1) / P;  // (a request with pages taken is granted)
    a.table[s * a.t_ss + held + (i - pre[s])] = a.free_pages[avail - 1 - i];
  }
  __threadfence_block();
  __syncthreads();
  if (own_slots) {
    const int64_t all = min(totals[2], a.T);
    for (int64_t x = tid; x < a.T; x += nt) {
      int64_t slot = -1;
      if (x < all) {
        const int s = find_last(cu, S, x);
        if (old[s] >= 0) slot = slot_of(a.table + s * a.t_ss, old[s] + (x - cu[s]), P);
      }
      a.slots[x] = slot;
    }
  } else {
    for (int s = tid; s < S; s += nt) {
      const int64_t end = s + 1 < S ? cu[s + 1] : min(totals[2], a.T);
      if (cu[s] < end) a.slots[cu[s]] = old[s] >= 0 ? slot_of(a.table + s * a.t_ss, old[s], P) : -1;
    }
  }
}

// The slots of every token.  cache_plan_kernel left each request's first one (written again
// here, with the same value): -1 where the request was refused.
__global__ __launch_bounds__(kSlotThreads) void cache_slots_kernel(CachePlanArgs a) {
  const int64_t x0 = (int64_t)blockIdx.x * kSlotThreads * kSlotPer + threadIdx.x;
  if (x0 >= a.T) return;
  const int64_t all = a.cu[a.S];
  int s = find_last(a.cu, a.S, min(x0, all));
#pragma unroll
  for (int i = 0; i < kSlotPer; i++) {
    const int64_t x = x0 + i * kSlotThreads;
    if (x >= a.T) return;
    int64_t slot = -1;
    if (x < all) {
      while (s + 1 < a.S && a.cu[s + 1] <= x) s++;
      const int c0 = a.cu[s];
      if (a.slots[c0] >= 0)
        slot = slot_of(a.table + s * a.t_ss, (int64_t)a.lens_out[s] - a.add[s] + (x - c0), a.P);
    }
    a.slots[x] = slot;
  }
}

}  // namespace

hipError_t launch_cache_plan(const CachePlanArgs& a, hipStream_t st) {
  const bool own = a.T <= kPlanOwnTokens;
  // threads for the requests and for the slots or pages to write
  int nt = a.S <= 64 && a.T <= 256 ? 64 : kPlanThreads;
  cache_plan_kernel<<<1, nt, 3 * sizeof(int32_t) * (size_t)a.S, st>>>(a, own);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || own) return e;
  const int64_t groups = (a.T + kSlotThreads * kSlotPer - 1) / (kSlotThreads * kSlotPer);
  cache_slots_kernel<<<(unsigned)groups, kSlotThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace moba
