// Block tables and slot maps of a serving step, from the requests' lengths.
//
// With h = ceil(len / P) pages held, a request that grows to len' takes ceil(len' / P) - h
// pages off the free list and one that ends gives its h back, so everything follows
// from three prefix sums over the requests (new tokens, pages given back, pages needed), done by
// one work-group: the whole step of a decode batch is a few hundred integers, bound by the
// latency of one launch and its chain of dependent loads (add and lens, the free list, the
// table).  The slots of a long prompt are the only bytes in quantity (8 per token, and 4 per
// page): past kPlanOwnTokens of them a second launch writes them over the whole chip, and, past
// kPlanOwnPages, the tables' new pages, where its work-groups have a thread for every request.
//
// Measured: 64 requests, one token each, two ending: 5.0 us (a launch that does nothing takes
// about 3); 1M tokens of 8 prompts into 16384 pages: 5.7 us, and 8.8 for their slots and
// pages (with the pages in the first launch, 12.4 and 6.1).
#include "cache_internal.h"

namespace moba {
namespace {

constexpr int kPlanOwnTokens = 8192;
constexpr int kPlanOwnPages = 65536;  // tokens, up to which the first launch takes their pages
constexpr int kPlanPer = 4;         // requests per thread at most, of kPlanThreads
constexpr int kPlanThreads = kPlanMaxRequests / kPlanPer;
constexpr int kLightTokens = 4;     // at most, of every request: none of them searches (a
                                    // page has at least 64, so they need one new page at most)
constexpr int kSlotThreads = 256;
constexpr int kSlotPer = 8;         // tokens per thread of the second launch

// Inclusive sum over the work-group's threads.  part: a word per wave, of this sum alone.
__device__ __forceinline__ int64_t group_scan(int64_t x, int64_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up((long long)x, d, 64);
    if (lane >= d) x += o;
  }
  if (lane == 63) part[wave] = x;
  __syncthreads();
  if (blockDim.x == 64) return x;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64 - 1; w++) x += w < wave ? part[w] : 0;
  return x;
}

// find_last for E values side by side.
template <int E>
__device__ __forceinline__ void find_last(const int32_t* pre, int n, const uint32_t* x, int* s) {
#pragma unroll
  for (int e = 0; e < E; e++) s[e] = 0;
  for (int step = 1 << (31 - __clz(n)); step > 0; step >>= 1) {
    int32_t p[E];
#pragma unroll
    for (int e = 0; e < E; e++) p[e] = pre[min(s[e] + step, n - 1)];
#pragma unroll
    for (int e = 0; e < E; e++) s[e] += s[e] + step < n && (uint32_t)p[e] <= x[e] ? step : 0;
  }
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

// x / P for a page of 1 to 4 tiles (a general division is 20 instructions, and one
// work-group divides for every page).
__device__ __forceinline__ uint32_t page_of(uint32_t x, int P) {
  const uint32_t t = x / kCacheTile;
  return P == kCacheTile ? t : P == 2 * kCacheTile ? t / 2 : P == 3 * kCacheTile ? t / 3 : t / 4;
}
// The slot of a page's token `at`.  Where a table or the free list has a negative entry, a negative
// one, and not a refused token's -1 (a request's first slot tells the second launch which it is).
__device__ __forceinline__ int64_t slot_in(int32_t page, int P, uint32_t at) {
  return (int64_t)page * P + (page >= 0 ? at : 0u);
}
// Pages of x tokens (x up to 2^31 - 1).
__device__ __forceinline__ uint32_t pages_of(uint32_t x, int P) { return page_of(x + P - 1, P); }

// put(i, s, get(i, s)) for the items i < n, s the request with pre[s] <= i.  A few items go
// one to a thread.  Many go 512 in a row to a wave, eight to a thread, all read before the
// first is put; where one request has all of them, as a long prompt does, it is searched
// for once (an own search for each made 16384 pages cost 14 us).
template <typename Get, typename Put>
__device__ __forceinline__ void each_item(const int32_t* pre, int S, uint32_t n, Get get, Put put) {
  const uint32_t tid = threadIdx.x, nt = blockDim.x, lane = tid & 63;
  if (n <= 2 * nt) {
    for (uint32_t i = tid; i < n; i += nt) {
      const int s = find_last(pre, S, i);
      put(i, s, get(i, s));
    }
    return;
  }
  for (uint32_t i0 = 8 * (tid & ~63u); i0 < n; i0 += 8 * nt) {
    const uint32_t end = min(i0 + 511, n - 1);
    const int s0 = __builtin_amdgcn_readfirstlane(find_last(pre, S, i0));
    const bool one = s0 + 1 >= S || (uint32_t)pre[s0 + 1] > end;
    uint32_t at[8];
    int s[8];
    int32_t x[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
      at[e] = min(i0 + 64 * e + lane, end);
      s[e] = s0;
    }
    if (!one) find_last<8>(pre, S, at, s);
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = get(at[e], s[e]);
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const uint32_t i = i0 + 64 * e + lane;
      if (i < n) put(i, s[e], x[e]);
    }
  }
}

// own_slots: this launch writes slots; otherwise only the one of each request's first
// token (where cache_slots_kernel finds whether the request was refused).  own_pages: it
// writes the new pages into the tables.
__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(CachePlanArgs a, bool own_slots,
                                                                  bool own_pages) {
  extern __shared__ int32_t lds[];
  __shared__ int64_t part[3][kPlanThreads / 64];
  __shared__ int64_t totals[3];  // pages given back, pages taken, new tokens
  __shared__ int nrefused, heavy;
  int32_t* pre = lds;             // [S] exclusive sums: pages given back, then pages taken
  int32_t* cu = lds + a.S;        // [S]
  int32_t* old = lds + 2 * a.S;   // [S] length before the step, ~length where nothing is granted
  const int tid = threadIdx.x, nt = blockDim.x, S = a.S, P = a.P;
  const int64_t cap = min((int64_t)a.W * P, (int64_t)INT32_MAX);  // (lengths are 32-bit)
  const int per = (S + nt - 1) / nt;  // <= kPlanPer
  const int s0 = tid * per;
  int64_t len[kPlanPer], tok[kPlanPer], need[kPlanPer];
  bool ended[kPlanPer], granted[kPlanPer];
  if (tid == 0) nrefused = heavy = 0;
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
    if (ended[i]) sum_back += pages_of((uint32_t)len[i], P);
  }
  const int64_t nfree = min(max((int64_t)*a.num_free, (int64_t)0), (int64_t)a.N);
  const int64_t in_tok = group_scan(sum_tok, part[0]);
  const int64_t in_back = group_scan(sum_back, part[1]);
  int64_t upto = in_tok - sum_tok;
#pragma unroll
  for (int i = 0; i < kPlanPer; i++) {
    upto += tok[i];
    if (ended[i] || len[i] + tok[i] > cap || upto > a.T) need[i] = -1;  // not to be granted
    else need[i] = pages_of((uint32_t)(len[i] + tok[i]), P) - pages_of((uint32_t)len[i], P);
    sum_need += max(need[i], (int64_t)0);
    if (tok[i] > kLightTokens) heavy = 1;
  }
  const int64_t in_need = group_scan(sum_need, part[2]);
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
  int32_t first_taken[kPlanPer], my_cu[kPlanPer];
#pragma unroll
  for (int i = 0; i < kPlanPer; i++) {
    first_taken[i] = (int32_t)min(w, avail);
    my_cu[i] = (int32_t)min(t, a.T);
    granted[i] = false;
    if (i >= per || s0 + i >= S) continue;
    const int s = s0 + i;
    pre[s] = (int32_t)min(b, back);
    cu[s] = my_cu[i];
    a.cu[s] = my_cu[i];
    t += tok[i];
    if (ended[i]) b += pages_of((uint32_t)len[i], P);
    w += max(need[i], (int64_t)0);
    granted[i] = need[i] >= 0 && (need[i] == 0 || w <= avail);
    if (granted[i] && need[i] > 0) taken = w;  // (w <= avail)
    old[s] = granted[i] ? (int32_t)len[i] : ~(int32_t)len[i];
    a.lens_out[s] = ended[i] ? 0 : (int32_t)(len[i] + (granted[i] ? tok[i] : 0));
    gone += !granted[i] && !ended[i];
  }
  if (gone) atomicAdd(&nrefused, gone);
  // w grows with s, so the pages taken are the largest granted sum
  if (taken > 0) atomicMax((long long*)&totals[1], (long long)taken);
  __syncthreads();
  const int64_t take = totals[1];
  if (tid == 0) {
    a.cu[S] = (int32_t)min(totals[2], a.T);
    *a.refused = nrefused;
    *a.num_free_out = (int32_t)(avail - take);
  }
  // pages of ended requests to the end of the free list
  if (back > 0) {
    each_item(pre, S, (uint32_t)back, [&](uint32_t i, int s) { return a.table[s * a.t_ss + (i - pre[s])]; },
              [&](uint32_t i, int, int32_t page) { a.free_pages[nfree + i] = page; });
    __threadfence_block();
    __syncthreads();
  }
  const int64_t all = min(totals[2], a.T);
  if (!heavy) {
    // a decode step: a request's few tokens lie on its last page and on one new page at most,
    // and its thread has all that is needed
    int32_t last_page[kPlanPer], new_page[kPlanPer];
#pragma unroll
    for (int i = 0; i < kPlanPer; i++) {
      last_page[i] = new_page[i] = 0;
      if (!granted[i] || tok[i] == 0) continue;
      if (len[i] % P) last_page[i] = a.table[(s0 + i) * a.t_ss + page_of((uint32_t)len[i], P)];
      if (need[i] > 0) new_page[i] = a.free_pages[avail - 1 - first_taken[i]];
    }
#pragma unroll
    for (int i = 0; i < kPlanPer; i++) {
      if (tok[i] == 0) continue;
      const uint32_t h = pages_of((uint32_t)len[i], P);
      if (granted[i] && need[i] > 0) a.table[(s0 + i) * a.t_ss + h] = new_page[i];
      for (int x = 0; x < (int)min(tok[i], a.T - my_cu[i]); x++) {
        const uint32_t pos = (uint32_t)len[i] + x, j = page_of(pos, P);
        a.slots[my_cu[i] + x] =
            granted[i] ? slot_in(j < h ? last_page[i] : new_page[i], P, pos - j * P) : -1;
      }
    }
    if (own_slots)
      for (int64_t x = all + tid; x < a.T; x += nt) a.slots[x] = -1;
    return;
  }
#pragma unroll
  for (int i = 0; i < kPlanPer; i++)
    if (i < per && s0 + i < S) pre[s0 + i] = first_taken[i];
  __syncthreads();
  // From here on table entries are written or read, never both: new pages are taken from
  // the free list wherever they are needed.
  const auto held = [&](int s) { return pages_of((uint32_t)old[s], P); };  // (of a granted one)
  const auto slot_of = [&](int s, uint32_t pos) {
    const uint32_t j = page_of(pos, P), h = held(s);
    const int page = j < h ? a.table[s * a.t_ss + j] : a.free_pages[avail - 1 - (pre[s] + (int64_t)(j - h))];
    return slot_in(page, P, pos - j * P);
  };
  if (own_pages)
    each_item(pre, S, (uint32_t)take, [&](uint32_t i, int) { return a.free_pages[avail - 1 - i]; },
              [&](uint32_t i, int s, int32_t page) {
                a.table[s * a.t_ss + held(s) + (i - pre[s])] = page;
              });
  if (own_slots) {
    for (int64_t x0 = tid; x0 < a.T; x0 += 8 * nt) {
      uint32_t at[8];
      int s[8];
      int64_t slot[8];
#pragma unroll
      for (int e = 0; e < 8; e++) at[e] = (uint32_t)min(x0 + e * nt, a.T - 1);
      find_last<8>(cu, S, at, s);
#pragma unroll
      for (int e = 0; e < 8; e++)
        slot[e] = at[e] < all && old[s[e]] >= 0 ? slot_of(s[e], (uint32_t)old[s[e]] + (at[e] - cu[s[e]])) : -1;
#pragma unroll
      for (int e = 0; e < 8; e++)
        if (x0 + e * nt < a.T) a.slots[x0 + e * nt] = slot[e];
    }
  } else {
    for (int s = tid; s < S; s += nt)
      if (cu[s] < (s + 1 < S ? cu[s + 1] : all))
        a.slots[cu[s]] = old[s] >= 0 ? slot_of(s, (uint32_t)old[s]) : -1;
  }
}

// The slots of every token.  cache_plan_kernel left each request's first one (written again
// here, with the same value): -1 where the request was refused.  PAGES (S <= kSlotThreads): and
// the new pages of the tables, from the free list, by the page's first token; where a
// request's begin on the list follows from the lengths.
template <bool PAGES>
__global__ __launch_bounds__(kSlotThreads) void cache_slots_kernel(CachePlanArgs a) {
  __shared__ int64_t part[kPlanThreads / 64];
  __shared__ int32_t before[kSlotThreads];  // pages that earlier requests take
  __shared__ int64_t taken;
  const int lane = threadIdx.x & 63, P = a.P;
  const int64_t w0 = ((int64_t)blockIdx.x * kSlotThreads + (threadIdx.x & ~63)) * kSlotPer;  // the wave's
  const int64_t all = a.cu[a.S];
  int64_t top = 0;  // pages on the free list before any was taken
  if constexpr (PAGES) {
    const int r = threadIdx.x;
    int64_t need = 0;
    if (r < a.S) {
      const int c = a.cu[r];
      const uint32_t now = (uint32_t)a.lens_out[r], tok = (uint32_t)max(a.add[r], 0);
      if (c < a.cu[r + 1] && a.slots[c] != -1) need = pages_of(now, P) - pages_of(now - tok, P);
    }
    const int64_t upto = group_scan(need, part);
    before[r] = (int32_t)(upto - need);
    if (r == kSlotThreads - 1) taken = upto;
    __syncthreads();
    top = *a.num_free_out + taken;
  }
  if (w0 >= a.T) return;
  // the requests of the wave's first and last token, 64 candidates at a time
  int lo = 0, hi = 0;
  for (int width = a.S; width > 1;) {
    const int step = (width + 63) / 64;
    const int64_t c0 = lo + lane * step < a.S && lane * step < width ? a.cu[lo + lane * step] : INT64_MAX;
    const int64_t c1 = hi + lane * step < a.S && lane * step < width ? a.cu[hi + lane * step] : INT64_MAX;
    lo += step * (max((int)__popcll(__ballot(c0 <= w0)), 1) - 1);
    hi += step * (max((int)__popcll(__ballot(c1 <= w0 + 64 * kSlotPer - 1)), 1) - 1);
    width = step;
  }
  // the slot of position pos of a granted request s that held h pages; its page for the table
  const auto slot_of = [&](int s, uint32_t pos, uint32_t h) {
    const uint32_t j = page_of(pos, P);
    int32_t* at = a.table + s * a.t_ss + j;
    int32_t page;
    if (PAGES && j >= h) {
      page = a.free_pages[top - 1 - (before[s] + (int64_t)(j - h))];
      if (pos == j * P) *at = page;
    } else {
      page = *at;
    }
    return slot_in(page, P, pos - j * P);
  };
  if (lo == hi && w0 + 64 * kSlotPer <= all) {  // one request's, as in a long prompt
    const int r = __builtin_amdgcn_readfirstlane(lo), begin = a.cu[r];
    const bool ok = a.slots[begin] != -1;
    const uint32_t old = (uint32_t)(a.lens_out[r] - a.add[r]);
    const uint32_t pos0 = old + (uint32_t)(w0 - begin) + lane, h = pages_of(old, P);
    int64_t slot[kSlotPer];
#pragma unroll
    for (int i = 0; i < kSlotPer; i++) slot[i] = ok ? slot_of(r, pos0 + 64 * i, h) : -1;
#pragma unroll
    for (int i = 0; i < kSlotPer; i++) a.slots[w0 + 64 * i + lane] = slot[i];
    return;
  }
  const int64_t x0 = w0 + lane * kSlotPer;
  int s = lo, c0 = 0;
  for (int last = hi; s < last;) {  // among them, this thread's first
    const int mid = (s + last + 1) >> 1;
    if (a.cu[mid] <= x0) s = mid; else last = mid - 1;
  }
  int64_t end = -1, old = 0;  // where request s ends; its length before the step
  uint32_t h = 0;
  bool granted = false;
  int64_t slot[kSlotPer];
#pragma unroll
  for (int i = 0; i < kSlotPer; i++) {
    const int64_t x = x0 + i;
    slot[i] = -1;
    if (x < all) {
      if (x >= end) {
        while (s + 1 < a.S && a.cu[s + 1] <= x) s++;
        c0 = a.cu[s];
        end = a.cu[s + 1];
        granted = a.slots[c0] != -1;
        old = (int64_t)a.lens_out[s] - a.add[s];
        if (granted) h = pages_of((uint32_t)old, P);
      }
      if (granted) slot[i] = slot_of(s, (uint32_t)(old + (x - c0)), h);
    }
  }
  if (x0 + kSlotPer <= a.T) {
    typedef int64_t Two __attribute__((ext_vector_type(2), aligned(8)));
#pragma unroll
    for (int i = 0; i < kSlotPer; i += 2) *reinterpret_cast<Two*>(a.slots + x0 + i) = Two{slot[i], slot[i + 1]};
    return;
  }
#pragma unroll
  for (int i = 0; i < kSlotPer; i++)
    if (x0 + i < a.T) a.slots[x0 + i] = slot[i];
}

}  // namespace

hipError_t launch_cache_plan(const CachePlanArgs& a, hipStream_t st) {
  const bool own = a.T <= kPlanOwnTokens;
  // New pages from one work-group, and from the second launch (whole calls): 10000 tokens
  // in 8 requests 11.5, 13.2 us, 32768 12.3, 12.4, 524288 14.1, 12.9; in 200 requests 10000 16.0,
  // 17.8, 131072 20.1, 16.8; 2M in 256 43, 20.
  const bool pages = a.T <= kPlanOwnPages || a.S > kSlotThreads;
  // threads for the requests, and for the pages and slots to write (64 tokens in 8 requests:
  // 4.9 us with 64 threads, 8.2 with 1024)
  const int nt = a.S <= 64 && a.T <= 256 ? 64 : a.S <= 256 && (!pages || a.T <= 16384) ? 256 : kPlanThreads;
  cache_plan_kernel<<<1, nt, 3 * sizeof(int32_t) * (size_t)a.S, st>>>(a, own, pages);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || own) return e;
  const unsigned groups = (unsigned)((a.T + kSlotThreads * kSlotPer - 1) / (kSlotThreads * kSlotPer));
  if (pages) cache_slots_kernel<false><<<groups, kSlotThreads, 0, st>>>(a);
  else cache_slots_kernel<true><<<groups, kSlotThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace moba
