// Staged tiles of the latent attention kernels (expanded form): 64 tokens of a wide part (128
// dims) or of the rotary part (64 dims), row-major in LDS, filled by global_load_lds_dwordx4 and read both
// as rows and transposed.
//
// Row r's 16-byte chunk c stands at chunk c ^ swizzle(r) of its row.  An operand read, 16 lanes on
// 16 consecutive rows at one chunk, then meets 16 distinct bank groups (LDS: 64 banks of 4 bytes, so 16
// chunks), and so do the windows of a transposed read (ds_read_b64_tr_b16: per 32 lanes 4 consecutive
// rows by 64 bytes).  Wide rows (16 chunks): 4 (r % 4) + (r / 4) % 4.  Rotary rows (8 chunks, two
// rows to the bank period): 4 (r / 2 % 2) + (r / 4) % 4.
#pragma once

#include "latent_internal.h"
#include "mfma_tile.h"

#include <type_traits>
#include <utility>

namespace moba {

constexpr int kWide = kLatTile * kNope / 8;     // 16-byte chunks of a wide tile (1024)
constexpr int kSlim = kLatTile * kRopeDim / 8;  // of a rotary one (512)

__device__ __forceinline__ int swz_wide(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }
__device__ __forceinline__ int swz_slim(int r) { return ((r & 2) << 1) | ((r >> 2) & 3); }

typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ s16x4 tr16(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}

__device__ __forceinline__ bf16x8 join16(s16x4 a, s16x4 b) {
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A pointer that all lanes hold alike, in scalar registers, for dma16_at.  A scalar register that a vector
// instruction wrote (here v_readfirstlane) may be the address of a memory access only five wait states on, and
// the compiler does not count them into inline assembly.
__device__ __forceinline__ const char* scalar_ptr(const void* p) {
  const char* s = uniform_ptr(static_cast<const char*>(p));
  asm volatile("s_nop 4" : "+s"(s));
  return s;
}

// A tensor's rows of one sequence (and head), wave-uniform.
struct Rows {
  const char* base;  // row 0 of the sequence
  uint32_t st;       // bytes between rows
  int len;           // rows of the sequence
};

// Lane's part of the DMA of tile i (64 rows; those past the sequence repeat its last one) by NW
// waves.  WIDE: 16 instructions of four rows, else 8 of eight rows; wave w issues w, w + NW, ..., here its x-th.
template <int NW, bool WIDE>
__device__ __forceinline__ void stage_part(const Rows& R, int i, u32x4* buf, int wave, int lane, int x) {
  constexpr int kCh = WIDE ? 16 : 8;
  const int r0 = i * kLatTile;
  const char* tile = R.base + (int64_t)r0 * R.st;
  const int last = R.len - 1 - r0;  // (a staged tile begins in the sequence)
  const int j = wave + NW * x, row = (64 / kCh) * j + lane / kCh;
  const int c = (lane % kCh) ^ (WIDE ? swz_wide(row) : swz_slim(row));
  dma16_at(tile, (uint32_t)min(row, last) * R.st + (uint32_t)c * 16, buf + 64 * j);
}

template <int NW, bool WIDE>
__device__ __forceinline__ void stage_tile(const Rows& R, int i, u32x4* buf, int wave, int lane) {
  static_assert((WIDE ? 16 : 8) % NW == 0, "whole instructions");
#pragma unroll
  for (int x = 0; x < (WIDE ? 16 : 8) / NW; x++) stage_part<NW, WIDE>(R, i, buf, wave, lane, x);
}

// Row operand: chunk c of row r (bytes).
__device__ __forceinline__ uint32_t at_wide(int r, int c) { return (uint32_t)(r * 256 + ((c ^ swz_wide(r)) * 16)); }
__device__ __forceinline__ uint32_t at_slim(int r, int c) { return (uint32_t)(r * 128 + ((c ^ swz_slim(r)) * 16)); }

// Transposed operand of a 32x32x16 product: lane qc, hh holds dim 32 dt + qc of the rows r0 + {0-3,
// 8-11} + 4 hh, r0 a multiple of 16: two reads, x = 0, 1.  Its address: row r0 + 4 hh + 8 x + i / 4
// at dims 32 dt + 16 (qc / 16) + 4 (i % 4), i = qc % 16.
struct TrLane {
  int row, chunk, half;  // of dt = 0, x = 0
};
__device__ __forceinline__ TrLane tr_lane(int qc, int hh) {
  const int i = qc & 15;
  return {4 * hh + (i >> 2), 2 * (qc >> 4) + ((i & 3) >> 1), 8 * (i & 1)};
}
__device__ __forceinline__ uint32_t tr_wide(const TrLane& t, int dt, int x) {
  return at_wide(t.row + 8 * x, 4 * dt + t.chunk) + t.half;
}
__device__ __forceinline__ uint32_t tr_slim(const TrLane& t, int dt, int x) {
  return at_slim(t.row + 8 * x, 4 * dt + t.chunk) + t.half;
}

// f(0), f(1), ... f(N - 1), the index a constant of the compiler.
template <int N>
using Index = std::integral_constant<int, N>;
template <typename F, int... X>
__device__ __forceinline__ void each_of(F& f, std::integer_sequence<int, X...>) {
  (f(Index<X>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  each_of(f, std::make_integer_sequence<int, N>());
}

// What a packed pair of bf16 leaves out of a and b, as such a pair.
__device__ __forceinline__ uint32_t rest_bf16(uint32_t pair, float a, float b) {
  return pack_bf16(a - __uint_as_float(pair << 16), b - __uint_as_float(pair & 0xffff0000u));
}

// ---- the backward's kernels: work-groups of 4 waves, one on a CU
constexpr int kLatBwdWaves = 4;
constexpr int kLatBwdDma = 10;     // DMA instructions a wave and tile: 4 + 4 + 2
constexpr int kSlicesAhead = 6;    // slices from an operand's reads to its product

// The end of a slice: nothing is moved over it.
__device__ __forceinline__ void slice_end() { __builtin_amdgcn_sched_barrier(0); }

// Places of work.  Sequence s's tiles of `rows` tokens begin at place cu[s] / rows + s, so that
// no table is needed: places(T, S) of them, some empty.
__host__ __device__ inline int64_t latent_places(int64_t T, int S, int rows) { return T / rows + S; }

struct Place {
  int64_t tok0;  // the sequence's first token
  int len;       // its tokens
  int t0;        // the tile's first token within the sequence
};

// Sequence s's first token and tokens: whatever cu holds, within [0, T).
__device__ __forceinline__ int64_t latent_span(const LatentArgs& a, int s, int* len) {
  const int64_t c0 = a.cu[s], c1 = a.cu[s + 1];
  const int64_t b = c0 < 0 ? 0 : c0 > a.T ? a.T : c0;
  const int64_t e = c1 < b ? b : c1 > a.T ? a.T : c1;
  *len = (int)(e - b);
  return b;
}

__device__ __forceinline__ bool latent_place(const LatentArgs& a, int64_t x, int rows, Place* p) {
  // the last sequence whose first place is at or before x: 64 of them looked at together
  int lo = 0;
  for (int n = a.S; n > 1;) {
    const int step = (n + 63) / 64, lane = threadIdx.x & 63, at = lo + lane * step;
    const bool before = lane * step < n && a.cu[min(at, a.S)] / rows + at <= x;
    const int k = max(0, __popcll(__builtin_amdgcn_ballot_w64(before)) - 1);
    lo += k * step;
    n = min(step, n - k * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  int len;
  const int64_t b = latent_span(a, lo, &len);
  const int64_t t0 = (x - (a.cu[lo] / rows + lo)) * rows;
  if (t0 < 0 || t0 >= len) return false;
  p->tok0 = uniform64(b);
  p->len = __builtin_amdgcn_readfirstlane(len);
  p->t0 = __builtin_amdgcn_readfirstlane((int)t0);
  return true;
}

// Sequence s's first tile.
__device__ __forceinline__ bool latent_first(const LatentArgs& a, int s, Place* p) {
  int len;
  p->tok0 = uniform64(latent_span(a, s, &len));
  p->len = __builtin_amdgcn_readfirstlane(len);
  p->t0 = 0;
  return p->len > 0;
}

// Pair r of (head, tile of kLatKeys tokens), those with the most tiles before them in their sequence first; of up to
// 64 sequences.  more: the tiles behind it.
__device__ __forceinline__ bool latent_ranked(const LatentArgs& a, uint32_t r, Place* p, int* h, int* more) {
  const int lane = threadIdx.x & 63;
  int64_t tok0 = 0;
  int len = 0;
  if (lane < a.S) tok0 = latent_span(a, lane, &len);
  const int n = (int)(((uint32_t)len + kLatKeys - 1) / kLatKeys);
  int level = n;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) level = max(level, __shfl_xor(level, d, 64));
  level = __builtin_amdgcn_readfirstlane(level);
  r = __builtin_amdgcn_readfirstlane(r);
  for (; level > 0; level--) {
    const uint64_t in = __builtin_amdgcn_ballot_w64(n >= level);
    const uint32_t c = (uint32_t)__popcll(in), all = c * (uint32_t)a.H;
    if (r >= all) {
      r -= all;
      continue;
    }
    const uint32_t i = r % c;
    const uint32_t before = (uint32_t)__popcll(in & ((1ull << lane) - 1));
    const uint64_t at = __builtin_amdgcn_ballot_w64(n >= level && before == i);
    const int s = __ffsll((unsigned long long)at) - 1;
    *h = (int)(r / c);
    p->tok0 = uniform64(__shfl(tok0, s, 64));
    p->len = __builtin_amdgcn_readlane(len, s);
    p->t0 = (level - 1) * kLatKeys;
    *more = __builtin_amdgcn_readlane(n, s) - level;
    return true;
  }
  return false;
}

// Work-group -> (head, place).  Work-groups go round-robin to the 8 XCDs; each XCD takes a
// contiguous run of (head, place) pairs, so that a head's keys and values stay in one L2.  The places
// of a head are taken longest first where heads divide among the XCDs, and else from both
// ends in turn, so that every run holds long and short ones.
struct Work {
  int h;
  int64_t place;
};
template <bool LAST_LONGEST>
__device__ __forceinline__ bool latent_work(const LatentArgs& a, int64_t places, Work* w) {
  const int64_t per = gridDim.x / 8;
  const int64_t x = (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8;
  if (x >= places * a.H) return false;
  w->h = (int)(x / places);
  int64_t y = x % places;  // 0: the longest
  if (a.H % 8 != 0) y = y % 2 ? places - 1 - y / 2 : y / 2;
  w->place = LAST_LONGEST ? places - 1 - y : y;
  return true;
}

inline unsigned latent_grid(const LatentArgs& a, int rows) {
  return (unsigned)((latent_places(a.T, a.S, rows) * a.H + 7) / 8 * 8);
}

}  // namespace moba
