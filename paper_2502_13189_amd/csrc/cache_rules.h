// Arithmetic on a request's length in the paged cache, for the device and the host (plain C++).
#pragma once

namespace moba {

constexpr int kCacheTile = 64;  // tokens of a V tile, and of a decode step

// Steps of `len` tokens, for every len >= 0 (len + 63 would pass 2^31 - 1 near its end).
constexpr int cache_steps(int len) { return len / kCacheTile + (len % kCacheTile != 0); }

}  // namespace moba
