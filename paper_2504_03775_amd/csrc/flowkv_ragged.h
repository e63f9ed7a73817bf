// Device helpers for calls over a ragged batch: new tokens that lie one request
// after another, request r's at offsets[r] .. offsets[r + 1].
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace flowkv {

// The last r in [0, n) with at(r) <= x (0 if there is none), the same in every
// lane of the wave; at() does not fall and x is uniform.  The lanes probe 64
// places at a time: one round of loads up to 64 requests, two up to 4096,
// where a bisection waits for each of its log2(n) loads.
template <class F>
__device__ __forceinline__ int32_t last_at_most(int32_t n, int64_t x, F at) {
  const int32_t ln = threadIdx.x & 63;
  int32_t lo = 0;
  while (n > 1) {
    const int32_t step = (n + 63) / 64;
    const int32_t i = ln * step;
    const uint64_t hit = __ballot(i < n && int64_t(at(lo + i)) <= x);
    // probe 0 counts as a hit whatever it holds
    const int32_t k = hit ? 63 - __builtin_clzll(hit) : 0;
    lo += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  return lo;
}

}  // namespace flowkv
