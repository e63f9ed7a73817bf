// How many splits of a length a request's tokens fill, on host and device.
#pragma once

#include <cstdint>

namespace flowkv {

// ceil(tokens / split) for tokens >= 0, split >= 1, both up to 2^31 - 1.  (tokens + split - 1
// would not fit into 32 bits.)
constexpr int32_t splits_of(int32_t tokens, int32_t split) {
  return tokens / split + (tokens % split > 0);
}

}  // namespace flowkv
