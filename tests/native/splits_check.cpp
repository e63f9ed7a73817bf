// The count of splits at the ends of 32 bits, against 64 (built with
// UndefinedBehaviorSanitizer by tests/test_chunk_plan_host.py, CPU only).
#include "flowkv_splits.h"

#include <cstdio>
#include <initializer_list>

int main() {
  int checks = 0;
  for (int64_t top : {int64_t(0), int64_t(1) << 11, int64_t(1) << 30, INT64_C(2147483647)})
    for (int64_t tokens = top - 200; tokens <= top + 200; ++tokens)
      for (int64_t split : {INT64_C(1), INT64_C(64), INT64_C(2048), INT64_C(1) << 29, INT64_C(1) << 30,
                            (INT64_C(1) << 30) + 64, INT64_C(2147483584), INT64_C(2147483647)}) {
        if (tokens < 0 || tokens > INT32_MAX) continue;
        const int64_t want = (tokens + split - 1) / split;
        if (flowkv::splits_of(int32_t(tokens), int32_t(split)) != want) {
          std::printf("%lld tokens in splits of %lld: %d, not %lld\n", (long long)tokens,
                      (long long)split, flowkv::splits_of(int32_t(tokens), int32_t(split)),
                      (long long)want);
          return 1;
        }
        ++checks;
      }
  std::printf("%d counts ok\n", checks);
}
