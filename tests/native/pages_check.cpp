// Block owners, forks and compaction of the allocator on seeded random streams, built
// with AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_pages_host.py (CPU
// only).  After every call the owners and the free count are what a plain count says.
// Exit status 0 = all checks passed.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "flowkv.h"

#define CHECK(cond)                                                            \
  do {                                                                         \
    if (!(cond)) {                                                             \
      std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); \
      std::exit(1);                                                            \
    }                                                                          \
  } while (0)

namespace {

void round_of(uint64_t seed) {
  std::mt19937_64 rng(seed);
  auto below = [&](int64_t n) { return n > 0 ? int64_t(rng() % uint64_t(n)) : 0; };
  const int32_t P = int32_t(below(200)), bs = 1 + int32_t(below(8));
  flowkv_allocator* a = nullptr;
  CHECK(flowkv_allocator_create(P, int32_t(below(3)), seed, &a) == FLOWKV_OK);
  std::vector<int32_t> own(size_t(P), 0);
  std::vector<std::vector<int32_t>> held;
  for (int step = 0; step < 80; ++step) {
    int64_t room = 0;
    for (int32_t o : own) room += o == 0;
    const int op = int(below(5));
    if (op == 0) {
      std::vector<int32_t> ids(size_t(below(room + 3)));
      const int rc = flowkv_alloc(a, int32_t(ids.size()), ids.data());
      CHECK(rc == (int64_t(ids.size()) > room ? FLOWKV_ENOSPC : FLOWKV_OK));
      if (rc) continue;
      for (int32_t b : ids) ++own[size_t(b)];
      held.push_back(ids);
    } else if (op == 1 && !held.empty()) {
      const size_t i = size_t(below(int64_t(held.size())));
      CHECK(flowkv_free(a, held[i].data(), int32_t(held[i].size())) == FLOWKV_OK);
      for (int32_t b : held[i]) --own[size_t(b)];
      held.erase(held.begin() + int64_t(i));
    } else if (op == 2 && !held.empty()) {
      const std::vector<int32_t> ids = held[size_t(below(int64_t(held.size())))];
      CHECK(flowkv_share(a, ids.data(), int32_t(ids.size())) == FLOWKV_OK);
      for (int32_t b : ids) ++own[size_t(b)];
      held.push_back(ids);
    } else if (op == 3 && !held.empty()) {
      const std::vector<int32_t>& ids = held[size_t(below(int64_t(held.size())))];
      const int64_t tokens = below(int64_t(ids.size()) * bs + 1);
      std::vector<int32_t> out(size_t((tokens + bs - 1) / bs));
      int32_t copy = -1;
      const int rc = flowkv_fork(a, ids.data(), int32_t(ids.size()), tokens, bs, out.data(), &copy);
      CHECK(rc == (tokens % bs && room == 0 ? FLOWKV_ENOSPC : FLOWKV_OK));
      if (rc) continue;
      CHECK(copy == tokens % bs);
      for (int32_t b : out) ++own[size_t(b)];
      held.push_back(out);
    } else if (op == 4) {
      std::vector<int32_t> src(size_t(P), 0), dst(size_t(P), 0);
      int32_t n = -1;
      const int rc = flowkv_compact(a, 0, nullptr, nullptr, &n);
      CHECK(rc == (n > 0 ? FLOWKV_ECAP : FLOWKV_OK));
      if (n > 0) CHECK(flowkv_compact(a, n - 1, src.data(), dst.data(), &n) == FLOWKV_ECAP);
      src.resize(size_t(n));
      dst.resize(size_t(n));
      CHECK(flowkv_compact(a, n, src.data(), dst.data(), &n) == FLOWKV_OK);
      std::vector<int32_t> name(size_t(P), 0);
      for (int32_t b = 0; b < P; ++b) name[size_t(b)] = b;
      for (size_t i = 0; i < size_t(n); ++i) {
        CHECK(own[size_t(src[i])] > 0 && own[size_t(dst[i])] == 0 && dst[i] < src[i]);
        std::swap(own[size_t(src[i])], own[size_t(dst[i])]);
        name[size_t(src[i])] = dst[i];
      }
      for (auto& ids : held)
        for (int32_t& b : ids) b = name[size_t(b)];
    }
    flowkv_alloc_stats st{};
    CHECK(flowkv_allocator_stats(a, &st) == FLOWKV_OK);
    int64_t free_blocks = 0;
    for (int32_t b = 0; b < P; ++b) {
      int32_t count = -1;
      CHECK(flowkv_owners(a, &b, 1, &count) == FLOWKV_OK && count == own[size_t(b)]);
      free_blocks += count == 0;
    }
    CHECK(st.free_blocks == free_blocks);
  }
  flowkv_allocator_destroy(a);
}

}  // namespace

int main(int argc, char** argv) {
  const int rounds = argc > 1 ? std::atoi(argv[1]) : 50;
  for (int i = 0; i < rounds; ++i) round_of(uint64_t(i) * 7919 + 1);
  std::printf("%d rounds ok\n", rounds);
}
