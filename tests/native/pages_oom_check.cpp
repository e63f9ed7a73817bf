// Host memory running out inside the allocator's calls: each allocation in turn fails, and
// the call either does all of its work or returns FLOWKV_ENOMEM and has changed nothing
// (built with AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_pages_oom_host.py,
// CPU only).
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <new>
#include <vector>

#include "flowkv.h"

namespace {
int64_t left = -1;                               // allocations until one fails; -1: none does
}
void* operator new(size_t n) {
  if (left == 0) throw std::bad_alloc();
  if (left > 0) --left;
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void* operator new(size_t n, const std::nothrow_t&) noexcept { return std::malloc(n ? n : 1); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

#define CHECK(cond)                                                            \
  do {                                                                         \
    if (!(cond)) {                                                             \
      std::printf("check failed at line %d: %s\n", __LINE__, #cond);           \
      std::exit(1);                                                            \
    }                                                                          \
  } while (0)

namespace {

constexpr int32_t kBlocks = 64;
int failed = 0;

flowkv_allocator* fragmented(int32_t policy) {
  flowkv_allocator* a = nullptr;
  CHECK(flowkv_allocator_create(kBlocks, policy, 5, &a) == FLOWKV_OK);
  std::vector<int32_t> ids(kBlocks), some;
  CHECK(flowkv_alloc(a, kBlocks, ids.data()) == FLOWKV_OK);
  for (int32_t b = 0; b < kBlocks; ++b)
    if (b % 3 == 1 || b / 8 == 3) some.push_back(b);
  CHECK(flowkv_free(a, some.data(), int32_t(some.size())) == FLOWKV_OK);
  return a;
}

// Owners, the summary of free space, and the blocks that allocations would get.
std::vector<int64_t> state(flowkv_allocator* a, bool drain) {
  std::vector<int64_t> s;
  for (int32_t b = 0; b < kBlocks; ++b) {
    int32_t n = -1;
    CHECK(flowkv_owners(a, &b, 1, &n) == FLOWKV_OK);
    s.push_back(n);
  }
  flowkv_alloc_stats st{};
  CHECK(flowkv_allocator_stats(a, &st) == FLOWKV_OK);
  s.insert(s.end(), {st.free_blocks, st.free_segments, st.largest_free});
  if (drain)
    for (int32_t b; flowkv_alloc(a, 1, &b) == FLOWKV_OK;) s.push_back(b);
  return s;
}

// `call` fails at each of its allocations in turn, and then succeeds.
void each(int32_t policy, const std::function<void(flowkv_allocator*)>& before,
          const std::function<int(flowkv_allocator*, std::vector<int32_t>&)>& call) {
  for (int64_t k = 0;; ++k) {
    CHECK(k < 1000);
    flowkv_allocator *a = fragmented(policy), *untouched = fragmented(policy);
    before(a);
    before(untouched);
    std::vector<int32_t> out(3 * kBlocks, -7);
    left = k;
    const int rc = call(a, out);
    left = -1;
    CHECK(rc == FLOWKV_OK || rc == FLOWKV_ENOMEM);
    if (rc != FLOWKV_OK) {
      ++failed;
      for (int32_t x : out) CHECK(x == -7);
      CHECK(state(a, true) == state(untouched, true));
    }
    flowkv_allocator_destroy(a);
    flowkv_allocator_destroy(untouched);
    if (rc == FLOWKV_OK) return;
  }
}

}  // namespace

int main() {
  const int32_t held[] = {0, 2, 3, 5};
  auto nothing = [](flowkv_allocator*) {};
  auto shared = [&](flowkv_allocator* a) { CHECK(flowkv_share(a, held, 2) == FLOWKV_OK); };
  for (int32_t policy :
       {FLOWKV_POLICY_SEGMENT, FLOWKV_POLICY_FIFO_SORTED, FLOWKV_POLICY_FIFO_SHUFFLED})
    for (int with = 0; with < 2; ++with) {
      std::function<void(flowkv_allocator*)> before = nothing;
      if (with) before = shared;
      each(policy, before, [&](flowkv_allocator* a, std::vector<int32_t>&) {
        return flowkv_share(a, held, 4);
      });
      each(policy, before, [&](flowkv_allocator* a, std::vector<int32_t>& out) {
        return flowkv_fork(a, held, 4, 14, 4, out.data(), &out[kBlocks]);
      });
      each(policy, before, [&](flowkv_allocator* a, std::vector<int32_t>& out) {
        return flowkv_alloc(a, 9, out.data());
      });
      each(policy, before, [&](flowkv_allocator* a, std::vector<int32_t>& out) {
        return flowkv_compact(a, kBlocks, out.data(), out.data() + kBlocks, &out[2 * kBlocks]);
      });
    }
  std::printf("%d failures ok\n", failed);
}
