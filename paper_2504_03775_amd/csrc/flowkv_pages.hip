// Writing into the pages of a pool, for gfx950 (MI355X): new tokens' K and V
// appended to their requests' blocks, and blocks copied within one pool.
//
// Both move bytes and interpret none.  The pool is either layout of FlowKV's
// Eq. 5 (arXiv 2504.03775, section 3.3).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <vector>

#include "flowkv.h"
#include "flowkv_device.h"
#include "flowkv_ragged.h"
#include "flowkv_status.h"

using flowkv::fail;
using flowkv::ok;

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) u32x4 gvec;
typedef __attribute__((address_space(1))) const u32x4 cgvec;

// ---- append --------------------------------------------------------------------

struct AppendArgs {
  char* kbase;              // the layer's K of block 0
  int64_t voff;             // V from K
  int64_t bstride;          // bytes between blocks
  const char* k;
  const char* v;
  int64_t k_stride, v_stride;   // bytes between tokens
  const int32_t* offsets;
  const int32_t* seq_lens;
  const int32_t* tables;
  int32_t n_tokens, n_req, max_blocks, pool_blocks, block_size;
  int32_t pieces;           // 16-byte pieces of a slot
};

// Token i of request r goes to position p = seq_lens[r] - new[r] + (i - offsets[r]),
// new[r] = offsets[r + 1] - offsets[r]: slot p % bs of block tables[r][p / bs].
// A token outside every request or with a negative position, past its block list
// or with a block outside the pool is dropped.
//
// Work: the 16-byte pieces of all tokens' K and V, in order; a wave takes 64
// consecutive ones, or twice 64 in a long call.  What bounds it: up to a few hundred
// tokens a launch and its dependent loads (the offsets, the length, the table
// entry), with the data's own loads under way meanwhile: 32 tokens of 8 KV heads of
// 128 take 2.9 us in a graph (3.2 with two pieces a lane, 4.1 with four).  A long
// call is bound by memory: 18,750 tokens of one KV head (19.2 MB read and written)
// 6.3 us, 6.9 with one piece a lane; the two are level at 2^18 pieces.
constexpr int kAppendThreads = 256;
constexpr int64_t kAppendFew = 1 << 18;              // pieces up to which a lane takes one

template <int kAppendUnroll>
__global__ __launch_bounds__(kAppendThreads) void kv_append(const AppendArgs a) {
  const int ln = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t first =
      (int64_t(blockIdx.x) * (kAppendThreads / 64) + wave) * (64 * kAppendUnroll);
  const uint32_t per = 2 * uint32_t(a.pieces);       // pieces of a token
  const int64_t items = int64_t(a.n_tokens) * per;
  if (first >= items) return;
  const int64_t last = std::min<int64_t>(first + 64 * kAppendUnroll, items) - 1;
  const int32_t t0 = int32_t(first / per), t1 = int32_t(last / per);
  const uint32_t rem0 = uint32_t(first - int64_t(t0) * per);

  u32x4 x[kAppendUnroll];
  int32_t token[kAppendUnroll];
  uint32_t piece[kAppendUnroll];                     // of K, then of V
#pragma unroll
  for (int u = 0; u < kAppendUnroll; ++u) {
    const int64_t i = first + u * 64 + ln;
    const uint32_t d = rem0 + u * 64 + ln;
    token[u] = i < items ? t0 + int32_t(d / per) : t1;
    piece[u] = i < items ? d % per : 0;
    const bool v = piece[u] >= uint32_t(a.pieces);
    const char* src = v ? a.v + token[u] * a.v_stride + int64_t(piece[u] - a.pieces) * 16
                        : a.k + token[u] * a.k_stride + int64_t(piece[u]) * 16;
    x[u] = *(cgvec*)src;
  }
  const int32_t r0 = flowkv::last_at_most(a.n_req, t0, [&](int32_t r) { return a.offsets[r]; });
  const int32_t r1 =
      t1 == t0 ? r0
               : flowkv::last_at_most(a.n_req, t1, [&](int32_t r) { return a.offsets[r]; });
  // no branch but the search's, so that the pieces' loads are under way together
  uint32_t slot[kAppendUnroll];
  int32_t id[kAppendUnroll];
  bool in[kAppendUnroll];
#pragma unroll
  for (int u = 0; u < kAppendUnroll; ++u) {
    int32_t r = r0;
    if (r1 != r0) {                                  // uniform
      int32_t hi = r1 + 1;                           // the last in [r0, r1] at most token
      while (hi - r > 1) {
        const int32_t mid = r + (hi - r) / 2;
        if (a.offsets[mid] <= token[u]) r = mid;
        else hi = mid;
      }
    }
    const int32_t begin = a.offsets[r], end = a.offsets[r + 1];
    const int64_t p = int64_t(a.seq_lens[r]) - (int64_t(end) - begin) + (token[u] - begin);
    const uint32_t b = uint32_t(p) / uint32_t(a.block_size);   // p < 2^31: below a length
    in[u] = first + u * 64 + ln < items && token[u] >= begin && token[u] < end && p >= 0 &&
            b < uint32_t(a.max_blocks);
    id[u] = a.tables[in[u] ? int64_t(r) * a.max_blocks + b : 0];
    slot[u] = uint32_t(p) - b * uint32_t(a.block_size);
  }
#pragma unroll
  for (int u = 0; u < kAppendUnroll; ++u) {
    if (!in[u] || id[u] < 0 || id[u] >= a.pool_blocks) continue;
    const bool v = piece[u] >= uint32_t(a.pieces);
    char* dst = a.kbase + (v ? a.voff : 0) + id[u] * a.bstride +
                (int64_t(slot[u]) * a.pieces + (v ? piece[u] - a.pieces : piece[u])) * 16;
    *(gvec*)dst = x[u];
  }
}

// ---- copies within a pool --------------------------------------------------------

struct PairOf {
  int32_t src, dst;
};
struct PairTokens {
  int32_t src, dst, tokens;
};

__device__ inline int32_t tokens_of(const PairOf&) { return 0; }
__device__ inline int32_t tokens_of(const PairTokens& r) { return r.tokens; }

template <class Rec, int kBases, int kRecs>
struct CopyArgs {
  typedef Rec Record;
  static constexpr int kMaxBases = kBases;
  static constexpr int kMaxRecs = kRecs;
  int64_t chunk_bytes, block_bytes;   // H, 2 L H
  int64_t num_blocks;
  int32_t n;                          // records
  int32_t num_layers;
  int32_t slot_pieces;                // 16-byte pieces of a slot (token counts only)
  int32_t chunk_pieces;               // the most that a record moves of a chunk
  int32_t tiles;                      // of a record, or of a plane
  int64_t perm_mul;
  char* base[kBases];
  Rec rec[kRecs];
};
// The records travel in the kernel arguments, as many as a 4 KiB segment holds
// beside the base pointers; a longer list takes several launches.
using CopyBM = CopyArgs<PairOf, 1, 460>;
using CopyLM = CopyArgs<PairOf, FLOWKV_MAX_LAYERS, 330>;
using CopyTokensBM = CopyArgs<PairTokens, 1, 300>;
using CopyTokensLM = CopyArgs<PairTokens, FLOWKV_MAX_LAYERS, 220>;
constexpr size_t kImplicitArgBytes = 256;
static_assert(sizeof(CopyBM) + kImplicitArgBytes <= 4096, "kernel arguments");
static_assert(sizeof(CopyLM) + kImplicitArgBytes <= 4096, "kernel arguments");
static_assert(sizeof(CopyTokensBM) + kImplicitArgBytes <= 4096, "kernel arguments");
static_assert(sizeof(CopyTokensLM) + kImplicitArgBytes <= 4096, "kernel arguments");

// The two kernels below move the same bytes: of each record the first `tokens`
// slots (all of them without token counts) of its 2 L chunks, in 16-byte pieces.
// Both are bound by memory.  A call that reads and writes up to 256 MiB takes the
// first, a larger one the second: of 2 MiB blocks (32 layers of 8 x 128, block-major)
// 60 take 38.0 us in the first and 40.0 in the second, 90 take 67.2 and 59.4, 1,000
// take 775 and 645 (6.5 TB/s); 24 partly filled ones 10.0 and 12.0 (calls one after another;
// the first kernel alone 7.1).
//
// The first: what it reads was written a moment ago as a rule (the block that a
// prompt ends in) and is looked for in the caches.  A record's pieces are one span,
// two pieces a lane, 512 lanes, a record's tiles together, records scattered
// (x -> x m mod n).
constexpr int kCopyThreads = 512;
constexpr int kCopyUnroll = 2;

template <class A, bool kLM>
__global__ __launch_bounds__(kCopyThreads) void kv_block_copy(const A a) {
  constexpr bool kTokens = sizeof(typename A::Record) == sizeof(PairTokens);
  __shared__ char* s_base[kLM ? FLOWKV_MAX_LAYERS : 1];
  const uint32_t t = blockIdx.x % uint32_t(a.tiles);
  const uint32_t i =
      uint32_t(uint64_t(blockIdx.x / uint32_t(a.tiles)) * uint64_t(a.perm_mul) % uint32_t(a.n));
  const int64_t src = a.rec[i].src, dst = a.rec[i].dst;
  uint32_t chunk = uint32_t(a.chunk_bytes / 16);     // pieces moved of a chunk
  if constexpr (kTokens) chunk = uint32_t(a.rec[i].tokens) * uint32_t(a.slot_pieces);
  const uint32_t span = chunk * 2u * uint32_t(a.num_layers);
  const uint32_t o0 = t * uint32_t(kCopyThreads * kCopyUnroll);
  if (o0 >= span) return;
  if constexpr (kLM) {
    for (uint32_t l = threadIdx.x; l < uint32_t(a.num_layers); l += kCopyThreads)
      s_base[l] = a.base[l];
    __syncthreads();
  }
  auto at = [&](int64_t block, uint32_t o) -> char* {
    if constexpr (!kLM && !kTokens) {
      return a.base[0] + block * a.block_bytes + int64_t(o) * 16;
    } else {
      const uint32_t c = o / chunk, w = o - c * chunk;
      if constexpr (kLM)
        return s_base[c >> 1] + (int64_t(c & 1) * a.num_blocks + block) * a.chunk_bytes +
               int64_t(w) * 16;
      else
        return a.base[0] + block * a.block_bytes + int64_t(c) * a.chunk_bytes + int64_t(w) * 16;
    }
  };
  u32x4 x[kCopyUnroll];
#pragma unroll
  for (int k = 0; k < kCopyUnroll; ++k) {
    const uint32_t o = o0 + k * kCopyThreads + threadIdx.x;
    if (o < span) x[k] = *(cgvec*)at(src, o);
  }
#pragma unroll
  for (int k = 0; k < kCopyUnroll; ++k) {
    const uint32_t o = o0 + k * kCopyThreads + threadIdx.x;
    if (o < span) __builtin_nontemporal_store(x[k], (gvec*)at(dst, o));
  }
}

// The second: one wave and one piece a lane to a workgroup, past the caches, so that
// the memory's channels are shared out in steps of 1 KiB.  (64 lanes x 1 piece: 643
// us at the 1,000 blocks above; 64 x 2: 711, 256 x 1: 713, 1,024 x 4: 716.)  A
// block-major record's tiles follow each other; a layer-major launch goes plane by
// plane (a layer's K, or its V), each plane's pieces of all records in order: 1,500
// blocks of 80 layers of 4 KiB chunks take 337 us (5.8 TB/s), block by block 384.
constexpr int kStreamThreads = 64;

template <class A, bool kLM>
__global__ __launch_bounds__(kStreamThreads) void kv_block_stream(const A a) {
  constexpr bool kTokens = sizeof(typename A::Record) == sizeof(PairTokens);
  const uint32_t t = blockIdx.x % uint32_t(a.tiles), u = blockIdx.x / uint32_t(a.tiles);
  const uint32_t o = t * kStreamThreads + threadIdx.x;
  const char* src;
  char* dst;
  if constexpr (kLM) {
    const uint32_t chunk = uint32_t(a.chunk_pieces);
    const uint32_t i = o / chunk, w = o - i * chunk;
    if (i >= uint32_t(a.n)) return;
    if constexpr (kTokens)
      if (w >= uint32_t(a.rec[i].tokens) * uint32_t(a.slot_pieces)) return;
    char* plane = a.base[u >> 1] + int64_t(u & 1) * a.num_blocks * a.chunk_bytes + int64_t(w) * 16;
    src = plane + int64_t(a.rec[i].src) * a.chunk_bytes;
    dst = plane + int64_t(a.rec[i].dst) * a.chunk_bytes;
  } else {
    const uint32_t i = uint32_t(uint64_t(u) * uint64_t(a.perm_mul) % uint32_t(a.n));
    const uint32_t chunk =
        uint32_t(kTokens ? tokens_of(a.rec[i]) * a.slot_pieces : a.chunk_pieces);
    if (o >= chunk * 2u * uint32_t(a.num_layers)) return;
    int64_t off = int64_t(o) * 16;
    if constexpr (kTokens) off = int64_t(o / chunk) * a.chunk_bytes + int64_t(o % chunk) * 16;
    src = a.base[0] + a.rec[i].src * a.block_bytes + off;
    dst = a.base[0] + a.rec[i].dst * a.block_bytes + off;
  }
  __builtin_nontemporal_store(__builtin_nontemporal_load((cgvec*)src), (gvec*)dst);
}

// The pool's descriptor, as every call here checks it.
int check_pool(const flowkv_pool* p) {
  if (!p) return fail(FLOWKV_EINVAL, "NULL pool");
  if (p->layout != FLOWKV_LAYOUT_LAYER_MAJOR && p->layout != FLOWKV_LAYOUT_BLOCK_MAJOR)
    return fail(FLOWKV_EINVAL, "unknown layout %d", p->layout);
  if (p->num_layers < 1 || p->num_layers > FLOWKV_MAX_LAYERS)
    return fail(FLOWKV_EINVAL, "%d layers, need 1..%d", p->num_layers, FLOWKV_MAX_LAYERS);
  if (p->num_blocks < 1) return fail(FLOWKV_EINVAL, "%d blocks", p->num_blocks);
  if (p->reserved != 0) return fail(FLOWKV_EINVAL, "reserved field not 0");
  if (p->chunk_bytes <= 0 || p->chunk_bytes % 16)
    return fail(FLOWKV_EINVAL, "chunk_bytes %lld not a positive multiple of 16",
                (long long)p->chunk_bytes);
  if (p->chunk_bytes >= (int64_t(1) << 31) / (2 * int64_t(p->num_layers)))
    return fail(FLOWKV_EINVAL, "block of %d x 2 chunks of %lld bytes, limit 2 GiB", p->num_layers,
                (long long)p->chunk_bytes);
  if (!p->layer_base) return fail(FLOWKV_EINVAL, "NULL layer_base");
  const int nb = p->layout == FLOWKV_LAYOUT_LAYER_MAJOR ? p->num_layers : 1;
  for (int i = 0; i < nb; ++i)
    if (!p->layer_base[i] || reinterpret_cast<uintptr_t>(p->layer_base[i]) % 16)
      return fail(FLOWKV_EINVAL, "pool base pointer %d NULL or not 16-byte aligned", i);
  return FLOWKV_OK;
}

}  // namespace

extern "C" int flowkv_append(const flowkv_pool* pool, int32_t layer, const void* k_dev,
                             int64_t k_stride, const void* v_dev, int64_t v_stride,
                             int64_t slot_bytes, int32_t n_tokens, int32_t n_req,
                             const int32_t* offsets_dev, const int32_t* block_tables_dev,
                             int32_t max_blocks, const int32_t* seq_lens_dev, void* hip_stream) {
  int rc = check_pool(pool);
  if (rc) return rc;
  if (layer < 0 || layer >= pool->num_layers)
    return fail(FLOWKV_EINVAL, "layer %d outside the pool's %d layers", layer, pool->num_layers);
  if (slot_bytes <= 0 || slot_bytes % 16 || pool->chunk_bytes % slot_bytes)
    return fail(FLOWKV_EINVAL,
                "slot of %lld bytes: need a multiple of 16 that divides chunk_bytes %lld",
                (long long)slot_bytes, (long long)pool->chunk_bytes);
  if (n_tokens < 0 || n_req < 0 || max_blocks < 0) return fail(FLOWKV_EINVAL, "negative sizes");
  if (n_tokens == 0 || n_req == 0 || max_blocks == 0) return ok();
  if (!k_dev || !v_dev || !offsets_dev || !seq_lens_dev || !block_tables_dev)
    return fail(FLOWKV_EINVAL, "NULL device pointer");
  if (reinterpret_cast<uintptr_t>(k_dev) % 16 || reinterpret_cast<uintptr_t>(v_dev) % 16 ||
      k_stride % 16 || v_stride % 16)
    return fail(FLOWKV_EINVAL, "K and V need 16-byte alignment and strides of whole 16 bytes");
  if (n_tokens > 1 && (k_stride < slot_bytes || v_stride < slot_bytes))
    return fail(FLOWKV_EINVAL, "token strides of %lld and %lld bytes, a token has %lld",
                (long long)k_stride, (long long)v_stride, (long long)slot_bytes);
  const bool lm = pool->layout == FLOWKV_LAYOUT_LAYER_MAJOR;
  AppendArgs a{};
  a.kbase = static_cast<char*>(pool->layer_base[lm ? layer : 0]) +
            (lm ? 0 : int64_t(layer) * 2 * pool->chunk_bytes);
  a.voff = lm ? int64_t(pool->num_blocks) * pool->chunk_bytes : pool->chunk_bytes;
  a.bstride = lm ? pool->chunk_bytes : 2 * int64_t(pool->num_layers) * pool->chunk_bytes;
  a.k = static_cast<const char*>(k_dev);
  a.v = static_cast<const char*>(v_dev);
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.offsets = offsets_dev;
  a.seq_lens = seq_lens_dev;
  a.tables = block_tables_dev;
  a.n_tokens = n_tokens;
  a.n_req = n_req;
  a.max_blocks = max_blocks;
  a.pool_blocks = pool->num_blocks;
  a.block_size = int32_t(pool->chunk_bytes / slot_bytes);
  a.pieces = int32_t(slot_bytes / 16);
  const int64_t items = int64_t(n_tokens) * 2 * a.pieces;
  const bool few = items <= kAppendFew;
  const int64_t per_group = int64_t(kAppendThreads) * (few ? 1 : 2);
  const int64_t groups = (items + per_group - 1) / per_group;
  if (groups * kAppendThreads > UINT32_MAX)          // lanes of a launch
    return fail(FLOWKV_EINVAL, "%d tokens of %lld bytes: too many for one call", n_tokens,
                (long long)slot_bytes);
  void* args[] = {&a};
  hipError_t e = hipLaunchKernel(
      few ? reinterpret_cast<const void*>(kv_append<1>)
          : reinterpret_cast<const void*>(kv_append<2>),
      dim3(unsigned(groups)), dim3(kAppendThreads), args, 0, static_cast<hipStream_t>(hip_stream));
  if (e == hipSuccess) e = hipGetLastError();
  if (e != hipSuccess) return fail(FLOWKV_EHIP, "append launch: %s", hipGetErrorString(e));
  return ok();
}

namespace {

// The destinations of a call: a table of twice their number or more, looked through from an
// ID's place on.  (A mark for each of the pool's blocks would go by the pool: 30 us a call at
// 2^20 blocks, 2 GiB at 2^31.)
class Destinations {
 public:
  explicit Destinations(int32_t n) {
    while ((int64_t(1) << bits_) < 2 * int64_t(n)) ++bits_;
    ids_.assign(size_t(1) << bits_, -1);
  }
  // where the ID is, or would be
  int32_t& at(int32_t id) {
    const size_t mask = ids_.size() - 1;
    size_t x = size_t(uint32_t(id) * 2654435769u >> (32 - bits_));
    while (ids_[x] != id && ids_[x] != -1) x = (x + 1) & mask;
    return ids_[x];
  }

 private:
  int bits_ = 1;
  std::vector<int32_t> ids_;
};

// Every destination once, and no destination among the sources: the pairs can
// then be copied in any order, in any number of launches.
int check_pairs(const int32_t* src, const int32_t* dst, int32_t n, int32_t blocks) {
  Destinations is_dst(n);
  for (int32_t i = 0; i < n; ++i) {
    for (const int32_t* ids : {src, dst})
      if (ids[i] < 0 || ids[i] >= blocks)
        return fail(FLOWKV_ERANGE, "block %d at position %d outside [0, %d)", ids[i], i, blocks);
    int32_t& place = is_dst.at(dst[i]);
    if (place == dst[i])
      return fail(FLOWKV_EDUP, "block %d is a destination twice (position %d)", dst[i], i);
    place = dst[i];
  }
  for (int32_t i = 0; i < n; ++i)
    if (is_dst.at(src[i]) == src[i])
      return fail(FLOWKV_EDUP, "block %d at position %d is a source and a destination", src[i], i);
  return FLOWKV_OK;
}

// Bytes read and written by a call up to which the first kernel takes it.
constexpr int64_t kCopyCached = int64_t(256) << 20;

template <class A, bool kLM>
int launch_copy(const flowkv_pool* p, const int32_t* src, const int32_t* dst,
                const int32_t* tokens, int32_t n, int64_t slot_bytes, void* stream) {
  constexpr bool kTokens = sizeof(typename A::Record) == sizeof(PairTokens);
  const int64_t span = 2 * int64_t(p->num_layers) * p->chunk_bytes;
  A a{};
  a.chunk_bytes = p->chunk_bytes;
  a.block_bytes = span;
  a.num_blocks = p->num_blocks;
  a.num_layers = p->num_layers;
  a.slot_pieces = int32_t(slot_bytes / 16);
  for (int i = 0; i < (kLM ? p->num_layers : 1); ++i)
    a.base[i] = static_cast<char*>(p->layer_base[i]);
  const int64_t planes = 2 * int64_t(p->num_layers);
  int64_t all = n * span;
  if constexpr (kTokens) {
    all = 0;
    for (int32_t i = 0; i < n; ++i) all += planes * tokens[i] * slot_bytes;
  }
  const bool stream_past = 2 * all > kCopyCached;
  for (int32_t at = 0; at < n;) {
    // a launch has fewer than 2^32 lanes, a piece each
    const int32_t m =
        int32_t(std::min<int64_t>({int64_t(n) - at, A::kMaxRecs,
                                   std::max<int64_t>(1, (int64_t(1) << 31) / (span / 16))}));
    int64_t most = kTokens ? 0 : p->chunk_bytes;       // moved of a chunk
    for (int32_t i = 0; i < m; ++i) {
      a.rec[i].src = src[at + i];
      a.rec[i].dst = dst[at + i];
      if constexpr (kTokens) {
        a.rec[i].tokens = tokens[at + i];
        most = std::max(most, tokens[at + i] * slot_bytes);
      }
    }
    at += m;
    if (most == 0) continue;
    const bool by_plane = kLM && stream_past;
    const int64_t pieces = most / 16 * (by_plane ? m : planes);
    const int64_t line = stream_past ? kStreamThreads : kCopyThreads * kCopyUnroll;
    a.n = m;
    a.chunk_pieces = int32_t(most / 16);
    a.tiles = int32_t((pieces + line - 1) / line);
    a.perm_mul = int64_t(2654435761ull % uint64_t(m));   // a prime above m: a bijection mod m
    void* args[] = {&a};
    hipError_t e = hipLaunchKernel(
        stream_past ? reinterpret_cast<const void*>(kv_block_stream<A, kLM>)
                    : reinterpret_cast<const void*>(kv_block_copy<A, kLM>),
        dim3(unsigned(a.tiles) * unsigned(by_plane ? planes : m)),
        dim3(stream_past ? kStreamThreads : kCopyThreads), args, 0,
        static_cast<hipStream_t>(stream));
    if (e == hipSuccess) e = hipGetLastError();
    if (e != hipSuccess) return fail(FLOWKV_EHIP, "block copy launch: %s", hipGetErrorString(e));
  }
  return ok();
}

int copy_impl(const flowkv_pool* pool, const int32_t* src_ids, const int32_t* dst_ids,
              const int32_t* tokens, int32_t n_blocks, int64_t slot_bytes, void* stream) {
  int rc = check_pool(pool);
  if (rc) return rc;
  if (n_blocks < 0) return fail(FLOWKV_EINVAL, "negative block count %d", n_blocks);
  if (tokens) {
    if (slot_bytes <= 0 || slot_bytes % 16 || pool->chunk_bytes % slot_bytes)
      return fail(FLOWKV_EINVAL,
                  "slot of %lld bytes: need a multiple of 16 that divides chunk_bytes %lld",
                  (long long)slot_bytes, (long long)pool->chunk_bytes);
    const int64_t bs = pool->chunk_bytes / slot_bytes;
    for (int32_t i = 0; i < n_blocks; ++i)
      if (tokens[i] < 0 || tokens[i] > bs)
        return fail(FLOWKV_EINVAL, "%d tokens at position %d, a block holds %lld", tokens[i], i,
                    (long long)bs);
  }
  if (n_blocks == 0) return ok();
  if (!src_ids || !dst_ids) return fail(FLOWKV_EINVAL, "NULL block list");
  rc = check_pairs(src_ids, dst_ids, n_blocks, pool->num_blocks);
  if (rc) return rc;
  const bool lm = pool->layout == FLOWKV_LAYOUT_LAYER_MAJOR;
  if (tokens)
    return lm ? launch_copy<CopyTokensLM, true>(pool, src_ids, dst_ids, tokens, n_blocks,
                                                slot_bytes, stream)
              : launch_copy<CopyTokensBM, false>(pool, src_ids, dst_ids, tokens, n_blocks,
                                                 slot_bytes, stream);
  return lm ? launch_copy<CopyLM, true>(pool, src_ids, dst_ids, nullptr, n_blocks, 16, stream)
            : launch_copy<CopyBM, false>(pool, src_ids, dst_ids, nullptr, n_blocks, 16, stream);
}

}  // namespace

extern "C" int flowkv_copy_blocks(const flowkv_pool* pool, const int32_t* src_ids,
                                  const int32_t* dst_ids, const int32_t* tokens,
                                  int32_t n_blocks, int64_t slot_bytes, void* hip_stream) {
  return flowkv::guarded([&] {
    return copy_impl(pool, src_ids, dst_ids, tokens, n_blocks, slot_bytes, hip_stream);
  });
}
