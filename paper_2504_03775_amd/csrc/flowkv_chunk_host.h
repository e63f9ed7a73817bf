// The host's part of attention of new tokens: the form, the split and the workspace of a
// call, the checks of its arguments, and its launches.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "flowkv.h"
#include "flowkv_chunk_kernels.h"
#include "flowkv_status.h"

namespace flowkv {
namespace chunk {

// The forms, by how many rows a request brings and how many workgroups there are.
struct Kind {
  int rows, threads, step;
  int per_cu[2];                                 // head_dim 64, 128, as below
  const void* fn[2];
  const void *cut[2], *join[2];                  // work by the lengths
};
template <class F64, class F128>
Kind kind_of(const void* fn64, const void* fn128, const void* cut64, const void* cut128,
             const void* join64, const void* join128) {
  static_assert(F64::kRows == F128::kRows && F64::kThreads == F128::kThreads &&
                F64::kStep == F128::kStep);
  return Kind{F64::kRows,
              F64::kThreads,
              F64::kStep,
              {F64::kPerCu, F128::kPerCu},
              {fn64, fn128},
              {cut64, cut128},
              {join64, join128}};
}
// The kernels of a call: 16 and 32 rows, 128 and 256 (128 x 128 and 256 x 64 a step).
struct Kernels {
  Kind kind[4];
  const void* merge[2][2];                       // head_dim; a wave or four a row
};
constexpr int kSplitUnit = 64;
// Whole tiles and a tail in pieces (cut_tiles): 32 steps at least, so that a round not begun is
// worth the search and the join; up to four rounds, and of the last one up to half in use, by the
// tiles to be expected (a request's last one half full); and tiles about as long as each other,
// 3 tokens cached for 5 new ones: the short ones under a prompt's diagonal fill the last round by
// themselves.  (us, whole tiles and with a tail, 32 heads of 128 on 8, new tokens behind cached
// ones.  Gains: 2,304 behind 4,000, 1.12 rounds, 272 and 224; 4,416, 2.16, 531 and 462; 8 of 320
// behind 2,200, 39 steps, 155 and 135; 24 of 125 behind 10,606, 1.5 rounds, 702 and 604.  Losses:
// 8 of 320 behind 700, 16 steps, 76 and 81; 4,096 behind 4,000, 2.0 rounds, 398 and 409; 8 of 960
// behind 1,700, 3.75, 316 and 336; through a window of 2,100 with nothing cached, 4,416, 155 and
// 165, 4 of 1,100, 71 and 87.)
constexpr int kTailRounds = 4;
constexpr int kTailSteps = 32;
constexpr int kFewSteps = 8;               // of 32 tokens, a CU

// x / d = (umulhi(x, m) + x) >> l with l = ceil(log2 d), m = floor(2^32 (2^l - d) / d) + 1.
inline void by_product(uint32_t d, uint32_t* magic, uint32_t* shift) {
  *shift = 0;
  while ((uint64_t(1) << *shift) < d) ++*shift;
  *magic = uint32_t((((uint64_t(1) << *shift) - d) << 32) / d + 1);
}

// From a table of the kernels: many<F>(cut), join<F>(), few<kDh, kC>(), merge<kDh, kWavesPer>().
template <class Table>
Kernels kernels_of() {
  typedef Form<64, 4, 2> A64;
  typedef Form<128, 4, 2> A128;
  typedef Form<64, 8, 1> B64;
  typedef Form<128, 8, 1> B128;
  return Kernels{
      {{16, kFewThreads, kFewTile, {},
        {Table::template few<64, 1>(), Table::template few<128, 1>()}, {}, {}},
       {32, kFewThreads, kFewTile, {},
        {Table::template few<64, 2>(), Table::template few<128, 2>()}, {}, {}},
       kind_of<A64, A128>(Table::template many<A64>(false), Table::template many<A128>(false),
                          Table::template many<A64>(true), Table::template many<A128>(true),
                          Table::template join<A64>(), nullptr),
       kind_of<B64, B128>(Table::template many<B64>(false), Table::template many<B128>(false),
                          Table::template many<B64>(true), Table::template many<B128>(true),
                          nullptr, Table::template join<B128>())},
      {{Table::template merge<64, 1>(), Table::template merge<64, 4>()},
       {Table::template merge<128, 1>(), Table::template merge<128, 4>()}}};
}

// Tile slots of a call, see first_tile.
inline int64_t tile_slots(int64_t n_tokens, int64_t n_req, int group, int rows) {
  return n_tokens * group / rows + n_req;
}

// Tiles of `rows` rows that the batch has at most.  (Where a request could have as many as there
// are slots, no product: it may pass 63 bits.)
inline int64_t tiles_of(int64_t n_tokens, int64_t n_req, int group, int64_t max_new, int rows) {
  const int64_t slots = tile_slots(n_tokens, n_req, group, rows);
  const int64_t each = (max_new * group + rows - 1) / rows;
  return n_req == 0 ? 0 : each >= slots ? slots : std::min(n_req * each, slots);
}

// The same without padding: of no more than max_new tokens a request.
inline int64_t used_slots(int64_t n_tokens, int64_t n_req, int group, int64_t max_new, int rows) {
  return tile_slots(std::min(n_tokens, n_req * max_new), n_req, group, rows);
}

// Whether the kernels that look at all lengths take a call: their tables' sizes, a tile's
// steps x kPieceTiles and all steps within 31 bits.
inline bool by_lengths(int64_t n_tokens, int64_t n_req, int group, int64_t max_new,
                       int64_t max_seq_len, const Kind& kind) {
  const int64_t slots = used_slots(n_tokens, n_req, group, max_new, kind.rows);
  const int64_t steps = (max_seq_len + kind.step - 1) / kind.step;
  return slots <= kPieceTiles && steps < 1 << 22 && slots * steps < 1 << 30;
}

struct Shape {
  int kind;
  int32_t split, splits, pieces;
  bool cut, order;                               // pieces by the lengths; tiles, the longest first
  bool tail;                                     // whole tiles, then pieces
  int64_t need;
};

// The most workspace that the library's rule asks for where requests bring more than 32
// rows: that of pieces, in which a batch's padding has no part.
constexpr int64_t kRuleBytes =
    int64_t(kCus) * 256 * (128 + 2) * sizeof(float) + (kPieceTiles + 1) * sizeof(float);

// The split that ends soonest by a simple count: the CUs' rounds over all tiles' splits, each
// as long as its tokens and `fixed` more (a workgroup's start and end), and the merge.  In
// few rows, 4 KiB of K and V a token: 5 new ones over 13,000, 8 KV heads, take 18.8 us in
// splits of 512 (208 workgroups), 21.6 of 256, 23.8 of 384 (272), 20.7 of 768; 8 requests of 4
// over up to 12,000 70.9 of 1,536 (512), 78.5 of 1,024, 86.0 of 2,048.
inline int32_t best_split(int64_t tiles, int64_t max_seq_len, int64_t fixed, int64_t most) {
  constexpr int64_t kUnit = 128, kMerge = 150;
  constexpr int kTried[] = {1,  2,  3,  4,  5,  6,  8,  10, 12,  16,
                            20, 24, 32, 40, 48, 64, 96, 128, 192, 256};
  int64_t best = kUnit;
  double least = INFINITY;
  for (const int n : kTried) {
    const int64_t even = ((max_seq_len + n - 1) / n + kUnit - 1) / kUnit * kUnit;
    const int64_t s = std::min(std::max(even, kUnit), most), k = (max_seq_len + s - 1) / s;
    const double rounds = std::ceil(double(tiles) * double(k) / kCus);   // (past 64 bits, maybe)
    const double time = rounds * double(s + fixed) + (k > 1 ? kMerge : 0);
    if (time < least) {
      least = time;
      best = s;
    }
    if (s == kUnit) break;
  }
  return int32_t(best);
}

// The most tokens that a tile goes through: all, or its rows' windows and the first ones.
struct Span {
  int32_t max_seq_len;
  int32_t window = 0, sinks = 0;                 // window 0: none
  int64_t of(int rows, int group) const {
    if (window == 0) return max_seq_len;
    // (rows of at most so many tokens, one after another)
    const int64_t tokens = (int64_t(rows) + group - 2) / group + 1;
    return std::min<int64_t>(max_seq_len, int64_t(sinks) + window + tokens - 1);
  }
};

// The form and the split of a call, and the workspace that it takes.
inline int plan_shape(const Kernels& kernels, int32_t n_tokens, int32_t n_req, int32_t q_heads,
                      int32_t kv_heads, int32_t head_dim, int32_t max_new, const Span& span,
                      int32_t split_tokens, bool tail, Shape* out) {
  const Kind* kKinds = kernels.kind;
  if (n_tokens < 0 || n_req < 0 || max_new < 0 || span.max_seq_len < 0)
    return fail(FLOWKV_EINVAL, "negative sizes");
  if (head_dim != 64 && head_dim != 128)
    return fail(FLOWKV_EINVAL, "head_dim %d: need 64 or 128", head_dim);
  if (kv_heads < 1 || q_heads < 1 || q_heads % kv_heads)
    return fail(FLOWKV_EINVAL, "q_heads %d not a multiple of kv_heads %d", q_heads, kv_heads);
  if (split_tokens < 0 || split_tokens % kSplitUnit)
    return fail(FLOWKV_EINVAL, "split_tokens %d: need 0 or a multiple of %d", split_tokens,
                kSplitUnit);
  const int group = q_heads / kv_heads;
  if (int64_t(n_tokens) * group > INT32_MAX - 512)
    return fail(FLOWKV_EINVAL, "%d tokens x %d query heads a KV head: need under 2^31 - 512",
                n_tokens, group);
  // A step of 256 rows x 64 tokens moves half as much as one of 128 x 128, and the smaller
  // tiles share out better where there are few.
  const int64_t t256 = tiles_of(n_tokens, n_req, group, max_new, 256) * kv_heads;
  const int64_t t128 = tiles_of(n_tokens, n_req, group, max_new, 128) * kv_heads;
  // Up to 32 rows a request, or few steps in all: 32 rows a workgroup and its waves apart in
  // the keys end soonest.  (60 tokens behind 140, 4 heads of 64 on 2: 7.5 us, in 128 rows
  // 9.8; 30 behind 500, 32 of 128 on 8: 12.7 and 19.3; but 1,000 behind none, 8 on 1: 29.0
  // and 22.7.)
  const int64_t t32 = tiles_of(n_tokens, n_req, group, max_new, 32) * kv_heads;
  const bool rule = split_tokens == 0, many = int64_t(max_new) * group > 32;
  auto length = [&](int kind) { return span.of(kKinds[kind].rows, group); };
  // records of even splits, past 63 bits: the most that 63 bits hold
  auto splits_of = [&](int kind, int32_t split) {
    return std::max<int64_t>((length(kind) + split - 1) / split, 1);
  };
  auto bytes_of = [&](int kind, int32_t split) {
    int64_t bytes = 0;
    if (splits_of(kind, split) > 1 &&            // (fewer than 2^62 rows)
        (__builtin_mul_overflow(int64_t(n_tokens) * q_heads,
                                int64_t((head_dim + 2) * sizeof(float)), &bytes) ||
         __builtin_mul_overflow(bytes, splits_of(kind, split), &bytes)))
      return INT64_MAX;
    return bytes;
  };
  auto by_pieces = [&](int kind, bool behind_whole) {
    out->kind = kind;
    out->cut = !behind_whole;
    out->tail = behind_whole;
    out->split = 0;
    out->splits = 1;
    out->pieces = kKinds[kind].per_cu[head_dim == 128] * kCus;
    out->need = (int64_t(out->pieces) * kKinds[kind].rows * (head_dim + 2) +
                 std::min<int64_t>(tile_slots(n_tokens, n_req, group, kKinds[kind].rows),
                                   kPieceTiles) + 1) * int64_t(sizeof(float));
    return FLOWKV_OK;
  };
  auto takes_lengths = [&](int kind) {
    return by_lengths(n_tokens, n_req, group, max_new, length(kind), kKinds[kind]);
  };
  constexpr int32_t kAll = INT32_MAX / kSplitUnit * kSplitUnit;
  const int cut_kind = head_dim == 128 ? 3 : 2;  // the form that has pieces
  out->cut = out->order = out->tail = false;
  if (split_tokens <= kFewSplit && !many) {
    out->kind = int64_t(max_new) * group > 16;
  } else if (rule && t32 <= kCus && t32 * ((length(1) + 31) / 32) <= kFewSteps * kCus &&
             bytes_of(1, best_split(std::max<int64_t>(t32, 1), length(1), 300, kFewSplit)) <=
                 kRuleBytes) {
    out->kind = 1;
  } else if (t256 >= kCus) {
    out->kind = 3;
  } else {
    const int64_t tiles = cut_kind == 3 ? t256 : t128, step = kKinds[cut_kind].step;
    if (rule && tiles < kCus && takes_lengths(cut_kind) &&
        tiles * ((length(cut_kind) + step - 1) / step) >= kCutSteps * kCus)
      return by_pieces(cut_kind, false);
    out->kind = 2;
  }
  const Kind& kind = kKinds[out->kind];
  // (the workspace of a tail is asked for wherever there might be one)
  int64_t asked = 0;
  if (tail && rule && out->kind == cut_kind && head_dim == 128 && takes_lengths(cut_kind)) {
    const int64_t round = int64_t(kind.per_cu[1]) * kCus;
    if (t256 > round && t256 <= kTailRounds * round &&
        length(cut_kind) >= int64_t(kTailSteps) * kind.step) {
      by_pieces(cut_kind, true);
      const int64_t rows = std::min(int64_t(n_tokens), int64_t(n_req) * max_new) * group;
      const int64_t half_full = (rows + (int64_t(n_req) + 2) * kind.rows / 2 - 1) / kind.rows;
      const int64_t last = std::min(t256, half_full * kv_heads) % round;
      const int64_t cached = span.max_seq_len - std::min(max_new, span.max_seq_len);
      if (last > 0 && 2 * last <= round && 5 * cached >= 3 * int64_t(max_new)) return FLOWKV_OK;
      out->tail = false;
      asked = out->need;
    }
  }
  if (rule && out->kind >= 2 && n_req > 1 && span.max_seq_len / 2 >= max_new &&
      (out->kind == 3 ? t256 : t128) > kCus && takes_lengths(out->kind)) {
    out->order = true;
    out->split = 0;
    out->splits = 1;
    out->pieces = 0;
    out->need = asked;
    return FLOWKV_OK;
  }
  if (rule) {
    const int64_t tiles =
        std::max<int64_t>(tiles_of(n_tokens, n_req, group, max_new, kind.rows) * kv_heads, 1);
    if (out->kind <= 1) split_tokens = best_split(tiles, length(out->kind), 300, kFewSplit);
    else split_tokens = tiles < kCus ? best_split(tiles, length(out->kind), 500, kAll) : kAll;
    // padding and few steps, as a rule: pieces, or the splits that the workspace has room for
    if (many && bytes_of(out->kind, split_tokens) > kRuleBytes) {
      if (takes_lengths(cut_kind)) return by_pieces(cut_kind, false);
      while (split_tokens < kAll && bytes_of(out->kind, split_tokens) > kRuleBytes)
        split_tokens = split_tokens < kAll / 2 ? 2 * split_tokens : kAll;
    }
  }
  out->split = split_tokens;
  const int64_t splits = splits_of(out->kind, split_tokens);
  out->need = std::max(bytes_of(out->kind, split_tokens), asked);
  out->splits = int32_t(splits);
  out->pieces = 0;
  if (out->need == INT64_MAX)
    return fail(FLOWKV_EINVAL, "%d splits: the workspace's size overflows", out->splits);
  return FLOWKV_OK;
}

// A call's arguments, as every entry point has them.
struct Call {
  const flowkv_pool* pool;
  int32_t layer;
  const void* q;
  int64_t q_stride;
  int32_t n_tokens, n_req, q_heads, kv_heads, head_dim;
  const int32_t *offsets, *tables;
  int32_t max_blocks;
  const int32_t* seq_lens;
  int32_t max_seq_len;
  float scale;
  void* out;
  void* workspace;
  int64_t workspace_bytes;
  hipStream_t stream;

  bool layer_major() const { return pool->layout == FLOWKV_LAYOUT_LAYER_MAJOR; }
  int64_t per_token() const { return int64_t(kv_heads) * head_dim * 2; }
  int64_t block_stride() const {
    return layer_major() ? pool->chunk_bytes : 2 * int64_t(pool->num_layers) * pool->chunk_bytes;
  }
  bool empty() const { return n_req == 0 || n_tokens == 0; }
};

inline int check_16_bits(int32_t dtype) {
  if (dtype != FLOWKV_BF16 && dtype != FLOWKV_FP16)
    return fail(FLOWKV_EINVAL, "element type %d: attention reads FLOWKV_BF16 or FLOWKV_FP16",
                dtype);
  return FLOWKV_OK;
}

inline int check_pool(const Call& c) {
  if (!c.pool) return fail(FLOWKV_EINVAL, "NULL pool");
  const flowkv_pool* pool = c.pool;
  if (pool->layout != FLOWKV_LAYOUT_LAYER_MAJOR && pool->layout != FLOWKV_LAYOUT_BLOCK_MAJOR)
    return fail(FLOWKV_EINVAL, "unknown layout %d", pool->layout);
  if (pool->num_layers < 1 || pool->num_layers > FLOWKV_MAX_LAYERS || pool->num_blocks < 1 ||
      !pool->layer_base)
    return fail(FLOWKV_EINVAL, "bad pool descriptor");
  if (c.layer < 0 || c.layer >= pool->num_layers)
    return fail(FLOWKV_EINVAL, "layer %d outside the pool's %d layers", c.layer,
                pool->num_layers);
  return FLOWKV_OK;
}

// What a call's shape (heads and sizes are checked by then) has to keep to.
inline int check_sizes(const Call& c) {
  const flowkv_pool* pool = c.pool;
  const int64_t per_token = c.per_token();
  if (pool->chunk_bytes <= 0 || pool->chunk_bytes % per_token)
    return fail(FLOWKV_EINVAL, "chunk_bytes %lld is not block_size x %d KV heads x %d of 2 bytes",
                (long long)pool->chunk_bytes, c.kv_heads, c.head_dim);
  const int64_t bs = pool->chunk_bytes / per_token, stride = c.block_stride();
  // one block stride under 4 GiB, as for decode attention; the kernel forms offsets in
  // 128-byte units (a head's row is one or two) of 32 bits
  if (stride >= (int64_t(1) << 32))
    return fail(FLOWKV_EINVAL, "block stride of %lld bytes: need under 4 GiB", (long long)stride);
  if (pool->num_blocks >= (int64_t(1) << 39) / stride)
    return fail(FLOWKV_EINVAL, "%d blocks %lld bytes apart: need under 512 GiB", pool->num_blocks,
                (long long)stride);
  if (c.max_blocks < 0 || int64_t(c.max_blocks) * bs > INT32_MAX)
    return fail(FLOWKV_EINVAL, "max_blocks %d x block_size %lld tokens: need 0 to 2^31 - 1",
                c.max_blocks, (long long)bs);
  // positions are formed in 32 bits past the last tile's end
  if (c.max_seq_len > INT32_MAX - 4096)
    return fail(FLOWKV_EINVAL, "max_seq_len %d: need at most 2^31 - 4097", c.max_seq_len);
  // (the kernels take it in powers of 2)
  if (!(c.scale > 0.f) || !std::isfinite(c.scale * kLog2e))
    return fail(FLOWKV_EINVAL, "bad scale");
  return FLOWKV_OK;
}

// The buffers of a call that has something to do.
inline int check_buffers(const Call& c, int64_t need) {
  if (!c.q || !c.offsets || !c.seq_lens || !c.out || (c.max_blocks > 0 && !c.tables))
    return fail(FLOWKV_EINVAL, "NULL device pointer");
  if (reinterpret_cast<uintptr_t>(c.q) % 16 || c.q_stride % 8)
    return fail(FLOWKV_EINVAL, "queries need 16-byte alignment and a stride of whole 16 bytes");
  if (c.n_tokens > 1 && c.q_stride < int64_t(c.q_heads) * c.head_dim)
    return fail(FLOWKV_EINVAL, "query stride of %lld elements, a token has %lld",
                (long long)c.q_stride, (long long)c.q_heads * c.head_dim);
  if (reinterpret_cast<uintptr_t>(c.out) % 8)
    return fail(FLOWKV_EINVAL, "output not 8-byte aligned");
  if (need > 0 && !c.workspace) return fail(FLOWKV_EINVAL, "NULL workspace");
  if (c.workspace_bytes < need)
    return fail(FLOWKV_ECAP, "workspace of %lld bytes, %lld needed",
                (long long)c.workspace_bytes, (long long)need);
  if (need > 0 && reinterpret_cast<uintptr_t>(c.workspace) % 4)
    return fail(FLOWKV_EINVAL, "workspace not 4-byte aligned");
  const int base = c.layer_major() ? c.layer : 0;
  if (!c.pool->layer_base[base] || reinterpret_cast<uintptr_t>(c.pool->layer_base[base]) % 16)
    return fail(FLOWKV_EINVAL, "pool base pointer %d NULL or not 16-byte aligned", base);
  return FLOWKV_OK;
}

// The kernels' arguments but for the form's.
inline void fill(const Call& c, ChunkArgs* a) {
  const flowkv_pool* pool = c.pool;
  const bool lm = c.layer_major();
  const int64_t bs = pool->chunk_bytes / c.per_token();
  a->kbase = static_cast<const char*>(pool->layer_base[lm ? c.layer : 0]) +
             (lm ? 0 : int64_t(c.layer) * 2 * pool->chunk_bytes);
  a->voff = lm ? int64_t(pool->num_blocks) * pool->chunk_bytes : pool->chunk_bytes;
  a->q = static_cast<const uint16_t*>(c.q);
  a->q_stride = c.q_stride;
  a->offsets = c.offsets;
  a->seq_lens = c.seq_lens;
  a->tables = c.tables;
  a->out = static_cast<uint16_t*>(c.out);
  a->ws = static_cast<float*>(c.workspace);
  a->bunits = uint32_t(c.block_stride() / 128);
  a->sunits = uint32_t(c.per_token() / 128);
  by_product(uint32_t(bs), &a->bs_magic, &a->bs_shift);
  by_product(uint32_t(c.q_heads / c.kv_heads), &a->g_magic, &a->g_shift);
  a->pool_blocks = pool->num_blocks;
  a->block_size = int32_t(bs);
  a->max_blocks = c.max_blocks;
  a->max_seq_len = c.max_seq_len;
  a->n_tokens = c.n_tokens;
  a->n_req = c.n_req;
  a->q_heads = c.q_heads;
  a->kv_heads = c.kv_heads;
  a->group = c.q_heads / c.kv_heads;
  a->scale_log2 = c.scale * kLog2e;
}

// Tile slots of a call's launch, workgroups of its merge (`one`: a wave per (new token, query
// head), where its lane groups hold all records at once), and whether their lanes are within 32
// bits.
struct Grid {
  int64_t tiles, merge;
  bool one, fits;
};
inline Grid grid_of(const Kernels& kernels, const Shape& sh, int64_t n_tokens, int64_t n_req,
                    int32_t q_heads, int32_t kv_heads, int head_dim) {
  const Kind& kind = kernels.kind[sh.kind];
  Grid g;
  g.tiles = tile_slots(n_tokens, n_req, q_heads / kv_heads, kind.rows);
  g.one = sh.splits <= kMergeChunk * 64 * 4 / head_dim;
  g.merge = g.one ? (n_tokens * q_heads + 3) / 4 : n_tokens * q_heads;
  g.fits = g.tiles * kv_heads <= UINT32_MAX / kind.threads / sh.splits &&
           (sh.splits <= 1 || g.merge <= UINT32_MAX / kMergeThreads);
  return g;
}

// Launches a call's kernels: its form's, and what joins its pieces or splits.  `args` begins
// with a ChunkArgs that fill() has been through.
template <class Args>
int launch(const Kernels& kernels, const Shape& sh, int32_t max_new, int head_dim, Args& a,
           hipStream_t stream) {
  const Kind& kind = kernels.kind[sh.kind];
  a.split_tokens = sh.split;
  a.splits = sh.splits;
  a.row_shift = 0;
  while (1 << a.row_shift < kind.rows) ++a.row_shift;
  const Grid size = grid_of(kernels, sh, a.n_tokens, a.n_req, a.q_heads, a.kv_heads, head_dim);
  const int64_t tiles = size.tiles, grid = tiles * a.kv_heads, merge = size.merge;
  if (!size.fits)
    return fail(FLOWKV_EINVAL, "%lld tiles of queries x %d splits: too many for one call",
                (long long)grid, sh.splits);
  a.tiles = int32_t(tiles);
  if (sh.cut || sh.order || sh.tail)
    a.tiles = int32_t(used_slots(a.n_tokens, a.n_req, a.group, max_new, kind.rows));
  a.pieces = sh.pieces;
  if constexpr (std::is_same_v<Args, SpanArgs>) a.tail = sh.tail;
  void* args[] = {&a};
  const int d128 = head_dim == 128;
  const int64_t groups =
      sh.tail  ? std::max(grid, int64_t(a.tiles) * a.kv_heads + sh.pieces)
      : sh.cut ? std::max<int64_t>(grid, sh.pieces)
               : grid * sh.splits;
  hipError_t e = hipLaunchKernel(sh.cut || sh.order || sh.tail ? kind.cut[d128] : kind.fn[d128],
                                 dim3(unsigned(groups)), dim3(unsigned(kind.threads)), args, 0,
                                 stream);
  if (e == hipSuccess && (sh.cut || sh.tail))
    e = hipLaunchKernel(kind.join[d128], dim3(unsigned(a.tiles * a.kv_heads * (kind.rows / 32))),
                        dim3(unsigned(2 * head_dim)), args, 0, stream);
  if (e == hipSuccess && sh.splits > 1)
    e = hipLaunchKernel(kernels.merge[d128][!size.one], dim3(unsigned(merge)), dim3(kMergeThreads),
                        args, 0, stream);
  if (e == hipSuccess) e = hipGetLastError();
  if (e != hipSuccess) return fail(FLOWKV_EHIP, "attention launch: %s", hipGetErrorString(e));
  return ok();
}

}  // namespace chunk
}  // namespace flowkv
