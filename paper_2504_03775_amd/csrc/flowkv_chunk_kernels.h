// Attention of a ragged batch's new tokens over a paged pool, for gfx950 (MI355X): the
// forms of a workgroup and what joins their parts, for the calls that differ in which cached
// tokens a row sees (flowkv_chunk.hip, flowkv_window.hip, flowkv_prefix.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "flowkv_ragged.h"
#include "flowkv_splits.h"

namespace flowkv {
namespace chunk {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(1))) const u32x4 cgvec4;
typedef __attribute__((address_space(1))) const u32x2 cgvec2;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2u __attribute__((ext_vector_type(2), aligned(4)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds4;

typedef __attribute__((address_space(1))) const void gvoid;
typedef __attribute__((address_space(3))) void lvoid;
typedef __attribute__((address_space(3))) u32x4 lvec;
typedef __attribute__((address_space(3))) uint8_t lbyte;

// CUs that a call is spread over (MI355X's, also where no device is asked).
constexpr int kCus = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;               // log2 of the largest unnormalised weight

// The element types: products, the rounding of two float32 to one word, and what an exponent
// of all ones is.  kLift: the weights' power of two.  fp16 weights below 2^-14 are rounded by
// up to 2^-25 whatever their size; lifted by 2^7 (the largest, 2^(kLazy + 7), is within fp16)
// that is 2^-32 of a weight of 1, and a million such tokens are off by 2^-12 of it together.
struct Bf16 {
  typedef bf16x8 Vec;
  static constexpr float kLift = 0.f;
  static constexpr uint32_t kOdd = 0x7f80u;
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
  }
  // float32 bits of a word's element
  template <int kHi>
  static __device__ __forceinline__ uint32_t widen(uint32_t w) {
    return kHi ? w & 0xffff0000u : w << 16;
  }
  static __device__ __forceinline__ f32x16 mfma(Vec a, Vec b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma(Vec a, Vec b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
struct Fp16 {
  typedef f16x8 Vec;
  static constexpr float kLift = 7.f;
  static constexpr uint32_t kOdd = 0x7c00u;
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2));
  }
  template <int kHi>
  static __device__ __forceinline__ uint32_t widen(uint32_t w) {
    return __builtin_bit_cast(
        uint32_t, float(__builtin_bit_cast(_Float16, uint16_t(kHi ? w >> 16 : w))));
  }
  static __device__ __forceinline__ f32x16 mfma(Vec a, Vec b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma(Vec a, Vec b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

struct ChunkArgs {
  const char* kbase;                    // the layer's K of block 0
  int64_t voff;                         // V from K
  const uint16_t* q;                    // a token's Hq x Dh values every q_stride
  int64_t q_stride;                     // in elements
  const int32_t* offsets;               // (n_req + 1)
  const int32_t* seq_lens;              // (n_req)
  const int32_t* tables;                // (n_req, max_blocks)
  uint16_t* out;                        // (n_tokens, Hq, Dh), of q's type
  float* ws;                            // the splits' records
  uint32_t bunits, sunits;              // 128-byte units between blocks, slots
  uint32_t bs_magic, bs_shift;          // division by block_size,
  uint32_t g_magic, g_shift;            // and by the group
  int32_t pool_blocks, block_size, max_blocks, max_seq_len;
  int32_t n_tokens, n_req, q_heads, kv_heads, group;
  int32_t row_shift;                    // query rows of a workgroup's tile: 2^row_shift
  int32_t tiles, split_tokens, splits;
  int32_t pieces;                       // work by the lengths: at most; 0: whole tiles
  float scale_log2;                     // scale * log2(e)
};

// What the calls through a window and over shared prefixes bring beside it.
struct SpanArgs : ChunkArgs {
  int32_t window, sinks;                // tokens seen up to a row's own; first ones always seen
  const int32_t* groups;                // (n_groups + 1) requests of shared prefixes
  const int32_t* prefix_lens;           // (n_groups)
  int32_t n_groups, max_prefix;
  int32_t tail;                         // the tiles behind the last whole round in pieces
  int32_t max_own;                      // tokens of a request behind its prefix
  int32_t first_split;                  // records of a row: [0, first_split) of its prefix,
  int32_t prefix_split;                 // this many tokens each, the others its own
  uint32_t prefix_items;                // Shared: workgroups of prefixes, of a KV head
};

// The kernel's arguments, loaded here and not before.
template <class A>
__device__ __forceinline__ A late_args() {
  auto p = (const __attribute__((address_space(4))) void*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  A a;
  __builtin_memcpy(&a, (const void*)p, sizeof(a));
  return a;
}

// What the calls differ in: the element type, which tokens a row sees, and whose rows make
// up a tile.
//   Causal    a request's rows, over all tokens up to each row's own (Alone: with a tail)
//   Windowed  the same, over the last `window` of them and the first `sinks`
//   Prefixed  the rows of a whole group of requests, over the prefix that they share
//   Shared    (few rows) the same in some workgroups, and in the others a request's rows, over
//             what is behind its group's prefix; what joins the two
template <class T_>
struct Causal {
  typedef T_ T;
  typedef ChunkArgs Args;
  static constexpr bool kWindow = false, kPrefix = false, kShared = false, kTail = false;
};
template <class T_>
struct Alone {
  typedef T_ T;
  typedef SpanArgs Args;
  static constexpr bool kWindow = false, kPrefix = false, kShared = false, kTail = true;
};
template <class T_>
struct Windowed {
  typedef T_ T;
  typedef SpanArgs Args;
  static constexpr bool kWindow = true, kPrefix = false, kShared = false, kTail = true;
};
template <class T_>
struct Prefixed {
  typedef T_ T;
  typedef SpanArgs Args;
  static constexpr bool kWindow = false, kPrefix = true, kShared = false, kTail = false;
};
template <class T_>
struct Shared {
  typedef T_ T;
  typedef SpanArgs Args;
  static constexpr bool kWindow = false, kPrefix = false, kShared = true, kTail = false;
};

__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// The requests of group g are group_at(g) .. group_at(g + 1) - 1, within the batch's whatever
// the caller's array holds.
__device__ __forceinline__ int32_t group_at(const SpanArgs& a, int32_t g) {
  const int32_t r = a.groups[g];
  return r < 0 ? 0 : r < a.n_req ? r : a.n_req;
}

// A tile's rows are those of a unit: a request, or a group of them.  The rows of a unit are its
// (new token, query head of the KV head's group) pairs, token by token; a tile is 2^row_shift of
// them.  Tile slot x of the batch: request r has the slots from floor(offsets[r] * G / rows) + r,
// which are enough for its rows whatever the offsets are, and at most n_tokens * G / rows +
// n_req in all: the grid needs no lengths on the host.
__device__ __forceinline__ int64_t first_tile(const ChunkArgs& a, int32_t r) {
  return (int64_t(a.offsets[r]) * a.group >> a.row_shift) + r;
}

// The token of a unit's row x (0 <= x < 2^31).
__device__ __forceinline__ int32_t token_of(const ChunkArgs& a, int32_t x) {
  return int32_t((__umulhi(uint32_t(x), a.g_magic) + uint32_t(x)) >> a.g_shift);
}

struct Request {
  int32_t r, begin, n_new;              // n_new 0: nothing to do
  int32_t base;                         // position of its first new token
  int32_t limit;                        // tokens that can be read at all
};

__device__ __forceinline__ Request request_at(const ChunkArgs& a, int32_t r) {
  Request q;
  q.r = r;
  q.begin = a.offsets[r];
  const int64_t n = int64_t(a.offsets[r + 1]) - q.begin;
  q.n_new = q.begin >= 0 && n > 0 && q.begin + n <= a.n_tokens ? int32_t(n) : 0;
  const int32_t len = a.seq_lens[r] > 0 ? a.seq_lens[r] : 0;
  q.base = len - q.n_new;
  const int32_t by_table = a.max_blocks * a.block_size;
  q.limit = len < by_table ? len : by_table;
  if (q.limit > a.max_seq_len) q.limit = a.max_seq_len;
  return q;
}

// The prefix of a group, as far as it can be read.
__device__ __forceinline__ int32_t prefix_of(const SpanArgs& a, int32_t g) {
  const int32_t by_table = a.max_blocks * a.block_size;
  const int32_t n = std::min(std::min(a.prefix_lens[g], a.max_prefix), by_table);
  return n > 0 ? n : 0;
}
// The same of the group that request r is in (0: in none).
__device__ __forceinline__ int32_t prefix_before(const SpanArgs& a, int32_t r) {
  if (a.n_groups == 0) return 0;
  const int32_t g =
      flowkv::last_at_most(a.n_groups, r, [&](int32_t i) { return group_at(a, i); });
  return group_at(a, g) <= r && r < group_at(a, g + 1) ? prefix_of(a, g) : 0;
}

// Item `want` of the tiles of all groups, each tile in splits of its group's prefix: which group,
// which of its items (-1: there are fewer).  The lanes count 64 groups at a time, so that the
// workgroups with something to do are the first of a launch, next to each other.  (Empty ones in
// turn with them go to the same shader engines each time and leave those idle: one group of 128
// rows in 26 splits took 37 us with a slot without rows beside each, 23 without.)  Past 64 groups
// each 64 are one more chain of loads: with single tokens on one KV head of 128, 64 groups of 4
// behind 1,000 take 22 us (each request by itself 35), 256 of 4 behind 500 49 (62), 512 of 2 59
// (63), 1,024 of 2 behind 300 109 (76).
// The group is a unit of rows: r is its first request, whose block list is read, base the one
// behind its last, and limit its prefix.  (All of it from the lane that has counted it: read
// again by the scalar unit it cost another chain of loads.)
struct Item {
  Request unit;
  int32_t at;
};
__device__ __forceinline__ Item find_item(const SpanArgs& a, uint32_t want) {
  constexpr int32_t kMany = 1 << 24;             // (more than a launch has workgroups: `want`
                                                 // is below, and 64 of them are below 2^31)
  const int ln = threadIdx.x & 63;
  int64_t before = 0;
  for (int32_t g0 = 0; g0 < a.n_groups; g0 += 64) {
    const int32_t g = g0 + ln;
    int32_t count = 0, r = 0, base = 0, begin = 0, end = 0, limit = 0;
    if (g < a.n_groups) {
      r = group_at(a, g);
      base = group_at(a, g + 1);
      limit = prefix_of(a, g);
      begin = a.offsets[r];
      end = a.offsets[base];
      const int64_t rows = (int64_t(end) - begin) * a.group;
      const int64_t tiles = rows > 0 ? (rows + (int64_t(1) << a.row_shift) - 1) >> a.row_shift : 0;
      const int64_t items =
          std::min<int64_t>(tiles, kMany) * splits_of(limit, a.prefix_split);
      count = items < kMany ? int32_t(items) : kMany;
    }
    int32_t sum = count;
    for (int off = 1; off < 64 && off < a.n_groups - g0; off *= 2) {
      const int32_t y = __shfl_up(sum, off);
      if (ln >= off) sum += y;
    }
    const uint64_t hit = __ballot(want < before + sum);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      auto of = [&](int32_t x) { return __builtin_amdgcn_readlane(x, l); };
      Request q;
      q.r = of(r);
      q.base = of(base);
      q.begin = of(begin);
      q.limit = of(limit);
      const int64_t n = int64_t(of(end)) - q.begin;
      q.n_new = q.r < q.base && q.begin >= 0 && n > 0 && q.begin + n <= a.n_tokens && q.limit > 0
                    ? int32_t(n) : 0;
      return Item{q, int32_t(want - before - of(sum - count))};
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  return Item{Request{}, -1};
}

// Item `at` of a group's: 8 splits of all tiles, tile by tile, then the next 8.  So the tiles of
// a split are 8 workgroups (of a KV head) apart, on one XCD and at the same time, and all but
// the first find its K and V in that XCD's L2.
__device__ __forceinline__ void place_item(const SpanArgs& a, const Request& q, int32_t at,
                                           int64_t* tile, int* split) {
  const uint32_t splits = uint32_t(splits_of(q.limit, a.prefix_split));
  const int64_t rows = int64_t(q.n_new) * a.group;
  const uint32_t tiles = uint32_t((rows + (int64_t(1) << a.row_shift) - 1) >> a.row_shift);
  if (tiles == 0 || splits == 0) {
    *tile = -1;
    return;
  }
  const uint32_t block = uint32_t(at) / (8 * tiles), rest = uint32_t(at) - block * 8 * tiles;
  const uint32_t wide = splits - 8 * block < 8 ? splits - 8 * block : 8;
  *tile = rest / wide;
  *split = int(8 * block + (rest - uint32_t(*tile) * wide));
}

// What new token i of a group sees of the prefix: all of it, unless the token lies in it.  Its
// request is first looked for where it would be if all had as many.
struct Guess {
  int32_t r, from, to, len;              // of that request: first tokens, its own and the next's
};
__device__ __forceinline__ Guess guess_at(const SpanArgs& a, int32_t r) {
  return Guess{r, a.offsets[r], a.offsets[r + 1], a.seq_lens[r]};
}
__device__ __forceinline__ int32_t likely(const Request& q, int32_t i) {
  return std::min(q.r + int32_t(float(i) * float(q.base - q.r) / float(q.n_new)), q.base - 1);
}
__device__ __forceinline__ int32_t seen_of_prefix(const SpanArgs& a, const Request& q, int32_t i,
                                                  Guess x) {
  const int32_t token = q.begin + i;
  if (x.from > token || x.to <= token) {
    int32_t r = q.r, hi = q.base;
    if (x.from > token) hi = x.r;
    else r = std::min(x.r + 1, hi - 1);
    while (hi - r > 1) {
      const int32_t mid = r + (hi - r) / 2;
      if (a.offsets[mid] <= token) r = mid;
      else hi = mid;
    }
    x = guess_at(a, r);
  }
  const int64_t count = int64_t(x.to) - x.from;
  const int32_t n_new = x.from >= 0 && count > 0 && x.from + count <= a.n_tokens ? int32_t(count) : 0;
  const int32_t n = (x.len > 0 ? x.len : 0) - n_new + (token - x.from) + 1;
  return n < 0 ? 0 : n < q.limit ? n : q.limit;
}

// Tokens that new token i of a request sees: those up to its own position.
__device__ __forceinline__ int32_t seen(const Request& q, int32_t i) {
  const int32_t n = q.base + i + 1;
  return n < 0 ? 0 : n < q.limit ? n : q.limit;
}

// The tokens that a tile goes through, counted without those that none of its rows sees:
// token x of the count is token x of the request below `sinks`, else x + shift.  All limits,
// splits and steps of a tile are in this count.
template <class P>
struct Reach {
  __device__ __forceinline__ Reach() {}
  int32_t sinks = 0, shift = 0;
  int32_t window = 0;                    // kWindow
  int32_t most = 0;                      // kShared
  __device__ __forceinline__ Reach(const typename P::Args& a, const Request& rq, int32_t row0) {
    if constexpr (P::kWindow) {
      // the window of the tile's first row on
      const int32_t p = rq.base + token_of(a, row0), low = (p > 0 ? p : 0) - a.window + 1;
      window = a.window;
      sinks = a.sinks;
      shift = low > sinks ? low - sinks : 0;
    }
    if constexpr (P::kShared) {              // (behind the prefix)
      shift = prefix_before(a, rq.r);
      most = a.max_own;
    }
  }
  // how many are below token n of the request
  __device__ __forceinline__ int32_t below(int32_t n) const {
    if constexpr (P::kWindow) return n <= sinks ? n : std::max(sinks, n - shift);
    else if constexpr (P::kShared) return std::min(std::max(n - shift, 0), most);
    else return n;
  }
  __device__ __forceinline__ uint32_t token(uint32_t x) const {
    if constexpr (P::kWindow) return x < uint32_t(sinks) ? x : x + uint32_t(shift);
    else if constexpr (P::kShared) return x + uint32_t(shift);
    else return x;
  }
  // the first that new token i sees, but for those below `sinks`
  __device__ __forceinline__ int32_t low(const Request& rq, int32_t i) const {
    if constexpr (P::kWindow) {
      const int32_t p = rq.base + i, from = (p > 0 ? p : 0) - window + 1;
      return from > shift ? from - shift : 0;
    } else {
      return 0;
    }
  }
};

// The end of what new token i of the unit sees, in the tile's count.
template <class P>
__device__ __forceinline__ int32_t end_of(const typename P::Args& a, const Request& rq,
                                          const Reach<P>& reach, int32_t i) {
  if constexpr (P::kPrefix) return seen_of_prefix(a, rq, i, guess_at(a, likely(rq, i)));
  else return reach.below(seen(rq, i));
}

// The workspace holds a record per (new token, query head, split): the weighted V
// (Dh floats) of all records first, then all records' (reference max, sum).
__device__ __forceinline__ int64_t record_at(const ChunkArgs& a, int64_t row, int split) {
  return row * a.splits + split;
}
__device__ __forceinline__ float* record_sums(const ChunkArgs& a, int dh, int64_t rec) {
  return a.ws + rec * dh;
}
__device__ __forceinline__ f32x2u* record_ml(const ChunkArgs& a, int dh, int64_t rec) {
  return reinterpret_cast<f32x2u*>(a.ws + int64_t(a.n_tokens) * a.q_heads * a.splits * dh) + rec;
}

// Takes infinities and NaN out of two elements; whether there was one.
template <class T>
__device__ __forceinline__ bool tame(uint32_t& w) {
  bool any = false;
  if ((w & T::kOdd) == T::kOdd) {
    w &= 0xffff0000u;
    any = true;
  }
  if ((w & T::kOdd << 16) == T::kOdd << 16) {
    w &= 0xffffu;
    any = true;
  }
  return any;
}

// What the parts of one row weigh when they are joined under reference m: a part that saw
// no token has a reference of -inf and a sum of 0 (one whose scores are all NaN has a sum
// of NaN, which stays).
__device__ __forceinline__ float part_weight(float mine, float sum, float m) {
  return mine == -INFINITY ? (sum == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(mine - m);
}

// Two parts with their weights.  (Which product is rounded before the sum is stated, not the
// compiler's choice: it has chosen otherwise for other calls of the same code.)
__device__ __forceinline__ float weighted(float x, float wx, float y, float wy) {
  return __builtin_fmaf(x, wx, y * wy);
}
__device__ __forceinline__ f32x4 weighted(f32x4 x, float wx, f32x4 y, float wy) {
  f32x4 r;
#pragma unroll
  for (int k = 0; k < 4; ++k) r[k] = weighted(x[k], wx, y[k], wy);
  return r;
}

// 16-byte piece p of token x's row is at place x kPc + (p ^ swizzle(x)) of a tile: so
// neither the operand reads (32 rows of K at one piece; V transposed, 4 rows of 32 dims)
// nor the rows' arrival meet in a bank.
template <int kPc>
__device__ __forceinline__ int k_swizzle(int x) {
  return kPc == 16 ? x & 15 : x >> 1 & 7;
}
template <int kPc>
__device__ __forceinline__ int v_swizzle(int x) {
  return kPc == 16 ? (x & 3) * 4 : (x >> 1 & 1) * 4;
}

// ---- many rows -----------------------------------------------------------------------
//
// One pass over the cached tokens: with a row's reference m and x = scale log2(e) q.K,
//   l = sum 2^(x - m),  O = sum 2^(x - m) V,  out = O / l,
// m being the largest x so far, or up to kLazy below it: O and l are scaled only when some x
// is more than that above m, so that most steps have no scaling (weights then reach 2^8,
// which costs neither float32 sums nor bf16 weights any relative precision).  Weights are
// rounded to bf16 for the matrix product, as any library's are; l sums them unrounded.
//
// S^T = K Q^T and O^T = V^T P^T: a query row is a lane's column in both, so that the maximum,
// the sum and the weights stay in the lane, and P needs no exchange between the products.
// K and V reach LDS straight from memory, the next step's while this one is worked on
// (through registers instead: a 13,000-token prompt 3.09 ms, not 1.49); V is read transposed
// by the LDS itself.
//
// What bounds it: 4 Dh operations a (row, token) on the matrix units beside an exponential
// and some ten vector operations, on a card that lowers its clock under this load (to about
// 1.8 of 2.4 GHz).  The 13,000-token prompt, 32 heads of 128 on 8, takes 1.29 to 1.38 ms by
// the card, 1.00 to 1.07 PFLOP/s (a library's product of 4,096^3 reaches 1.13, of 16,384^3
// 1.34); 20,000 tokens, 8 heads of 64 on 4, 524 us, 0.78, where exponentials take as long as
// products.  A lone step
// is bound by its load (a CU alone draws about 45 bytes a nanosecond) and its latencies:
// 1.7 us for 256 rows x 64 tokens of 128.
//
// The form of a workgroup: kRw waves side by side in rows (32 each), kKw in keys; a wave
// takes kTile cached tokens a step.
constexpr int kTile = 64;
template <int kDh_, int kRw_, int kKw_>
struct Form {
  static constexpr int kDh = kDh_, kRw = kRw_, kKw = kKw_;
  static constexpr int kWaves = kRw * kKw, kThreads = 64 * kWaves;
  static constexpr int kRows = 32 * kRw;
  // Workgroups on a CU at once.  At 64 dims two fit into the registers (128 a lane, with the
  // operands of one product read ahead, not of 8), and hide each other's latencies: 16
  // prompts of 500 to 3,000 tokens, 8 heads on 4, 140 us, not 160.
  static constexpr int kPerCu = kDh == 64 ? 2 : 1;
  static constexpr int kAhead = kDh == 64 ? 1 : 8;
  static constexpr int kStep = kTile * kKw;         // tokens of a step
  static constexpr int kPc = kDh / 8;            // 16-byte pieces of a row
  static constexpr int kLd = kStep * kPc / kThreads;  // 16-byte loads of a step's K, or V, a lane
  static constexpr int kLdRows = kThreads / kPc;      // tokens of one such load
  static constexpr int kGroup = kThreads / kStep;     // steps whose places are found at once
  // (the swizzles repeat with 16 rows; a group's places are found in its predecessor's
  // first step, and read from two steps before they are used)
  static_assert(kGroup >= 3 && kLdRows % 16 == 0);
};

// What a wave carries through the steps.
template <class F, class P>
struct Wave {
  typedef typename P::T T;
  typedef typename T::Vec Vec;
  static constexpr int kPc = F::kPc;
  static constexpr int kI = F::kDh / 16;         // MFMA steps of K.q
  static constexpr int kB = F::kDh / 32;         // blocks of 32 dims
  static constexpr int kN = kTile / 32;             // blocks of 32 tokens
  Vec q[kI];
  f32x16 o[kB];
  float mref, lsum;                              // of the lane's row; lsum of its own half's tokens
  float scale_log2;
  int half;
  uint32_t ka[kI], va[kB];                       // LDS places of the operand reads in a step's rows
  int32_t lim;                                   // tokens that the lane's row sees,
  int32_t wlim, wleast;                          // at most and at least that one of the wave's sees
  int32_t sinks, low, wlow, wfirst;              // kWindow: where it begins to, the last and the
                                                 // first of the wave's to

  __device__ __forceinline__ void place_reads(int ln, int kw) {
    half = ln >> 5;
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      const int x = kw * kTile + (ln & 31);
      ka[i] = (x * kPc + ((2 * i + half) ^ k_swizzle<kPc>(x))) * 16;
    }
#pragma unroll
    for (int d = 0; d < kB; ++d) {
      const int x = kw * kTile + 4 * half + (ln & 15) / 4;
      const int col = 32 * d + 16 * (ln >> 4 & 1) + 4 * (ln & 3);   // dim
      va[d] = (x * kPc + ((col >> 3) ^ v_swizzle<kPc>(x))) * 16 + (col >> 2 & 1) * 8;
    }
  }
  // Operands: dims 16 i + 8 half of token 32 b + ln % 32; and of V, transposed, dim
  // 32 d + ln % 32 of the 8 tokens of k-step j that the scores' lanes hold.
  __device__ __forceinline__ u32x4 keys(const lvec* k, int b, int i) const {
    return *(const lvec*)((const lbyte*)k + ka[i] + b * 32 * kPc * 16);
  }
  __device__ __forceinline__ u32x4 values(const lvec* v, int d, int j) const {
    const lbyte* p = (const lbyte*)v + va[d];
    const u32x2 lo = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + j * 16 * kPc * 16)));
    const u32x2 hi = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + (j * 16 + 8) * kPc * 16)));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  }

  // S^T = K Q^T: rows are tokens, columns query rows.  The operands of kAhead products are
  // read ahead.
  __device__ __forceinline__ void scores(f32x16 (&s)[kN], const lvec* k) const {
    constexpr int kM = kN * kI, kAhead = F::kAhead;
    u32x4 w[kM];
#pragma unroll
    for (int b = 0; b < kN; ++b) s[b] = f32x16{};
#pragma unroll
    for (int m = 0; m < kAhead; ++m) w[m] = keys(k, m / kI, m % kI);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int m = 0; m < kM; ++m) {
      if (m + kAhead < kM) w[m + kAhead] = keys(k, (m + kAhead) / kI, (m + kAhead) % kI);
      s[m / kI] = T::mfma(__builtin_bit_cast(Vec, w[m]), q[m % kI], s[m / kI]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // The weights of the scores of the tokens from t on, as the B operand of P.V: a lane
  // holds of its row what the operand wants of it, so they change no lane.
  __device__ __forceinline__ void weigh(f32x16 (&s)[kN], int32_t t, uint64_t dead,
                                        u32x4 (&p)[2 * kN]) {
    bool masked = t + kTile > wleast || dead;
    if constexpr (P::kWindow) masked |= t < wlow && t + kTile > sinks;
    if (masked) {
      const int32_t last = lim - t - 4 * half;
      const int32_t always = sinks - t - 4 * half, first = low - t - 4 * half;
      const uint64_t d = dead >> (4 * half);
#pragma unroll
      for (int b = 0; b < kN; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int x = 32 * b + 8 * (i / 4) + i % 4;
          if (x >= last || (d >> x & 1) || (P::kWindow && x >= always && x < first))
            s[b][i] = -INFINITY;
        }
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < kN; ++b)
#pragma unroll
      for (int i = b == 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
    mx *= scale_log2;
    // the reference moves only where some score is more than kLazy above it
    if (__any(mx > mref + kLazy)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (mx > mref + kLazy) {
        const float c = __builtin_amdgcn_exp2f(mref - mx);
        mref = mx;
        lsum *= c;
#pragma unroll
        for (int b = 0; b < kB; ++b) o[b] *= c;
      }
    }
    float mu = mref == -INFINITY ? 0.f : mref;
    if constexpr (T::kLift != 0) mu -= T::kLift;
#pragma unroll
    for (int b = 0; b < kN; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[b][i], scale_log2, -mu));
        const float y = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], scale_log2, -mu));
        lsum += x + y;
        p[2 * b + i / 8][i % 8 / 2] = T::pack(x, y);
      }
  }

  // O^T += V^T P^T: rows are dims.
  __device__ __forceinline__ void add(const lvec* v, const u32x4 (&p)[2 * kN]) {
#pragma unroll
    for (int j = 0; j < 2 * kN; ++j)
#pragma unroll
      for (int d = 0; d < kB; ++d)
        o[d] = T::mfma(__builtin_bit_cast(Vec, values(v, d, j)), __builtin_bit_cast(Vec, p[j]),
                       o[d]);
  }
};

// Where the rows of the workgroup's K and V are, kThreads tokens at a time (a group): their
// places in the pool in 128-byte units, and which of 64 tokens have a block outside it.
template <class F>
struct Places {
  uint32_t at[2 * F::kThreads];
  uint64_t dead[2 * F::kWaves];
  uint32_t odd[2];                               // where V lost a value: a bit per 64th, below
  int32_t least[F::kWaves];                      // kPrefix: the least that a row of a wave sees
};

template <class F, class P>
struct Source {
  Reach<P> reach;
  const char* base;                              // the head's K of block 0
  int64_t voff;
  const int32_t* table;
  uint32_t bs, bs_magic, bs_shift, bunits, sunits;
  int32_t pool_blocks, s0, s1;
  int tid, wave;
  uint32_t kpiece, vpiece;                       // the lane's bytes of a row,
  uint32_t row;                                  // and its first row of a step
  Places<F>* places;
  uint32_t u[F::kLd];                            // the places of the step that is sent next
  int32_t next_block;
  uint32_t next_slot;
  bool next_in;

  // a lane's token of a group: its block ID and slot
  __device__ __forceinline__ void fetch(int group) {
    const uint32_t t = uint32_t(s0) + uint32_t(group) * F::kThreads + uint32_t(tid);
    const uint32_t x = reach.token(t);
    const uint32_t b = uint32_t((uint64_t(__umulhi(x, bs_magic)) + x) >> bs_shift);
    next_slot = x - b * bs;
    next_in = t < uint32_t(s1);
    next_block = table[next_in ? b : 0];         // (s1 lies within the block list)
  }
  // a token that cannot be read has the place of the pool's first row
  __device__ __forceinline__ void place(int group) const {
    const bool good = next_in & (uint32_t(next_block) < uint32_t(pool_blocks));
    const uint64_t dead = __ballot(next_in & !good);
    const uint32_t at = uint32_t(next_block) * bunits + next_slot * sunits;
    places->at[(group & 1) * F::kThreads + tid] = good ? at : 0;
    if ((tid & 63) == 0) places->dead[(group & 1) * F::kWaves + wave] = dead;
  }
  __device__ __forceinline__ bool any_dead(int group) const {
    return __any((tid & 63) < F::kWaves &&
                 places->dead[(group & 1) * F::kWaves + tid % F::kWaves] != 0);
  }
  // which of the tile's tokens have a block outside the pool; x: its first, counted from s0
  __device__ __forceinline__ uint64_t dead(int32_t x) const {
    const uint64_t d = places->dead[x / 64 % (2 * F::kWaves)];
    return uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(d >> 32)))) << 32 |
           uint32_t(__builtin_amdgcn_readfirstlane(int(d)));
  }
  // whether token x, counted from s0, is not one of the pool: behind s1, or in a missing block
  __device__ __forceinline__ bool lost(int32_t x) const {
    return x >= s1 - s0 || (places->dead[x / 64 % (2 * F::kWaves)] >> (x % 64) & 1);
  }
  // The lane's places of step i.
  __device__ __forceinline__ void look(int i) {
#pragma unroll
    for (int e = 0; e < F::kLd; ++e)
      u[e] = places->at[i % (2 * F::kGroup) * F::kStep + row + e * F::kLdRows];
  }
  // The rows at the lane's places on their way to LDS, with no register between.  An
  // instruction fills 64 consecutive 16-byte places, so a lane's place is fixed, and the
  // swizzle is in which piece of the row it reads.
  __device__ __forceinline__ void send(lvec* k, lvec* v) const {
#pragma unroll
    for (int e = 0; e < F::kLd; ++e) {
      const uint64_t off = uint64_t(u[e]) * 128;
      const int to = e * F::kThreads + wave * 64;
      __builtin_amdgcn_global_load_lds((gvoid*)(base + (off + kpiece)), (lvoid*)(k + to), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((gvoid*)(base + voff + (off + vpiece)), (lvoid*)(v + to), 16,
                                       0, 0);
    }
  }
};

// ---- work by the lengths ------------------------------------------------------------
//
// The host sees only the longest request.  Two kinds of call have every workgroup look at
// all lengths first (about 3 us), and find what it does from them by itself:
//   - fewer tiles than CUs, but long ones: a tile's steps are cut into pieces, one to a
//     workgroup, no longer than need be for all of them to be on the CUs at once.  (With one length
//     of split for contexts of 500 to 9,000 tokens, or under the causal diagonal, some CUs
//     have nothing while others go round twice.)  Tiles in more than one piece are joined
//     from their records by a second kernel.  Chunks of 100 to 700 tokens beside 20 single
//     ones over up to 8,000 cached, 8 heads of 128 on one KV head: 67 us, by even splits 78
//     at best; 512 tokens behind 8,000, 32 heads on 8: 86 and 92; 4,000 behind none, 8 on 1:
//     60 and 68.  With few steps the even splits are faster: 256 behind 4,000, 32 on 8: 37,
//     in pieces 39.
//   - more tiles than CUs, of requests with much in the cache: whole tiles, the longest
//     first, so that the last ones to end are short.  4 chunks of 100 to 600 tokens beside 36
//     single ones over 100 to 6,600, 32 heads on 8: 251 us, in the requests' order 326.
//     (Prompts with nothing cached gain nothing: the diagonal orders each of them.)
// A third kind, where tiles are long and a few rounds of the CUs (kTail): as many whole tiles as
// fill rounds, the longest first, and the rest of them in pieces, one round more.  (16 prompts of
// 50 to 700 tokens behind 3,000 and 5,000, 20 heads of 128 on 4, 560 tiles on 256 CUs: 403 us, in
// whole tiles, three rounds, 465 on the same card.)
constexpr int kPieceTiles = 512;           // most tile slots, and requests, of such a call
constexpr int kPieceLeast = 2;             // steps
constexpr int kCutSteps = 16;              // steps a CU, were all tiles the longest, from which on

struct Mine {                              // what a workgroup does; pieces 0: nothing
  Request rq;
  int32_t row0, split, pieces;
};

struct Cut {
  int32_t start[kPieceTiles];              // a request's first tile slot
  union {                                  // of a tile slot
    alignas(16) float steps[kPieceTiles];
    alignas(16) uint32_t key[kPieceTiles];
  };
  int32_t part[2][8];
  int32_t length;
  Mine mine;
};

// Pieces of a tile (steps >= 0, whole), by the reciprocal of their length: at the exact
// multiples it may give one more, the same one wherever it is asked.
__device__ __forceinline__ float pieces_of(float steps, float inv) {
  return ceilf(steps * inv);
}

// The workspace of a call in pieces: a record a piece, its rows as the waves hold them:
// register 4 j + i of lane l of dim block b at (j * 64 + l) * 4 + i; then the rows'
// (reference, sum); then the pieces of one KV head before each tile slot.
template <class F>
__device__ __forceinline__ float* piece_sums(const ChunkArgs& a, int64_t rec, int rw, int b) {
  return a.ws + ((rec * F::kRw + rw) * (F::kDh / 32) + b) * 1024;
}
template <class F>
__device__ __forceinline__ f32x2u* piece_ml(const ChunkArgs& a, int64_t rec, int rw) {
  return reinterpret_cast<f32x2u*>(a.ws + int64_t(F::kPerCu) * kCus * F::kRows * F::kDh) +
         (rec * F::kRw + rw) * 32;
}
template <class F>
__device__ __forceinline__ int32_t* piece_first(const ChunkArgs& a) {
  return reinterpret_cast<int32_t*>(a.ws + int64_t(F::kPerCu) * kCus * F::kRows * (F::kDh + 2));
}

// The workgroup's number.  Where two are on a CU at once and that is all there are, the
// second ones come in reverse, the shortest beside the longest.
template <class F>
__device__ __forceinline__ uint32_t paired() {
  const uint32_t id = blockIdx.x, n = gridDim.x;
  return F::kPerCu == 2 && id >= uint32_t(kCus) && n <= 2 * kCus ? n - 1 - (id - kCus) : id;
}

// Finds the workgroup's tile, or its piece of one, and the KV head; kPieceTiles lanes, one
// to a tile slot (slots are counted from the first request's token here: rows before it,
// or behind the last request, are padding and have none).  The first workgroup leaves the
// pieces before each slot in the workspace.
template <class F, class P>
__device__ __forceinline__ Mine cut_tiles(const typename P::Args& a, Cut& c, int& g,
                                          int32_t& record) {
  static_assert(F::kThreads == kPieceTiles);
  const int tid = threadIdx.x, ln = tid & 63, wave = tid >> 6;
  const int32_t first = a.offsets[0];
  Mine mine;
  mine.pieces = 0;
  if ((int64_t(a.offsets[a.n_req]) - first) * a.group / F::kRows + a.n_req > a.tiles) {
    // More rows than the host was told of (max_new): whole tiles, in the batch's order.
    if (a.pieces && blockIdx.x == 0)
      for (int32_t i = tid; i <= a.tiles; i += F::kThreads) piece_first<F>(a)[i] = 0;
    g = int(blockIdx.x % uint32_t(a.kv_heads));
    const int32_t slot = int32_t(blockIdx.x / uint32_t(a.kv_heads));
    mine.rq = request_at(
        a, flowkv::last_at_most(a.n_req, slot, [&](int32_t i) { return first_tile(a, i); }));
    const int64_t local = int64_t(slot) - first_tile(a, mine.rq.r);
    if (local >= 0 && local * F::kRows < int64_t(mine.rq.n_new) * a.group) mine.pieces = 1;
    mine.row0 = int32_t(local) * F::kRows;
    mine.split = 0;
    return mine;
  }
  uint32_t id = a.pieces ? blockIdx.x : paired<F>();
  bool tail = false;
  if constexpr (P::kTail) tail = a.tail != 0;
  const uint32_t slots = uint32_t(a.tiles * a.kv_heads);
  // (padding's; with a tail, fewer than `pieces` whole tiles and as many pieces are behind)
  if (id >= (tail ? slots + uint32_t(a.pieces) : std::max(slots, uint32_t(a.pieces)))) return mine;
  // (at most kPieceTiles x kRows rows: 32 bits hold what valid offsets give)
  if (tid < a.n_req)
    c.start[tid] = int32_t(uint32_t(a.offsets[tid] - first) * uint32_t(a.group) / F::kRows) + tid;
  if (tid == 0) {
    c.length = INT32_MAX;
    c.mine.pieces = 0;
  }
  __syncthreads();
  int32_t n = 0;                                 // steps
  if (tid < a.tiles) {
    int32_t r = 0, hi = a.n_req;
    while (hi - r > 1) {
      const int32_t mid = r + (hi - r) / 2;
      if (c.start[mid] <= tid) r = mid;
      else hi = mid;
    }
    mine.rq = request_at(a, r);
    const int32_t rows = mine.rq.n_new * a.group;
    mine.row0 = (tid - c.start[r]) * F::kRows;
    if (mine.row0 >= 0 && mine.row0 < rows) {
      const int32_t end = std::min(mine.row0 + F::kRows, rows);
      const Reach<P> reach(a, mine.rq, mine.row0);
      const int32_t limit = reach.below(seen(mine.rq, token_of(a, end - 1)));
      n = limit > F::kStep ? (limit + F::kStep - 1) / F::kStep : 1;
    }
  }
  int32_t whole = INT32_MAX;                     // with a tail: whole tiles of a KV head
  if (a.pieces == 0 || tail) {                   // each counts the longer ones
    const uint32_t key = uint32_t(n) * kPieceTiles + uint32_t(tid);
    c.key[tid] = key;
    if (tail) {
      const int32_t some = __popcll(__ballot(n > 0));
      if (ln == 0) c.part[0][wave] = some;
    }
    __syncthreads();
    if (tail) {
      int32_t all = 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) all += c.part[0][w];
      whole = all * a.kv_heads / a.pieces * a.pieces / a.kv_heads;
    }
    g = int(id % uint32_t(a.kv_heads));
    if (n > 0) {
      int32_t before = 0;
#pragma unroll 4
      for (int32_t i = 0; i < a.tiles; i += 4) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(&c.key[i]);
        before += x[0] > key;
        before += x[1] > key;
        before += x[2] > key;
        before += x[3] > key;
      }
      if (tail && before < whole) n = 0;         // (not one of the tail's)
      if (before < whole && before == int32_t(id / uint32_t(a.kv_heads))) {
        mine.split = 0;
        mine.pieces = 1;
        c.mine = mine;
      }
    }
    __syncthreads();
  }
  if (a.pieces != 0 && (!tail || id >= uint32_t(whole * a.kv_heads))) {
    if (tail) id -= uint32_t(whole * a.kv_heads);
    c.steps[tid] = float(n);
    int32_t sum = n, most = n;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
      sum += __shfl_xor(sum, off);
      most = std::max(most, __shfl_xor(most, off));
    }
    if (ln == 0) {
      c.part[0][wave] = sum;
      c.part[1][wave] = most;
    }
    __syncthreads();
    sum = most = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      sum += c.part[0][w];
      most = std::max(most, c.part[1][w]);
    }
    // a lane tries a length: the least one that leaves few enough pieces
    constexpr int kTries = F::kThreads / 2;
    const int32_t each = std::max(a.pieces / a.kv_heads, 1);
    const int32_t least = std::max((sum + each - 1) / each, kPieceLeast);
    const int32_t by = most > least ? (most - least + kTries - 1) / kTries : 1;
    const int32_t tried = least + tid * by;
    if (tid < kTries && tried - by < most) {
      const float inv = tried >= most ? 0.f : 1.f / float(tried);
      float pieces = 0.f;
#pragma unroll 4
      for (int32_t i = 0; i < a.tiles; i += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(&c.steps[i]);
        pieces += (pieces_of(x[0], inv) + pieces_of(x[1], inv)) +
                  (pieces_of(x[2], inv) + pieces_of(x[3], inv));
      }
      if (pieces <= float(each)) atomicMin(&c.length, tried);
    }
    __syncthreads();
    const int32_t length = c.length;
    mine.pieces =
        n == 0 ? 0 : length >= most ? 1 : int32_t(pieces_of(float(n), 1.f / float(length)));
    sum = mine.pieces;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
      const int32_t y = __shfl_up(sum, off);
      if (ln >= off) sum += y;
    }
    if (ln == 63) c.part[0][wave] = sum;
    __syncthreads();
    int32_t total = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      if (w < wave) sum += c.part[0][w];
      total += c.part[0][w];
    }
    // an XCD's workgroups have pieces in a row
    record = int32_t(id) < a.pieces ? int32_t(id) % 8 * (a.pieces / 8) + int32_t(id) / 8
                                    : int32_t(id);
    if (record == 0) {
      if (tid == 0) piece_first<F>(a)[0] = 0;
      if (tid < a.tiles) piece_first<F>(a)[tid + 1] = sum;
    }
    g = uniform(total ? record / total : 0);
    mine.split = record - g * total - (sum - mine.pieces);
    if (mine.split >= 0 && mine.split < mine.pieces && g < a.kv_heads) c.mine = mine;
    __syncthreads();
  }
  mine.rq = {uniform(c.mine.rq.r), uniform(c.mine.rq.begin), uniform(c.mine.rq.n_new),
             uniform(c.mine.rq.base), uniform(c.mine.rq.limit)};
  mine.row0 = uniform(c.mine.row0);
  mine.split = uniform(c.mine.split);
  mine.pieces = uniform(c.mine.pieces);
  return mine;
}

template <class F, bool kCut, class P>
__device__ __forceinline__ void attend_many(const typename P::Args& a) {
  typedef Wave<F, P> W;
  typedef typename P::T T;
  constexpr int kDh = F::kDh, kPc = F::kPc, kStep = F::kStep, kB = W::kB;
  const int tid = threadIdx.x, ln = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % F::kRw, kw = wave / F::kRw;
  const int half = ln >> 5, c32 = ln & 31;

  int g;
  int32_t row0, split, record = 0, pieces = 1;
  Request rq;
  if constexpr (kCut) {
    __shared__ Cut c;
    const Mine mine = cut_tiles<F, P>(a, c, g, record);
    if (mine.pieces == 0) return;
    rq = mine.rq;
    row0 = mine.row0;
    split = mine.split;
    pieces = mine.pieces;
  } else {
    const uint32_t id = paired<F>();
    g = int(id % uint32_t(a.kv_heads));
    const uint32_t rest = id / uint32_t(a.kv_heads);
    int64_t local;
    if constexpr (P::kPrefix) {
      const Item item = find_item(a, rest);
      if (item.at < 0) return;
      rq = item.unit;
      place_item(a, rq, item.at, &local, &split);
    } else {
      split = int(rest / uint32_t(a.tiles));
      const int slot = a.tiles - 1 - int(rest % uint32_t(a.tiles));  // the longest first
      rq = request_at(
          a, flowkv::last_at_most(a.n_req, slot, [&](int32_t i) { return first_tile(a, i); }));
      local = int64_t(slot) - first_tile(a, rq.r);
    }
    if (local < 0 || local * F::kRows >= int64_t(rq.n_new) * a.group) return;
    row0 = int32_t(local) * F::kRows;
  }
  const int32_t rows = rq.n_new * a.group, row_end = std::min(row0 + F::kRows, rows);
  const Reach<P> reach(a, rq, row0);
  int32_t tile_limit, tile_least;
  if constexpr (P::kPrefix) {
    tile_limit = tile_least = rq.limit;
  } else {
    tile_limit = end_of<P>(a, rq, reach, token_of(a, row_end - 1));
    tile_least = end_of<P>(a, rq, reach, token_of(a, row0));
  }
  // (from here on no row has tokens behind the first ones that it does not see any more)
  const int32_t tile_low = P::kWindow ? reach.low(rq, token_of(a, row_end - 1)) : 0;
  int32_t length = a.split_tokens;
  if constexpr (kCut)                            // (a piece's, of as many even ones)
    length = (tile_limit + pieces * F::kStep - 1) / (pieces * F::kStep) * F::kStep;
  const int32_t s0 = split * length;
  if (!kCut && split > 0 && s0 >= tile_limit) return;   // (split 0 writes what sees nothing)
  const int32_t s1 = tile_limit - s0 > length ? s0 + length : tile_limit;
  const bool direct = kCut ? pieces == 1 : !P::kPrefix && tile_limit <= length;

  __shared__ alignas(16) u32x4 sk0[kStep * kPc], sk1[kStep * kPc], sv0[kStep * kPc],
      sv1[kStep * kPc];
  __shared__ Places<F> places;

  const int lr = tid / kPc, lp = tid % kPc;
  Source<F, P> src{reach};
  src.base = a.kbase + g * kDh * 2;
  src.voff = a.voff;
  src.table = a.tables + int64_t(rq.r) * a.max_blocks;
  src.bs = uint32_t(a.block_size);
  src.bs_magic = a.bs_magic;
  src.bs_shift = a.bs_shift;
  src.bunits = a.bunits;
  src.sunits = a.sunits;
  src.pool_blocks = a.pool_blocks;
  src.s0 = s0;
  src.s1 = s1;
  src.tid = tid;
  src.wave = wave;
  src.row = lr;
  src.kpiece = 16 * (lp ^ k_swizzle<kPc>(lr));
  src.vpiece = 16 * (lp ^ v_swizzle<kPc>(lr));
  src.places = &places;

  // The first step is on its way while the query rows are looked up and loaded (chunk
  // attention has it behind them).
  constexpr bool kEarly = !std::is_same_v<typename P::Args, ChunkArgs>;
  bool next_dead = false, suspect = false;       // a block is missing in the next group of
                                                 // steps; in it or in this one
  auto start = [&] {
    src.fetch(0);
    src.place(0);
    if (tid < 2) places.odd[tid] = 0;
    __syncthreads();
    suspect = next_dead = src.any_dead(0);
    src.look(0);
    src.send((lvec*)sk0, (lvec*)sv0);
    src.look(1);
  };
  if constexpr (kEarly) {
    if (s0 < s1) start();
  }

  // this lane's query row, as a column of S^T
  const int32_t wrow = row0 + rw * 32, row = wrow + c32;
  const bool live = row < rows;
  const int32_t qi = live ? token_of(a, row) : 0;
  const int32_t qh = live ? row - qi * a.group : 0;
  const int64_t token = int64_t(rq.begin) + qi;
  const int32_t head = g * a.group + qh;
  W w;
  w.place_reads(ln, kw);
  w.scale_log2 = a.scale_log2;
  w.lim = live ? end_of<P>(a, rq, reach, qi) : 0;
  const bool any_row = wrow < rows;              // (the wave may hold no row)
  if constexpr (P::kPrefix) {
    int32_t most = w.lim, least = live ? w.lim : rq.limit;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
      most = std::max(most, __shfl_xor(most, off));
      least = std::min(least, __shfl_xor(least, off));
    }
    w.wlim = uniform(most);
    w.wleast = uniform(least);
  } else {
    w.wlim = uniform(any_row ? end_of<P>(a, rq, reach, token_of(a, std::min(wrow + 31, rows - 1)))
                             : 0);
    w.wleast = uniform(any_row ? end_of<P>(a, rq, reach, token_of(a, wrow)) : 0);
  }
  w.sinks = w.low = w.wlow = w.wfirst = 0;
  if constexpr (P::kWindow) {
    w.sinks = reach.sinks;
    w.low = reach.low(rq, qi);
    w.wlow = uniform(reach.low(rq, token_of(a, std::min(wrow + 31, rows - 1))));
    w.wfirst = uniform(reach.low(rq, token_of(a, std::min(wrow, rows - 1))));
  }
#pragma unroll
  for (int i = 0; i < W::kI; ++i) {
    u32x4 x = {0, 0, 0, 0};
    if (live) x = *(cgvec4*)(a.q + token * a.q_stride + int64_t(head) * kDh + 16 * i + 8 * half);
    w.q[i] = __builtin_bit_cast(typename T::Vec, x);
  }
#pragma unroll
  for (int b = 0; b < kB; ++b) w.o[b] = f32x16{};
  w.mref = -INFINITY;
  w.lsum = 0.f;

  // Where some row does not see some token, or a block is missing, an infinity or a NaN
  // in V would reach a row as 0 x inf: such values are taken out of the step's rows by the
  // lanes that brought them, and added at the end to the rows that see them.  (What lies at
  // the place of a row that does not exist counts for nothing.)  Which 64ths of the
  // workgroup's tokens, 2^odd_shift each, such values were in, is kept: the end looks
  // through those alone.
  auto odd_shift = [&] { return std::max(0, 26 - __builtin_clz((s1 - s0 - 1) | 1)); };
  auto landed = [&](lvec* v, int32_t t0) {
    __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0)
    bool all_seen = t0 + kStep <= tile_least;
    if constexpr (P::kWindow) all_seen &= t0 >= tile_low || t0 + kStep <= reach.sinks;
    if (__builtin_expect(all_seen && !suspect, 1)) return;
#pragma unroll
    for (int e = 0; e < F::kLd; ++e) {
      const int32_t t = t0 + int32_t(src.row) + e * F::kLdRows;
      u32x4 x = v[e * F::kThreads + tid];
      bool any = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t y = x[i];
        any |= tame<T>(y);
        x[i] = y;
      }
      if (any) {
        v[e * F::kThreads + tid] = x;
        const int bit = (t - s0) >> odd_shift();
        if (!src.lost(t - s0)) atomicOr(&places.odd[bit >> 5], 1u << (bit & 31));
      }
    }
  };

  if (s0 < s1) {                                 // uniform
    int i = 0;
    auto step = [&](int32_t t0, lvec* __restrict__ k, lvec* __restrict__ v, lvec* __restrict__ k_to,
                    lvec* __restrict__ v_to) {
      const bool more = t0 + kStep < s1;
      const bool find = i % F::kGroup == 0;      // the next group's places
      if (more) src.send(k_to, v_to);
      if (find) src.fetch(i / F::kGroup + 1);
      const int32_t t = t0 + kw * kTile;
      bool some = t < w.wlim && t < s1;
      if constexpr (P::kWindow) some &= t + kTile > w.wfirst || t < w.sinks;
      if (some) {
        f32x16 s[W::kN];
        u32x4 p[2 * W::kN];
        w.scores(s, k);
        w.weigh(s, t, __builtin_expect(suspect, 0) ? src.dead(t - s0) : 0, p);
        w.add(v, p);
      }
      src.look(i + 2);
      if (find) src.place(i / F::kGroup + 1);
      if (more) landed(v_to, t0 + kStep);
      __syncthreads();
      if (find) {
        suspect = next_dead;
        next_dead = src.any_dead(i / F::kGroup + 1);
        suspect |= next_dead;
      }
      ++i;
    };
    lvec *const k0 = (lvec*)sk0, *const k1 = (lvec*)sk1, *const v0 = (lvec*)sv0,
                *const v1 = (lvec*)sv1;
    if constexpr (!kEarly) start();
    if constexpr (P::kPrefix) {
      if (ln == 0) places.least[wave] = w.wleast;
      __syncthreads();
#pragma unroll
      for (int x = 0; x < F::kWaves; ++x) tile_least = std::min(tile_least, places.least[x]);
      tile_least = uniform(tile_least);
    }
    landed(v0, s0);
    __syncthreads();
    for (int32_t t0 = s0; t0 < s1; t0 += 2 * kStep) {
      step(t0, k0, v0, k1, v1);
      if (t0 + kStep < s1) step(t0 + kStep, k1, v1, k0, v0);
    }
  }
  // (the arguments and the lane's row again: the loop has no registers left for them)
  const typename P::Args e = late_args<typename P::Args>();
  const int lane = int(__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)));
  const int hi = lane >> 5;
  uint64_t odd = 0;
  if (s0 < s1)
    odd = uint64_t(uint32_t(uniform(int32_t(places.odd[1])))) << 32 |
          uint32_t(uniform(int32_t(places.odd[0])));
  float lsum = w.lsum + __shfl_xor(w.lsum, 32);
  float mref = w.mref;
  if constexpr (F::kKw > 1) {
    // The waves of other keys bring their sums to the first ones', through LDS, kR blocks of
    // dims at a time: register j of lane l at place 64 j + l.
    constexpr int kFit = int(sizeof(sk0)) / (F::kRw * 64 * 16 * int(sizeof(float)));
    constexpr int kR = kFit < kB ? kFit : kB;
    static_assert(kR >= 1 && kB % kR == 0 && sizeof(sk1) >= F::kRw * 2 * 64 * sizeof(float));
    float* const sums = reinterpret_cast<float*>(sk0) + rw * (kR * 16 * 64) + lane;
    float* const ml = reinterpret_cast<float*>(sk1) + rw * 128 + lane;
    for (int from = 1; from < F::kKw; ++from) {
      float c1 = 0.f, c2 = 0.f;
#pragma unroll
      for (int b0 = 0; b0 < kB; b0 += kR) {
        if (kw == from) {
#pragma unroll
          for (int j = 0; j < 16 * kR; ++j) sums[64 * j] = w.o[b0 + j / 16][j % 16];
          if (b0 == 0) {
            ml[0] = mref;
            ml[64] = lsum;
          }
        }
        __syncthreads();
        if (kw == 0) {
          if (b0 == 0) {
            const float m2 = ml[0], l2 = ml[64], m = fmaxf(mref, m2);
            c1 = part_weight(mref, lsum, m);
            c2 = part_weight(m2, l2, m);
            mref = m;
            lsum = weighted(lsum, c1, l2, c2);
          }
#pragma unroll
          for (int j = 0; j < 16 * kR; ++j)
            w.o[b0 + j / 16][j % 16] =
                weighted(w.o[b0 + j / 16][j % 16], c1, sums[64 * j], c2);
        }
        __syncthreads();
      }
    }
    if (kw > 0) return;
  }
  // the rows of V of the marked 64ths, 64 pieces of 16 bytes at a time
  for (; odd; odd &= odd - 1) {
    constexpr int kPer = 64 / kPc;
    const int32_t from = s0 + (__builtin_ctzll(odd) << odd_shift());
    const int32_t to = std::min(s1 - from, 1 << odd_shift()) + from;
    for (int32_t t0 = from; t0 < to; t0 += kPer) {
      const int32_t t = t0 + lane / kPc;
      const int32_t token = int32_t(reach.token(uint32_t(t < to ? t : from)));
      const int32_t blk = src.table[token / e.block_size];
      uint32_t at = 0;                           // in 128-byte units, as in the loop
      bool any = false;
      if (t < to && blk >= 0 && blk < e.pool_blocks) {
        at = uint32_t(blk) * e.bunits + uint32_t(token % e.block_size) * e.sunits;
        const u32x4 x = *(cgvec4*)(src.base + e.voff + uint64_t(at) * 128 + lane % kPc * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t y = x[i];
          any |= tame<T>(y);
        }
      }
      for (uint64_t hit = __ballot(any); hit;) { // a token with such a value
        const int x = __builtin_ctzll(hit) / kPc;
        hit &= ~(((uint64_t(1) << kPc) - 1) << (x * kPc));
        const char* v = src.base + e.voff +
                        uint64_t(uint32_t(__builtin_amdgcn_readlane(int(at), x * kPc))) * 128;
        bool sees = t0 + x < w.lim;
        if constexpr (P::kWindow) sees &= t0 + x < w.sinks || t0 + x >= w.low;
        bool full = true;                        // with NaN, which stays
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) full &= w.o[b][i] != w.o[b][i];
        if (!__any(sees && !full)) {
          // later tokens are seen by no other rows, or by those whose window begins behind x
          if (P::kWindow && __any(t0 + x < w.lim && !full)) continue;
          odd = 0;
          t0 = to;
          break;
        }
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u32x2 y = *(cgvec2*)(v + (32 * b + 8 * j + 4 * hi) * 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t z = i % 2 ? T::template widen<1>(y[i / 2]) : T::template widen<0>(y[i / 2]);
              if (sees && (z & 0x7f800000u) == 0x7f800000u)
                w.o[b][4 * j + i] += __uint_as_float(z);
            }
          }
      }
    }
  }
  if (kCut && !direct && any_row) {
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4u*>(piece_sums<F>(e, record, rw, b) + (j * 64 + lane) * 4) =
            f32x4u{w.o[b][4 * j], w.o[b][4 * j + 1], w.o[b][4 * j + 2], w.o[b][4 * j + 3]};
    if (hi == 0) piece_ml<F>(e, record, rw)[lane & 31] = f32x2u{mref, lsum};
  }
  const int32_t late_row = wrow + (lane & 31);     // of the request
  if (late_row >= rows) return;
  const int32_t new_token = token_of(e, late_row);
  const int64_t orow = (int64_t(rq.begin) + new_token) * e.q_heads + g * e.group +
                       (late_row - new_token * e.group);
  if (direct) {
    const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const u32x2 x = {T::pack(w.o[b][i] * inv, w.o[b][i + 1] * inv),
                         T::pack(w.o[b][i + 2] * inv, w.o[b][i + 3] * inv)};
        *reinterpret_cast<u32x2*>(e.out + orow * kDh + 32 * b + 2 * i + 4 * hi) = x;
      }
  } else if constexpr (!kCut) {
    const int64_t rec = record_at(e, orow, split);
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4u*>(record_sums(e, kDh, rec) + 32 * b + 2 * i + 4 * hi) =
            f32x4u{w.o[b][i], w.o[b][i + 1], w.o[b][i + 2], w.o[b][i + 3]};
    if (hi == 0) *record_ml(e, kDh, rec) = f32x2u{mref, lsum};
  }
}

// Joins the records of the tiles that are in more than one piece: a wave per 32 rows and
// 32 dims.
template <class F, class T>
__device__ __forceinline__ void join_pieces(const ChunkArgs& a) {
  const int ln = threadIdx.x & 63, half = ln >> 5, c32 = ln & 31;
  const int b = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = int(blockIdx.x % F::kRw);
  const uint32_t rest = blockIdx.x / F::kRw;
  const int g = int(rest % uint32_t(a.kv_heads)), slot = int(rest / uint32_t(a.kv_heads));
  const int32_t* first = piece_first<F>(a);
  const int32_t total = first[a.tiles], from = first[slot], to = first[slot + 1];
  if (to - from < 2) return;                     // written already
  const int32_t base = a.offsets[0];             // (as cut_tiles counts)
  auto start = [&](int32_t i) {
    return (int64_t(a.offsets[i] - base) * a.group >> a.row_shift) + i;
  };
  const int32_t r = flowkv::last_at_most(a.n_req, slot, start);
  const Request rq = request_at(a, r);
  const int64_t row = (int64_t(slot) - start(r)) * F::kRows + rw * 32 + c32;
  const bool live = row >= 0 && row < int64_t(rq.n_new) * a.group;
  if (!__any(live)) return;
  float m = -INFINITY, l = 0.f;
  f32x4 x[4] = {};
  constexpr int kAhead = 4;                      // records under way
  for (int32_t w = from; w < to; w += kAhead) {
    f32x2u ml[kAhead];
    f32x4 y[kAhead][4];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {           // (past the end: the last record, not used)
      const int64_t rec = int64_t(g) * total + std::min(w + k, to - 1);
      ml[k] = piece_ml<F>(a, rec, rw)[c32];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        y[k][j] =
            *reinterpret_cast<const f32x4u*>(piece_sums<F>(a, rec, rw, b) + (j * 64 + ln) * 4);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (w + k >= to) break;
      const float mm = fmaxf(m, ml[k][0]);
      const float c1 = part_weight(m, l, mm), c2 = part_weight(ml[k][0], ml[k][1], mm);
      m = mm;
      l = weighted(l, c1, ml[k][1], c2);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = weighted(x[j], c1, y[k][j], c2);
    }
  }
  if (!live) return;
  const int32_t qi = token_of(a, int32_t(row));
  const int64_t orow =
      (int64_t(rq.begin) + qi) * a.q_heads + g * a.group + (int32_t(row) - qi * a.group);
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const u32x2 y = {T::pack(x[j][0] * inv, x[j][1] * inv), T::pack(x[j][2] * inv, x[j][3] * inv)};
    *reinterpret_cast<u32x2*>(a.out + orow * F::kDh + 32 * b + 8 * j + 4 * half) = y;
  }
}

// ---- few rows ----------------------------------------------------------------------
//
// A request of a few new tokens reads every cached K and V for a handful of rows: that is
// bound by HBM, as the decode step is, and wants many loads in flight rather than many rows
// per byte.  A workgroup takes 16 rows, as the 16 columns of S^T, or twice 16, and each of
// its four waves tiles of 32 tokens of its own, four tiles apart, with no barrier between:
//   - K and V rows arrive whole in registers (16 lanes a row of K; a lane of group q4 =
//     lane / 16 has V of the tokens 4 e + q4, e = 0..7), the next tile's while this one is
//     worked on;
//   - K goes through the wave's part of LDS into the A operand, row m of half gg being
//     token 16 gg + 4 (m % 4) + m / 4: a lane's scores are then those of the tokens whose
//     V it holds, and P and V are operands of P.V where they are.
// 24 requests of 2 to 8 tokens over 2,000 to 16,000, 32 heads of 128 on 8 (915 MB), in 32 rows
// take 179 us with the merge, 5.1 TB/s; 64 of one token over 500 to 4,000, in 16 rows, 115 us
// (128 rows a workgroup, one split: 166).  K and V are read once and past the caches.
constexpr int kFewWaves = 4;
constexpr int kFewThreads = 64 * kFewWaves;
constexpr int kFewTile = 32;
constexpr int kFewSplit = 2048;            // most tokens of a workgroup: their places are in LDS

template <int kDh, int kC>
struct FewLds {
  static constexpr int kRows = 16 * kC;
  uint32_t at[kFewSplit];                  // a tile's token 4 e + q4 at 8 q4 + e, in 128-byte units
  // K's staging, a tile per wave; after the loop the waves' weighted sums
  alignas(16) uint8_t area[kFewWaves * kRows * kDh * sizeof(float)];
  uint32_t dead[kFewSplit / kFewTile];
  uint32_t odd[2];                         // tiles whose V lost an infinity or a NaN
  float m[kFewWaves][kRows], l[kFewWaves][kRows];
  int32_t lim[kRows];
  int32_t low[kRows];                      // kWindow
  static_assert(kFewWaves * kFewTile * kDh * 2 <= sizeof(area) && kFewSplit / kFewTile <= 64);
};

__device__ __forceinline__ uint32_t pair_hi(uint32_t lo, uint32_t hi) {
  return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
}
__device__ __forceinline__ uint32_t pair_lo(uint32_t lo, uint32_t hi) {
  return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// Workgroups on a CU at once.
constexpr int few_per_cu(int dh, int c) { return (dh == 64 ? 4 : 3) - (c - 1); }

template <int kDh, int kC, class P>
__device__ __forceinline__ void attend_few(const typename P::Args& a) {
  typedef typename P::T T;
  typedef typename T::Vec Vec;
  constexpr int kFewRows = 16 * kC;
  constexpr int kI = kDh / 32;                   // MFMA steps of K.q
  constexpr int kT = kDh / 16;                   // dims a lane owns in P.V
  constexpr int kVW = kT / 2;                    // V words per token and lane
  constexpr int kPc = kDh / 8;                   // 16-byte pieces of a K row
  constexpr int kKL = kFewTile * kPc / 64;       // K loads of a tile and lane
  typedef uint32_t VT __attribute__((ext_vector_type(kVW)));
  typedef __attribute__((address_space(1))) const VT cgv;
  const int tid = threadIdx.x, ln = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q4 = ln >> 4, c16 = ln & 15;

  const uint32_t id = blockIdx.x;
  const int g = int(id % uint32_t(a.kv_heads));
  const uint32_t rest = id / uint32_t(a.kv_heads);
  int split = 0;
  int32_t length = a.split_tokens;
  Request rq{};
  int64_t local = -1;
  bool of_prefix = false;                        // kShared: a group's rows, over its prefix
  if constexpr (P::kShared) of_prefix = rest < a.prefix_items;
  if (of_prefix) {
    if constexpr (P::kShared) {
      const Item item = find_item(a, rest);
      if (item.at < 0) return;
      length = a.prefix_split;
      rq = item.unit;
      place_item(a, rq, item.at, &local, &split);
    }
  } else {
    uint32_t at = rest;
    if constexpr (P::kShared) at -= a.prefix_items;
    split = int(at / uint32_t(a.tiles));
    const int slot = int(at % uint32_t(a.tiles));
    rq = request_at(
        a, flowkv::last_at_most(a.n_req, slot, [&](int32_t i) { return first_tile(a, i); }));
    local = int64_t(slot) - first_tile(a, rq.r);
  }
  if (local < 0 || local * kFewRows >= int64_t(rq.n_new) * a.group) return;
  const int32_t row0 = int32_t(local) * kFewRows, rows = rq.n_new * a.group;
  Reach<P> reach;
  int32_t tile_limit = rq.limit, tile_least = rq.limit;
  if (!of_prefix) {
    reach = Reach<P>(a, rq, row0);
    tile_limit = end_of<P>(a, rq, reach, token_of(a, std::min(row0 + kFewRows, rows) - 1));
    tile_least = end_of<P>(a, rq, reach, token_of(a, row0));
  }
  const int32_t tile_low =
      P::kWindow ? reach.low(rq, token_of(a, std::min(row0 + kFewRows, rows) - 1)) : 0;
  const int32_t s0 = split * length;
  if (split > 0 && s0 >= tile_limit) return;
  const int32_t s1 = tile_limit - s0 > length ? s0 + length : tile_limit;
  const bool direct = !P::kShared && tile_limit <= length;
  const int n_tiles = (s1 - s0 + kFewTile - 1) / kFewTile;

  __shared__ FewLds<kDh, kC> lds;
  const int32_t* table = a.tables + int64_t(rq.r) * a.max_blocks;
  auto entry_of = [&](int x, uint32_t* within) {
    const uint32_t t = reach.token(uint32_t(s0 + x));
    const uint32_t b = uint32_t((uint64_t(__umulhi(t, a.bs_magic)) + t) >> a.bs_shift);
    *within = t - b * uint32_t(a.block_size);
    return s0 + x < s1 ? int32_t(b) : 0;         // (s1 lies within the block list)
  };
  auto place = [&](int x, int32_t blk, uint32_t within) {
    const bool good = s0 + x < s1 && blk >= 0 && blk < a.pool_blocks;
    const uint64_t dead = __ballot(!good);
    lds.at[(x & -kFewTile) + (x & 3) * 8 + (x >> 2 & 7)] =
        good ? uint32_t(blk) * a.bunits + within * a.sunits : 0;
    if (ln % kFewTile == 0) lds.dead[x / kFewTile] = uint32_t(dead >> ln);
  };
  u32x4* const s_k = reinterpret_cast<u32x4*>(lds.area + wave * (kFewTile * kDh * 2));
  u32x4 kw[kKL];
  VT vw[8];
  constexpr int kStride = 64 / kPc;              // tokens of one K load
  const int kt = ln / kPc, kp = ln % kPc;
  const char* const kbase = a.kbase + g * kDh * 2 + 16 * kp;
  const char* const vbase = a.kbase + a.voff + g * kDh * 2 + c16 * (kVW * 4);
  auto swz = [](int token) { return (token * kPc >> 4) & (kPc - 1); };
  // Rows are read once, past the caches; those of a prefix again, by its other tiles.  (With a
  // branch on what a workgroup does, its own rows past the caches too, 32 samples behind 13,000
  // tokens took 41.4 us, not 37.3.)
  auto load_k = [&](int tile) {
#pragma unroll
    for (int e = 0; e < kKL; ++e) {
      const int x = kt + e * kStride;            // token of the tile
      const auto at =
          (cgvec4*)(kbase + uint64_t(lds.at[tile * kFewTile + (x & 3) * 8 + (x >> 2)]) * 128);
      if constexpr (P::kShared) kw[e] = *at;
      else kw[e] = __builtin_nontemporal_load(at);
    }
  };
  auto load_v = [&](int tile) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const auto at = (cgv*)(vbase + uint64_t(lds.at[tile * kFewTile + 8 * q4 + e]) * 128);
      if constexpr (P::kShared) vw[e] = *at;
      else vw[e] = __builtin_nontemporal_load(at);
    }
  };
  int32_t lim[kC], low[kC], qi[kC];
  bool live[kC];
  Vec qb[kC][kI];
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    const int32_t row = row0 + 16 * c + c16;
    live[c] = row < rows;
    qi[c] = live[c] ? token_of(a, row) : 0;
  }
  auto load_q = [&](int c) {
    const int32_t qh = live[c] ? row0 + 16 * c + c16 - qi[c] * a.group : 0;
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      u32x4 x = {0, 0, 0, 0};
      // (kShared: a lane without a row has the first one's, which its column keeps to itself)
      if (P::kShared || live[c])
        x = *(cgvec4*)(a.q + (int64_t(rq.begin) + qi[c]) * a.q_stride +
                       (g * a.group + qh) * int64_t(kDh) + 32 * i + 8 * q4);
      qb[c][i] = __builtin_bit_cast(Vec, x);
    }
  };
  auto limit = [&](int c, int32_t l) {
    lim[c] = live[c] ? l : 0;
    if (tid < 16) lds.lim[16 * c + tid] = lim[c];
    if constexpr (P::kWindow) {
      low[c] = reach.low(rq, qi[c]);
      if (tid < 16) lds.low[16 * c + tid] = low[c];
    }
  };
  if (tid < 2) lds.odd[tid] = 0;
  if constexpr (P::kShared) {
    // One link of loads before K and V: the block list, the rows' requests and the queries are
    // under way together, so without branches between them.
    constexpr int kPlaces = kFewSplit / kFewThreads;
    int32_t blk[kPlaces];
    uint32_t within[kPlaces];
    const int32_t* const from = n_tiles > 0 ? table : a.offsets;   // (no list where none is seen)
#pragma unroll
    for (int e = 0; e < kPlaces; ++e) blk[e] = from[entry_of(tid + e * kFewThreads, &within[e])];
    Guess one[kC];
#pragma unroll
    for (int c = 0; c < kC; ++c) one[c] = guess_at(a, of_prefix ? likely(rq, qi[c]) : rq.r);
#pragma unroll
    for (int c = 0; c < kC; ++c) load_q(c);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < kPlaces; ++e) place(tid + e * kFewThreads, blk[e], within[e]);
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      limit(c, of_prefix ? seen_of_prefix(a, rq, qi[c], one[c]) : end_of<P>(a, rq, reach, qi[c]));
      if (of_prefix) {
        int32_t least = live[c] ? lim[c] : rq.limit;
#pragma unroll
        for (int off = 1; off < 16; off *= 2) least = std::min(least, __shfl_xor(least, off));
        tile_least = std::min(tile_least, uniform(least));
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      limit(c, end_of<P>(a, rq, reach, qi[c]));
      load_q(c);
    }
    for (int x = tid; x < n_tiles * kFewTile; x += kFewThreads) {
      uint32_t within;
      const int32_t blk = table[entry_of(x, &within)];
      place(x, blk, within);
    }
    __syncthreads();
  }
  if (wave < n_tiles) {
    load_k(wave);
    load_v(wave);
  }
  f32x4 o[kC][kT];
  float mref[kC], lsum[kC];                      // of the column's row; this lane's tokens
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    mref[c] = -INFINITY;
    lsum[c] = 0.f;
#pragma unroll
    for (int t = 0; t < kT; ++t) o[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int tile = wave; tile < n_tiles; tile += kFewWaves) {
    // (past the wave's last tile: its own again, so that as many loads are under way)
    const int next = tile + kFewWaves < n_tiles ? tile + kFewWaves : tile;
#pragma unroll
    for (int e = 0; e < kKL; ++e) {
      const int x = kt + e * kStride;
      s_k[x * kPc + (kp ^ swz(x))] = kw[e];
    }
    __builtin_amdgcn_wave_barrier();
    const int kr[2] = {4 * (c16 & 3) + (c16 >> 2), 16 + 4 * (c16 & 3) + (c16 >> 2)};
    Vec ka[2][kI];
#pragma unroll
    for (int gg = 0; gg < 2; ++gg)
#pragma unroll
      for (int i = 0; i < kI; ++i)
        ka[gg][i] = __builtin_bit_cast(Vec, s_k[kr[gg] * kPc + ((4 * i + q4) ^ swz(kr[gg]))]);
    f32x4 s[kC][2];
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int gg = 0; gg < 2; ++gg) {
        s[c][gg] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kI; ++i)
          s[c][gg] = T::mfma(ka[gg][i], qb[c][i], s[c][gg]);
      }
    __builtin_amdgcn_sched_barrier(0);
    load_k(next);
    __builtin_amdgcn_sched_barrier(0);
    const int32_t t0 = s0 + tile * kFewTile;
    const uint32_t dead = __builtin_amdgcn_readfirstlane(lds.dead[tile]) >> q4;   // bit 4 e
    bool masked = t0 + kFewTile > tile_least || __any(dead != 0);                 // uniform
    if constexpr (P::kWindow) masked |= t0 < tile_low && t0 + kFewTile > reach.sinks;
    u32x4 p[kC];
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      if (masked) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (t0 + 4 * e + q4 >= lim[c] || (dead >> (4 * e) & 1) ||
              (P::kWindow && t0 + 4 * e + q4 >= reach.sinks && t0 + 4 * e + q4 < low[c]))
            s[c][e >> 2][e & 3] = -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3])),
                       fmaxf(fmaxf(s[c][1][0], s[c][1][1]), fmaxf(s[c][1][2], s[c][1][3]))) *
                 a.scale_log2;
      if (__any(mx > mref[c] + kLazy)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        float f = 1.f;
        if (mx > mref[c] + kLazy) {
          f = __builtin_amdgcn_exp2f(mref[c] - mx);
          mref[c] = mx;
        }
        lsum[c] *= f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float fx = __shfl(f, 4 * q4 + x);
#pragma unroll
          for (int t = 0; t < kT; ++t) o[c][t][x] *= fx;
        }
      }
      float mu = mref[c] == -INFINITY ? 0.f : mref[c];
      if constexpr (T::kLift != 0) mu -= T::kLift;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[c][i >> 1][2 * i & 3], a.scale_log2, -mu));
        const float y =
            __builtin_amdgcn_exp2f(fmaf(s[c][i >> 1][(2 * i & 3) + 1], a.scale_log2, -mu));
        lsum[c] += x + y;
        p[c][i] = T::pack(x, y);
      }
    }
    if (masked) {                                // 0 x inf is not 0
      bool odd = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (dead >> (4 * e) & 1) vw[e] = VT{};
#pragma unroll
        for (int i = 0; i < kVW; ++i) {
          uint32_t x = vw[e][i];
          odd |= tame<T>(x);
          vw[e][i] = x;
        }
      }
      if (odd) atomicOr(&lds.odd[tile >> 5], 1u << (tile & 31));
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int m = 0; m < kVW; ++m) {
      u32x4 w[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[0][i] = pair_lo(vw[2 * i][m], vw[2 * i + 1][m]);
        w[1][i] = pair_hi(vw[2 * i][m], vw[2 * i + 1][m]);
      }
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          o[c][2 * m + h] = T::mfma(__builtin_bit_cast(Vec, p[c]), __builtin_bit_cast(Vec, w[h]),
                                    o[c][2 * m + h]);
    }
    __builtin_amdgcn_sched_barrier(0);
    load_v(next);
  }

#pragma unroll
  for (int c = 0; c < kC; ++c) {
    lsum[c] += __shfl_xor(lsum[c], 16);
    lsum[c] += __shfl_xor(lsum[c], 32);
    if (q4 == 0) {
      lds.m[wave][16 * c + c16] = mref[c];
      lds.l[wave][16 * c + c16] = lsum[c];
    }
  }
  __syncthreads();                               // every wave is past the loop: the area is free
  const uint64_t odd = uint64_t(uint32_t(uniform(int32_t(lds.odd[1])))) << 32 |
                       uint32_t(uniform(int32_t(lds.odd[0])));
  float* const s_o = reinterpret_cast<float*>(lds.area);   // [wave][row][dim]
#pragma unroll
  for (int c = 0; c < kC; ++c)
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int t = 0; t < kT; t += 4)
        *reinterpret_cast<f32x4*>(
            &s_o[(wave * kFewRows + 16 * c + 4 * q4 + x) * kDh + kT * c16 + t]) =
            f32x4{o[c][t][x], o[c][t + 1][x], o[c][t + 2][x], o[c][t + 3][x]};
  __syncthreads();
  // a row's dims 4 at a time
  for (int i = tid; i < kFewRows * kDh / 4; i += kFewThreads) {
    const int h = i / (kDh / 4), d = i % (kDh / 4) * 4;
    if (row0 + h >= rows) break;
    float M = -INFINITY, L = 0.f;
    f32x4 A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) M = fmaxf(M, lds.m[w][h]);
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float wt = part_weight(lds.m[w][h], lds.l[w][h], M);
      L += lds.l[w][h] * wt;
      A += *reinterpret_cast<const f32x4*>(&s_o[(w * kFewRows + h) * kDh + d]) * wt;
    }
    // infinities and NaN of the tokens that the row sees, until it is all NaN
    for (uint64_t left = odd; left; left &= left - 1) {
      const int tile = __builtin_ctzll(left);
      const int32_t sees = lds.lim[h] - s0 - tile * kFewTile;
      if (sees <= 0 || (A[0] != A[0] && A[1] != A[1] && A[2] != A[2] && A[3] != A[3])) break;
      const uint32_t gone = lds.dead[tile];
#pragma unroll 8
      for (int x = 0; x < kFewTile; ++x) {
        const u32x2 y = *(cgvec2*)(a.kbase + a.voff + (g * kDh + d) * 2 +
                                   uint64_t(lds.at[tile * kFewTile + (x & 3) * 8 + (x >> 2)]) * 128);
        if (x >= sees || (gone >> x & 1)) continue;
        if constexpr (P::kWindow) {
          const int32_t t = s0 + tile * kFewTile + x;
          if (t >= reach.sinks && t < lds.low[h]) continue;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t z = k % 2 ? T::template widen<1>(y[k / 2]) : T::template widen<0>(y[k / 2]);
          if ((z & 0x7f800000u) == 0x7f800000u) A[k] += __uint_as_float(z);
        }
      }
    }
    const int32_t qi = token_of(a, row0 + h);
    const int64_t orow =
        (int64_t(rq.begin) + qi) * a.q_heads + g * a.group + (row0 + h - qi * a.group);
    if (direct) {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      const u32x2 x = {T::pack(A[0] * inv, A[1] * inv), T::pack(A[2] * inv, A[3] * inv)};
      *reinterpret_cast<u32x2*>(a.out + orow * kDh + d) = x;
    } else {
      int64_t rec = record_at(a, orow, split);
      if constexpr (P::kShared) rec += of_prefix ? 0 : a.first_split;
      *reinterpret_cast<f32x4u*>(record_sums(a, kDh, rec) + d) = A;
      if (d == 0) *record_ml(a, kDh, rec) = f32x2u{M, L};
    }
  }
}

// Joins the splits' records of the rows whose tile has more than one: a wave, or the four
// of a workgroup, per (new token, query head), Dh / 4 lanes a record, kMergeChunk records
// of a lane group under way at once.  A launch and three dependent loads bound it: 4.0 us for
// 5 tokens x 32 heads x 26 splits.
constexpr int kMergeThreads = 256;
constexpr int kMergeChunk = 8;

struct Running {
  float m, l;
  f32x4 v;
};
__device__ __forceinline__ Running join(const Running& a, const Running& b) {
  Running r;
  r.m = fmaxf(a.m, b.m);
  const float wa = part_weight(a.m, a.l, r.m), wb = part_weight(b.m, b.l, r.m);
  r.l = weighted(a.l, wa, b.l, wb);
  r.v = weighted(a.v, wa, b.v, wb);
  return r;
}

template <int kDh, int kWavesPer, class P>
__device__ __forceinline__ void merge_splits(const typename P::Args& a) {
  typedef typename P::T T;
  constexpr int kLanes = kDh / 4, kParts = 64 * kWavesPer / kLanes;
  const int ln = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t orow = kWavesPer == 1 ? int64_t(blockIdx.x) * 4 + wave : int64_t(blockIdx.x);
  if (orow >= int64_t(a.n_tokens) * a.q_heads) return;
  const int32_t token = int32_t(uint32_t(orow) / uint32_t(a.q_heads));   // (orow < 2^26)
  const int32_t head = int32_t(orow) - token * a.q_heads;
  const int32_t r =
      flowkv::last_at_most(a.n_req, token, [&](int32_t i) { return a.offsets[i]; });
  const Request rq = request_at(a, r);
  const int32_t i = token - rq.begin;
  if (i < 0 || i >= rq.n_new) return;
  // the tile that the row was in, as its workgroups saw it
  const int32_t row = i * a.group + int32_t(uint32_t(head) % uint32_t(a.group));
  const Reach<P> reach(a, rq, row >> a.row_shift << a.row_shift);
  if constexpr (!P::kShared) {
    const int32_t end = std::min(((row >> a.row_shift) + 1) << a.row_shift, rq.n_new * a.group);
    const int32_t tile_limit = end_of<P>(a, rq, reach, token_of(a, end - 1));
    if (tile_limit <= a.split_tokens) return;    // written already
  }
  int32_t n = flowkv::splits_of(end_of<P>(a, rq, reach, i), a.split_tokens);
  int32_t before = 0;                            // kShared: the prefix's records
  if constexpr (P::kShared) {
    before = flowkv::splits_of(std::min(std::max(rq.base + i + 1, 0), reach.shift), a.prefix_split);
    n += before;
  }
  const int64_t rec = orow * a.splits;
  // record s: those of the prefix, then those behind them
  auto at_of = [&](int32_t s) {
    if constexpr (P::kShared) return s < before ? s : s - before + a.first_split;
    else return s;
  };
  const int tid = kWavesPer == 1 ? ln : threadIdx.x;
  const float* sums = record_sums(a, kDh, rec) + 4 * (tid % kLanes);
  const f32x2u* ml = record_ml(a, kDh, rec);
  Running x{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
  for (int32_t s = tid / kLanes; s < n; s += kParts * kMergeChunk) {
    Running y[kMergeChunk];
#pragma unroll
    for (int j = 0; j < kMergeChunk; ++j) {      // (past the end: the first record, not used)
      const int32_t at = s + j * kParts < n ? at_of(s + j * kParts) : at_of(0);
      const f32x2u m = ml[at];
      y[j] = Running{m[0], m[1], *reinterpret_cast<const f32x4u*>(sums + int64_t(at) * kDh)};
    }
#pragma unroll
    for (int j = 0; j < kMergeChunk; ++j)
      if (s + j * kParts < n) x = join(x, y[j]);
  }
#pragma unroll
  for (int off = kLanes; off < 64; off *= 2) {
    Running y;
    y.m = __shfl_xor(x.m, off);
    y.l = __shfl_xor(x.l, off);
#pragma unroll
    for (int k = 0; k < 4; ++k) y.v[k] = __shfl_xor(x.v[k], off);
    x = join(x, y);
  }
  if constexpr (kWavesPer > 1) {
    __shared__ float s_ml[kWavesPer][2];
    __shared__ f32x4 s_v[kWavesPer][kLanes];
    if (ln < kLanes) s_v[wave][ln] = x.v;
    if (ln == 0) {
      s_ml[wave][0] = x.m;
      s_ml[wave][1] = x.l;
    }
    __syncthreads();
    if (threadIdx.x >= kLanes) return;
    x = Running{s_ml[0][0], s_ml[0][1], s_v[0][ln]};
#pragma unroll
    for (int k = 1; k < kWavesPer; ++k) x = join(x, Running{s_ml[k][0], s_ml[k][1], s_v[k][ln]});
  }
  if (ln < kLanes) {
    const float inv = x.l == 0.f ? 0.f : 1.f / x.l;
    const u32x2 y = {T::pack(x.v[0] * inv, x.v[1] * inv), T::pack(x.v[2] * inv, x.v[3] * inv)};
    *reinterpret_cast<u32x2*>(a.out + orow * kDh + 4 * ln) = y;
  }
}

}  // namespace chunk
}  // namespace flowkv
