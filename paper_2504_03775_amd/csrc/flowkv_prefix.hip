// Attention of new tokens for requests that share a long prefix, over the paged cache, for
// gfx950 (MI355X).
//
// Requests whose block lists begin with the same blocks (flowkv_share, flowkv_fork) read the
// same K and V there.  The softmax over a row's tokens falls into a part over the prefix and
// one over the tokens behind it, each with its own reference and sum:
//   out = (2^(m1 - m) O1 + 2^(m2 - m) O2) / (2^(m1 - m) l1 + 2^(m2 - m) l2),  m = max(m1, m2)
// The first is done for the rows of all the group's requests together, so that the prefix is
// read once a group and its products fill whole tiles; the second for each request.  The
// parts' records are joined in a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "flowkv.h"
#include "flowkv_chunk_host.h"
#include "flowkv_chunk_kernels.h"
#include "flowkv_status.h"

using flowkv::fail;
using flowkv::ok;

namespace {

using namespace flowkv::chunk;

// ---- over a group's prefix, over what is behind it, and their join ----------------------

// Few rows: both in one launch.  A tile of 16 or 32 rows of a group reads the prefix through its
// XCD's L2, so what its CU draws bounds it, some 45 bytes a nanosecond.  32 single tokens behind
// 13,000, 32 heads of 128 on 8: 27 us, of them 2 to find the group, 3 to look up its block list and
// rows and 18 for 52 steps of 32 tokens (four tiles of 32 rows draw 213 MB between them, 46 bytes a
// nanosecond and CU; 1.4 us for each of a wave's 13 steps), 2 for its records; 4 more of join.
// Behind 4,000 and 100 to 2,500 of their own, 64 of them: 88 us, memory's 60 and the last
// workgroups' end.
template <int kDh, int kC, class T>
__global__ __launch_bounds__(kFewThreads, few_per_cu(kDh, kC))
void prefix_attn_few(const SpanArgs a) {
  attend_few<kDh, kC, Shared<T>>(a);
}
// Many rows: prefixes alone.
template <class F, class T>
__global__ __launch_bounds__(F::kThreads, 2 * F::kPerCu)
void prefix_attn(const SpanArgs a) {
  attend_many<F, false, Prefixed<T>>(a);
}
template <int kDh, int kWavesPer, class T>
__global__ __launch_bounds__(kMergeThreads) void prefix_attn_merge(const SpanArgs a) {
  merge_splits<kDh, kWavesPer, Shared<T>>(a);
}

// ---- each request by itself ----------------------------------------------------------------

template <class F, bool kCut, class T>
__global__ __launch_bounds__(F::kThreads, 2 * F::kPerCu)
void alone_attn(const SpanArgs a) {
  attend_many<F, kCut, Alone<T>>(a);
}
template <class F, class T>
__global__ __launch_bounds__(2 * F::kDh) void alone_attn_join(const SpanArgs a) {
  join_pieces<F, T>(a);
}
template <int kDh, int kC, class T>
__global__ __launch_bounds__(kFewThreads, few_per_cu(kDh, kC))
void alone_attn_few(const SpanArgs a) {
  attend_few<kDh, kC, Alone<T>>(a);
}
template <int kDh, int kWavesPer, class T>
__global__ __launch_bounds__(kMergeThreads) void alone_attn_merge(const SpanArgs a) {
  merge_splits<kDh, kWavesPer, Alone<T>>(a);
}

template <class T>
struct AloneTable {
  template <class F>
  static const void* many(bool cut) {
    return cut ? reinterpret_cast<const void*>(alone_attn<F, true, T>)
               : reinterpret_cast<const void*>(alone_attn<F, false, T>);
  }
  template <class F>
  static const void* join() {
    return reinterpret_cast<const void*>(alone_attn_join<F, T>);
  }
  template <int kDh, int kC>
  static const void* few() {
    return reinterpret_cast<const void*>(alone_attn_few<kDh, kC, T>);
  }
  template <int kDh, int kWavesPer>
  static const void* merge() {
    return reinterpret_cast<const void*>(alone_attn_merge<kDh, kWavesPer, T>);
  }
};

const Kernels& alone(int32_t dtype) {
  static const Kernels bf16 = kernels_of<AloneTable<Bf16>>(),
                       fp16 = kernels_of<AloneTable<Fp16>>();
  return dtype == FLOWKV_BF16 ? bf16 : fp16;
}

// ---- the host's part -----------------------------------------------------------------------

struct Parts {
  const void* few[2][2];       // 16, 32 rows; head_dim
  const void* many[2];         // 128 rows; head_dim
  const void* merge[2][2];     // head_dim; a wave or four a row
};
template <class T>
Parts parts_of() {
  auto ptr = [](void (*fn)(SpanArgs)) { return reinterpret_cast<const void*>(fn); };
  return Parts{{{ptr(prefix_attn_few<64, 1, T>), ptr(prefix_attn_few<128, 1, T>)},
                {ptr(prefix_attn_few<64, 2, T>), ptr(prefix_attn_few<128, 2, T>)}},
               {ptr(prefix_attn<Form<64, 4, 2>, T>), ptr(prefix_attn<Form<128, 4, 2>, T>)},
               {{ptr(prefix_attn_merge<64, 1, T>), ptr(prefix_attn_merge<64, 4, T>)},
                {ptr(prefix_attn_merge<128, 1, T>), ptr(prefix_attn_merge<128, 4, T>)}}};
}
const Parts& parts(int32_t dtype) {
  static const Parts bf16 = parts_of<Bf16>(), fp16 = parts_of<Fp16>();
  return dtype == FLOWKV_BF16 ? bf16 : fp16;
}

// Bytes of prefixes that tiles of 32 rows of a group read less than its requests would, each by
// itself, from which on the join's launch is worth it.  (In a graph, us shared and each by itself.
// 8 KV heads of 128: 2 requests behind 5,000 tokens, 20 MiB saved, 12.7 and 12.7; behind 8,000,
// 31 MiB, 14.4 and 15.9; 16 behind 500, 27 MiB, 13.7 and 12.5; behind 1,000, 55 MiB, 14.3 and
// 15.4; 4 behind 8,000, 94 MiB, 14.7 and 29.3; one KV head: 16 behind 2,000, 12 MiB, 14.0 and
// 11.4; 48 behind 1,500, 26 MiB, 14.3 and 14.1.  So up to some 50 MiB the one or the other may be
// sooner, by up to 4 us: few long reads gain early, many short ones late.  Requests of no group
// count as if they shared: the host does not know them.)
constexpr int64_t kLeastSaved = int64_t(24) << 20;
// Rows a request, on average, up to which it is: the tiles of all of them are then few beside
// those of the requests; and where the longest brings four times as many and more, so that most
// bring few.  (us, each by itself and shared.  8 KV heads of 128, groups of 4, 64 requests of 16
// tokens, 64 rows, behind 2,000, 111 and 102, behind 8,000, 335 and 207; of 17, 101 and 143, 310
// and 277; of 32, 123 and 181, 359 and 390.  63 single tokens beside one of 17, 5 rows a request,
// behind 4,000, 169 and 36; beside one of 512, 36 rows, 221 and 113, behind 1,000 80 and 67, behind
// 500 55 and 60; beside one of 1,500, 98 rows, behind 2,000 183 and 192, behind 4,000 303 and 252;
// beside one of 2,048, 132 rows, 351 and 381.  One KV head, groups of 8: the 63 beside one of 512,
// 72 rows, 66 and 45, beside one of 850, 114 rows, 74 and 68.)
constexpr int64_t kMostRows = 64, kMostRowsMixed = 112;
// Bytes that they read, through their L2s, from which on tiles of 128 rows in a launch of their
// own are sooner done: they are bound by the matrix units, at less than half of the time.  (64
// requests behind 13,000 tokens, 426 MB: 45.0 and 44.7 us; 128: 81 and 65; 250: 152 and 108; 250
// behind 2,000, 260 MB: 54 and 62.)
constexpr int64_t kMostRead = int64_t(400) << 20;

struct Plan {
  bool shared;                 // false: each request by itself, `sh`
  Shape sh;
  int few_rows;                // of a tile behind a prefix, 16 or 32
  int many_rows;               // of a tile over a prefix, in a launch of its own; 0: few_rows
  int32_t prefix_split, own_split;
  int64_t prefix_splits, own_splits;             // records of a row
  int64_t prefix_items, own_tiles;               // tile slots of prefixes, and behind them
  int64_t merge;                                 // workgroups of the join,
  bool one, fits;                                // a wave a row; lanes of a launch in 32 bits
  int64_t need;
  int prefix_rows() const { return many_rows ? many_rows : few_rows; }
};

int plan(int32_t n_tokens, int32_t n_req, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
         int32_t n_groups, int32_t max_new, int32_t max_group, int32_t max_own,
         int32_t max_prefix, int32_t split_tokens, Plan* out) {
  if (n_groups < 0 || max_group < 0 || max_own < 0 || max_prefix < 0)
    return fail(FLOWKV_EINVAL, "negative sizes");
  const int64_t longest = int64_t(max_prefix) + max_own;
  if (longest > INT32_MAX - 4096)
    return fail(FLOWKV_EINVAL, "%lld tokens of a prefix and behind it: need at most 2^31 - 4097",
                (long long)longest);
  const bool groups = n_groups > 0 && max_prefix > 0;
  // (its checks of the sizes hold for either way; with split_tokens and groups the plan is shared)
  const int rc = plan_shape(alone(FLOWKV_BF16), n_tokens, n_req, q_heads, kv_heads, head_dim,
                            max_new, Span{int32_t(longest)}, groups ? 0 : split_tokens, true,
                            &out->sh);
  if (rc) return rc;
  if (split_tokens < 0 || split_tokens % kSplitUnit)
    return fail(FLOWKV_EINVAL, "split_tokens %d: need 0 or a multiple of %d", split_tokens,
                kSplitUnit);
  const int group = q_heads / kv_heads;
  const int64_t one = int64_t(max_new) * group;  // rows of a request, at most
  auto tiles_at = [&](int64_t units, int64_t most_new, int rows) {
    return std::max<int64_t>(tiles_of(n_tokens, units, group, most_new, rows) * kv_heads, 1);
  };
  const int64_t rows =                           // of all requests, no padding; on average
      std::min(int64_t(n_tokens), int64_t(n_req) * max_new) * group;
  const int64_t each = rows / std::max(n_req, 1);
  const int64_t tiles32 = tiles_of(n_tokens, n_groups, group, max_group, 32);
  const int64_t alone32 = tiles_of(n_tokens, n_req, group, max_new, 32);
  // (in double: tiles of it pass 63 bits where max_prefix is set to the most there can be)
  const double prefix_bytes = double(max_prefix) * kv_heads * head_dim * 4;
  out->shared = groups &&
                (split_tokens > 0 ||
                 (rows <= (one >= 4 * each ? kMostRowsMixed : kMostRows) * n_req &&
                  double(alone32 - tiles32) * prefix_bytes >= double(kLeastSaved)));
  // Tiles of 32 rows halve what a prefix is read, with two workgroups a CU instead of three.
  const bool many = split_tokens > kFewSplit ||
                    (split_tokens == 0 && double(tiles32) * prefix_bytes >= double(kMostRead));
  out->few_rows = (many || int64_t(max_group) * group <= 16) && one <= 16 ? 16 : 32;
  out->many_rows = many ? 128 : 0;
  constexpr int64_t kAll = INT32_MAX / kSplitUnit * kSplitUnit;
  auto split_of = [&](int64_t tiles, int32_t tokens, int64_t fixed, int64_t most) {
    if (split_tokens > 0) return int32_t(std::min<int64_t>(split_tokens, most));
    return best_split(tiles, tokens, fixed, most);
  };
  const int64_t prefix_tiles = tiles_at(n_groups, max_group, out->prefix_rows());
  out->prefix_split = split_of(prefix_tiles, max_prefix, out->many_rows ? 500 : 300,
                               out->many_rows ? kAll : kFewSplit);
  out->own_split = split_of(tiles_at(n_req, max_new, out->few_rows), max_own, 300, kFewSplit);
  auto splits_of = [](int32_t tokens, int32_t split) {
    return std::max<int64_t>((int64_t(tokens) + split - 1) / split, 1);
  };
  out->prefix_splits = splits_of(max_prefix, out->prefix_split);
  out->own_splits = splits_of(max_own, out->own_split);
  const int64_t splits = out->prefix_splits + out->own_splits;
  const int64_t out_rows = int64_t(n_tokens) * q_heads;
  out->one = splits <= kMergeChunk * 64 * 4 / head_dim;
  out->merge = out->one ? (out_rows + 3) / 4 : out_rows;
  out->prefix_items = tile_slots(n_tokens, n_groups, group, out->prefix_rows());
  out->own_tiles = tile_slots(n_tokens, n_req, group, out->few_rows);
  // lanes of a launch in 32 bits: workgroups of prefixes and behind them, of a KV head
  auto left = [&](int64_t most, int64_t items, int64_t each) {     // negative: too many
    return each <= most && items <= most / each ? most - items * each : -1;
  };
  const int64_t most = UINT32_MAX / kFewThreads / kv_heads;
  const int64_t room =
      left(many ? UINT32_MAX / 512 / kv_heads : most, out->prefix_items, out->prefix_splits);
  out->fits = splits <= INT32_MAX && out->merge <= UINT32_MAX / kMergeThreads &&
              left(many && room >= 0 ? most : room, out->own_tiles, out->own_splits) >= 0;
  const bool overflows = __builtin_mul_overflow(out_rows, int64_t((head_dim + 2) * sizeof(float)),
                                                &out->need) ||
                         __builtin_mul_overflow(out->need, splits, &out->need);
  // (the rule takes no plan that is refused where the other is not)
  if (split_tokens == 0 && (overflows || !out->fits) &&
      grid_of(alone(FLOWKV_BF16), out->sh, n_tokens, n_req, q_heads, kv_heads, head_dim).fits)
    out->shared = false;
  if (!out->shared) {
    out->need = out->sh.need;
    return FLOWKV_OK;
  }
  if (overflows)
    return fail(FLOWKV_EINVAL, "%lld splits: the workspace's size overflows", (long long)splits);
  return FLOWKV_OK;
}

int row_shift(int rows) {
  int shift = 0;
  while (1 << shift < rows) ++shift;
  return shift;
}

int launch_parts(int32_t dtype, const Plan& p, int head_dim, SpanArgs& a, hipStream_t stream) {
  const Parts& fn = parts(dtype);
  const int d128 = head_dim == 128, kv = a.kv_heads;
  const int64_t splits = p.prefix_splits + p.own_splits;
  if (!p.fits)
    return fail(FLOWKV_EINVAL,
                "%lld tiles of prefixes x %lld splits, %lld behind them x %lld: too many for one "
                "call", (long long)p.prefix_items, (long long)p.prefix_splits,
                (long long)p.own_tiles, (long long)p.own_splits);
  a.splits = int32_t(splits);
  a.first_split = int32_t(p.prefix_splits);
  a.prefix_split = p.prefix_split;
  void* args[] = {&a};
  hipError_t e = hipSuccess;
  if (p.many_rows) {
    a.split_tokens = p.prefix_split;
    a.row_shift = row_shift(p.many_rows);
    e = hipLaunchKernel(fn.many[d128],
                        dim3(unsigned(p.prefix_items * p.prefix_splits * kv)), dim3(512), args, 0,
                        stream);
  }
  a.prefix_items = p.many_rows ? 0 : uint32_t(p.prefix_items * p.prefix_splits);
  a.split_tokens = p.own_split;
  a.row_shift = row_shift(p.few_rows);
  a.tiles = int32_t(p.own_tiles);
  if (e == hipSuccess)
    e = hipLaunchKernel(fn.few[p.few_rows == 32][d128],
                        dim3(unsigned((a.prefix_items + p.own_tiles * p.own_splits) * kv)),
                        dim3(kFewThreads), args, 0, stream);
  if (e == hipSuccess)
    e = hipLaunchKernel(fn.merge[d128][!p.one], dim3(unsigned(p.merge)), dim3(kMergeThreads), args,
                        0, stream);
  if (e == hipSuccess) e = hipGetLastError();
  if (e != hipSuccess)
    return fail(FLOWKV_EHIP, "prefix attention launch: %s", hipGetErrorString(e));
  return ok();
}

}  // namespace

extern "C" int flowkv_prefix_attention_workspace(int32_t n_tokens, int32_t n_req, int32_t q_heads,
                                                 int32_t kv_heads, int32_t head_dim,
                                                 int32_t n_groups, int32_t max_new,
                                                 int32_t max_group, int32_t max_own,
                                                 int32_t max_prefix, int32_t split_tokens,
                                                 int64_t* bytes) {
  if (!bytes) return fail(FLOWKV_EINVAL, "NULL output");
  Plan p;
  const int rc = plan(n_tokens, n_req, q_heads, kv_heads, head_dim, n_groups, max_new, max_group,
                      max_own, max_prefix, split_tokens, &p);
  if (rc) return rc;
  *bytes = p.need;
  return ok();
}

extern "C" int flowkv_prefix_attention(
    const flowkv_pool* pool, int32_t layer, int32_t dtype, const void* q_dev, int64_t q_stride,
    int32_t n_tokens, int32_t n_req, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
    const int32_t* offsets_dev, const int32_t* block_tables_dev, int32_t max_blocks,
    const int32_t* seq_lens_dev, int32_t n_groups, const int32_t* groups_dev,
    const int32_t* prefix_lens_dev, int32_t max_new, int32_t max_group, int32_t max_own,
    int32_t max_prefix, float scale, int32_t split_tokens, void* out_dev, void* workspace_dev,
    int64_t workspace_bytes, void* hip_stream) {
  Call c = {pool,        layer,       q_dev,         q_stride,        n_tokens,
            n_req,       q_heads,     kv_heads,      head_dim,        offsets_dev,
            block_tables_dev,         max_blocks,    seq_lens_dev,    0,
            scale,       out_dev,     workspace_dev, workspace_bytes,
            static_cast<hipStream_t>(hip_stream)};
  int rc = check_pool(c);
  if (rc) return rc;
  rc = check_16_bits(dtype);
  if (rc) return rc;
  Plan p;
  rc = plan(n_tokens, n_req, q_heads, kv_heads, head_dim, n_groups, max_new, max_group, max_own,
            max_prefix, split_tokens, &p);
  if (rc) return rc;
  c.max_seq_len = max_prefix + max_own;
  rc = check_sizes(c);
  if (rc) return rc;
  if (c.empty()) return ok();
  if (n_groups > 0 && (!groups_dev || !prefix_lens_dev))
    return fail(FLOWKV_EINVAL, "NULL device pointer");
  rc = check_buffers(c, p.need);
  if (rc) return rc;
  SpanArgs a{};
  fill(c, &a);
  a.groups = groups_dev;
  a.prefix_lens = prefix_lens_dev;
  a.n_groups = n_groups;
  a.max_prefix = max_prefix;
  a.max_own = max_own;
  if (p.shared) return launch_parts(dtype, p, head_dim, a, c.stream);
  return launch(alone(dtype), p.sh, max_new, head_dim, a, c.stream);
}
