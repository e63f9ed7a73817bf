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

template <class F, class P>
__global__ __launch_bounds__(F::kThreads, 2 * F::kPerCu)
void prefix_attn(const SpanArgs a) {
  attend_many<F, false, P>(a);
}
template <int kDh, int kC, class P>
__global__ __launch_bounds__(kFewThreads, few_per_cu(kDh, kC))
void prefix_attn_few(const SpanArgs a) {
  attend_few<kDh, kC, P>(a);
}
// Behind the prefix: four waves, or eight where there are no more workgroups than CUs.
template <int kDh, int kC, int kWaves, class P>
__global__ __launch_bounds__(64 * kWaves, kWaves == kFewWaves ? few_per_cu(kDh, kC) : 2)
void prefix_attn_own(const SpanArgs a) {
  attend_few<kDh, kC, P, kFewOwn, kWaves>(a);
}
template <int kDh, int kWavesPer, class T>
__global__ __launch_bounds__(kMergeThreads) void prefix_attn_merge(const SpanArgs a) {
  merge_splits<kDh, kWavesPer, Own<T>>(a);
}

// ---- each request by itself ----------------------------------------------------------------

template <class F, bool kCut>
__global__ __launch_bounds__(F::kThreads, 2 * F::kPerCu)
void alone_attn(const ChunkArgs a) {
  attend_many<F, kCut, Causal<Fp16>>(a);
}
template <class F>
__global__ __launch_bounds__(2 * F::kDh) void alone_attn_join(const ChunkArgs a) {
  join_pieces<F, Fp16>(a);
}
template <int kDh, int kC>
__global__ __launch_bounds__(kFewThreads, few_per_cu(kDh, kC))
void alone_attn_few(const ChunkArgs a) {
  attend_few<kDh, kC, Causal<Fp16>>(a);
}
template <int kDh, int kWavesPer>
__global__ __launch_bounds__(kMergeThreads) void alone_attn_merge(const ChunkArgs a) {
  merge_splits<kDh, kWavesPer, Causal<Fp16>>(a);
}

struct Alone {
  template <class F>
  static const void* many(bool cut) {
    return cut ? reinterpret_cast<const void*>(alone_attn<F, true>)
               : reinterpret_cast<const void*>(alone_attn<F, false>);
  }
  template <class F>
  static const void* join() {
    return reinterpret_cast<const void*>(alone_attn_join<F>);
  }
  template <int kDh, int kC>
  static const void* few() {
    return reinterpret_cast<const void*>(alone_attn_few<kDh, kC>);
  }
  template <int kDh, int kWavesPer>
  static const void* merge() {
    return reinterpret_cast<const void*>(alone_attn_merge<kDh, kWavesPer>);
  }
};

const Kernels& alone(int32_t dtype) {
  static const Kernels fp16 = kernels_of<Alone>();
  return dtype == FLOWKV_BF16 ? causal_bf16() : fp16;
}

// ---- the host's part -----------------------------------------------------------------------

// The forms of the parts, as Kernels has them; 256 rows for prefixes alone.
struct Parts {
  const void* prefix[4][2];
  const void* own[3][2];
  const void* own_wide[2][2];                    // eight waves
  const void* merge[2][2];
};
template <class T>
Parts parts_of() {
  auto ptr = [](void (*fn)(SpanArgs)) { return reinterpret_cast<const void*>(fn); };
  typedef Prefixed<T> P;
  typedef Own<T> O;
  return Parts{{{ptr(prefix_attn_few<64, 1, P>), ptr(prefix_attn_few<128, 1, P>)},
                {ptr(prefix_attn_few<64, 2, P>), ptr(prefix_attn_few<128, 2, P>)},
                {ptr(prefix_attn<Form<64, 4, 2>, P>), ptr(prefix_attn<Form<128, 4, 2>, P>)},
                {ptr(prefix_attn<Form<64, 8, 1>, P>), ptr(prefix_attn<Form<128, 8, 1>, P>)}},
               {{ptr(prefix_attn_own<64, 1, 4, O>), ptr(prefix_attn_own<128, 1, 4, O>)},
                {ptr(prefix_attn_own<64, 2, 4, O>), ptr(prefix_attn_own<128, 2, 4, O>)},
                {ptr(prefix_attn<Form<64, 4, 2>, O>), ptr(prefix_attn<Form<128, 4, 2>, O>)}},
               {{ptr(prefix_attn_own<64, 1, 8, O>), ptr(prefix_attn_own<128, 1, 8, O>)},
                {ptr(prefix_attn_own<64, 2, 8, O>), ptr(prefix_attn_own<128, 2, 8, O>)}},
               {{ptr(prefix_attn_merge<64, 1, T>), ptr(prefix_attn_merge<64, 4, T>)},
                {ptr(prefix_attn_merge<128, 1, T>), ptr(prefix_attn_merge<128, 4, T>)}}};
}
const Parts& parts(int32_t dtype) {
  static const Parts bf16 = parts_of<Bf16>(), fp16 = parts_of<Fp16>();
  return dtype == FLOWKV_BF16 ? bf16 : fp16;
}

// Forms of a part: rows of a tile, threads.
constexpr int kRows[4] = {16, 32, 128, 256};
constexpr int kThreads[4] = {kFewThreads, kFewThreads, 512, 512};
constexpr int kWideThreads = 512;

struct Plan {
  bool shared;                 // false: each request by itself, `sh`
  Shape sh;
  int prefix_kind, own_kind;
  bool wide;                                     // eight waves behind the prefix
  int32_t prefix_split, own_split;
  int64_t prefix_splits, own_splits;             // records of a row
  int64_t need;
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
  // (its checks of the sizes hold for either way)
  const int rc = plan_shape(alone(FLOWKV_BF16), n_tokens, n_req, q_heads, kv_heads, head_dim,
                            max_new, Span{int32_t(longest)}, 0, &out->sh);
  if (rc) return rc;
  if (split_tokens < 0 || split_tokens % kSplitUnit)
    return fail(FLOWKV_EINVAL, "split_tokens %d: need 0 or a multiple of %d", split_tokens,
                kSplitUnit);
  const int group = q_heads / kv_heads;
  const int64_t together = int64_t(max_group) * group, one = int64_t(max_new) * group;
  out->shared = n_groups > 0 && max_prefix > 0 &&
                (split_tokens > 0 || (n_req > n_groups && one <= 128 && max_prefix >= 512));
  if (!out->shared) {
    out->need = out->sh.need;
    return FLOWKV_OK;
  }
  out->prefix_kind = together <= 16 ? 0 : together <= 32 ? 1 : 2;
  if (tiles_of(n_tokens, n_groups, group, max_group, 256) * kv_heads >= kCus) out->prefix_kind = 3;
  out->own_kind = one <= 16 ? 0 : one <= 64 ? 1 : 2;
  constexpr int64_t kAll = INT32_MAX / kSplitUnit * kSplitUnit;
  auto tiles_at = [&](int kind, int64_t units, int64_t most_new) {
    return std::max<int64_t>(tiles_of(n_tokens, units, group, most_new, kRows[kind]) * kv_heads,
                             1);
  };
  auto split_of = [&](int kind, int64_t tiles, int32_t tokens, int64_t most) {
    if (kind > 1) most = kAll;
    if (split_tokens > 0) return int32_t(std::min<int64_t>(split_tokens, most));
    return best_split(tiles, tokens, kind <= 1 ? 300 : 500, most);
  };
  const int64_t own_tiles = tiles_at(out->own_kind, n_req, max_new);
  out->prefix_split = split_of(out->prefix_kind, tiles_at(out->prefix_kind, n_groups, max_group),
                               max_prefix, kFewSplit);
  out->own_split = split_of(out->own_kind, own_tiles, max_own, kFewOwn);
  auto splits_of = [](int32_t tokens, int32_t split) {
    return std::max<int64_t>((int64_t(tokens) + split - 1) / split, 1);
  };
  out->prefix_splits = splits_of(max_prefix, out->prefix_split);
  out->own_splits = splits_of(max_own, out->own_split);
  out->wide = out->own_kind <= 1 && own_tiles * out->own_splits <= kCus;
  if (__builtin_mul_overflow(int64_t(n_tokens) * q_heads,
                             int64_t((head_dim + 2) * sizeof(float)), &out->need) ||
      __builtin_mul_overflow(out->need, out->prefix_splits + out->own_splits, &out->need))
    return fail(FLOWKV_EINVAL, "%lld splits: the workspace's size overflows",
                (long long)(out->prefix_splits + out->own_splits));
  return FLOWKV_OK;
}

// A part of units (requests or groups): its workgroups, or a failure where they are too many.
int part_grid(const ChunkArgs& a, int kind, int threads, int64_t n_units, int64_t splits,
              int64_t* grid) {
  const int64_t tiles = tile_slots(a.n_tokens, n_units, a.group, kRows[kind]) * a.kv_heads;
  if (tiles > UINT32_MAX / threads / splits)  // lanes of a launch in 32 bits
    return fail(FLOWKV_EINVAL, "%lld tiles of queries x %lld splits: too many for one call",
                (long long)tiles, (long long)splits);
  *grid = tiles * splits;
  return FLOWKV_OK;
}

hipError_t launch_part(const void* fn, int kind, int threads, int64_t grid, int64_t splits,
                       int32_t split_tokens, SpanArgs& a, hipStream_t stream) {
  a.split_tokens = split_tokens;
  a.tiles = int32_t(grid / splits / a.kv_heads);
  a.row_shift = 0;
  while (1 << a.row_shift < kRows[kind]) ++a.row_shift;
  void* args[] = {&a};
  return hipLaunchKernel(fn, dim3(unsigned(grid)), dim3(unsigned(threads)), args, 0,
                         stream);
}

int launch_parts(int32_t dtype, const Plan& p, int head_dim, SpanArgs& a, hipStream_t stream) {
  const Parts& fn = parts(dtype);
  const int d128 = head_dim == 128;
  const int64_t splits = p.prefix_splits + p.own_splits;
  const int64_t out_rows = int64_t(a.n_tokens) * a.q_heads;
  const bool one = splits <= kMergeChunk * 64 * 4 / head_dim;
  const int64_t merge = one ? (out_rows + 3) / 4 : out_rows;
  if (merge > UINT32_MAX / kMergeThreads || splits > INT32_MAX)
    return fail(FLOWKV_EINVAL, "%lld rows of output x %lld splits: too many for one call",
                (long long)out_rows, (long long)splits);
  int64_t prefix_grid, own_grid;
  const int prefix_threads = kThreads[p.prefix_kind];
  const int own_threads = p.wide ? kWideThreads : kThreads[p.own_kind];
  int rc = part_grid(a, p.prefix_kind, prefix_threads, a.n_groups, p.prefix_splits, &prefix_grid);
  if (rc) return rc;
  rc = part_grid(a, p.own_kind, own_threads, a.n_req, p.own_splits, &own_grid);
  if (rc) return rc;
  a.splits = int32_t(splits);
  a.first_split = int32_t(p.prefix_splits);
  a.prefix_split = p.prefix_split;
  void* args[] = {&a};
  hipError_t e = launch_part(fn.prefix[p.prefix_kind][d128], p.prefix_kind, prefix_threads,
                             prefix_grid, p.prefix_splits, p.prefix_split, a, stream);
  if (e == hipSuccess)
    e = launch_part(p.wide ? fn.own_wide[p.own_kind][d128] : fn.own[p.own_kind][d128], p.own_kind,
                    own_threads, own_grid, p.own_splits, p.own_split, a, stream);
  // (one split behind the prefix, of few rows: its workgroup joins them)
  if (e == hipSuccess && (p.own_splits > 1 || p.own_kind > 1))
    e = hipLaunchKernel(fn.merge[d128][!one], dim3(unsigned(merge)), dim3(kMergeThreads), args, 0,
                        stream);
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
  return launch<ChunkArgs>(alone(dtype), p.sh, max_new, head_dim, a, c.stream);
}
