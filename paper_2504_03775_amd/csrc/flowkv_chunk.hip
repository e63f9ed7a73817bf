// Attention of a chunk of new tokens over the paged cache, for gfx950 (MI355X).
//
// The prefill counterpart of decode attention (FlowKV, arXiv 2504.03775, section
// 3.3: attention reads the pool in either layout of Eq. 5 through a request's
// block list): each request brings some new tokens whose K and V are in the pool
// already, and query i of them attends to every token up to its own position.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "flowkv.h"
#include "flowkv_chunk_host.h"
#include "flowkv_chunk_kernels.h"
#include "flowkv_status.h"

using flowkv::fail;
using flowkv::ok;

namespace {

using namespace flowkv::chunk;

typedef Causal<Bf16> Policy;

template <class F, bool kCut>
__global__ __launch_bounds__(F::kThreads, 2 * F::kPerCu)
void chunk_attn(const ChunkArgs a) {
  attend_many<F, kCut, Policy>(a);
}
template <class F>
__global__ __launch_bounds__(2 * F::kDh) void chunk_attn_join(const ChunkArgs a) {
  join_pieces<F, Bf16>(a);
}
template <int kDh, int kC>
__global__ __launch_bounds__(kFewThreads, few_per_cu(kDh, kC))
void chunk_attn_few(const ChunkArgs a) {
  attend_few<kDh, kC, Policy>(a);
}
template <int kDh, int kWavesPer>
__global__ __launch_bounds__(kMergeThreads) void chunk_attn_merge(const ChunkArgs a) {
  merge_splits<kDh, kWavesPer, Policy>(a);
}

struct Table {
  template <class F>
  static const void* many(bool cut) {
    return cut ? reinterpret_cast<const void*>(chunk_attn<F, true>)
               : reinterpret_cast<const void*>(chunk_attn<F, false>);
  }
  template <class F>
  static const void* join() {
    return reinterpret_cast<const void*>(chunk_attn_join<F>);
  }
  template <int kDh, int kC>
  static const void* few() {
    return reinterpret_cast<const void*>(chunk_attn_few<kDh, kC>);
  }
  template <int kDh, int kWavesPer>
  static const void* merge() {
    return reinterpret_cast<const void*>(chunk_attn_merge<kDh, kWavesPer>);
  }
};

const Kernels& kernels() {
  static const Kernels k = kernels_of<Table>();
  return k;
}

}  // namespace

extern "C" int flowkv_chunk_attention_workspace(int32_t n_tokens, int32_t n_req, int32_t q_heads,
                                                int32_t kv_heads, int32_t head_dim,
                                                int32_t max_new, int32_t max_seq_len,
                                                int32_t split_tokens, int64_t* bytes) {
  if (!bytes) return fail(FLOWKV_EINVAL, "NULL output");
  Shape sh;
  const int rc = plan_shape(kernels(), n_tokens, n_req, q_heads, kv_heads, head_dim, max_new,
                            Span{max_seq_len}, split_tokens, false, &sh);
  if (rc) return rc;
  *bytes = sh.need;
  return ok();
}

extern "C" int flowkv_chunk_attention(const flowkv_pool* pool, int32_t layer, const void* q_dev,
                                      int64_t q_stride, int32_t n_tokens, int32_t n_req,
                                      int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                      const int32_t* offsets_dev, const int32_t* block_tables_dev,
                                      int32_t max_blocks, const int32_t* seq_lens_dev,
                                      int32_t max_new, int32_t max_seq_len, float scale,
                                      int32_t split_tokens, void* out_dev, void* workspace_dev,
                                      int64_t workspace_bytes, void* hip_stream) {
  const Call c = {pool,        layer,       q_dev,         q_stride,        n_tokens,
                  n_req,       q_heads,     kv_heads,      head_dim,        offsets_dev,
                  block_tables_dev,         max_blocks,    seq_lens_dev,    max_seq_len,
                  scale,       out_dev,     workspace_dev, workspace_bytes,
                  static_cast<hipStream_t>(hip_stream)};
  int rc = check_pool(c);
  if (rc) return rc;
  Shape sh;
  rc = plan_shape(kernels(), n_tokens, n_req, q_heads, kv_heads, head_dim, max_new,
                  Span{max_seq_len}, split_tokens, false, &sh);
  if (rc) return rc;
  rc = check_sizes(c);
  if (rc) return rc;
  if (c.empty()) return ok();
  rc = check_buffers(c, sh.need);
  if (rc) return rc;
  ChunkArgs a{};
  fill(c, &a);
  return launch(kernels(), sh, max_new, head_dim, a, c.stream);
}
