// Attention of new tokens through a sliding window, with a few first tokens that stay
// visible, over the paged cache, for gfx950 (MI355X).
//
// A new token at position p sees token t <= p if t > p - window or t < sinks.  The forms are
// those of attention over all of the cache (flowkv_chunk_kernels.h).  A tile of rows goes
// through the first `sinks` tokens and then those from its first row's window on, counted
// without the gap between: steps, splits and pieces know nothing of it, only the lookup of a
// token's place does.  Rows of a tile differ by a few tokens in where their window begins;
// the steps that lie across it are masked as those across the diagonal are.
//
// What bounds it: few rows, HBM (32 single tokens through a window of 4,096, 8 KV heads of 128,
// 514 MB: 91 us, 5.65 TB/s, and 5 of join); many rows, the matrix and vector units by turns, as
// over all of the cache (13,000 tokens, 32 heads of 128 on 8, window 4,096: 748 to 802 us by the
// card, 0.92 to 0.98 PFLOP/s).
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

template <class F, bool kCut, class T>
__global__ __launch_bounds__(F::kThreads, 2 * F::kPerCu)
void window_attn(const SpanArgs a) {
  attend_many<F, kCut, Windowed<T>>(a);
}
template <class F, class T>
__global__ __launch_bounds__(2 * F::kDh) void window_attn_join(const SpanArgs a) {
  join_pieces<F, T>(a);
}
template <int kDh, int kC, class T>
__global__ __launch_bounds__(kFewThreads, few_per_cu(kDh, kC))
void window_attn_few(const SpanArgs a) {
  attend_few<kDh, kC, Windowed<T>>(a);
}
template <int kDh, int kWavesPer, class T>
__global__ __launch_bounds__(kMergeThreads) void window_attn_merge(const SpanArgs a) {
  merge_splits<kDh, kWavesPer, Windowed<T>>(a);
}

template <class T>
struct Table {
  template <class F>
  static const void* many(bool cut) {
    return cut ? reinterpret_cast<const void*>(window_attn<F, true, T>)
               : reinterpret_cast<const void*>(window_attn<F, false, T>);
  }
  template <class F>
  static const void* join() {
    return reinterpret_cast<const void*>(window_attn_join<F, T>);
  }
  template <int kDh, int kC>
  static const void* few() {
    return reinterpret_cast<const void*>(window_attn_few<kDh, kC, T>);
  }
  template <int kDh, int kWavesPer>
  static const void* merge() {
    return reinterpret_cast<const void*>(window_attn_merge<kDh, kWavesPer, T>);
  }
};

const Kernels& kernels(int32_t dtype) {
  static const Kernels bf16 = kernels_of<Table<Bf16>>(), fp16 = kernels_of<Table<Fp16>>();
  return dtype == FLOWKV_BF16 ? bf16 : fp16;
}

int plan(int32_t n_tokens, int32_t n_req, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
         int32_t max_new, int32_t max_seq_len, int32_t window, int32_t sinks,
         int32_t split_tokens, Shape* out) {
  if (window < 1 || sinks < 0)
    return fail(FLOWKV_EINVAL, "window of %d tokens and %d first ones: need 1 and 0 at least",
                window, sinks);
  return plan_shape(kernels(FLOWKV_BF16), n_tokens, n_req, q_heads, kv_heads, head_dim, max_new,
                    Span{max_seq_len, window, sinks}, split_tokens, true, out);
}

}  // namespace

extern "C" int flowkv_window_attention_workspace(int32_t n_tokens, int32_t n_req, int32_t q_heads,
                                                 int32_t kv_heads, int32_t head_dim,
                                                 int32_t max_new, int32_t max_seq_len,
                                                 int32_t window, int32_t sinks,
                                                 int32_t split_tokens, int64_t* bytes) {
  if (!bytes) return fail(FLOWKV_EINVAL, "NULL output");
  Shape sh;
  const int rc = plan(n_tokens, n_req, q_heads, kv_heads, head_dim, max_new, max_seq_len, window,
                      sinks, split_tokens, &sh);
  if (rc) return rc;
  *bytes = sh.need;
  return ok();
}

extern "C" int flowkv_window_attention(
    const flowkv_pool* pool, int32_t layer, int32_t dtype, const void* q_dev, int64_t q_stride,
    int32_t n_tokens, int32_t n_req, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
    const int32_t* offsets_dev, const int32_t* block_tables_dev, int32_t max_blocks,
    const int32_t* seq_lens_dev, int32_t max_new, int32_t max_seq_len, int32_t window,
    int32_t sinks, float scale, int32_t split_tokens, void* out_dev, void* workspace_dev,
    int64_t workspace_bytes, void* hip_stream) {
  const Call c = {pool,        layer,       q_dev,         q_stride,        n_tokens,
                  n_req,       q_heads,     kv_heads,      head_dim,        offsets_dev,
                  block_tables_dev,         max_blocks,    seq_lens_dev,    max_seq_len,
                  scale,       out_dev,     workspace_dev, workspace_bytes,
                  static_cast<hipStream_t>(hip_stream)};
  int rc = check_pool(c);
  if (rc) return rc;
  rc = check_16_bits(dtype);
  if (rc) return rc;
  Shape sh;
  rc = plan(n_tokens, n_req, q_heads, kv_heads, head_dim, max_new, max_seq_len, window, sinks,
            split_tokens, &sh);
  if (rc) return rc;
  rc = check_sizes(c);
  if (rc) return rc;
  if (c.empty()) return ok();
  rc = check_buffers(c, sh.need);
  if (rc) return rc;
  SpanArgs a{};
  fill(c, &a);
  a.window = window;
  a.sinks = sinks;
  return launch(kernels(dtype), sh, max_new, head_dim, a, c.stream);
}
