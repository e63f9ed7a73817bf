// New tokens' K and V appended to their requests' blocks with K, and the queries, rotated by
// their positions on the way, for gfx950 (MI355X).
//
// A position's angles come as a row of float32 cosines and sines.  Each pair (a, b) of a head's
// first rot_dim dims, with its angle's c and s, becomes
//   a' = a c - b s,  b' = a s + b c
// in float32, rounded once; the dims behind stay.  Pairs are dims (j, j + rot_dim / 2), or
// neighbours (2 j, 2 j + 1).  Without this call q and K are read and written once more.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "flowkv.h"
#include "flowkv_ragged.h"
#include "flowkv_status.h"

using flowkv::fail;
using flowkv::ok;

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(1))) u32x4 gvec;
typedef __attribute__((address_space(1))) const u32x4 cgvec;

struct RotateArgs {
  char* kbase;                    // the layer's K of block 0
  int64_t voff;                   // V from K
  int64_t bstride;                // bytes between blocks
  const char *q, *k, *v;
  char* q_out;
  int64_t q_stride, q_out_stride, k_stride, v_stride;   // bytes between tokens
  const float* angles;            // (n_positions, rot_dim): cosines, then sines
  const int32_t *offsets, *seq_lens, *tables;
  int32_t n_tokens, n_req, max_blocks, pool_blocks, block_size;
  int32_t q_heads, kv_heads, pieces;                    // 16-byte pieces of a head
  int32_t n_positions, rot_dim;
};

// 16-byte pieces of each type as float32, and back.
struct Bf16 {
  static constexpr int kPer = 8;
  static __device__ __forceinline__ void widen(u32x4 x, float (&y)[kPer]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = __uint_as_float(x[i] << 16);
      y[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 round(const float (&y)[kPer]) {
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = __builtin_bit_cast(
          uint32_t, __builtin_convertvector(f32x2{y[2 * i], y[2 * i + 1]}, bf16x2));
    return x;
  }
};
struct Fp16 {
  static constexpr int kPer = 8;
  static __device__ __forceinline__ void widen(u32x4 x, float (&y)[kPer]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = x[i];
      const f16x2 h = __builtin_bit_cast(f16x2, w);
      y[2 * i] = float(h[0]);
      y[2 * i + 1] = float(h[1]);
    }
  }
  static __device__ __forceinline__ u32x4 round(const float (&y)[kPer]) {
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = __builtin_bit_cast(
          uint32_t, __builtin_convertvector(f32x2{y[2 * i], y[2 * i + 1]}, f16x2));
    return x;
  }
};
struct F32 {
  static constexpr int kPer = 4;
  static __device__ __forceinline__ void widen(u32x4 x, float (&y)[kPer]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __uint_as_float(x[i]);
  }
  static __device__ __forceinline__ u32x4 round(const float (&y)[kPer]) {
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(y[i]);
    return x;
  }
};

// Work: units of two 16-byte pieces of a head, a lane each, heads of q, then of K, then of V,
// token by token.  A rotated unit holds kPer pairs whole: pieces x and x + half (pairs half a
// rotation apart), or 2 x and 2 x + 1 (neighbours), with kPer cosines and as many sines.
constexpr int kThreads = 256;

template <class T, bool kNeighbours>
__global__ __launch_bounds__(kThreads) void kv_rotate(const RotateArgs a) {
  constexpr int kPer = T::kPer;
  const int ln = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t first = (int64_t(blockIdx.x) * (kThreads / 64) + wave) * 64;
  const uint32_t per_head = uint32_t(a.pieces + 1) / 2;
  const uint32_t per = uint32_t(a.q_heads + 2 * a.kv_heads) * per_head;    // units of a token
  const int64_t items = int64_t(a.n_tokens) * per;
  if (first >= items) return;
  const int64_t last = std::min<int64_t>(first + 64, items) - 1;
  const int32_t t0 = int32_t(first / per), t1 = int32_t(last / per);
  const bool some = first + ln < items;
  const uint32_t d = uint32_t(first - int64_t(t0) * per) + ln;
  const int32_t token = some ? t0 + int32_t(d / per) : t1;
  const uint32_t unit = some ? d % per : 0;
  const uint32_t head = unit / per_head, x = unit % per_head;
  const bool is_q = head < uint32_t(a.q_heads);
  const bool is_v = head >= uint32_t(a.q_heads + a.kv_heads);
  const uint32_t h = is_q ? head : head - a.q_heads - (is_v ? a.kv_heads : 0);
  const uint32_t half = uint32_t(a.rot_dim) / (2 * kPer);                  // pieces
  const bool turned = !is_v && x < half;
  const uint32_t p0 = turned && !kNeighbours ? x : 2 * x;
  const uint32_t p1 = turned && !kNeighbours ? x + half : 2 * x + 1;
  const bool two = p1 < uint32_t(a.pieces);
  const char* src = is_q   ? a.q + token * a.q_stride
                    : is_v ? a.v + token * a.v_stride
                           : a.k + token * a.k_stride;
  src += int64_t(h) * a.pieces * 16;
  u32x4 y0 = *(cgvec*)(src + p0 * 16), y1 = {};
  if (two) y1 = *(cgvec*)(src + p1 * 16);

  // the lane's request: among those of the wave's tokens
  int32_t r = flowkv::last_at_most(a.n_req, t0, [&](int32_t i) { return a.offsets[i]; });
  if (t1 != t0) {
    int32_t hi = flowkv::last_at_most(a.n_req, t1, [&](int32_t i) { return a.offsets[i]; }) + 1;
    while (hi - r > 1) {
      const int32_t mid = r + (hi - r) / 2;
      if (a.offsets[mid] <= token) r = mid;
      else hi = mid;
    }
  }
  const int32_t begin = a.offsets[r], end = a.offsets[r + 1];
  const int64_t p = int64_t(a.seq_lens[r]) - (int64_t(end) - begin) + (token - begin);
  if (!some || token < begin || token >= end || p < 0 || p >= a.n_positions) return;
  char* dst;
  if (is_q) {
    dst = a.q_out + token * a.q_out_stride + int64_t(h) * a.pieces * 16;
  } else {
    const uint32_t b = uint32_t(p) / uint32_t(a.block_size);
    if (b >= uint32_t(a.max_blocks)) return;
    const int32_t id = a.tables[int64_t(r) * a.max_blocks + b];
    if (id < 0 || id >= a.pool_blocks) return;
    const uint32_t slot = uint32_t(p) - b * uint32_t(a.block_size);
    dst = a.kbase + (is_v ? a.voff : 0) + id * a.bstride +
          (int64_t(slot) * a.kv_heads + h) * a.pieces * 16;
  }
  if (turned) {
    float c[kPer], s[kPer];
    const float* row = a.angles + p * a.rot_dim + x * kPer;
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
      const f32x4u u = *reinterpret_cast<const f32x4u*>(row + i);
      const f32x4u v = *reinterpret_cast<const f32x4u*>(row + a.rot_dim / 2 + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[i + j] = u[j];
        s[i + j] = v[j];
      }
    }
    float f0[kPer], f1[kPer];
    T::widen(y0, f0);
    T::widen(y1, f1);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      float& u = kNeighbours ? (i < kPer / 2 ? f0[2 * i] : f1[2 * i - kPer]) : f0[i];
      float& w = kNeighbours ? (i < kPer / 2 ? f0[2 * i + 1] : f1[2 * i + 1 - kPer]) : f1[i];
      const float turned_u = u * c[i] - w * s[i];
      w = u * s[i] + w * c[i];
      u = turned_u;
    }
    y0 = T::round(f0);
    y1 = T::round(f1);
  }
  *(gvec*)(dst + p0 * 16) = y0;
  if (two) *(gvec*)(dst + p1 * 16) = y1;
}

template <class T>
const void* kernel(bool neighbours) {
  return neighbours ? reinterpret_cast<const void*>(kv_rotate<T, true>)
                    : reinterpret_cast<const void*>(kv_rotate<T, false>);
}

}  // namespace

extern "C" int flowkv_append_rotated(
    const flowkv_pool* pool, int32_t layer, int32_t dtype, const void* q_dev, int64_t q_stride,
    void* q_out_dev, int64_t q_out_stride, const void* k_dev, int64_t k_stride,
    const void* v_dev, int64_t v_stride, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
    const float* cos_sin_dev, int32_t n_positions, int32_t rot_dim, int32_t interleaved,
    int32_t n_tokens, int32_t n_req, const int32_t* offsets_dev, const int32_t* block_tables_dev,
    int32_t max_blocks, const int32_t* seq_lens_dev, void* hip_stream) {
  const int rc = flowkv::check_pool(pool);
  if (rc) return rc;
  if (layer < 0 || layer >= pool->num_layers)
    return fail(FLOWKV_EINVAL, "layer %d outside the pool's %d layers", layer, pool->num_layers);
  if (dtype != FLOWKV_BF16 && dtype != FLOWKV_FP16 && dtype != FLOWKV_F32)
    return fail(FLOWKV_EINVAL, "unknown element type %d", dtype);
  if (q_heads < 0 || kv_heads < 1 || head_dim < 1)
    return fail(FLOWKV_EINVAL, "%d query heads, %d KV heads, head_dim %d", q_heads, kv_heads,
                head_dim);
  const int64_t e = dtype == FLOWKV_F32 ? 4 : 2, head = head_dim * e, slot = kv_heads * head;
  if (head % 16 || pool->chunk_bytes % slot)
    return fail(FLOWKV_EINVAL,
                "heads of %lld bytes: need a multiple of 16 whose %d KV heads divide chunk_bytes "
                "%lld", (long long)head, kv_heads, (long long)pool->chunk_bytes);
  if (rot_dim < 1 || rot_dim > head_dim || rot_dim * e % 32)
    return fail(FLOWKV_EINVAL, "rot_dim %d of %d: need a whole number of 32 bytes", rot_dim,
                head_dim);
  if (interleaved != 0 && interleaved != 1)
    return fail(FLOWKV_EINVAL, "interleaved %d: need 0 or 1", interleaved);
  if (n_tokens < 0 || n_req < 0 || max_blocks < 0 || n_positions < 0)
    return fail(FLOWKV_EINVAL, "negative sizes");
  const int64_t per = (int64_t(q_heads) + 2 * int64_t(kv_heads)) * ((head / 16 + 1) / 2);
  if (per > INT32_MAX / 2)
    return fail(FLOWKV_EINVAL, "%d query and %d KV heads: too many", q_heads, kv_heads);
  if (n_tokens == 0 || n_req == 0 || n_positions == 0) return ok();
  if (!k_dev || !v_dev || !cos_sin_dev || !offsets_dev || !seq_lens_dev ||
      (max_blocks > 0 && !block_tables_dev) || (q_heads > 0 && (!q_dev || !q_out_dev)))
    return fail(FLOWKV_EINVAL, "NULL device pointer");
  const struct {
    const void* at;
    int64_t stride, heads;
  } rows[] = {{k_dev, k_stride, kv_heads}, {v_dev, v_stride, kv_heads},
              {q_dev, q_stride, q_heads}, {q_out_dev, q_out_stride, q_heads}};
  for (const auto& x : rows) {
    if (x.heads == 0) continue;
    if (reinterpret_cast<uintptr_t>(x.at) % 16 || x.stride % (16 / e))
      return fail(FLOWKV_EINVAL, "rows need 16-byte alignment and strides of whole 16 bytes");
    if (n_tokens > 1 && x.stride < x.heads * head_dim)
      return fail(FLOWKV_EINVAL, "token stride of %lld elements, a token has %lld",
                  (long long)x.stride, (long long)x.heads * head_dim);
  }
  if (reinterpret_cast<uintptr_t>(cos_sin_dev) % 4)
    return fail(FLOWKV_EINVAL, "cosines not 4-byte aligned");
  const int64_t items = int64_t(n_tokens) * per;
  const int64_t groups = (items + kThreads - 1) / kThreads;
  if (groups * kThreads > UINT32_MAX)                // lanes of a launch
    return fail(FLOWKV_EINVAL, "%d tokens of %lld units: too many for one call", n_tokens,
                (long long)per);
  const bool lm = pool->layout == FLOWKV_LAYOUT_LAYER_MAJOR;
  RotateArgs a{};
  a.kbase = static_cast<char*>(pool->layer_base[lm ? layer : 0]) +
            (lm ? 0 : int64_t(layer) * 2 * pool->chunk_bytes);
  a.voff = lm ? int64_t(pool->num_blocks) * pool->chunk_bytes : pool->chunk_bytes;
  a.bstride = lm ? pool->chunk_bytes : 2 * int64_t(pool->num_layers) * pool->chunk_bytes;
  a.q = static_cast<const char*>(q_dev);
  a.k = static_cast<const char*>(k_dev);
  a.v = static_cast<const char*>(v_dev);
  a.q_out = static_cast<char*>(q_out_dev);
  a.q_stride = q_stride * e;
  a.q_out_stride = q_out_stride * e;
  a.k_stride = k_stride * e;
  a.v_stride = v_stride * e;
  a.angles = cos_sin_dev;
  a.offsets = offsets_dev;
  a.seq_lens = seq_lens_dev;
  a.tables = block_tables_dev;
  a.n_tokens = n_tokens;
  a.n_req = n_req;
  a.max_blocks = max_blocks;
  a.pool_blocks = pool->num_blocks;
  a.block_size = int32_t(pool->chunk_bytes / slot);
  a.q_heads = q_heads;
  a.kv_heads = kv_heads;
  a.pieces = int32_t(head / 16);
  a.n_positions = n_positions;
  a.rot_dim = rot_dim;
  void* args[] = {&a};
  const void* fn = dtype == FLOWKV_BF16   ? kernel<Bf16>(interleaved)
                   : dtype == FLOWKV_FP16 ? kernel<Fp16>(interleaved)
                                          : kernel<F32>(interleaved);
  hipError_t rc2 = hipLaunchKernel(fn, dim3(unsigned(groups)), dim3(kThreads), args, 0,
                                   static_cast<hipStream_t>(hip_stream));
  if (rc2 == hipSuccess) rc2 = hipGetLastError();
  if (rc2 != hipSuccess)
    return fail(FLOWKV_EHIP, "rotated append launch: %s", hipGetErrorString(rc2));
  return ok();
}
