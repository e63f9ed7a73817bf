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
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(1))) u32x4 gvec;
typedef __attribute__((address_space(1))) const u32x4 cgvec;

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

// x / d = (umulhi(x, m) + x) >> l with l = ceil(log2 d), m = floor(2^32 (2^l - d) / d) + 1.
struct Divisor {
  uint32_t magic, shift;
};
__device__ __forceinline__ uint32_t div(uint32_t x, Divisor d) {
  return uint32_t((uint64_t(__umulhi(x, d.magic)) + x) >> d.shift);
}
Divisor divisor(uint32_t d) {
  Divisor r{0, 0};
  while ((uint64_t(1) << r.shift) < d) ++r.shift;
  r.magic = uint32_t((((uint64_t(1) << r.shift) - d) << 32) / d + 1);
  return r;
}

// Work: units of two 16-byte pieces of a head; a lane takes one, or the same one of kHeads heads
// next to each other (which share their cosines and sines), heads of q, then of K, then of V,
// token by token.  A rotated unit is pieces x and x + half of the rotated dims, kPer pairs half
// a rotation apart or two times kPer / 2 neighbours; an unrotated one is two pieces half of the
// unrotated ones apart.  So 16 bytes of neighbouring lanes lie together in every store.
//
// What bounds it: short calls, a launch and its chain of loads (offsets, length, angles; the rows'
// own are under way meanwhile): 32 tokens of 48 heads of 128 3.3 us in a graph.  Long ones memory:
// 17,679 tokens of 10 heads, 99.6 MB, 16.7 to 17.5 us by the card, 5.7 to 5.9 TB/s; in float32, 190
// MB, 30.8 us, 6.2.  (With divisions for the products, one
// head a lane and pairs of pieces next to each other 20.2.)
constexpr int kThreads = 256;

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
  uint32_t items, per, per_head;  // lanes' items in all, of a token, of a head
  Divisor by_per, by_per_head, by_block;
};

template <class T, bool kNeighbours, int kHeads, bool kPast>
__global__ __launch_bounds__(kThreads) void kv_rotate(const RotateArgs a) {
  constexpr int kPer = T::kPer;
  const int ln = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t first = (blockIdx.x * (kThreads / 64) + wave) * 64;
  if (first >= a.items) return;
  const uint32_t last = std::min(first + 63, a.items - 1);
  const int32_t t0 = int32_t(div(first, a.by_per)), t1 = int32_t(div(last, a.by_per));
  const bool some = first + ln <= last;
  const uint32_t d = first - uint32_t(t0) * a.per + uint32_t(ln);
  const uint32_t dt = some ? div(d, a.by_per) : uint32_t(t1 - t0);
  const int32_t token = t0 + int32_t(dt);
  const uint32_t unit = some ? d - dt * a.per : 0;
  const uint32_t j = div(unit, a.by_per_head), x = unit - j * a.per_head;
  const uint32_t half = uint32_t(a.rot_dim) / (2 * kPer);                  // pieces
  const uint32_t heads = uint32_t(a.q_heads + 2 * a.kv_heads), kv = uint32_t(a.kv_heads);
  const bool turning = x < half;
  u32x4 y[kHeads][2];
  uint32_t p0[kHeads], p1[kHeads], h[kHeads];
  bool is_q[kHeads], is_v[kHeads], turned[kHeads], here[kHeads], two[kHeads];
#pragma unroll
  for (int e = 0; e < kHeads; ++e) {
    const uint32_t head = j * kHeads + e;
    here[e] = head < heads;
    is_q[e] = head < uint32_t(a.q_heads);
    is_v[e] = head >= uint32_t(a.q_heads) + kv;
    h[e] = is_q[e] ? head : head - uint32_t(a.q_heads) - (is_v[e] ? kv : 0);
    turned[e] = !is_v[e] && turning;
    // (behind the rotated dims the units go on from 2 half)
    const uint32_t rest = !turning ? half : 0;
    p0[e] = is_v[e] ? x : x + rest;
    p1[e] = is_v[e] ? x + a.per_head : x + (turning ? half : a.per_head);
    two[e] = p1[e] < uint32_t(a.pieces);
    const char* src = is_q[e]   ? a.q + token * a.q_stride
                      : is_v[e] ? a.v + token * a.v_stride
                                : a.k + token * a.k_stride;
    src += int64_t(h[e] * uint32_t(a.pieces)) * 16;
    y[e][0] = y[e][1] = u32x4{};
    if (here[e]) {
      y[e][0] = *(cgvec*)(src + p0[e] * 16);
      if (two[e]) y[e][1] = *(cgvec*)(src + p1[e] * 16);
    }
  }

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
  const int64_t pos = int64_t(a.seq_lens[r]) - (int64_t(end) - begin) + (token - begin);
  if (!some || token < begin || token >= end || pos < 0 || pos >= a.n_positions) return;
  const uint32_t p = uint32_t(pos);
  float c[kPer], s[kPer];
  if (turning) {
    // neighbours: of piece x, then of piece x + half
    const float* row = a.angles + int64_t(p) * a.rot_dim + x * (kNeighbours ? kPer / 2 : kPer);
    constexpr int kLoad = kNeighbours ? kPer / 2 : 4;
    typedef float Load __attribute__((ext_vector_type(kLoad), aligned(4)));
#pragma unroll
    for (int i = 0; i < kPer; i += kLoad) {
      const float* at = row + (kNeighbours && i ? half * (kPer / 2) : uint32_t(i));
      const Load u = *reinterpret_cast<const Load*>(at);
      const Load w = *reinterpret_cast<const Load*>(at + a.rot_dim / 2);
#pragma unroll
      for (int k = 0; k < kLoad; ++k) {
        c[i + k] = u[k];
        s[i + k] = w[k];
      }
    }
  }
  const uint32_t b = div(p, a.by_block);
  int32_t id = -1;                                       // of the token's block
  if (b < uint32_t(a.max_blocks)) id = a.tables[int64_t(r) * a.max_blocks + b];
  const bool kept = id >= 0 && id < a.pool_blocks;
  char* const slot = a.kbase + id * a.bstride +
                     int64_t((p - b * uint32_t(a.block_size)) * kv) * a.pieces * 16;
#pragma unroll
  for (int e = 0; e < kHeads; ++e) {
    if (!here[e] || !(is_q[e] || kept)) continue;
    if (turned[e]) {
      float f0[kPer], f1[kPer];
      T::widen(y[e][0], f0);
      T::widen(y[e][1], f1);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        float& u = kNeighbours ? (i < kPer / 2 ? f0[2 * i] : f1[2 * i - kPer]) : f0[i];
        float& w = kNeighbours ? (i < kPer / 2 ? f0[2 * i + 1] : f1[2 * i + 1 - kPer]) : f1[i];
        const float turned_u = u * c[i] - w * s[i];
        w = u * s[i] + w * c[i];
        u = turned_u;
      }
      y[e][0] = T::round(f0);
      y[e][1] = T::round(f1);
    }
    char* dst = is_q[e] ? a.q_out + token * a.q_out_stride : slot + (is_v[e] ? a.voff : 0);
    dst += int64_t(h[e] * uint32_t(a.pieces)) * 16;
    if constexpr (!kPast) {
      *(gvec*)(dst + p0[e] * 16) = y[e][0];
      if (two[e]) *(gvec*)(dst + p1[e] * 16) = y[e][1];
    } else {
      __builtin_nontemporal_store(y[e][0], (gvec*)(dst + p0[e] * 16));
      if (two[e]) __builtin_nontemporal_store(y[e][1], (gvec*)(dst + p1[e] * 16));
    }
  }
}

// Units up to which a lane takes one: they then are on the CUs at once.  And bytes written from
// which on they go past the caches.  (us past them and through, in a graph: 10 heads of 128 in
// blocks of 16, 10 MiB 5.5 and 6.2, 29 MiB 11.8 and 13.1, 146 MiB 54.6 and 59.8; 17,679 tokens of
// them, 43 MiB, 17.5 and 18.2; 16 heads of 64 in blocks of 7, 17 MiB, 9.7 and 9.2.  With attention
// through a window behind it, which then finds K, V and q in the L2s, 32 MiB together: 15 MiB 68.1
// and 68.1, 29 MiB 96.6 and 95.1, 98.2 and 96.9, 38 MiB 94.4 and 93.8.)
constexpr int64_t kRotateFew = 1 << 17;
constexpr int64_t kRotatePast = int64_t(32) << 20;

enum Variant { kOneHead, kTwoHeads, kTwoHeadsPast };

template <class T, bool kNeighbours>
const void* kernel(Variant v) {
  return v == kOneHead    ? reinterpret_cast<const void*>(kv_rotate<T, kNeighbours, 1, false>)
         : v == kTwoHeads ? reinterpret_cast<const void*>(kv_rotate<T, kNeighbours, 2, false>)
                          : reinterpret_cast<const void*>(kv_rotate<T, kNeighbours, 2, true>);
}
template <class T>
const void* kernel(bool neighbours, Variant v) {
  return neighbours ? kernel<T, true>(v) : kernel<T, false>(v);
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
  const int64_t e = dtype == FLOWKV_F32 ? 4 : 2, head = head_dim * e;
  if (head % 16 || kv_heads > pool->chunk_bytes / head || pool->chunk_bytes % (kv_heads * head))
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
  const int64_t heads = int64_t(q_heads) + 2 * int64_t(kv_heads), per_head = (head / 16 + 1) / 2;
  if (heads * per_head > INT32_MAX / 2)
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
  const Variant variant = n_tokens * heads * per_head <= kRotateFew ? kOneHead
                          : n_tokens * heads <= kRotatePast / head  ? kTwoHeads
                                                                    : kTwoHeadsPast;
  const int64_t per = (variant == kOneHead ? heads : (heads + 1) / 2) * per_head;
  const int64_t items = n_tokens * per;
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
  a.block_size = int32_t(pool->chunk_bytes / (kv_heads * head));
  a.q_heads = q_heads;
  a.kv_heads = kv_heads;
  a.pieces = int32_t(head / 16);
  a.n_positions = n_positions;
  a.rot_dim = rot_dim;
  a.items = uint32_t(items);
  a.per = uint32_t(per);
  a.per_head = uint32_t(per_head);
  a.by_per = divisor(a.per);
  a.by_per_head = divisor(a.per_head);
  a.by_block = divisor(uint32_t(a.block_size));
  void* args[] = {&a};
  const void* fn = dtype == FLOWKV_BF16   ? kernel<Bf16>(interleaved, variant)
                   : dtype == FLOWKV_FP16 ? kernel<Fp16>(interleaved, variant)
                                          : kernel<F32>(interleaved, variant);
  hipError_t rc2 = hipLaunchKernel(fn, dim3(unsigned(groups)), dim3(kThreads), args, 0,
                                   static_cast<hipStream_t>(hip_stream));
  if (rc2 == hipSuccess) rc2 = hipGetLastError();
  if (rc2 != hipSuccess)
    return fail(FLOWKV_EHIP, "rotated append launch: %s", hipGetErrorString(rc2));
  return ok();
}
