// Attention of a chunk of new tokens over the paged cache, for gfx950 (MI355X).
//
// The prefill counterpart of decode attention (FlowKV, arXiv 2504.03775, section
// 3.3: attention reads the pool in either layout of Eq. 5 through a request's
// block list): each request brings some new tokens whose K and V are in the pool
// already, and query i of them attends to every token up to its own position.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "flowkv.h"
#include "flowkv_device.h"
#include "flowkv_ragged.h"
#include "flowkv_status.h"

using flowkv::fail;
using flowkv::ok;

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(1))) const u32x4 cgvec4;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2u __attribute__((ext_vector_type(2), aligned(4)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds4;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 32 * kWaves;         // query rows of a workgroup's tile
constexpr int kKeys = 64;                  // cached tokens of a step
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;               // log2 of the largest unnormalised weight

struct ChunkArgs {
  const char* kbase;                    // the layer's K of block 0
  int64_t voff;                         // V from K
  const uint16_t* q;                    // a token's Hq x Dh values every q_stride
  int64_t q_stride;                     // in elements
  const int32_t* offsets;               // (n_req + 1)
  const int32_t* seq_lens;              // (n_req)
  const int32_t* tables;                // (n_req, max_blocks)
  uint16_t* out;                        // (n_tokens, Hq, Dh) bf16
  float* ws;                            // the splits' records
  uint32_t bunits, sunits;              // 128-byte units between blocks, slots
  uint32_t bs_magic, bs_shift;          // division by block_size
  int32_t pool_blocks, block_size, max_blocks, max_seq_len;
  int32_t n_tokens, n_req, q_heads, kv_heads, group;
  int32_t tiles, split_tokens, splits;
  float scale_log2;                     // scale * log2(e)
};

// The rows of a request are its (new token, query head of the group) pairs,
// token by token; a tile is kRows of them.  Tile slot x of the batch: request r
// has the slots from floor(offsets[r] * G / kRows) + r, which are enough for its
// rows whatever the offsets are, and at most n_tokens * G / kRows + n_req in all:
// the grid needs no lengths on the host.
__device__ __forceinline__ int64_t first_tile(const ChunkArgs& a, int32_t r) {
  return int64_t(a.offsets[r]) * a.group / kRows + r;
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

// Tokens that new token i sees: those up to its own position.
__device__ __forceinline__ int32_t seen(const Request& q, int32_t i) {
  const int32_t n = q.base + i + 1;
  return n < 0 ? 0 : n < q.limit ? n : q.limit;
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

__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
}

// 16 bytes that a staged row of a token that cannot be read is made of.
__device__ const u32x4 g_zeros = {0, 0, 0, 0};

template <int kDh>
struct ChunkLds {
  alignas(16) u32x4 k[kKeys * kDh / 8];
  alignas(16) u32x4 v[kKeys * kDh / 8];
};

typedef __attribute__((address_space(1))) const void gvoid;
typedef __attribute__((address_space(3))) void lvoid;

template <int kDh>
__global__ __launch_bounds__(kThreads, 2) void chunk_attn(const ChunkArgs a) {
  constexpr int kPc = kDh / 8;                   // 16-byte pieces of a row
  constexpr int kI = kDh / 16;                   // MFMA steps of K.q
  constexpr int kB = kDh / 32;                   // blocks of 32 dims
  constexpr int kLd = kKeys * kPc / kThreads;    // 16-byte loads of a tile's K, and V, a lane
  constexpr int kLdRows = kThreads / kPc;        // tokens of one such load
  const int tid = threadIdx.x, ln = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = ln >> 5, c32 = ln & 31;

  const uint32_t id = blockIdx.x;
  const int g = int(id % uint32_t(a.kv_heads));
  const uint32_t rest = id / uint32_t(a.kv_heads);
  const int split = int(rest / uint32_t(a.tiles));
  const int slot = a.tiles - 1 - int(rest % uint32_t(a.tiles));  // the longest first
  const int32_t r =
      flowkv::last_at_most(a.n_req, slot, [&](int32_t i) { return first_tile(a, i); });
  const Request rq = request_at(a, r);
  const int64_t local = int64_t(slot) - first_tile(a, r);
  const int64_t rows = int64_t(rq.n_new) * a.group;
  const int64_t row0 = local * kRows;
  if (local < 0 || row0 >= rows) return;
  const int64_t row_end = row0 + kRows < rows ? row0 + kRows : rows;
  const int32_t tile_limit = seen(rq, int32_t((row_end - 1) / a.group));
  const int32_t tile_least = seen(rq, int32_t(row0 / a.group));
  const int32_t s0 = split * a.split_tokens;
  if (split > 0 && s0 >= tile_limit) return;     // (split 0 writes the rows that see nothing)
  const int32_t s1 = tile_limit - s0 > a.split_tokens ? s0 + a.split_tokens : tile_limit;
  const bool direct = tile_limit <= a.split_tokens;

  // this lane's query row, as a column of S^T
  const int64_t row = row0 + wave * 32 + c32;
  const bool live = row < rows;
  const int32_t qi = live ? int32_t(row / a.group) : 0;
  const int32_t qh = live ? int32_t(row - int64_t(qi) * a.group) : 0;
  const int32_t lim = live ? seen(rq, qi) : 0;
  const int64_t token = int64_t(rq.begin) + qi;
  const int32_t head = g * a.group + qh;
  // what the wave's rows see at least and at most (it may hold no row)
  const int64_t wrow = row0 + wave * 32;
  const bool any_row = wrow < rows;
  const int32_t wlast = any_row ? int32_t((wrow + 31 < rows ? wrow + 31 : rows - 1) / a.group) : 0;
  const int32_t wlim = __builtin_amdgcn_readfirstlane(any_row ? seen(rq, wlast) : 0);
  const int32_t wleast =
      __builtin_amdgcn_readfirstlane(any_row ? seen(rq, int32_t(wrow / a.group)) : 0);

  bf16x8 qb[kI];
#pragma unroll
  for (int i = 0; i < kI; ++i) {
    u32x4 w = {0, 0, 0, 0};
    if (live)
      w = *(cgvec4*)(a.q + token * a.q_stride + head * kDh + 16 * i + 8 * half);
    qb[i] = __builtin_bit_cast(bf16x8, w);
  }

  __shared__ ChunkLds<kDh> lds0, lds1;

  // Staging: K and V rows go from memory to LDS directly.  An instruction fills 64
  // consecutive 16-byte places, so a lane's place is fixed, token lr + e kLdRows and
  // piece lp of its row, and the swizzle is in which piece it reads.
  const int lr = tid / kPc, lp = tid % kPc;
  const int32_t* table = a.tables + int64_t(r) * a.max_blocks;
  const char* kp = a.kbase + g * kDh * 2 + 16 * (lp ^ (kPc == 16 ? lr & 15 : lr >> 1 & 7));
  const char* vp = a.kbase + a.voff + g * kDh * 2 +
                   16 * (lp ^ (kPc == 16 ? (lr & 3) * 4 : (lr >> 1 & 1) * 4));
  const char* const zeros = reinterpret_cast<const char*>(&g_zeros);
  // lane ln's token of a tile: block ID, and its row's place in the pool in 128-byte
  // units (all ones: it cannot be read)
  uint32_t next_slot;
  int32_t next_block;
  bool next_in;
  auto fetch = [&](int32_t t0) {
    const uint32_t t = uint32_t(t0 + ln);
    const uint32_t b = uint32_t((uint64_t(__umulhi(t, a.bs_magic)) + t) >> a.bs_shift);
    next_slot = t - b * uint32_t(a.block_size);
    next_in = int32_t(t) < s1;
    next_block = table[next_in ? b : 0];         // (s1 lies within the block list)
  };
  uint64_t dead, next_dead;                      // tokens of a tile whose block is outside
  auto stage = [&](ChunkLds<kDh>& to) {
    const bool good = next_in && next_block >= 0 && next_block < a.pool_blocks;
    next_dead = __ballot(next_in && !good);
    const uint32_t at =
        good ? uint32_t(next_block) * a.bunits + next_slot * a.sunits : 0xffffffffu;
#pragma unroll
    for (int e = 0; e < kLd; ++e) {
      const uint32_t u = __shfl(at, lr + e * kLdRows);
      const uint64_t off = uint64_t(u) * 128;
      const char* ks = u != 0xffffffffu ? kp + off : zeros;
      const char* vs = u != 0xffffffffu ? vp + off : zeros;
      const int place = e * kThreads + wave * 64;
      __builtin_amdgcn_global_load_lds((gvoid*)ks, (lvoid*)(to.k + place), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((gvoid*)vs, (lvoid*)(to.v + place), 16, 0, 0);
    }
  };

  f32x16 o[kB];
#pragma unroll
  for (int b = 0; b < kB; ++b) o[b] = f32x16{};
  float mref = -INFINITY, lsum = 0.f;            // of the lane's row; its own half of the tokens

  // Where some row does not see some token, an infinity or a NaN in V would reach it as
  // 0 x inf: such values are taken out of the tile, and added at the end to the rows
  // that see them.
  bool odd = false;
  auto clean = [&](ChunkLds<kDh>& lds) {
#pragma unroll
    for (int e = 0; e < kLd; ++e) {
      u32x4 w = lds.v[e * kThreads + tid];
      bool any = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x7f80u) == 0x7f80u) {
          w[i] &= 0xffff0000u;
          any = true;
        }
        if ((w[i] & 0x7f800000u) == 0x7f800000u) {
          w[i] &= 0xffffu;
          any = true;
        }
      }
      if (any) lds.v[e * kThreads + tid] = w;
      odd |= any;
    }
    __syncthreads();
  };

  auto step = [&](int32_t t0, ChunkLds<kDh>& lds, ChunkLds<kDh>& other) {
    dead = next_dead;
    if (t0 + kKeys > tile_least) clean(lds);     // uniform
    if (t0 + kKeys < s1) {
      stage(other);
      fetch(t0 + 2 * kKeys);
    }
    if (t0 < wlim) {
      // S^T = K Q^T: rows are tokens, columns query rows
      f32x16 s[2] = {f32x16{}, f32x16{}};
      u32x4 w[2][kI];
      auto k_at = [&](int b, int i) {
        const int x = 32 * b + c32;
        return lds.k[x * kPc + ((2 * i + half) ^ (kPc == 16 ? x & 15 : x >> 1 & 7))];
      };
#pragma unroll
      for (int i = 0; i < kI; ++i) w[0][i] = k_at(0, i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kI; ++i) {
        w[1][i] = k_at(1, i);
        s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w[0][i]), qb[i],
                                                       s[0], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < kI; ++i)
        s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w[1][i]), qb[i],
                                                       s[1], 0, 0, 0);
      if (t0 + kKeys > wleast || dead) {
        const int32_t last = lim - t0 - 4 * half;
        const uint64_t d = dead >> (4 * half);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int x = 32 * b + 8 * (i / 4) + i % 4;
            if (x >= last || (d >> x & 1)) s[b][i] = -INFINITY;
          }
      }
      float mx = s[0][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[0][i]);
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[1][i]);
      mx *= a.scale_log2;
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
      const float mu = mref == -INFINITY ? 0.f : mref;
      u32x4 p[4];                                // k-step j: the B operand
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[b][i], a.scale_log2, -mu));
          const float y = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], a.scale_log2, -mu));
          lsum += x + y;
          p[2 * b + i / 8][i % 8 / 2] = pack_bf16(x, y);
        }
      // O^T += V^T P^T: rows are dims.  V is read transposed
      auto v_at = [&](int b, int j) {
        const int x = 16 * j + 4 * half + (ln & 15) / 4;
        const int col = 32 * b + 16 * (ln >> 4 & 1) + 4 * (ln & 3);   // dim
        const int at = x * kPc + ((col >> 3) ^ (kPc == 16 ? (x & 3) * 4 : (x >> 1 & 1) * 4));
        lds4* base = (lds4*)(reinterpret_cast<const uint16_t*>(lds.v) + at * 8 + (col & 4));
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(base);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(base + 8 * kPc * 2);
        return u32x4{__builtin_bit_cast(u32x2, lo)[0], __builtin_bit_cast(u32x2, lo)[1],
                     __builtin_bit_cast(u32x2, hi)[0], __builtin_bit_cast(u32x2, hi)[1]};
      };
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int b = 0; b < kB; ++b)
          o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v_at(b, j)),
                                                         __builtin_bit_cast(bf16x8, p[j]), o[b], 0,
                                                         0, 0);
    }
    __syncthreads();
  };
  if (s0 < s1) {
    fetch(s0);
    stage(lds0);
    fetch(s0 + kKeys);
  }
  __syncthreads();
  for (int32_t t0 = s0; t0 < s1; t0 += 2 * kKeys) {
    step(t0, lds0, lds1);
    if (t0 + kKeys < s1) step(t0 + kKeys, lds1, lds0);
  }

  if (__syncthreads_or(odd)) {
    for (int32_t t = std::max(tile_least / kKeys * kKeys, s0); t < s1; ++t) {
      const int32_t b = table[t / a.block_size];
      if (b < 0 || b >= a.pool_blocks) continue;
      const char* v = a.kbase + a.voff + g * kDh * 2 +
                      (int64_t(b) * a.bunits + int64_t(t % a.block_size) * a.sunits) * 128;
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t y = uint32_t(reinterpret_cast<const uint16_t*>(
                                 v)[32 * b + 8 * (i / 4) + 4 * half + i % 4])
                             << 16;
          if ((y & 0x7f800000u) == 0x7f800000u && t < lim) o[b][i] += __uint_as_float(y);
        }
    }
  }
  lsum += __shfl_xor(lsum, 32);
  if (!live) return;
  const int64_t orow = token * a.q_heads + head;
  if (direct) {
    const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const u32x2 w = {pack_bf16(o[b][i] * inv, o[b][i + 1] * inv),
                         pack_bf16(o[b][i + 2] * inv, o[b][i + 3] * inv)};
        *reinterpret_cast<u32x2*>(a.out + orow * kDh + 32 * b + 2 * i + 4 * half) = w;
      }
  } else {
    const int64_t rec = record_at(a, orow, split);
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4u*>(record_sums(a, kDh, rec) + 32 * b + 2 * i + 4 * half) =
            f32x4u{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
    if (half == 0) *record_ml(a, kDh, rec) = f32x2u{mref, lsum};
  }
}

// Joins the splits' records of the rows whose tile has more than one: a wave per
// (new token, query head), Dh / 4 lanes a record.
template <int kDh>
__global__ __launch_bounds__(kThreads) void chunk_attn_merge(const ChunkArgs a) {
  constexpr int kLanes = kDh / 4, kParts = 64 / kLanes;
  const int ln = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t orow = int64_t(blockIdx.x) * kWaves + wave;
  if (orow >= int64_t(a.n_tokens) * a.q_heads) return;
  const int32_t token = int32_t(orow / a.q_heads), head = int32_t(orow - int64_t(token) * a.q_heads);
  const int32_t r =
      flowkv::last_at_most(a.n_req, token, [&](int32_t i) { return a.offsets[i]; });
  const Request rq = request_at(a, r);
  const int32_t i = token - rq.begin;
  if (i < 0 || i >= rq.n_new) return;
  // the tile that the row was in, as its workgroups saw it
  const int64_t row = int64_t(i) * a.group + head % a.group;
  const int64_t end = std::min<int64_t>((row / kRows + 1) * kRows, int64_t(rq.n_new) * a.group);
  const int32_t tile_limit = seen(rq, int32_t((end - 1) / a.group));
  if (tile_limit <= a.split_tokens) return;      // written already
  const int32_t n = (seen(rq, i) + a.split_tokens - 1) / a.split_tokens;
  const int64_t rec = record_at(a, orow, 0);
  const float* sums = record_sums(a, kDh, rec) + 4 * (ln % kLanes);
  const f32x2u* ml = record_ml(a, kDh, rec);
  float m = -INFINITY, l = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int32_t s = ln / kLanes; s < n; s += kParts) {
    const f32x2u x = ml[s];
    const f32x4u y = *reinterpret_cast<const f32x4u*>(sums + int64_t(s) * kDh);
    // (a split whose scores are all NaN has a max of -inf, and a sum of NaN)
    if (x[0] == -INFINITY && x[1] == 0.f) continue;
    const float mn = fmaxf(m, x[0]);
    const float c = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - mn);
    const float w = x[0] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(x[0] - mn);
    m = mn;
    l = l * c + x[1] * w;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = v[k] * c + y[k] * w;
  }
#pragma unroll
  for (int off = kLanes; off < 64; off *= 2) {
    const float m2 = __shfl_xor(m, off), l2 = __shfl_xor(l, off);
    const float mn = fmaxf(m, m2);
    const float c = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - mn);
    const float w = m2 == -INFINITY ? (l2 == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m2 - mn);
    l = l * c + l2 * w;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = v[k] * c + __shfl_xor(v[k], off) * w;
    m = mn;
  }
  if (ln < kLanes) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const u32x2 w = {pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
    *reinterpret_cast<u32x2*>(a.out + orow * kDh + 4 * ln) = w;
  }
}

// Tokens a split takes where the caller leaves it to the library.
int32_t auto_split(int64_t n_tokens, int32_t n_req, int32_t kv_heads, int32_t group,
                   int32_t max_new, int32_t max_seq_len) {
  const int64_t by_req = int64_t(n_req) * ((int64_t(max_new) * group + kRows - 1) / kRows);
  const int64_t tiles = std::min(by_req, n_tokens * group / kRows + n_req) * kv_heads;
  const int64_t want = tiles >= 256 ? 1 : (512 + tiles - 1) / std::max<int64_t>(tiles, 1);
  int64_t s = (int64_t(max_seq_len) + want - 1) / want;
  s = std::max<int64_t>((s + kKeys - 1) / kKeys * kKeys, 4 * kKeys);
  return int32_t(std::min<int64_t>(s, (int64_t(INT32_MAX) / kKeys) * kKeys));
}

struct Shape {
  int32_t split, splits;
  int64_t need;
};

// The split of a call and the workspace that it takes.
int plan_shape(int32_t n_tokens, int32_t n_req, int32_t q_heads, int32_t kv_heads,
               int32_t head_dim, int32_t max_new, int32_t max_seq_len, int32_t split_tokens,
               Shape* out) {
  if (n_tokens < 0 || n_req < 0 || max_new < 0 || max_seq_len < 0)
    return fail(FLOWKV_EINVAL, "negative sizes");
  if (head_dim != 64 && head_dim != 128)
    return fail(FLOWKV_EINVAL, "head_dim %d: need 64 or 128", head_dim);
  if (kv_heads < 1 || q_heads < 1 || q_heads % kv_heads)
    return fail(FLOWKV_EINVAL, "q_heads %d not a multiple of kv_heads %d", q_heads, kv_heads);
  if (split_tokens < 0 || split_tokens % kKeys)
    return fail(FLOWKV_EINVAL, "split_tokens %d: need 0 or a multiple of %d", split_tokens, kKeys);
  if (split_tokens == 0)
    split_tokens =
        auto_split(n_tokens, n_req, kv_heads, q_heads / kv_heads, max_new, max_seq_len);
  out->split = split_tokens;
  out->splits = int32_t((int64_t(max_seq_len) + split_tokens - 1) / split_tokens);
  if (out->splits < 1) out->splits = 1;
  out->need = 0;
  if (out->splits > 1 &&
      __builtin_mul_overflow(int64_t(n_tokens) * q_heads * (head_dim + 2) * int64_t(sizeof(float)),
                             int64_t(out->splits), &out->need))
    return fail(FLOWKV_EINVAL, "%d splits: the workspace's size overflows", out->splits);
  return FLOWKV_OK;
}

}  // namespace

extern "C" int flowkv_chunk_attention_workspace(int32_t n_tokens, int32_t n_req, int32_t q_heads,
                                                int32_t kv_heads, int32_t head_dim,
                                                int32_t max_new, int32_t max_seq_len,
                                                int32_t split_tokens, int64_t* bytes) {
  if (!bytes) return fail(FLOWKV_EINVAL, "NULL output");
  Shape sh;
  const int rc = plan_shape(n_tokens, n_req, q_heads, kv_heads, head_dim, max_new, max_seq_len,
                            split_tokens, &sh);
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
  if (!pool) return fail(FLOWKV_EINVAL, "NULL pool");
  if (pool->layout != FLOWKV_LAYOUT_LAYER_MAJOR && pool->layout != FLOWKV_LAYOUT_BLOCK_MAJOR)
    return fail(FLOWKV_EINVAL, "unknown layout %d", pool->layout);
  if (pool->num_layers < 1 || pool->num_layers > FLOWKV_MAX_LAYERS || pool->num_blocks < 1 ||
      !pool->layer_base)
    return fail(FLOWKV_EINVAL, "bad pool descriptor");
  if (layer < 0 || layer >= pool->num_layers)
    return fail(FLOWKV_EINVAL, "layer %d outside the pool's %d layers", layer, pool->num_layers);
  Shape sh;
  int rc = plan_shape(n_tokens, n_req, q_heads, kv_heads, head_dim, max_new, max_seq_len,
                      split_tokens, &sh);
  if (rc) return rc;
  const int64_t per_token = int64_t(kv_heads) * head_dim * 2;
  if (pool->chunk_bytes <= 0 || pool->chunk_bytes % per_token)
    return fail(FLOWKV_EINVAL, "chunk_bytes %lld is not block_size x %d KV heads x %d bf16",
                (long long)pool->chunk_bytes, kv_heads, head_dim);
  const int64_t bs = pool->chunk_bytes / per_token;
  const bool lm = pool->layout == FLOWKV_LAYOUT_LAYER_MAJOR;
  const int64_t stride = lm ? pool->chunk_bytes : 2 * int64_t(pool->num_layers) * pool->chunk_bytes;
  // one block stride under 4 GiB, as for decode attention; the kernel forms offsets in
  // 128-byte units (a head's row is one or two) of 32 bits
  if (stride >= (int64_t(1) << 32))
    return fail(FLOWKV_EINVAL, "block stride of %lld bytes: need under 4 GiB", (long long)stride);
  if (pool->num_blocks >= (int64_t(1) << 39) / stride)
    return fail(FLOWKV_EINVAL, "%d blocks %lld bytes apart: need under 512 GiB", pool->num_blocks,
                (long long)stride);
  if (max_blocks < 0 || int64_t(max_blocks) * bs > INT32_MAX)
    return fail(FLOWKV_EINVAL, "max_blocks %d x block_size %lld tokens: need 0 to 2^31 - 1",
                max_blocks, (long long)bs);
  // positions are formed in 32 bits past the last tile's end
  if (max_seq_len > INT32_MAX - 4096)
    return fail(FLOWKV_EINVAL, "max_seq_len %d: need at most 2^31 - 4097", max_seq_len);
  if (!(scale > 0.f) || !std::isfinite(scale)) return fail(FLOWKV_EINVAL, "bad scale");
  if (n_req == 0 || n_tokens == 0) return ok();
  if (!q_dev || !offsets_dev || !seq_lens_dev || !out_dev || (max_blocks > 0 && !block_tables_dev))
    return fail(FLOWKV_EINVAL, "NULL device pointer");
  if (reinterpret_cast<uintptr_t>(q_dev) % 16 || q_stride % 8)
    return fail(FLOWKV_EINVAL, "queries need 16-byte alignment and a stride of whole 16 bytes");
  if (n_tokens > 1 && q_stride < int64_t(q_heads) * head_dim)
    return fail(FLOWKV_EINVAL, "query stride of %lld elements, a token has %lld",
                (long long)q_stride, (long long)q_heads * head_dim);
  if (reinterpret_cast<uintptr_t>(out_dev) % 8)
    return fail(FLOWKV_EINVAL, "output not 8-byte aligned");
  if (sh.need > 0 && !workspace_dev) return fail(FLOWKV_EINVAL, "NULL workspace");
  if (workspace_bytes < sh.need)
    return fail(FLOWKV_ECAP, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
                (long long)sh.need);
  if (sh.need > 0 && reinterpret_cast<uintptr_t>(workspace_dev) % 4)
    return fail(FLOWKV_EINVAL, "workspace not 4-byte aligned");
  const int base = lm ? layer : 0;
  if (!pool->layer_base[base] || reinterpret_cast<uintptr_t>(pool->layer_base[base]) % 16)
    return fail(FLOWKV_EINVAL, "pool base pointer %d NULL or not 16-byte aligned", base);

  ChunkArgs a{};
  a.kbase = static_cast<const char*>(pool->layer_base[base]) +
            (lm ? 0 : int64_t(layer) * 2 * pool->chunk_bytes);
  a.voff = lm ? int64_t(pool->num_blocks) * pool->chunk_bytes : pool->chunk_bytes;
  a.q = static_cast<const uint16_t*>(q_dev);
  a.q_stride = q_stride;
  a.offsets = offsets_dev;
  a.seq_lens = seq_lens_dev;
  a.tables = block_tables_dev;
  a.out = static_cast<uint16_t*>(out_dev);
  a.ws = static_cast<float*>(workspace_dev);
  a.bunits = uint32_t(stride / 128);
  a.sunits = uint32_t(per_token / 128);
  // q = (umulhi(t, m) + t) >> l with l = ceil(log2 bs), m = floor(2^32 (2^l - bs) / bs) + 1
  while ((int64_t(1) << a.bs_shift) < bs) ++a.bs_shift;
  a.bs_magic = uint32_t((((uint64_t(1) << a.bs_shift) - uint64_t(bs)) << 32) / uint64_t(bs) + 1);
  a.pool_blocks = pool->num_blocks;
  a.block_size = int32_t(bs);
  a.max_blocks = max_blocks;
  a.max_seq_len = max_seq_len;
  a.n_tokens = n_tokens;
  a.n_req = n_req;
  a.q_heads = q_heads;
  a.kv_heads = kv_heads;
  a.group = q_heads / kv_heads;
  a.split_tokens = sh.split;
  a.splits = sh.splits;
  a.scale_log2 = scale * kLog2e;
  const int64_t tiles = int64_t(n_tokens) * a.group / kRows + n_req;
  const int64_t grid = tiles * kv_heads;
  const int64_t merge = (int64_t(n_tokens) * q_heads + kWaves - 1) / kWaves;
  if (grid > INT32_MAX / sh.splits || merge > INT32_MAX)
    return fail(FLOWKV_EINVAL, "%lld tiles of queries x %d splits: too many for one call",
                (long long)grid, sh.splits);
  a.tiles = int32_t(tiles);
  void* args[] = {&a};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const void* fn = head_dim == 64 ? reinterpret_cast<const void*>(chunk_attn<64>)
                                  : reinterpret_cast<const void*>(chunk_attn<128>);
  hipError_t e = hipLaunchKernel(fn, dim3(unsigned(grid * sh.splits)), dim3(kThreads), args, 0, st);
  if (e == hipSuccess && sh.splits > 1) {
    fn = head_dim == 64 ? reinterpret_cast<const void*>(chunk_attn_merge<64>)
                        : reinterpret_cast<const void*>(chunk_attn_merge<128>);
    e = hipLaunchKernel(fn, dim3(unsigned(merge)), dim3(kThreads), args, 0, st);
  }
  if (e == hipSuccess) e = hipGetLastError();
  if (e != hipSuccess) return fail(FLOWKV_EHIP, "chunk attention launch: %s", hipGetErrorString(e));
  return ok();
}
