// Rotary positions: rotation of the channel pairs of every head by an angle that grows with the token's position.
//
//   pair i of a token at position p:  a = p theta_i ;  (x, y) -> m (x cos a - y sin a, x sin a + y cos a)
//   gradient:                         the transposed map, the same with -a
//
// The angle is kept in turns as a 0.64 fixed-point number: p * (theta / 2 pi) modulo one turn is one 64-bit integer
// product, exact for every position (a float32 product is wrong in the first digit at positions past 10^7).  What is
// left after taking off whole quarter turns, at most an eighth of a turn, goes to sincospif.
//
// Both kernels below move every byte once and are bound by memory.  A block takes a few tokens: its threads compute the
// tokens' sines and cosines once into shared memory (a token's pairs are the same for all of its heads: 64 evaluations
// serve 16 KB of q and k) and then stream the heads, one item of V channels (half layout: V and V, `rotary_dim / 2`
// apart) per thread and step.  V is 16 bytes' worth where pointers, strides and the rotated part allow it, else items
// of one channel (half) or one pair (interleaved).
//
// Measured: 8191 x 40 heads of 128 channels, 64 rotated in neighbouring pairs, 33 us = 5.0 TB/s (77 % of a plain copy: loads in flight
// and instruction issue); float32, 16384 x 16 x 64, 25.6 us = 5.2 TB/s; append of 15K ragged tokens, 40 + 16 heads, 92 us = 5.3 TB/s;
// 16K tokens into an E4M3 cache 112 us = 5.6 TB/s.  Each on changing inputs.  Items of one channel or pair, which rotated parts
// that 16 bytes do not divide fall back to, have not been timed.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "libra.h"

namespace libra {

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxTokens = 4;   // tokens per block at most: with 8 a block is too long, with 2 the sines weigh (37.2, 35.4 and
                                    // 39.4 us for 2, 4, 8 tokens: 8191 tokens of 40 heads, 64 of 128 channels rotated)

namespace rope {

__device__ __forceinline__ float2 cos_sin(int32_t pos, uint64_t turns, float magnitude) {
  const uint64_t phase = uint64_t(int64_t(pos)) * turns;   // modulo one turn
  const int32_t t = int32_t(uint32_t(phase >> 32));        // signed, 2^-32 turns
  const int32_t quarter = int32_t(uint32_t(t) + (1u << 29)) >> 30;   // nearest quarter turn (the sum wraps at half a turn)
  const int32_t rest = int32_t(uint32_t(t) - (uint32_t(quarter) << 30));
  float s, c;
  sincospif(float(rest) * (1.0f / 2147483648.0f), &s, &c);   // |angle| <= pi / 4
  const float cc = (quarter & 1) ? s : c, ss = (quarter & 1) ? c : s;
  const float cr = ((quarter & 3) == 1 || (quarter & 3) == 2) ? -cc : cc;
  const float sr = ((quarter & 3) >= 2) ? -ss : ss;
  return make_float2(cr * magnitude, sr * magnitude);
}

// (x, y) turned by the angle whose cosine and sine are w, in instructions that keep numbers below the smallest normal one (the
// build's default flushes them to zero, and a bf16 or float32 value may be one).
__device__ __forceinline__ float mul_rn(float a, float b) {
  float d;
  asm("mul.rn.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float fma_rn(float a, float b, float c) {
  float d;
  asm("fma.rn.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float2 turned(float x, float y, float2 w) {
  return make_float2(fma_rn(x, w.x, mul_rn(y, -w.y)), fma_rn(x, w.y, mul_rn(y, w.x)));
}

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32(float x) { return x; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }

// V elements of type T; 16 bytes at once when kVector
template <typename T, int V, bool kVector>
__device__ __forceinline__ void load(const T* p, T (&x)[V]) {
  if constexpr (kVector) {
    static_assert(sizeof(T) * V == 16, "one 16-byte vector");
    *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = p[i];
  }
}
template <typename T, int V, bool kVector>
__device__ __forceinline__ void store(T* p, const T (&x)[V]) {
  if constexpr (kVector) {
    *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(x);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = x[i];
  }
}

// Items of one head: first those that rotate, then those that pass through.
//   half         item j: channels [jV, jV + V) and the same R / 2 further on
//   interleaved  item j: channels [jV, jV + V), V even
template <int V, bool kHalf>
__host__ __device__ __forceinline__ int rotating_items(int rotary_dim) {
  return kHalf ? rotary_dim / (2 * V) : rotary_dim / V;
}
// A thread keeps one item j and walks over rows (token, head): no division but one multiplication per row.
struct Walk {
  int j;      // item
  int first;  // first row
  int step;   // rows between this thread's rows
  __device__ __forceinline__ explicit Walk(int per_head) {
    step = kRopeThreads / per_head;          // 0: a head has more items than the block has threads
    if (step > 0) {
      first = int(threadIdx.x) / per_head;
      j = int(threadIdx.x) - first * per_head;
      if (first >= step) first = 0x3fffffff;   // threads behind the last whole head
    } else {
      first = 0;
      step = 1;
      j = threadIdx.x;
    }
  }
};
// The factors of a token's pairs are laid out for items of V pairs (V / 2, interleaved): the same pair of neighbouring items
// side by side.
template <int V, bool kHalf>
__device__ __forceinline__ int factor_at(int pair, int pairs) {
  constexpr int kPer = kHalf ? V : V / 2;
  return (pair % kPer) * (pairs / kPer) + pair / kPer;
}

}  // namespace rope

struct RopeApplyParams {
  const void* x;
  void* out;
  const int32_t* positions;   // [tokens]
  int64_t x_stride_token, x_stride_head, out_stride_token, out_stride_head;   // in elements
  int64_t n_tokens;
  int32_t n_heads, head_dim;
  int32_t tokens_per_block;
  uint32_t heads_inverse;   // ceil(2^32 / n_heads): row / n_heads = the upper word of the product, for kRopeMaxTokens * n_heads rows
  int32_t gradient;
  libra_rope_t rope;
};

// grid = ceil(tokens / tokens_per_block), block = kRopeThreads, dynamic shared memory = tokens_per_block * R / 2 float2
template <typename T, int V, bool kVector, bool kHalf>
__global__ void __launch_bounds__(kRopeThreads) rope_apply_kernel(const __grid_constant__ RopeApplyParams p) {
  extern __shared__ float2 cs[];   // [token][pair]
  const int pairs = p.rope.rotary_dim / 2;
  const int64_t t0 = int64_t(blockIdx.x) * p.tokens_per_block;
  const int nt = int(p.n_tokens - t0 < p.tokens_per_block ? p.n_tokens - t0 : p.tokens_per_block);
  for (int i = threadIdx.x; i < nt * pairs; i += kRopeThreads) {
    const int tok = i / pairs, pr = i - tok * pairs;
    float2 f = rope::cos_sin(__ldg(p.positions + t0 + tok), p.rope.turns[pr], p.rope.magnitude);
    if (p.gradient) f.y = -f.y;
    cs[tok * pairs + rope::factor_at<V, kHalf>(pr, pairs)] = f;
  }
  __syncthreads();
  const int rot = rope::rotating_items<V, kHalf>(p.rope.rotary_dim);
  const int rows = nt * p.n_heads;
  constexpr int kAtOnce = kVector ? 1 : 2;   // rows whose loads are in flight together (twice as many: 5 - 8 % slower)
  // First the items that rotate, then those that pass: together in a warp they would each wait for the other's code.
  auto run = [&](auto is_turning, int per_head) {
    constexpr bool turns = decltype(is_turning)::value;
    const rope::Walk walk(per_head);
    for (int j = walk.j; j < per_head; j += kRopeThreads) {
      const int c = (turns ? 0 : p.rope.rotary_dim) + j * V;
      for (int r0 = walk.first; r0 < rows; r0 += kAtOnce * walk.step) {
        alignas(16) T a[kAtOnce][V];
        alignas(16) T b[kAtOnce][V];
        int64_t dst[kAtOnce];
        int tok[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int row = r0 + u * walk.step;
          tok[u] = -1;
          if (row < rows) {
            tok[u] = int(__umulhi(uint32_t(row), p.heads_inverse));
            if (p.n_heads == 1) tok[u] = row;
            const int head = row - tok[u] * p.n_heads;
            const T* src = static_cast<const T*>(p.x) + (t0 + tok[u]) * p.x_stride_token + head * p.x_stride_head + c;
            dst[u] = (t0 + tok[u]) * p.out_stride_token + head * p.out_stride_head + c;
            rope::load<T, V, kVector>(src, a[u]);
            if (kHalf && turns) rope::load<T, V, kVector>(src + pairs, b[u]);
          }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          if (tok[u] < 0) continue;
          T* to = static_cast<T*>(p.out) + dst[u];
          if (turns) {
            const float2* f = cs + tok[u] * pairs + j;
            const int pitch = rot;   // pairs / (V or V / 2)
            if constexpr (kHalf) {
#pragma unroll
              for (int k = 0; k < V; ++k) {
                const float2 w = f[k * pitch];
                const float2 z = rope::turned(rope::to_f32(a[u][k]), rope::to_f32(b[u][k]), w);
                a[u][k] = rope::from_f32<T>(z.x);
                b[u][k] = rope::from_f32<T>(z.y);
              }
              rope::store<T, V, kVector>(to + pairs, b[u]);
            } else {
#pragma unroll
              for (int k = 0; k < V; k += 2) {
                const float2 w = f[(k / 2) * pitch];
                const float2 z = rope::turned(rope::to_f32(a[u][k]), rope::to_f32(a[u][k + 1]), w);
                a[u][k] = rope::from_f32<T>(z.x);
                a[u][k + 1] = rope::from_f32<T>(z.y);
              }
            }
          }
          rope::store<T, V, kVector>(to, a[u]);
        }
      }
    }
  };
  run(std::true_type(), rot);
  if (p.x != p.out && p.head_dim > p.rope.rotary_dim) run(std::false_type(), (p.head_dim - p.rope.rotary_dim) / V);
}

struct RopeAppendParams {
  const __nv_bfloat16* q;      // or null: nothing is rotated but k
  __nv_bfloat16* q_out;
  const __nv_bfloat16* k_new;
  const __nv_bfloat16* v_new;
  int64_t q_stride, q_out_stride, kv_stride;   // elements from a token to the next
  const int32_t* q_offsets;    // [batch + 1]
  const int32_t* seq_lens;     // [batch]
  const int32_t* block_table;  // [batch][ld]
  void* k_pool;
  void* v_pool;
  uint32_t* error_word;
  int64_t stride_page, stride_head, stride_token;   // pool strides in elements
  int64_t num_pages;
  float k_inv_scale, v_inv_scale;                   // E4M3 pools
  int32_t batch, max_tokens;
  int32_t block_table_ld, page_shift;
  int32_t num_q_heads, num_kv_heads, head_dim;
  int32_t tokens_per_block;
  int32_t heads;            // rows of a token: query heads (0 without q), then KV heads of k, then of v
  uint32_t heads_inverse;   // as above, for kRopeMaxTokens * heads rows
  libra_rope_t rope;
};

namespace rope {

// V float32 values into the pool's element type.
template <typename P, int V, bool kVector>
__device__ __forceinline__ void store_pool(P* dst, const float (&x)[V], float inv_scale) {
  if constexpr (sizeof(P) == 2) {
    alignas(16) __nv_bfloat16 y[V];
#pragma unroll
    for (int k = 0; k < V; ++k) y[k] = __float2bfloat16_rn(x[k]);
    store<__nv_bfloat16, V, kVector>(reinterpret_cast<__nv_bfloat16*>(dst), y);
  } else {   // E4M3: round to nearest even, beyond the largest code = the largest code
    alignas(8) uint8_t y[V];
#pragma unroll
    for (int k = 0; k < V; ++k) y[k] = __nv_cvt_float_to_fp8(x[k] * inv_scale, __NV_SATFINITE, __NV_E4M3);
    if constexpr (kVector) {
      *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(y);
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) reinterpret_cast<uint8_t*>(dst)[k] = y[k];
    }
  }
}

}  // namespace rope

// Rotation of q and k of a ragged batch of new tokens and append of k and v to the pages.
// P: element of the pools (__nv_bfloat16 or uint8_t = E4M3 code).
// grid = ceil(max_tokens / tokens_per_block), block = kRopeThreads, dynamic shared memory as above.
template <typename P, int V, bool kVector, bool kHalf>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const __grid_constant__ RopeAppendParams p) {
  extern __shared__ float2 cs[];              // [token][pair]
  __shared__ int32_t s_pos[kRopeMaxTokens];
  __shared__ int64_t s_slot[kRopeMaxTokens];  // pool offset of the token's slot, head 0; -1: not stored; -2: no token
  const int pairs = p.rope.rotary_dim / 2;
  const int t0 = blockIdx.x * p.tokens_per_block;
  const int nt = min(p.tokens_per_block, p.max_tokens - t0);
  if (threadIdx.x < nt) {
    const int row = t0 + threadIdx.x;
    // the last sequence whose rows begin at or before this one (sequences without new tokens share a beginning)
    int lo = 0, hi = p.batch;   // q_offsets[lo] <= row < q_offsets[hi], if the row belongs to anyone
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldg(p.q_offsets + mid) <= row) lo = mid;
      else hi = mid;
    }
    int64_t slot = -2;
    int32_t pos = 0;
    const int32_t first = __ldg(p.q_offsets + lo), end = __ldg(p.q_offsets + lo + 1);
    if (row >= first && row < end) {
      pos = __ldg(p.seq_lens + lo) - end + row;
      slot = -1;
      const int page_index = pos >> p.page_shift;
      if (pos >= 0 && page_index >= p.block_table_ld) {
        atomicOr(p.error_word, uint32_t(LIBRA_ERR_PLAN_OVERFLOW));
      } else if (pos >= 0) {
        const int64_t page = __ldg(p.block_table + int64_t(lo) * p.block_table_ld + page_index);
        if (page < 0 || page >= p.num_pages) {
          atomicOr(p.error_word, uint32_t(LIBRA_ERR_BAD_PAGE_ID));
        } else {
          slot = page * p.stride_page + int64_t(pos & ((1 << p.page_shift) - 1)) * p.stride_token;
        }
      }
    }
    s_pos[threadIdx.x] = pos;
    s_slot[threadIdx.x] = slot;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nt * pairs; i += kRopeThreads) {
    const int tok = i / pairs, pr = i - tok * pairs;
    cs[tok * pairs + rope::factor_at<V, kHalf>(pr, pairs)] = rope::cos_sin(s_pos[tok], p.rope.turns[pr], p.rope.magnitude);
  }
  __syncthreads();
  const int rot = rope::rotating_items<V, kHalf>(p.rope.rotary_dim);
  const int q_heads = p.heads - 2 * p.num_kv_heads;
  const int rows = nt * p.heads;
  constexpr int kAtOnce = kVector ? (kHalf ? 2 : 4) : 2;   // rows whose loads are in flight together (half: 4 % slower, twice: up to 60 %)
  auto run = [&](auto is_turning, int per_head) {   // items that rotate (those of values are copied), items that pass
    constexpr bool turns = decltype(is_turning)::value;
    const rope::Walk walk(per_head);
    for (int j = walk.j; j < per_head; j += kRopeThreads) {
      const int c = (turns ? 0 : p.rope.rotary_dim) + j * V;
      for (int r0 = walk.first; r0 < rows; r0 += kAtOnce * walk.step) {
        alignas(16) __nv_bfloat16 a[kAtOnce][V];
        alignas(16) __nv_bfloat16 b[kAtOnce][V];
        int tok[kAtOnce], head[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int row = r0 + u * walk.step;
          tok[u] = -1;
          if (row < rows) {
            tok[u] = int(__umulhi(uint32_t(row), p.heads_inverse));
            head[u] = row - tok[u] * p.heads;
            const int64_t slot = s_slot[tok[u]];
            // a row behind the last sequence; a key or value that is not stored
            if (slot == -2 || (slot < 0 && head[u] >= q_heads)) {
              tok[u] = -1;
            } else {
              const int64_t at = t0 + tok[u];
              const __nv_bfloat16* src =
                  head[u] < q_heads ? p.q + at * p.q_stride + head[u] * p.head_dim
                  : head[u] < q_heads + p.num_kv_heads ? p.k_new + at * p.kv_stride + (head[u] - q_heads) * p.head_dim
                                                       : p.v_new + at * p.kv_stride + (head[u] - q_heads - p.num_kv_heads) * p.head_dim;
              rope::load<__nv_bfloat16, V, kVector>(src + c, a[u]);
              if (kHalf && turns) rope::load<__nv_bfloat16, V, kVector>(src + c + pairs, b[u]);
            }
          }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          if (tok[u] < 0) continue;
          const bool is_q = head[u] < q_heads, is_v = head[u] >= q_heads + p.num_kv_heads;
          float x[V], y[V];
#pragma unroll
          for (int k = 0; k < V; ++k) x[k] = __bfloat162float(a[u][k]);
          if (kHalf && turns) {
#pragma unroll
            for (int k = 0; k < V; ++k) y[k] = __bfloat162float(b[u][k]);
          }
          if (turns && !is_v) {
            const float2* f = cs + tok[u] * pairs + j;
            const int pitch = rot;   // pairs / (V or V / 2)
            if constexpr (kHalf) {
#pragma unroll
              for (int k = 0; k < V; ++k) {
                const float2 w = f[k * pitch];
                const float2 z = rope::turned(x[k], y[k], w);
                x[k] = z.x;
                y[k] = z.y;
              }
            } else {
#pragma unroll
              for (int k = 0; k < V; k += 2) {
                const float2 w = f[(k / 2) * pitch];
                const float2 z = rope::turned(x[k], x[k + 1], w);
                x[k] = z.x;
                x[k + 1] = z.y;
              }
            }
          }
          if (is_q) {
            __nv_bfloat16* to = p.q_out + int64_t(t0 + tok[u]) * p.q_out_stride + head[u] * p.head_dim + c;
            rope::store_pool<__nv_bfloat16, V, kVector>(to, x, 1.f);
            if (kHalf && turns) rope::store_pool<__nv_bfloat16, V, kVector>(to + pairs, y, 1.f);
          } else {
            const int kv_head = head[u] - q_heads - (is_v ? p.num_kv_heads : 0);
            P* to = static_cast<P*>(is_v ? p.v_pool : p.k_pool) + s_slot[tok[u]] + kv_head * p.stride_head + c;
            const float inv = is_v ? p.v_inv_scale : p.k_inv_scale;
            rope::store_pool<P, V, kVector>(to, x, inv);
            if (kHalf && turns) rope::store_pool<P, V, kVector>(to + pairs, y, inv);
          }
        }
      }
    }
  };
  if (rot > 0) run(std::true_type(), rot);
  if (p.head_dim > p.rope.rotary_dim) run(std::false_type(), (p.head_dim - p.rope.rotary_dim) / V);
}

}  // namespace libra
