// Norm of every head of q and k, rotation by position in the same pass, and the gradient of both.
//
//   r = 1 / sqrt(mean(x^2) + eps),   y = R(a) (w x r)          x: one head of one token, w: one weight per channel, R(a): the
//                                                              rotation of rope_kernel.cuh at the token's position
//   g = R(a)^T dy,   dw = sum over tokens and heads of g x r,   dx = r (w g - x r mean(w g x r))
//
// Arithmetic in float32, one rounding to the type.  Neither r nor the normalised x is kept for the gradient: x has to be read there
// in any case.  The two sums of a row of the gradient, of x^2 and of w g x, are found in the same pass.
//
// Every byte moves once; memory bounds it.  Work is shared out by warps, without a barrier of the block: a unit is a few rows (heads)
// of one token and one kind (q, k, v).  A row is held by a group of neighbouring lanes, each with one item of two 16-byte vectors
// whose channels turn together (half layout: R / 2 apart), so that a row's sums take one reduction within the group and nothing goes
// through shared memory but the cosines, which the warp's lanes work out together once a unit.  Rows that this does not fit (rotated
// parts that 16 bytes do not divide, addresses off a 16-byte boundary, heads of more items than a warp has lanes) go through
// shared memory, row by row, in the kernels at the end.
//
// dw is summed in registers along a warp's rows, then over the warps and the blocks in a fixed order: the same bits every time.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "libra.h"
#include "rope_kernel.cuh"

namespace libra {

constexpr int kNormThreads = 256, kNormWarps = kNormThreads / 32;
constexpr int kNormRows = 2;      // rows of a group of lanes whose loads are in flight together
constexpr int kNormAnyThreads = 128, kNormAnyWarps = kNormAnyThreads / 32;   // the kernels that go through shared memory

struct NormKind {         // q, k or v
  const void* x;
  const void* grad;       // gradient: of the output
  const void* weight;     // null: no norm and, for v, no rotation
  void* out;              // gradient: of x
  int64_t x_token, x_head, grad_token, grad_head, out_token, out_head;   // in elements
  int32_t n_heads;        // 0: absent
  int32_t units;          // of a token
};

struct NormParams {
  NormKind kind[3];
  const int32_t* positions;
  const int32_t* slots;        // append: of every row, -1: not stored
  const int32_t* n_rows;       // append: rows there are, or null
  uint32_t* error_word;
  float* partial;              // gradient: [block][head_dim]
  int64_t n_tokens;
  int64_t num_slots;           // append
  int64_t stride_page, stride_head, stride_token;   // of the pools, in elements
  float k_inv_scale, v_inv_scale;
  float eps, inv_dim;
  int32_t head_dim, page_shift;
  int32_t units;               // of a token, of all kinds
  int32_t items, lanes;        // of a row; lanes: the power of two that holds them
  int32_t first_blocks;        // gradient: blocks [0, first_blocks) take kind 0, the others kind 1
  libra_rope_t rope;
};

namespace norm {

using rope::fma_rn;
using rope::mul_rn;

template <typename T> constexpr int kVec = 16 / int(sizeof(T));

// Channel of an item's first vector, whether it is turned, and the second vector's (head_dim and beyond: there is none).
//   half         items that turn: [iV, iV + V) and the same R / 2 on; then the rest in neighbouring pairs of vectors
//   interleaved  2 V channels on end
template <int V, bool kHalf>
struct Item {
  int c0, c1;
  bool turn0, turn1;
  __device__ __forceinline__ Item(int i, int rotary) {
    const int turning = kHalf ? rotary / (2 * V) : 0;
    if (kHalf && i < turning) {
      c0 = i * V;
      c1 = c0 + rotary / 2;
    } else {
      c0 = (kHalf ? rotary : 0) + (i - turning) * 2 * V;
      c1 = c0 + V;
    }
    turn0 = c0 < rotary;
    turn1 = c1 < rotary;
  }
};

// The token's cosines and sines into the warp's part of shared memory: item i's V pairs as V / 2 vectors, vector j of all items
// side by side.
template <int V>
__device__ __forceinline__ void turn_factors(float2* cs, const uint64_t* turns, int pairs, int row_items, int32_t pos, float magnitude, int lane) {
  for (int pr = lane; pr < pairs; pr += 32) {
    const int item = pr / V, j = (pr % V) / 2;
    cs[2 * (j * row_items + item) + (pr & 1)] = rope::cos_sin(pos, turns[pr], magnitude);
  }
}
template <int V>
__device__ __forceinline__ void load_factors(float2 (&w)[V], const float2* cs, int row_items, int item) {
#pragma unroll
  for (int j = 0; j < V / 2; ++j) {
    const float4 f = reinterpret_cast<const float4*>(cs)[j * row_items + item];
    w[2 * j] = make_float2(f.x, f.y);
    w[2 * j + 1] = make_float2(f.z, f.w);
  }
}

template <typename T, int V>
__device__ __forceinline__ void unpack(const uint4& raw, float* f) {
  const T* t = reinterpret_cast<const T*>(&raw);
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = rope::to_f32(t[i]);
}
template <typename T, int V>
__device__ __forceinline__ uint4 packed(const float* f) {
  uint4 raw;
  T* t = reinterpret_cast<T*>(&raw);
#pragma unroll
  for (int i = 0; i < V; ++i) t[i] = rope::from_f32<T>(f[i]);
  return raw;
}

// Turns an item's channels (back: by the negative angle).
template <int V, bool kHalf, bool kBack>
__device__ __forceinline__ void turn(float (&y)[2 * V], const Item<V, kHalf>& it, const float2 (&w)[V]) {
  auto pair = [&](float& a, float& b, float2 f) {
    const float2 z = rope::turned(a, b, kBack ? make_float2(f.x, -f.y) : f);
    a = z.x;
    b = z.y;
  };
  if constexpr (kHalf) {
    if (it.turn0) {
#pragma unroll
      for (int i = 0; i < V; ++i) pair(y[i], y[V + i], w[i]);
    }
  } else {
    if (it.turn0) {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) pair(y[2 * i], y[2 * i + 1], w[i]);
    }
    if (it.turn1) {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) pair(y[V + 2 * i], y[V + 2 * i + 1], w[V / 2 + i]);
    }
  }
}

__device__ __forceinline__ float group_sum(float x, int lanes) {
  for (int off = lanes >> 1; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
  return x;
}

// A warp's walk over units: unit u of the launch is unit u % units of token u / units.
struct Units {
  int64_t token;
  int32_t unit;
  __device__ __forceinline__ Units(int64_t first, int32_t units) : token(first / units), unit(int32_t(first - token * units)) {}
  __device__ __forceinline__ void advance(int64_t tokens, int32_t rest, int32_t units) {
    token += tokens;
    unit += rest;
    if (unit >= units) {
      unit -= units;
      ++token;
    }
  }
};

// Offset of a row's slot in the pools; -1: the row is not stored.
__device__ __forceinline__ int64_t slot_offset(const NormParams& p, int64_t row) {
  const int32_t slot = __ldg(p.slots + row);
  if (slot == -1) return -1;
  if (slot < 0 || slot >= p.num_slots) {
    atomicOr(p.error_word, uint32_t(LIBRA_ERR_BAD_PAGE_ID));
    return -1;
  }
  return int64_t(slot >> p.page_shift) * p.stride_page + int64_t(slot & ((1 << p.page_shift) - 1)) * p.stride_token;
}

}  // namespace norm

// T: type of the rows; P: of the pools (append).  Any number of blocks; shared memory: the cosines.
template <typename T, typename P, bool kHalf, bool kAppend>
__global__ void __launch_bounds__(kNormThreads, 4) norm_rope_kernel(const __grid_constant__ NormParams p) {
  using namespace norm;
  constexpr int V = kVec<T>;
  __shared__ uint64_t turns[LIBRA_ROPE_MAX_PAIRS];
  __shared__ alignas(16) float2 factors[kNormWarps][LIBRA_ROPE_MAX_PAIRS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int R = p.rope.rotary_dim, pairs = R / 2;
  for (int i = threadIdx.x; i < pairs; i += kNormThreads) turns[i] = p.rope.turns[i];
  if constexpr (kAppend) asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  float2* const cs = factors[warp];
  const int item = lane & (p.lanes - 1), group = lane / p.lanes, groups = 32 / p.lanes;
  const bool on = item < p.items;
  const int turn_items = (pairs + V - 1) / V;
  const Item<V, kHalf> it(item, R);
  const bool two = it.c1 < p.head_dim;
  int64_t n_tokens = p.n_tokens;
  if (kAppend && p.n_rows) n_tokens = min(n_tokens, int64_t(*p.n_rows));
  const int64_t stride = int64_t(gridDim.x) * kNormWarps, first = int64_t(blockIdx.x) * kNormWarps + warp;
  const int64_t by_tokens = stride / p.units;
  const int32_t by_rest = int32_t(stride - by_tokens * p.units);
  for (Units u(first, p.units); u.token < n_tokens; u.advance(by_tokens, by_rest, p.units)) {
    int unit = u.unit, kd = 0;
    if (unit >= p.kind[0].units) {
      unit -= p.kind[0].units;
      kd = 1;
      if (unit >= p.kind[1].units) {
        unit -= p.kind[1].units;
        kd = 2;
      }
    }
    const NormKind& kind = p.kind[kd];
    const int head0 = unit * (kNormRows * groups) + group;
    const T* const src = static_cast<const T*>(kind.x) + u.token * kind.x_token;
    uint4 raw[kNormRows][2];
#pragma unroll
    for (int k = 0; k < kNormRows; ++k) {
      const int head = head0 + k * groups;
      raw[k][0] = raw[k][1] = make_uint4(0, 0, 0, 0);
      if (on && head < kind.n_heads) {
        const T* const row = src + head * kind.x_head;
        raw[k][0] = *reinterpret_cast<const uint4*>(row + it.c0);
        if (two) raw[k][1] = *reinterpret_cast<const uint4*>(row + it.c1);
      }
    }
    const bool pool = kAppend && kd > 0;
    const int64_t at = pool ? slot_offset(p, u.token) : u.token * kind.out_token;
    const bool normed = kind.weight != nullptr, turned = !(kAppend && kd == 2) && R > 0;
    float w[2 * V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) w[i] = 1.f;
    if (normed && on) {
      unpack<T, V>(__ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(kind.weight) + it.c0)), w);
      if (two) unpack<T, V>(__ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(kind.weight) + it.c1)), w + V);
    }
    float2 f[V];
    if (turned) {
      __syncwarp();   // the unit before has read its own
      turn_factors<V>(cs, turns, pairs, turn_items, __ldg(p.positions + u.token), p.rope.magnitude, lane);
      __syncwarp();
      load_factors<V>(f, cs, turn_items, min(item, max(turn_items - 1, 0)));
    }
#pragma unroll
    for (int k = 0; k < kNormRows; ++k) {
      const int head = head0 + k * groups;
      float y[2 * V];
      unpack<T, V>(raw[k][0], y);
      unpack<T, V>(raw[k][1], y + V);
      if (normed) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) sum = fmaf(y[i], y[i], sum);
        sum = group_sum(sum, p.lanes);
        const float r = __frsqrt_rn(fmaf(sum, p.inv_dim, p.eps));
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) y[i] = mul_rn(mul_rn(y[i], r), w[i]);
      }
      if (turned) turn<V, kHalf, false>(y, it, f);
      if (!on || head >= kind.n_heads) continue;
      if (!pool) {
        T* const row = static_cast<T*>(kind.out) + at + head * kind.out_head;
        *reinterpret_cast<uint4*>(row + it.c0) = packed<T, V>(y);
        if (two) *reinterpret_cast<uint4*>(row + it.c1) = packed<T, V>(y + V);
      } else if (at >= 0) {
        if constexpr (kAppend) {
          P* const row = static_cast<P*>(kind.out) + at + head * p.stride_head;
          const float inv = kd == 1 ? p.k_inv_scale : p.v_inv_scale;
          rope::store_pool<P, V, true>(row + it.c0, *reinterpret_cast<const float(*)[V]>(y), inv);
          if (two) rope::store_pool<P, V, true>(row + it.c1, *reinterpret_cast<const float(*)[V]>(y + V), inv);
        }
      }
    }
  }
}

// One kind a block; the rows' channels are summed into partial[block].
template <typename T, bool kHalf>
__global__ void __launch_bounds__(kNormThreads, 2) norm_rope_gradient_kernel(const __grid_constant__ NormParams p) {
  using namespace norm;
  constexpr int V = kVec<T>;
  __shared__ uint64_t turns[LIBRA_ROPE_MAX_PAIRS];
  __shared__ alignas(16) float2 factors[kNormWarps][LIBRA_ROPE_MAX_PAIRS];
  extern __shared__ float sums[];   // [warps][head_dim]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int R = p.rope.rotary_dim, pairs = R / 2;
  for (int i = threadIdx.x; i < pairs; i += kNormThreads) turns[i] = p.rope.turns[i];
  __syncthreads();
  float2* const cs = factors[warp];
  const int kd = int(blockIdx.x) < p.first_blocks ? 0 : 1;
  const int block = kd == 0 ? blockIdx.x : blockIdx.x - p.first_blocks;
  const int blocks = kd == 0 ? p.first_blocks : gridDim.x - p.first_blocks;
  const NormKind& kind = p.kind[kd];
  const int item = lane & (p.lanes - 1), group = lane / p.lanes, groups = 32 / p.lanes;
  const bool on = item < p.items;
  const int turn_items = (pairs + V - 1) / V;
  const Item<V, kHalf> it(item, R);
  const bool two = it.c1 < p.head_dim;
  float w[2 * V], acc[2 * V];
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) w[i] = acc[i] = 0.f;
  if (on) {
    unpack<T, V>(__ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(kind.weight) + it.c0)), w);
    if (two) unpack<T, V>(__ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(kind.weight) + it.c1)), w + V);
  }
  const int64_t stride = int64_t(blocks) * kNormWarps, first = int64_t(block) * kNormWarps + warp;
  const int64_t by_tokens = stride / kind.units;
  const int32_t by_rest = int32_t(stride - by_tokens * kind.units);
  for (Units u(first, kind.units); u.token < p.n_tokens; u.advance(by_tokens, by_rest, kind.units)) {
    const int head0 = u.unit * (kNormRows * groups) + group;
    const T* const src = static_cast<const T*>(kind.x) + u.token * kind.x_token;
    const T* const grad = static_cast<const T*>(kind.grad) + u.token * kind.grad_token;
    uint4 raw[kNormRows][2], graw[kNormRows][2];
#pragma unroll
    for (int k = 0; k < kNormRows; ++k) {
      const int head = head0 + k * groups;
      raw[k][0] = raw[k][1] = graw[k][0] = graw[k][1] = make_uint4(0, 0, 0, 0);
      if (on && head < kind.n_heads) {
        const T* const row = src + head * kind.x_head;
        const T* const grow = grad + head * kind.grad_head;
        raw[k][0] = *reinterpret_cast<const uint4*>(row + it.c0);
        graw[k][0] = *reinterpret_cast<const uint4*>(grow + it.c0);
        if (two) {
          raw[k][1] = *reinterpret_cast<const uint4*>(row + it.c1);
          graw[k][1] = *reinterpret_cast<const uint4*>(grow + it.c1);
        }
      }
    }
    float2 f[V];
    if (R > 0) {
      __syncwarp();
      turn_factors<V>(cs, turns, pairs, turn_items, __ldg(p.positions + u.token), p.rope.magnitude, lane);
      __syncwarp();
      load_factors<V>(f, cs, turn_items, min(item, max(turn_items - 1, 0)));
    }
#pragma unroll
    for (int k = 0; k < kNormRows; ++k) {
      const int head = head0 + k * groups;
      float x[2 * V], g[2 * V];
      unpack<T, V>(raw[k][0], x);
      unpack<T, V>(raw[k][1], x + V);
      unpack<T, V>(graw[k][0], g);
      unpack<T, V>(graw[k][1], g + V);
      if (R > 0) turn<V, kHalf, true>(g, it, f);
      float square = 0.f, dot = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) {
        square = fmaf(x[i], x[i], square);
        dot = fmaf(mul_rn(g[i], w[i]), x[i], dot);
      }
      square = group_sum(square, p.lanes);
      dot = group_sum(dot, p.lanes);
      if (!on || head >= kind.n_heads) continue;
      const float r = __frsqrt_rn(fmaf(square, p.inv_dim, p.eps));
      const float mean = mul_rn(mul_rn(dot, p.inv_dim), r);   // of w g x r
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) {
        const float n = mul_rn(x[i], r);
        acc[i] = fma_rn(g[i], n, acc[i]);
        g[i] = mul_rn(r, fma_rn(-n, mean, mul_rn(g[i], w[i])));
      }
      T* const row = static_cast<T*>(kind.out) + u.token * kind.out_token + head * kind.out_head;
      *reinterpret_cast<uint4*>(row + it.c0) = packed<T, V>(g);
      if (two) *reinterpret_cast<uint4*>(row + it.c1) = packed<T, V>(g + V);
    }
  }
  // groups of a warp, then the warps
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) {
    for (int off = p.lanes; off < 32; off <<= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], off);
  }
  if (on && group == 0) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sums[warp * p.head_dim + it.c0 + i] = acc[i];
      if (two) sums[warp * p.head_dim + it.c1 + i] = acc[V + i];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < p.head_dim; c += kNormThreads) {
    float s = 0.f;
    for (int i = 0; i < kNormWarps; ++i) s += sums[i * p.head_dim + c];
    p.partial[int64_t(blockIdx.x) * p.head_dim + c] = s;
  }
}

struct NormSumParams {
  const float* partial;
  float* out[2];
  int32_t head_dim;
  int32_t begin[3];   // blocks of each kind
};

constexpr int kNormSumSlices = 32;

// The blocks' sums: grid = (ceil(head_dim / 32), kinds), 32 channels x 32 slices of the blocks
__global__ void __launch_bounds__(32 * kNormSumSlices) norm_sum_kernel(const NormSumParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ float part[kNormSumSlices][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  float s = 0.f;
  if (c < p.head_dim) {
    for (int b = p.begin[blockIdx.y] + slice; b < p.begin[blockIdx.y + 1]; b += kNormSumSlices) s += p.partial[int64_t(b) * p.head_dim + c];
  }
  part[slice][threadIdx.x & 31] = s;
  __syncthreads();
  if (slice == 0 && c < p.head_dim) {
    s = 0.f;
    for (int i = 0; i < kNormSumSlices; ++i) s += part[i][threadIdx.x];
    p.out[blockIdx.y][c] = s;
  }
}

// ---------------------------------------------------------------------------------------------- rows through shared memory
// One row a warp, V channels a lane and step (16 bytes, or one).  Unit = one row.
// Dynamic shared memory: [warps][head_dim] floats (gradient: three times that)
template <typename T, typename P, int V, bool kVector, bool kHalf, bool kAppend>
__global__ void __launch_bounds__(kNormAnyThreads) norm_rope_any_kernel(const __grid_constant__ NormParams p) {
  using namespace norm;
  extern __shared__ float rows[];
  __shared__ uint64_t turns[LIBRA_ROPE_MAX_PAIRS];
  __shared__ float2 factors[kNormAnyWarps][LIBRA_ROPE_MAX_PAIRS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = p.head_dim;
  const int R = p.rope.rotary_dim, pairs = R / 2;
  for (int i = threadIdx.x; i < pairs; i += kNormAnyThreads) turns[i] = p.rope.turns[i];
  if constexpr (kAppend) asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  float* const row = rows + warp * D;
  float2* const cs = factors[warp];
  int64_t n_tokens = p.n_tokens;
  if (kAppend && p.n_rows) n_tokens = min(n_tokens, int64_t(*p.n_rows));
  const int64_t stride = int64_t(gridDim.x) * kNormAnyWarps, first = int64_t(blockIdx.x) * kNormAnyWarps + warp;
  const int64_t by_tokens = stride / p.units;
  const int32_t by_rest = int32_t(stride - by_tokens * p.units);
  for (Units u(first, p.units); u.token < n_tokens; u.advance(by_tokens, by_rest, p.units)) {
    int head = u.unit, kd = 0;
    if (head >= p.kind[0].units) {
      head -= p.kind[0].units;
      kd = 1;
      if (head >= p.kind[1].units) {
        head -= p.kind[1].units;
        kd = 2;
      }
    }
    const NormKind& kind = p.kind[kd];
    const T* const src = static_cast<const T*>(kind.x) + u.token * kind.x_token + head * kind.x_head;
    const bool pool = kAppend && kd > 0;
    const int64_t at = pool ? slot_offset(p, u.token) : u.token * kind.out_token;
    const bool normed = kind.weight != nullptr, turned = !(kAppend && kd == 2) && R > 0;
    __syncwarp();   // the row before has been read
    if (turned) {
      const int32_t pos = __ldg(p.positions + u.token);
      for (int i = lane; i < pairs; i += 32) cs[i] = rope::cos_sin(pos, turns[i], p.rope.magnitude);
    }
    float sum = 0.f;
    for (int c = lane * V; c < D; c += 32 * V) {
      alignas(16) T x[V];
      rope::load<T, V, kVector>(src + c, x);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float y = rope::to_f32(x[i]);
        row[c + i] = y;
        sum = fmaf(y, y, sum);
      }
    }
    float r = 1.f;
    if (normed) r = __frsqrt_rn(fmaf(group_sum(sum, 32), p.inv_dim, p.eps));
    __syncwarp();
    auto value = [&](int c) {
      return normed ? mul_rn(mul_rn(row[c], r), rope::to_f32(static_cast<const T*>(kind.weight)[c])) : row[c];
    };
    for (int c = lane * V; c < D; c += 32 * V) {
      float y[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int ch = c + i;
        if (turned && ch < R) {
          const bool second = kHalf ? ch >= pairs : (ch & 1);
          const int other = kHalf ? (second ? ch - pairs : ch + pairs) : ch ^ 1;
          const float2 f = cs[kHalf ? (second ? ch - pairs : ch) : ch >> 1];
          const float2 z = second ? rope::turned(value(other), value(ch), f) : rope::turned(value(ch), value(other), f);
          y[i] = second ? z.y : z.x;
        } else {
          y[i] = value(ch);
        }
      }
      if (!pool) {
        alignas(16) T t[V];
#pragma unroll
        for (int i = 0; i < V; ++i) t[i] = rope::from_f32<T>(y[i]);
        rope::store<T, V, kVector>(static_cast<T*>(kind.out) + at + head * kind.out_head + c, t);
      } else if (at >= 0) {
        if constexpr (kAppend) {
          rope::store_pool<P, V, kVector>(static_cast<P*>(kind.out) + at + head * p.stride_head + c, y, kd == 1 ? p.k_inv_scale : p.v_inv_scale);
        }
      }
    }
  }
}

template <typename T, int V, bool kVector, bool kHalf>
__global__ void __launch_bounds__(kNormAnyThreads) norm_rope_gradient_any_kernel(const __grid_constant__ NormParams p) {
  using namespace norm;
  extern __shared__ float rows[];
  __shared__ uint64_t turns[LIBRA_ROPE_MAX_PAIRS];
  __shared__ float2 factors[kNormAnyWarps][LIBRA_ROPE_MAX_PAIRS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = p.head_dim;
  const int R = p.rope.rotary_dim, pairs = R / 2;
  for (int i = threadIdx.x; i < pairs; i += kNormAnyThreads) turns[i] = p.rope.turns[i];
  float* const sums = rows + warp * D;                            // [warps][D]: a lane's channels are its own
  float* const xs = rows + (kNormAnyWarps + warp) * D;
  float* const gs = rows + (2 * kNormAnyWarps + warp) * D;
  for (int c = threadIdx.x; c < kNormAnyWarps * D; c += kNormAnyThreads) rows[c] = 0.f;
  __syncthreads();
  float2* const cs = factors[warp];
  const int kd = int(blockIdx.x) < p.first_blocks ? 0 : 1;
  const int block = kd == 0 ? blockIdx.x : blockIdx.x - p.first_blocks;
  const int blocks = kd == 0 ? p.first_blocks : gridDim.x - p.first_blocks;
  const NormKind& kind = p.kind[kd];
  const T* const weight = static_cast<const T*>(kind.weight);
  const int64_t stride = int64_t(blocks) * kNormAnyWarps, first = int64_t(block) * kNormAnyWarps + warp;
  const int64_t by_tokens = stride / kind.units;
  const int32_t by_rest = int32_t(stride - by_tokens * kind.units);
  for (Units u(first, kind.units); u.token < p.n_tokens; u.advance(by_tokens, by_rest, kind.units)) {
    const int head = u.unit;
    const T* const src = static_cast<const T*>(kind.x) + u.token * kind.x_token + head * kind.x_head;
    const T* const grad = static_cast<const T*>(kind.grad) + u.token * kind.grad_token + head * kind.grad_head;
    __syncwarp();
    if (R > 0) {
      const int32_t pos = __ldg(p.positions + u.token);
      for (int i = lane; i < pairs; i += 32) cs[i] = rope::cos_sin(pos, turns[i], p.rope.magnitude);
    }
    float square = 0.f;
    for (int c = lane * V; c < D; c += 32 * V) {
      alignas(16) T x[V];
      alignas(16) T g[V];
      rope::load<T, V, kVector>(src + c, x);
      rope::load<T, V, kVector>(grad + c, g);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float y = rope::to_f32(x[i]);
        xs[c + i] = y;
        gs[c + i] = rope::to_f32(g[i]);
        square = fmaf(y, y, square);
      }
    }
    __syncwarp();
    auto back = [&](int ch) {   // the gradient, turned back
      if (ch >= R) return gs[ch];
      const bool second = kHalf ? ch >= pairs : (ch & 1);
      const int other = kHalf ? (second ? ch - pairs : ch + pairs) : ch ^ 1;
      const float2 f = cs[kHalf ? (second ? ch - pairs : ch) : ch >> 1], b = make_float2(f.x, -f.y);
      const float2 z = second ? rope::turned(gs[other], gs[ch], b) : rope::turned(gs[ch], gs[other], b);
      return second ? z.y : z.x;
    };
    float dot = 0.f;
    for (int c = lane * V; c < D; c += 32 * V) {
#pragma unroll
      for (int i = 0; i < V; ++i) dot = fmaf(mul_rn(back(c + i), rope::to_f32(weight[c + i])), xs[c + i], dot);
    }
    const float r = __frsqrt_rn(fmaf(group_sum(square, 32), p.inv_dim, p.eps));
    const float mean = mul_rn(mul_rn(group_sum(dot, 32), p.inv_dim), r);
    for (int c = lane * V; c < D; c += 32 * V) {
      alignas(16) T t[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float n = mul_rn(xs[c + i], r), g = back(c + i);
        sums[c + i] = fma_rn(g, n, sums[c + i]);
        t[i] = rope::from_f32<T>(mul_rn(r, fma_rn(-n, mean, mul_rn(g, rope::to_f32(weight[c + i])))));
      }
      rope::store<T, V, kVector>(static_cast<T*>(kind.out) + u.token * kind.out_token + head * kind.out_head + c, t);
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < D; c += kNormAnyThreads) {
    float s = 0.f;
    for (int i = 0; i < kNormAnyWarps; ++i) s += rows[i * D + c];
    p.partial[int64_t(blockIdx.x) * D + c] = s;
  }
}

}  // namespace libra
