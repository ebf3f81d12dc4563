// Norm of every head of q and k, rotation by position in the same pass, and the gradient of both.
//
//   r = 1 / sqrt(mean(x^2) + eps),   y = R(a) (w x r)          x: one head of one token, w: one weight per channel, R(a): the
//                                                              rotation of rope_kernel.cuh at the token's position
//   g = R(a)^T dy,   dw = sum over tokens and heads of g x r,   dx = r (w g - x r mean(w g x r))
//
// Arithmetic in float32, one rounding to the type.  Neither r nor the normalised x is kept for the gradient: x has to be read there
// in any case.  A row of the gradient takes two sums, of x^2 and then of w g x r: every value on the way is one of the formula's.
//
// Every byte moves once; memory bounds it.  A step is the rows (heads) of one token and one kind (q, k, v) that a warp holds at once: a
// row is held by a group of neighbouring lanes, each with one item of two vectors (of 16 bytes, or 8) whose channels turn together (half layout:
// R / 2 apart), so that a row's sum takes one reduction within the group (the gradient's two) and nothing but cosines goes from lane to lane.  Every warp
// takes a run of consecutive steps, without a barrier of the block: a token's cosines and sines are worked out once in the run, by all
// lanes, and multiplied by the weights into four factors a pair, so that norm, weight and rotation are six multiplications a pair, two
// pairs an instruction.  Rows that this does not fit (rotated parts or heads that the items do not divide, addresses off a 16-byte boundary, heads of
// more items than a warp has lanes) are held whole in shared memory, one a warp, in the kernels at the end.
//
// The kernels may be launched while the one before still runs and wait for it first (programmatic dependent launch).  What that one may
// have written - positions, slots, weights too - is therefore read by ordinary loads: the read-only path's could be moved ahead of the wait.
//
// dw is summed in registers along a warp's run, then over the warps and the blocks in a fixed order: the same bits every time.
//
// Measured (device, changing inputs): 8191 tokens of 40 + 8 heads of 128, fp16, half of each rotated, 36 us = 5.6 TB/s; 16384 of the same
// in bf16, all channels rotated in halves, 68 - 74 us = 5.4 - 5.9 TB/s; 8192 tokens of 32 + 8 heads in float32 63 us = 5.3 TB/s; gradient of
// 16384 tokens of 32 + 8 heads, bf16, 85.5 us = 5.9 TB/s, of which 2 - 3 are the sums of the blocks (a kernel of its own; with both sums
// of a row in one reduction, of w g x, which leaves float32's range where the result does not: 82.4); the same bytes in float32 91 us; 16K
// tokens of 64 + 8 heads into an E4M3 cache 109 us = 5.8 TB/s.  A step is 215 instructions forward and 317 backward; with few heads a
// token's own share of them (factors, addresses) shows: 8192 tokens of 16 + 4 heads 20 us, 4.2 TB/s.  q and k of 64 tokens: 3 us.
// What did not do as well, on the three above (us): rows straight into registers, two a lane 41 / 128 / 157 (spills), four 43 / 158 / 143;
// every 32nd row a warp's, with the factors in shared memory 55 / 134 / 208; interleaved items of two neighbouring vectors 53 for the
// first (each sector asked for twice); gradient blocks for q or k alone 106.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "libra.h"
#include "ptx.cuh"
#include "rope_kernel.cuh"

namespace libra {

constexpr int kNormThreads = 128, kNormWarps = kNormThreads / 32;   // forward
constexpr int kNormBlocks = 4;                                      // of them a multiprocessor: no spills (5: 96 registers and spills, 3 - 20 % slower)
// Gradient: one block a multiprocessor, as many warps as the registers of its build allow without spills (168 and 128; four blocks of
// 128 threads at 16 bits, which spill: 16384 tokens of 32 + 8 heads 93 -> 119 us)
template <typename T> constexpr int kNormGradThreads = sizeof(T) == 4 ? 512 : 384;
constexpr int kNormAhead = 5, kNormGradAhead = 5;                   // steps in a warp's ring
constexpr int kNormGradStepBytes = 4 * 512;
constexpr int kNormAnyThreads = 128, kNormAnyWarps = kNormAnyThreads / 32;           // the kernels that hold a row in shared memory

struct NormKind {         // q, k or v
  const void* x;
  const void* grad;       // gradient: of the output
  const void* weight;     // null: no norm and, for v, no rotation
  void* out;              // gradient: of x
  int64_t x_token, x_head, grad_token, grad_head, out_token, out_head;   // in elements
  int32_t n_heads;        // 0: absent
  int32_t steps;          // of a token
};

struct NormParams {
  NormKind kind[3];
  const int32_t* positions;
  const int32_t* slots;        // append: of every row, -1: not stored
  const int32_t* n_rows;       // append: rows there are, or null
  uint32_t* error_word;
  float* partial;              // gradient: [block][kinds][head_dim]
  int64_t n_tokens;
  int64_t num_slots;           // append
  int64_t stride_page, stride_head, stride_token;   // of the pools, in elements
  float k_inv_scale, v_inv_scale;
  float eps, inv_dim;
  int32_t head_dim, page_shift;
  int32_t steps;               // of a token, of all kinds
  int32_t items, lanes_shift;  // of a row, and the power of two of lanes that holds them
  libra_rope_t rope;
};

namespace norm {

using rope::fma_rn;
using rope::mul_rn;

// An item's two vectors, at channels c0 and c1.  Vector 0 (1) of neighbouring items is neighbouring, so that the lanes' accesses fill
// whole sectors.
//   half         c1 = c0 + R / 2: the first and the second channels of V pairs; behind the items that turn, vectors of the rest
//   interleaved  any two vectors: V / 2 pairs each, the even elements and the odd ones
template <int V, bool kHalf>
struct Item {
  int c0, c1;        // c1 >= head_dim: there is none
  bool turn0, turn1;
  __device__ __forceinline__ Item(int i, int items, int rotary) {
    const int turning = kHalf ? rotary / (2 * V) : 0;
    if (kHalf && i < turning) {
      c0 = i * V;
      c1 = c0 + rotary / 2;
    } else {
      c0 = (kHalf ? rotary : 0) + (i - turning) * V;
      c1 = c0 + (items - turning) * V;
    }
    turn0 = c0 < rotary;
    turn1 = c1 < rotary;
  }
};

__device__ __forceinline__ uint64_t bits(float2 a) { return *reinterpret_cast<const uint64_t*>(&a); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
  return *reinterpret_cast<const float2*>(&d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)));
  return *reinterpret_cast<const float2*>(&d);
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 minus(float2 a) { return make_float2(-a.x, -a.y); }

// A vector of V elements of type T, 8 or 16 bytes, as it lies in memory
template <typename T, int V>
struct Raw {
  static constexpr int kWords = V * int(sizeof(T)) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kWords == 4) set(*reinterpret_cast<const uint4*>(p));
    else set(*reinterpret_cast<const uint2*>(p));
  }
  __device__ __forceinline__ void load_shared(uint32_t at) {
    if constexpr (kWords == 4) {
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
    } else {
      asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
    }
  }
  __device__ __forceinline__ void store(void* p) const {
    if constexpr (kWords == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  }
  __device__ __forceinline__ void unpack(float (&f)[V]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        if constexpr (std::is_same<T, __half>::value) {
          const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
          f[2 * i] = t.x;
          f[2 * i + 1] = t.y;
        } else {
          f[2 * i] = __uint_as_float(w[i] << 16);
          f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
      }
    }
  }
  __device__ __forceinline__ explicit Raw(const float (&f)[V]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
      else if constexpr (std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
      else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
    }
  }
  __device__ __forceinline__ Raw() {}

 private:
  __device__ __forceinline__ void set(uint4 v) { w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
  __device__ __forceinline__ void set(uint2 v) { w[0] = v.x; w[1] = v.y; }
};
// Codes of E4M3: round to nearest even, beyond the largest code = the largest code
template <int V>
__device__ __forceinline__ void store_e4m3(void* p, const float (&f)[V], float inv_scale) {
  uint32_t w[V / 4];
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(w[i])
        : "f"(f[4 * i] * inv_scale), "f"(f[4 * i + 1] * inv_scale), "f"(f[4 * i + 2] * inv_scale), "f"(f[4 * i + 3] * inv_scale));
  }
  if constexpr (V == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(p) = w[0];
}

// The two vectors of an item as its pairs' first (a) and second (b) channels, two pairs a register pair; and back.
template <int V, bool kHalf>
__device__ __forceinline__ void to_pairs(const float (&v0)[V], const float (&v1)[V], float2 (&a)[V / 2], float2 (&b)[V / 2]) {
#pragma unroll
  for (int i = 0; i < V / 2; ++i) {
    if constexpr (kHalf) {
      a[i] = make_float2(v0[2 * i], v0[2 * i + 1]);
      b[i] = make_float2(v1[2 * i], v1[2 * i + 1]);
    } else {
      const float* v = 4 * i < V ? v0 + 4 * i : v1 + (4 * i - V);
      a[i] = make_float2(v[0], v[2]);
      b[i] = make_float2(v[1], v[3]);
    }
  }
}
template <int V, bool kHalf>
__device__ __forceinline__ void from_pairs(const float2 (&a)[V / 2], const float2 (&b)[V / 2], float (&v0)[V], float (&v1)[V]) {
#pragma unroll
  for (int i = 0; i < V / 2; ++i) {
    if constexpr (kHalf) {
      v0[2 * i] = a[i].x;
      v0[2 * i + 1] = a[i].y;
      v1[2 * i] = b[i].x;
      v1[2 * i + 1] = b[i].y;
    } else {
      float* v = 4 * i < V ? v0 + 4 * i : v1 + (4 * i - V);
      v[0] = a[i].x;
      v[2] = a[i].y;
      v[1] = b[i].x;
      v[3] = b[i].y;
    }
  }
}

// The token's cosines and sines, worked out by the warp into its part of shared memory as vectors (cos, cos, sin, sin) of two pairs.
// An item (interleaved: a vector of channels) has kPer of them; vector j of all items lies side by side.
template <int V, bool kHalf>
struct Factors {
  static constexpr int kPer = kHalf ? V / 2 : V / 4;
  float4* at;
  int units;   // items, or vectors of channels, that turn
  __device__ __forceinline__ Factors(float4* where, int rotary) : at(where), units(rotary / (2 * kPer) / 2) {}
  __device__ __forceinline__ void make(const uint64_t* turns, int pairs, int32_t pos, float magnitude, int lane) const {
    __syncwarp();   // the token before has been read
    float* const f = reinterpret_cast<float*>(at);
    for (int pr = lane; pr < pairs; pr += 32) {
      const float2 w = rope::cos_sin(pos, turns[pr], magnitude);
      const int m = pr >> 1;
      float* const to = f + 4 * ((m % kPer) * units + m / kPer) + (pr & 1);
      to[0] = w.x;
      to[2] = w.y;
    }
    __syncwarp();
  }
  __device__ __forceinline__ void load(int item, const Item<V, kHalf>& it, float2 (&c)[V / 2], float2 (&s)[V / 2]) const {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      const bool there = kHalf || j < kPer ? it.turn0 : it.turn1;
      const float4 w = there ? at_pair(item, it, j) : make_float4(1.f, 1.f, 0.f, 0.f);
      c[j] = make_float2(w.x, w.y);
      s[j] = make_float2(w.z, w.w);
    }
  }
  // of register pair k of an item that turns
  __device__ __forceinline__ float4 at_pair(int item, const Item<V, kHalf>& it, int k) const {
    return at[(k % kPer) * units + (kHalf ? item : (k < kPer ? it.c0 : it.c1) / V)];
  }
  // turning(k) or passing(k) for every register pair k of an item
  template <typename F, typename G>
  static __device__ __forceinline__ void each(const Item<V, kHalf>& it, const F& turning, const G& passing) {
#pragma unroll
    for (int part = 0; part < V / 2 / kPer; ++part) {
      if (part == 0 ? it.turn0 : it.turn1) {
#pragma unroll
        for (int k = part * kPer; k < (part + 1) * kPer; ++k) turning(k);
      } else {
#pragma unroll
        for (int k = part * kPer; k < (part + 1) * kPer; ++k) passing(k);
      }
    }
  }
};

// Sums over a group of lanes (a power of two of them)
template <int N>
__device__ __forceinline__ void group_sums(float (&x)[N], int lanes) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    if (lanes > off) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], off);
    }
  }
}
__device__ __forceinline__ float group_sum(float x, int lanes) {
  float y[1] = {x};
  group_sums(y, lanes);
  return y[0];
}

// 1 / sqrt(m): the approximation and a Newton step; 0 for infinity.  m r first, which is a normal number: half of the smallest m is none
// and would be flushed to zero.
__device__ __forceinline__ float inverse_root(float m) {
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(m));
  const float better = r * fmaf(-0.5f * (m * r), r, 1.5f);
  return m == INFINITY ? 0.f : better;
}

template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
  if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void st_shared_zero(uint32_t at) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
}

// The steps of warp `me` of `warps`: a run of consecutive ones, step s of the launch being step s % steps of token s / steps.
struct Run {
  int32_t token, step, left;
  __device__ __forceinline__ Run(int64_t n_tokens, int32_t steps, uint32_t warps, uint32_t me) {
    const int64_t all = n_tokens * steps;
    if (all <= 0x7fffffff) {   // a division of 64 bits takes a hundred instructions
      const uint32_t run = (uint32_t(all) + warps - 1) / warps;
      const int64_t begin = int64_t(me) * run;
      left = int32_t(max(int64_t(0), min(int64_t(run), all - begin)));
      token = left > 0 ? int32_t(uint32_t(begin) / uint32_t(steps)) : 0;
      step = left > 0 ? int32_t(uint32_t(begin) - uint32_t(token) * uint32_t(steps)) : 0;
    } else {
      const int64_t run = (all + warps - 1) / warps, begin = me * run;
      left = int32_t(max(int64_t(0), min(run, all - begin)));
      token = left > 0 ? int32_t(begin / steps) : 0;
      step = left > 0 ? int32_t(begin - int64_t(token) * steps) : 0;
    }
  }
};

// A warp's walk over rows: row u of the launch is row u % units of token u / units.
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
__device__ __forceinline__ int64_t slot_offset(const NormParams& p, int32_t slot) {
  if (slot == -1) return -1;
  if (slot < 0 || slot >= p.num_slots) {
    atomicOr(p.error_word, uint32_t(LIBRA_ERR_BAD_PAGE_ID));
    return -1;
  }
  return int64_t(slot >> p.page_shift) * p.stride_page + int64_t(slot & ((1 << p.page_shift) - 1)) * p.stride_token;
}

}  // namespace norm

// T: type of the rows; P: of the pools (append); V: elements of a vector, 16 bytes or 8 (half layout of 16-bit rows whose R / 2 only these divide).
template <typename T, typename P, int V, bool kHalf, bool kAppend>
__global__ void __launch_bounds__(kNormThreads, kNormBlocks) norm_rope_kernel(const __grid_constant__ NormParams p) {
  using namespace norm;
  constexpr uint32_t kStep = 1024, kRing = kNormAhead * kStep;   // two vectors a lane, 16 bytes apart from the next lane's
  constexpr int kBytes = V * int(sizeof(T));
  __shared__ uint64_t turns[LIBRA_ROPE_MAX_PAIRS];
  __shared__ alignas(16) float4 factors[kNormWarps][LIBRA_ROPE_MAX_PAIRS / 2];
  __shared__ alignas(16) uint8_t rings[kNormWarps][kRing];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int R = p.rope.rotary_dim, pairs = R / 2;
  for (int i = threadIdx.x; i < pairs; i += kNormThreads) turns[i] = p.rope.turns[i];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lanes = 1 << p.lanes_shift, item = lane & (lanes - 1), group = lane >> p.lanes_shift, groups_shift = 5 - p.lanes_shift, groups = 1 << groups_shift;
  const bool on = item < p.items;
  const Item<V, kHalf> it(item, p.items, R);
  const Factors<V, kHalf> turn(factors[warp], R);
  const bool two = on && it.c1 < p.head_dim;
  int64_t n_tokens = p.n_tokens;
  if (kAppend && p.n_rows) n_tokens = max(int64_t(0), min(n_tokens, int64_t(*p.n_rows)));
  const Run run(n_tokens, p.steps, gridDim.x * kNormWarps, blockIdx.x * kNormWarps + warp);
  int left = run.left;

  struct Part {   // of the run: heads of one token and one kind
    int kind, head0, steps, rows;   // this lane's first head, steps, rows of this lane's group
  };
  auto part_of = [&](int step, int most) {
    Part x;
    x.kind = 0;
    if (step >= p.kind[0].steps) {
      step -= p.kind[0].steps;
      x.kind = 1;
      if (kAppend && step >= p.kind[1].steps) {
        step -= p.kind[1].steps;
        x.kind = 2;
      }
    }
    x.steps = min(most, p.kind[x.kind].steps - step);
    x.head0 = (step << groups_shift) + group;
    x.rows = on ? min(x.steps, (p.kind[x.kind].n_heads - x.head0 + groups - 1) >> groups_shift) : 0;
    return x;
  };
  int token = run.token, step = run.step;

  // ---- the copies, kNormAhead - 1 steps ahead.  Lanes and vectors that hold nothing are zero from the start.
  const uint32_t ring = dev::smem_u32(rings[warp]) + lane * 16;
#pragma unroll
  for (int i = 0; i < 2 * kNormAhead; ++i) {
    if (i & 1 ? !two : !on) st_shared_zero(ring + i * 512);
  }
  int ask_token = token;
  int ask_step = step, ask_left = left, ask_steps = 0, ask_rows = 0;
  const T* ask_src = nullptr;
  int64_t ask_hop = 0;
  auto ask = [&](uint32_t at) {
    if (ask_steps == 0 && ask_left > 0) {
      const Part x = part_of(ask_step, ask_left);
      const NormKind& kind = p.kind[x.kind];
      ask_src = static_cast<const T*>(kind.x) + int64_t(ask_token) * kind.x_token + x.head0 * kind.x_head + it.c0;
      ask_hop = groups * kind.x_head;
      ask_steps = x.steps;
      ask_rows = x.rows;
      ask_left -= x.steps;
      ask_step += x.steps;
      if (ask_step == p.steps) {
        ask_step = 0;
        ++ask_token;
      }
    }
    if (ask_rows > 0) {
      copy_async<kBytes>(ring + at, ask_src);
      if (two) copy_async<kBytes>(ring + at + 512, ask_src + (it.c1 - it.c0));
    }
    ask_src += ask_hop;
    --ask_rows;
    --ask_steps;
  };
#pragma unroll
  for (int i = 0; i < kNormAhead - 1; ++i) {
    if (i < left) ask(i * kStep);
    copies_commit();
  }

  int32_t pos = pairs > 0 && left > 0 ? p.positions[token] : 0, slot = kAppend && left > 0 ? p.slots[token] : 0;
  __syncthreads();   // `turns`, while the first rows are on their way
  bool new_token = true;
  uint32_t place = 0;
#pragma unroll 1
  while (left > 0) {
    const Part x = part_of(step, left);
    const NormKind& kind = p.kind[x.kind];
    const bool pool = kAppend && x.kind > 0, plain = kAppend && x.kind == 2, normed = kind.weight != nullptr;
    left -= x.steps;
    step += x.steps;
    const bool ends = step == p.steps;
    // the token after this one, while there is time
    const int after = ends && left > 0 ? token + 1 : token;
    const int32_t next_pos = pairs > 0 ? p.positions[after] : 0, next_slot = kAppend ? p.slots[after] : 0;
    int64_t at = pool ? slot_offset(p, slot) : int64_t(token) * kind.out_token;     // of the output, in elements
    int rows = at >= 0 ? x.rows : 0;
    const int64_t out_head = pool ? p.stride_head : kind.out_head, hop = groups * out_head;
    at += x.head0 * out_head;
    float2 aa[V / 2], ab[V / 2], ba[V / 2], bb[V / 2];                      // y_a = aa a + ab b, y_b = ba a + bb b
    if (!plain) {
      if (new_token && pairs > 0) turn.make(turns, pairs, pos, p.rope.magnitude, lane);
      new_token = false;
      float w0[V], w1[V];
#pragma unroll
      for (int k = 0; k < V; ++k) w0[k] = w1[k] = 1.f;
      Raw<T, V> w;
      if (normed && on) {
        w.load(static_cast<const T*>(kind.weight) + it.c0);
        w.unpack(w0);
      }
      if (normed && two) {
        w.load(static_cast<const T*>(kind.weight) + it.c1);
        w.unpack(w1);
      }
      to_pairs<V, kHalf>(w0, w1, aa, bb);
      if (it.turn0 || it.turn1) {
        float2 c[V / 2], s[V / 2];
        turn.load(item, it, c, s);
#pragma unroll
        for (int k = 0; k < V / 2; ++k) {
          ba[k] = mul2(s[k], aa[k]);
          ab[k] = minus(mul2(s[k], bb[k]));
          aa[k] = mul2(c[k], aa[k]);
          bb[k] = mul2(c[k], bb[k]);
        }
      }
    }
#pragma unroll 1
    for (int j = 0; j < x.steps; ++j) {
      copies_wait<kNormAhead - 2>();
      Raw<T, V> raw0, raw1;
      raw0.load_shared(ring + place);
      raw1.load_shared(ring + place + 512);
      if (ask_left > 0 || ask_steps > 0) ask(place == 0 ? kRing - kStep : place - kStep);   // where the step before was
      copies_commit();
      place = place == kRing - kStep ? 0 : place + kStep;
      float v0[V], v1[V];
      if (!plain || sizeof(P) == 1) {
        raw0.unpack(v0);
        raw1.unpack(v1);
      }
      if (!plain) {
        float2 a[V / 2], b[V / 2];
        to_pairs<V, kHalf>(v0, v1, a, b);
        if (normed) {
          float2 sum = both(0.f), more = both(0.f);
#pragma unroll
          for (int k = 0; k < V / 2; ++k) {
            sum = fma2(a[k], a[k], sum);
            more = fma2(b[k], b[k], more);
          }
          const float2 r = both(inverse_root(fmaf(group_sum((sum.x + more.x) + (sum.y + more.y), lanes), p.inv_dim, p.eps)));
#pragma unroll
          for (int k = 0; k < V / 2; ++k) {
            a[k] = mul2(a[k], r);
            b[k] = mul2(b[k], r);
          }
        }
        turn.each(it, [&](int k) {
          const float2 y = fma2(a[k], aa[k], mul2(b[k], ab[k]));
          b[k] = fma2(a[k], ba[k], mul2(b[k], bb[k]));
          a[k] = y;
        }, [&](int k) {
          a[k] = mul2(a[k], aa[k]);
          b[k] = mul2(b[k], bb[k]);
        });
        from_pairs<V, kHalf>(a, b, v0, v1);
      }
      if (j < rows) {
        if (!pool) {
          T* const row = static_cast<T*>(kind.out) + at;
          Raw<T, V>(v0).store(row + it.c0);
          if (two) Raw<T, V>(v1).store(row + it.c1);
        } else if constexpr (kAppend) {
          P* const row = static_cast<P*>(kind.out) + at;
          if constexpr (sizeof(P) == 1) {
            const float inv = plain ? p.v_inv_scale : p.k_inv_scale;
            store_e4m3<V>(row + it.c0, v0, inv);
            if (two) store_e4m3<V>(row + it.c1, v1, inv);
          } else {   // values as they came
            (plain ? raw0 : Raw<T, V>(v0)).store(row + it.c0);
            if (two) (plain ? raw1 : Raw<T, V>(v1)).store(row + it.c1);
          }
        }
      }
      at += hop;
    }
    if (ends) {
      step = 0;
      ++token;
      new_token = true;
      pos = next_pos;
      slot = next_slot;
    }
  }
}

// The rows' channels are summed into partial[block], q's and then k's.  Dynamic shared memory: the rings, and float [warps][2][head_dim]
// in their place at the end
template <typename T, int V, bool kHalf>
__global__ void __launch_bounds__(kNormGradThreads<T>, 1) norm_rope_gradient_kernel(const __grid_constant__ NormParams p) {
  using namespace norm;
  constexpr int kThreads = kNormGradThreads<T>, kWarps = kThreads / 32, kBytes = V * int(sizeof(T));
  constexpr uint32_t kStep = kNormGradStepBytes, kRing = kNormGradAhead * kStep;   // two vectors of x and two of the gradient a lane
  __shared__ uint64_t turns[LIBRA_ROPE_MAX_PAIRS];
  __shared__ alignas(16) float4 factors[kWarps][LIBRA_ROPE_MAX_PAIRS / 2];
  extern __shared__ __align__(16) uint8_t rings[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int R = p.rope.rotary_dim, pairs = R / 2;
  for (int i = threadIdx.x; i < pairs; i += kThreads) turns[i] = p.rope.turns[i];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lanes = 1 << p.lanes_shift, item = lane & (lanes - 1), group = lane >> p.lanes_shift, groups_shift = 5 - p.lanes_shift, groups = 1 << groups_shift;
  const bool on = item < p.items;
  const Item<V, kHalf> it(item, p.items, R);
  const Factors<V, kHalf> turn(factors[warp], R);
  const bool two = on && it.c1 < p.head_dim;
  float2 wa[V / 2], wb[V / 2], acca[2][V / 2], accb[2][V / 2];   // the kind's weights; sums of both
#pragma unroll
  for (int k = 0; k < V / 2; ++k) acca[0][k] = accb[0][k] = acca[1][k] = accb[1][k] = both(0.f);
  const Run run(p.n_tokens, p.steps, gridDim.x * kWarps, blockIdx.x * kWarps + warp);
  int token = run.token, step = run.step, left = run.left;

  struct Part {   // of the run: heads of one token and one kind
    int kind, head0, steps, rows;   // this lane's first head, steps, rows of this lane's group
  };
  auto part_of = [&](int at, int most) {
    Part x;
    x.kind = at >= p.kind[0].steps ? 1 : 0;
    if (x.kind) at -= p.kind[0].steps;
    x.steps = min(most, p.kind[x.kind].steps - at);
    x.head0 = (at << groups_shift) + group;
    x.rows = on ? min(x.steps, (p.kind[x.kind].n_heads - x.head0 + groups - 1) >> groups_shift) : 0;
    return x;
  };
  const uint32_t ring = dev::smem_u32(rings) + warp * kRing + lane * 16;
#pragma unroll
  for (int i = 0; i < 4 * kNormGradAhead; ++i) {
    if (i & 1 ? !two : !on) st_shared_zero(ring + i * 512);
  }
  int ask_token = token;
  int ask_step = step, ask_left = left, ask_steps = 0, ask_rows = 0;
  const T *ask_src = nullptr, *ask_grad = nullptr;
  int64_t src_hop = 0, grad_hop = 0;
  auto ask = [&](uint32_t at) {
    if (ask_steps == 0) {
      const Part x = part_of(ask_step, ask_left);
      const NormKind& kind = p.kind[x.kind];
      ask_src = static_cast<const T*>(kind.x) + int64_t(ask_token) * kind.x_token + x.head0 * kind.x_head + it.c0;
      ask_grad = static_cast<const T*>(kind.grad) + int64_t(ask_token) * kind.grad_token + x.head0 * kind.grad_head + it.c0;
      src_hop = groups * kind.x_head;
      grad_hop = groups * kind.grad_head;
      ask_steps = x.steps;
      ask_rows = x.rows;
      ask_left -= x.steps;
      ask_step += x.steps;
      if (ask_step == p.steps) {
        ask_step = 0;
        ++ask_token;
      }
    }
    if (ask_rows > 0) {
      copy_async<kBytes>(ring + at, ask_src);
      copy_async<kBytes>(ring + at + 1024, ask_grad);
      if (two) {
        copy_async<kBytes>(ring + at + 512, ask_src + (it.c1 - it.c0));
        copy_async<kBytes>(ring + at + 1536, ask_grad + (it.c1 - it.c0));
      }
    }
    ask_src += src_hop;
    ask_grad += grad_hop;
    --ask_rows;
    --ask_steps;
  };
#pragma unroll
  for (int i = 0; i < kNormGradAhead - 1; ++i) {
    if (i < left) ask(i * kStep);
    copies_commit();
  }
  int32_t pos = pairs > 0 && left > 0 ? p.positions[token] : 0;
  __syncthreads();   // `turns`, while the first rows are on their way
  bool new_token = true;
  uint32_t place = 0;
#pragma unroll 1
  while (left > 0) {
    const Part x = part_of(step, left);
    const NormKind& kind = p.kind[x.kind];
    left -= x.steps;
    step += x.steps;
    const bool ends = step == p.steps;
    const int32_t next_pos = pairs > 0 ? p.positions[ends && left > 0 ? token + 1 : token] : 0;
    T* out = static_cast<T*>(kind.out) + int64_t(token) * kind.out_token + x.head0 * kind.out_head;
    const int64_t out_hop = groups * kind.out_head;
    {
      float w0[V], w1[V];
#pragma unroll
      for (int k = 0; k < V; ++k) w0[k] = w1[k] = 0.f;
      Raw<T, V> w;
      if (on) {
        w.load(static_cast<const T*>(kind.weight) + it.c0);
        w.unpack(w0);
      }
      if (two) {
        w.load(static_cast<const T*>(kind.weight) + it.c1);
        w.unpack(w1);
      }
      to_pairs<V, kHalf>(w0, w1, wa, wb);
    }
    if (new_token && pairs > 0) turn.make(turns, pairs, pos, p.rope.magnitude, lane);
    new_token = false;
#pragma unroll 1
    for (int j = 0; j < x.steps; ++j) {
      copies_wait<kNormGradAhead - 2>();
      float2 xa[V / 2], xb[V / 2], ga[V / 2], gb[V / 2];
      float v0[V], v1[V];
      Raw<T, V> raw;
      raw.load_shared(ring + place);
      raw.unpack(v0);
      raw.load_shared(ring + place + 512);
      raw.unpack(v1);
      to_pairs<V, kHalf>(v0, v1, xa, xb);
      raw.load_shared(ring + place + 1024);
      raw.unpack(v0);
      raw.load_shared(ring + place + 1536);
      raw.unpack(v1);
      to_pairs<V, kHalf>(v0, v1, ga, gb);
      if (ask_left > 0 || ask_steps > 0) ask(place == 0 ? kRing - kStep : place - kStep);   // where the step before was
      copies_commit();
      place = place == kRing - kStep ? 0 : place + kStep;
      turn.each(it, [&](int k) {   // back; the factors are read anew: kept in registers they cost more
        const float4 f = turn.at_pair(item, it, k);
        const float2 c = make_float2(f.x, f.y), s = make_float2(f.z, f.w);
        const float2 g = fma2(ga[k], c, mul2(gb[k], s));
        gb[k] = fma2(gb[k], c, mul2(ga[k], minus(s)));
        ga[k] = g;
      }, [](int) {});
      float2 square = both(0.f), more = both(0.f);
#pragma unroll
      for (int k = 0; k < V / 2; ++k) {
        square = fma2(xa[k], xa[k], square);
        more = fma2(xb[k], xb[k], more);
      }
      const float r = inverse_root(fmaf(group_sum((square.x + more.x) + (square.y + more.y), lanes), p.inv_dim, p.eps));
      const float2 r2 = both(r);
      const bool there = j < x.rows;
      // x r and w g take the places of x and g; the sum of w g x r is of these: w g x may have no place in float32 where they do
#pragma unroll
      for (int k = 0; k < V / 2; ++k) {
        xa[k] = mul2(xa[k], r2);
        xb[k] = mul2(xb[k], r2);
      }
      if (there) {
        if (x.kind == 0) {
#pragma unroll
          for (int k = 0; k < V / 2; ++k) {
            acca[0][k] = fma2(ga[k], xa[k], acca[0][k]);
            accb[0][k] = fma2(gb[k], xb[k], accb[0][k]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < V / 2; ++k) {
            acca[1][k] = fma2(ga[k], xa[k], acca[1][k]);
            accb[1][k] = fma2(gb[k], xb[k], accb[1][k]);
          }
        }
      }
      float2 dot = both(0.f), dots = both(0.f);
#pragma unroll
      for (int k = 0; k < V / 2; ++k) {
        ga[k] = mul2(ga[k], wa[k]);
        gb[k] = mul2(gb[k], wb[k]);
        dot = fma2(ga[k], xa[k], dot);
        dots = fma2(gb[k], xb[k], dots);
      }
      const float2 mean2 = both(-(group_sum((dot.x + dots.x) + (dot.y + dots.y), lanes) * p.inv_dim));   // minus the mean of w g x r
      if (there) {
#pragma unroll
        for (int k = 0; k < V / 2; ++k) {
          ga[k] = mul2(fma2(xa[k], mean2, ga[k]), r2);
          gb[k] = mul2(fma2(xb[k], mean2, gb[k]), r2);
        }
        from_pairs<V, kHalf>(ga, gb, v0, v1);
        Raw<T, V>(v0).store(out + it.c0);
        if (two) Raw<T, V>(v1).store(out + it.c1);
      }
      out += out_hop;
    }
    if (ends) {
      step = 0;
      ++token;
      new_token = true;
      pos = next_pos;
    }
  }
  // groups of a warp, then the warps
  copies_wait<0>();
  __syncthreads();
  float* const sums = reinterpret_cast<float*>(rings);
  const int kinds = p.kind[1].n_heads > 0 ? 2 : 1;
#pragma unroll
  for (int kd = 0; kd < 2; ++kd) {
    float acc0[V], acc1[V];
    from_pairs<V, kHalf>(acca[kd], accb[kd], acc0, acc1);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      for (int off = lanes; off < 32; off <<= 1) {
        acc0[k] += __shfl_xor_sync(0xffffffffu, acc0[k], off);
        acc1[k] += __shfl_xor_sync(0xffffffffu, acc1[k], off);
      }
      if (on && group == 0 && kd < kinds) {
        sums[(warp * kinds + kd) * p.head_dim + it.c0 + k] = acc0[k];
        if (two) sums[(warp * kinds + kd) * p.head_dim + it.c1 + k] = acc1[k];
      }
    }
  }
  __syncthreads();
  const int channels = kinds * p.head_dim;
  for (int ch = threadIdx.x; ch < channels; ch += kThreads) {
    float sum = 0.f;
    for (int i = 0; i < kWarps; ++i) sum += sums[i * channels + ch];
    p.partial[int64_t(blockIdx.x) * channels + ch] = sum;
  }
}

struct NormSumParams {
  const float* partial;   // [blocks][kinds][head_dim]
  float* out[2];
  int32_t head_dim, channels;   // of all kinds
  int32_t blocks;
};

constexpr int kNormSumSlices = 32;

// The blocks' sums: grid = ceil(channels / 32), 32 channels x 32 slices of the blocks
__global__ void __launch_bounds__(32 * kNormSumSlices) norm_sum_kernel(const NormSumParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ float part[kNormSumSlices][33];
  const int ch = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  float s = 0.f;
  if (ch < p.channels) {
#pragma unroll 4
    for (int b = slice; b < p.blocks; b += kNormSumSlices) s += p.partial[int64_t(b) * p.channels + ch];
  }
  part[slice][threadIdx.x & 31] = s;
  __syncthreads();
  if (slice == 0 && ch < p.channels) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kNormSumSlices; ++i) s += part[i][threadIdx.x];
    (ch < p.head_dim ? p.out[0] : p.out[1] - p.head_dim)[ch] = s;
  }
}

// ---------------------------------------------------------------------------------------------- rows through shared memory
// One row a warp, V channels a lane and step (16 bytes, or one).  Unit = one row.
// Dynamic shared memory: [warps][head_dim] floats (gradient: two more, and one for each kind)
template <typename T, typename P, int V, bool kVector, bool kHalf, bool kAppend>
__global__ void __launch_bounds__(kNormAnyThreads) norm_rope_any_kernel(const __grid_constant__ NormParams p) {
  using namespace norm;
  extern __shared__ float rows[];
  __shared__ uint64_t turns[LIBRA_ROPE_MAX_PAIRS];
  __shared__ float2 factors[kNormAnyWarps][LIBRA_ROPE_MAX_PAIRS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = p.head_dim;
  const int R = p.rope.rotary_dim, pairs = R / 2;
  for (int i = threadIdx.x; i < pairs; i += kNormAnyThreads) turns[i] = p.rope.turns[i];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  float* const row = rows + warp * D;
  float2* const cs = factors[warp];
  int64_t n_tokens = p.n_tokens;
  if (kAppend && p.n_rows) n_tokens = min(n_tokens, int64_t(*p.n_rows));
  const int64_t stride = int64_t(gridDim.x) * kNormAnyWarps, first = int64_t(blockIdx.x) * kNormAnyWarps + warp;
  const int64_t by_tokens = stride / p.steps;
  const int32_t by_rest = int32_t(stride - by_tokens * p.steps);
  for (Units u(first, p.steps); u.token < n_tokens; u.advance(by_tokens, by_rest, p.steps)) {
    int head = u.unit, kd = 0;
    if (head >= p.kind[0].steps) {
      head -= p.kind[0].steps;
      kd = 1;
      if (head >= p.kind[1].steps) {
        head -= p.kind[1].steps;
        kd = 2;
      }
    }
    const NormKind& kind = p.kind[kd];
    const T* const src = static_cast<const T*>(kind.x) + u.token * kind.x_token + head * kind.x_head;
    const bool pool = kAppend && kd > 0;
    const int64_t at = pool ? slot_offset(p, p.slots[u.token]) : u.token * kind.out_token;
    const bool normed = kind.weight != nullptr, turned = !(kAppend && kd == 2) && R > 0;
    __syncwarp();   // the row before has been read
    if (turned) {
      const int32_t pos = p.positions[u.token];
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
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int kinds = p.kind[1].n_heads > 0 ? 2 : 1, channels = kinds * D;
  float* const xs = rows + (kinds * kNormAnyWarps + warp) * D;
  float* const gs = xs + kNormAnyWarps * D;
  for (int c = threadIdx.x; c < kNormAnyWarps * channels; c += kNormAnyThreads) rows[c] = 0.f;
  __syncthreads();
  float2* const cs = factors[warp];
  const int64_t stride = int64_t(gridDim.x) * kNormAnyWarps, first = int64_t(blockIdx.x) * kNormAnyWarps + warp;
  const int64_t by_tokens = stride / p.steps;
  const int32_t by_rest = int32_t(stride - by_tokens * p.steps);
  for (Units u(first, p.steps); u.token < p.n_tokens; u.advance(by_tokens, by_rest, p.steps)) {
    const int kd = u.unit >= p.kind[0].steps ? 1 : 0, head = u.unit - (kd ? p.kind[0].steps : 0);
    const NormKind& kind = p.kind[kd];
    const T* const weight = static_cast<const T*>(kind.weight);
    float* const sums = rows + (warp * kinds + kd) * D;   // a lane's channels are its own
    const T* const src = static_cast<const T*>(kind.x) + u.token * kind.x_token + head * kind.x_head;
    const T* const grad = static_cast<const T*>(kind.grad) + u.token * kind.grad_token + head * kind.grad_head;
    __syncwarp();
    if (R > 0) {
      const int32_t pos = p.positions[u.token];
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
    const float r = __frsqrt_rn(fmaf(group_sum(square, 32), p.inv_dim, p.eps));
    float dot = 0.f;   // of w g x r; w g x may have no place in float32
    for (int c = lane * V; c < D; c += 32 * V) {
#pragma unroll
      for (int i = 0; i < V; ++i) dot = fmaf(mul_rn(back(c + i), rope::to_f32(weight[c + i])), mul_rn(xs[c + i], r), dot);
    }
    const float mean = mul_rn(group_sum(dot, 32), p.inv_dim);
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
  for (int c = threadIdx.x; c < channels; c += kNormAnyThreads) {
    float s = 0.f;
    for (int i = 0; i < kNormAnyWarps; ++i) s += rows[i * channels + c];
    p.partial[int64_t(blockIdx.x) * channels + c] = s;
  }
}

}  // namespace libra
