// Causal attention of packed chunks of new tokens over the paged KV cache (sm_100a).
//
// For one item (up to 256 flattened query rows of one sequence and KV head, row = query token x head of the group) and a
// range of cached tokens, in steps of 128 tokens:
//
//   S = Q K^T          tcgen05.mma, Q and K tiles in shared memory, S (128 x 128 fp32) in tensor memory
//   P = 2^(S c - m c)  in registers, one row per thread; rounded to 16 bits and put where S was
//   O += P V           tcgen05.mma, P from tensor memory, V tile in shared memory, O (128 x D fp32) in tensor memory
//
// with the running maximum m and sum l of an online softmax.  m is raised, and O and l scaled, only when a tile's maximum
// exceeds it by more than 2^8 (the probabilities then lie below 2^8 instead of 1, which 16-bit and fp32 numbers hold as
// well), so that O stays untouched in tensor memory for most steps.
//
// Rounding P to one 16-bit number per weight (bf16: off by at most 2^-8 of it, 2.3e-3 of the result's norm instead of 1.7e-3 for a
// result rounded once) is the price of a single product with V.  The decode kernel takes two terms, its tensor cores being idle;
// here a second product would add half to the time of the large cases.  The sum l is of the unrounded weights, so lse is exact
// to float32.
//
// Roles of a block's warps: 0-3 and 4-7 softmax of row tiles 0 and 1 (and loading Q, writing the output), 9 the tensor-core
// instructions, 8, 10 and 11 the copies; over an E4M3 cache 12-15 convert K and V.  While one tile's rows are in the softmax
// the tensor cores work on the other's.  An item of at most 128 rows has one row tile: then both softmax groups take it, one the
// even steps and one the odd ones, and their results are merged in shared memory at the end.
//
// What bounds it.  A step of two row tiles is 2048 cycles of the tensor cores at D = 128, as many of the exponential unit (16 a
// cycle) and as many of shared memory (128 bytes a cycle for Q, K and V operands and the copies).  4096 new tokens on 12288,
// 64 / 8 heads: 1.44 ms = 1333 TFLOP/s in short runs, 80 % of a plain bf16 matrix product's burst rate (1663); the products and
// copies alone take 1.17 ms, without the exponentials it is 1.39.  In runs of a tenth of a second and more the power cap holds the
// clock at 1.62 GHz: 1.66 ms = 1160 TFLOP/s.  Three tokens on eight trajectories of 32K: 187 us = 5.7 TB/s of the cache (165 us
// when the same inputs are read again).  Over an E4M3 cache the
// conversion adds 96 KB of shared-memory traffic a step: 10 - 15 % slower than bf16 where arithmetic bounds.
//
// Copies: one tiled TMA load per page (16, 32 or 64 tokens) and 64 channels, 128-byte swizzle, into a ring of tiles.  Pages
// past the range are not read; what their rows of V hold is overwritten with zeros (0 x NaN would reach the result), scores
// past a row's limit are set to -inf by selection.
//
// E4M3 cache: the codes arrive as bytes and are converted to fp16 (exact).  q goes to fp16 too, every row multiplied by a
// power of two that brings its largest element to 2^10 .. 2^11: elements 2^-25 below it and larger stay exact, the rest are off
// by at most 2^-35 of it.  P is rounded to fp16.
//
// Every wait is bounded; the first one that runs out sets the block's stop flag and the error word, and every role leaves.  Once all
// have, the copies and products under way are waited for (bounded), before the block's memory goes to another.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "chunk_plan.hpp"
#include "chunk_ring.hpp"
#include "libra.h"
#include "ptx.cuh"

namespace libra {

struct ChunkParams {
  const __nv_bfloat16* q;
  int64_t q_stride;
  const int32_t* block_table;
  __nv_bfloat16* out;
  float* lse;                 // or null
  const uint32_t* serial_at;  // the plan in the workspace: its serial number, its items
  const int4* items;
  float* partial_o;           // [partial row][KV head][D]
  float* partial_lse;         // [partial row][KV head]
  uint32_t* error_word;
  int64_t num_pages;
  uint32_t serial;
  int32_t num_items;
  int32_t num_q_heads, num_kv_heads, group;
  uint32_t group_inverse;     // ceil(2^16 / group): v / group = v * group_inverse >> 16 for v < 4096
  int32_t block_table_ld;
  int32_t page_shift;
  int32_t pos_head, pos_page, pos_token;
  float scale_log2;           // sm_scale * log2(e) * k_scale
  float v_scale;
};

template <int D, bool kFp8>
struct ChunkShape {
  static constexpr int kTileBytes = kChunkKvTile * D * 2;      // a tile of K or V (and of Q) as the tensor cores read it
  static constexpr int kRawBytes = kChunkKvTile * D;           // the same as E4M3 codes
  static constexpr int kStages = kFp8 ? (D == 128 ? 3 : 6) : (D == 128 ? 5 : 8);
  static constexpr int kRawStages = kFp8 ? (D == 128 ? 4 : 8) : 0;
  // An item with one row tile leaves the second Q tile's place free: the ring is one stage longer then, and begins there.
  static constexpr int kSoloStages = kStages < 8 ? kStages + 1 : kStages;
  // Quarters of a step's probabilities that the product with V starts on (the other one: 1 - 2 % slower)
  static constexpr int kPEarly = kFp8 ? 3 : 2;
  static constexpr int kThreads = kFp8 ? 512 : 384;
  // registers a thread of each role: together what the launch brings (384 x 168, 512 x 128)
  static constexpr int kSoftmaxRegs = kFp8 ? 184 : 224, kIssueRegs = kFp8 ? 72 : 56, kConvertRegs = 72;
  static constexpr int kLaunchRegs = kFp8 ? 512 * 128 : 384 * 168;
  static_assert(256 * kSoftmaxRegs + 128 * kIssueRegs + (kFp8 ? 128 * kConvertRegs : 0) <= kLaunchRegs, "setmaxnreg would wait");
  // dynamic shared memory: Q tiles | ring | raw ring | floats | barriers
  static constexpr int kRing = 2 * kTileBytes;
  static constexpr int kRaw = kRing + kStages * kTileBytes;
  static constexpr int kFloats = kRaw + kRawStages * kRawBytes;   // 2 x 128 row factors, 2 x 128 (m, l) of the merge
  static constexpr int kBars = kFloats + 4 * 128 * 4;
  static constexpr int kDynamicBytes = kBars + 512;
  static_assert(kDynamicBytes <= 227 * 1024, "shared memory of a block");
};

namespace chunk {

using namespace dev;

// barriers, in 8-byte slots after the floats
constexpr int kBarFull = 0, kBarEmpty = 8, kBarRawFull = 16, kBarRawEmpty = 24, kBarQ = 32, kBarS = 34, kBarP = 36, kBarPTail = 38,
              kBarO = 40, kBarMergeFree = 42, kBarMergeFull = 43, kBarDrain = 44, kBarTail = 45, kNumBars = 48;
constexpr int kLoaders = kChunkLoaders;   // warps 8, 10 and 11
constexpr int kDrainTries = 4096;   // of the waits that end a block early, some 2 us each
constexpr int kSlotStop = 48, kSlotTmem = 49;   // the stop flag and the tensor-memory address live in two more slots

struct Stop {   // how a wait that ran out ends the block
  uint32_t flag;                // shared-memory address
  uint32_t* const& error_word;  // in the kernel's parameters
  __device__ __forceinline__ bool set() const {
    uint32_t v;
    asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(v) : "r"(flag) : "memory");
    return v != 0;
  }
  __device__ __forceinline__ void raise() const {
    asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(flag), "r"(1u) : "memory");
    atomicOr(error_word, uint32_t(LIBRA_ERR_WAIT_TIMEOUT));
  }
};

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, const Stop& stop) {
  for (uint32_t i = 0; i < kWaitLimit; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if (stop.set()) return false;
  }
  stop.raise();
  return false;
}
// The whole warp waits; in the usual case, the barrier is through already, with a single test.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, const Stop& stop) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, wait(bar, parity, stop));
}
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// ---- tensor memory and tensor-core instructions
__device__ __forceinline__ void tmem_alloc(uint32_t dst_smem, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t addr, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 16 or 32 columns of this warp's 32 lanes: register i of a thread is column i of its lane
__device__ __forceinline__ void tmem_ld16(float* r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
        "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_ld32(float* r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
        "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]),
        "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]),
        "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// Uses of these registers come after the wait that precedes this in the program.
template <int N>
__device__ __forceinline__ void settle(float* r) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+f"(r[i]));
}

// Shared-memory matrix descriptor, 128-byte swizzle.  K-major tiles (Q, K: channels contiguous): `sbo` is the distance of
// 8-row groups and `lbo` is not read.  MN-major tiles (V: the channels are the N of the product): `lbo` is the distance of
// 64-channel groups, `sbo` that of 8-token groups.
// The address field counts 16 bytes, so that a step within a tile is an addition to the lower word.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);   // sbo 1024, descriptor version, 128-byte swizzle
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t lbo) { return (addr >> 4) | ((lbo >> 4) << 16); }
__device__ __forceinline__ uint64_t smem_desc(uint32_t low) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(low), "r"(kDescHigh));
  return d;
}
// Instruction descriptor: fp32 accumulation, 16-bit operands (bf16 or fp16), M = 128
template <bool kBf16>
__host__ __device__ constexpr uint32_t instr_desc(int n, bool b_mn_major) {
  return (1u << 4) | (kBf16 ? (1u << 7) | (1u << 10) : 0u) | (b_mn_major ? 1u << 16 : 0u) | (uint32_t(n >> 3) << 17) |
         (uint32_t(kChunkTileRows >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(accumulate))
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(uint32_t(accumulate))
      : "memory");
}
// Completes on `bar` once everything this thread has issued to the tensor cores is done.
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ bool elect_one() {   // one lane of a converged warp
  uint32_t pred;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(pred));
  return pred != 0;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }

// Two floats at once, and the largest of three.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t d;
  asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;"
      : "=l"(d)
      : "l"(*reinterpret_cast<const uint64_t*>(&a)), "l"(*reinterpret_cast<const uint64_t*>(&b)), "l"(*reinterpret_cast<const uint64_t*>(&c)));
  return *reinterpret_cast<const float2*>(&d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t d;
  asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<const uint64_t*>(&a)), "l"(*reinterpret_cast<const uint64_t*>(&b)));
  return *reinterpret_cast<const float2*>(&d);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.ftz.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

template <bool kBf16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  uint32_t d;
  if constexpr (kBf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// Byte offset of 16-byte chunk c16 of row r in a tile of 128 rows: [D / 64][128 rows][128 bytes], 128-byte swizzle
__device__ __forceinline__ uint32_t swizzled(int r, int c16) {
  return uint32_t(((c16 >> 3) << 14) + (r << 7) + (((c16 & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ void st_shared(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Eight bf16 of a row that kLanes neighbouring lanes hold -> fp16, the row multiplied by the power of two that brings its
// largest element to 2^10 .. 2^11; `down` undoes it.
template <int kLanes>
__device__ __forceinline__ uint4 scaled_half_row(uint4 v, float& down) {
  float f[8];
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    most = fmaxf(most, fmaxf(fabsf(f[2 * i]), fabsf(f[2 * i + 1])));
  }
#pragma unroll
  for (int off = kLanes / 2; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
  // exponent of the largest element, kept where both factors are normal numbers; not finite: as it is
  const int e = max(int((__float_as_uint(most) >> 23) & 255) - 127, -107);
  const float up = e == 128 ? 1.f : __uint_as_float(uint32_t(127 + 10 - e) << 23);
  down = e == 128 ? 1.f : __uint_as_float(uint32_t(127 - 10 + e) << 23);
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = pack<false>(f[2 * i] * up, f[2 * i + 1] * up);
  return make_uint4(h[0], h[1], h[2], h[3]);
}

__device__ __forceinline__ uint4 ld_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// One unit of work as every role sees it.
struct ChunkUnit {
  int b, q_start, row0, n_rows, kv_begin, kv_end, ctx, slot;
  int head;    // KV head
  int steps;   // of 128 cached tokens
  bool solo;   // one row tile, the softmax groups take turns on the steps
  // Tile i of the ring, in the order in which the products need them: K of step 0, then V of a step and K of the next by turns;
  // solo: K runs one step further ahead.
  __device__ __forceinline__ bool is_v(int i) const { return solo ? i > 0 && ((i & 1) == 0 || i == 2 * steps - 1) : (i & 1); }
  __device__ __forceinline__ int step_of(int i) const { return solo ? (is_v(i) ? (i == 2 * steps - 1 ? steps - 1 : (i >> 1) - 1) : (i + 1) >> 1) : i >> 1; }
  // steps of row tile (softmax group) t
  __device__ __forceinline__ int steps_of(int t) const { return solo ? (steps + 1 - t) >> 1 : steps; }
};
__device__ __forceinline__ int4 load_again(const int4* at) {   // not merged with another load of the same address
  int4 v;
  asm volatile("ld.global.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(at));
  return v;
}
__device__ __forceinline__ uint32_t load_again(const uint32_t* at) {
  uint32_t v;
  asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(at));
  return v;
}
__device__ __forceinline__ int item_of(const ChunkParams& p) { return min(int(blockIdx.y + blockIdx.z * 65535u), p.num_items - 1); }
__device__ __forceinline__ void touch_unit(const ChunkParams& p) {
  asm volatile("{\n\t.reg .b32 v;\n\tld.global.b32 v, [%0];\n\t}" ::"l"(p.items + 2 * item_of(p)));
}
// Row r of an item: its token within the sequence's chunk and its head within the group.  One division for the item's first
// row, the rest by multiplication.
struct RowMap {
  int token0, rest;
  __device__ __forceinline__ RowMap(const ChunkParams& p, int row0) : token0(row0 / p.group), rest(row0 - token0 * p.group) {}
  __device__ __forceinline__ void at(const ChunkParams& p, int r, int& token, int& head) const {
    const int v = rest + r, t = int((uint32_t(v) * p.group_inverse) >> 16);
    token = token0 + t;
    head = v - t * p.group;
  }
};
// grid = (KV heads, items up to 65535, the rest by z): the heads of an item run side by side, they share its pages
__device__ __forceinline__ ChunkUnit load_unit(const ChunkParams& p) {
  const int item = item_of(p);
  const int4 a = load_again(p.items + 2 * item), c = load_again(p.items + 2 * item + 1);
  ChunkUnit x;
  x.b = a.x; x.q_start = a.y; x.row0 = a.z; x.n_rows = a.w;
  x.kv_begin = c.x; x.kv_end = c.y; x.ctx = c.z; x.slot = c.w;
  x.head = blockIdx.x;
  x.steps = (x.kv_end - x.kv_begin + kChunkKvTile - 1) / kChunkKvTile;
  x.solo = x.n_rows <= kChunkTileRows;
  return x;
}

}  // namespace chunk

template <int D, bool kFp8>
__global__ void __launch_bounds__(ChunkShape<D, kFp8>::kThreads, 1)
chunk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
             const __grid_constant__ ChunkParams p) {
  using namespace chunk;
  using Shape = ChunkShape<D, kFp8>;
  constexpr bool kBf16 = !kFp8;
  constexpr uint32_t kTmemColumns = 512;                  // S0 | S1 | O0 | O1, 128 columns each (O: D of them)
  extern __shared__ __align__(1024) uint8_t smem[];   // the 128-byte swizzle counts rows from 1024-byte boundaries
  const uint32_t base = smem_u32(smem);
  const uint32_t q_tiles = base, raw = base + Shape::kRaw;
  auto bar = [&](int i) { return base + uint32_t(Shape::kBars + 8 * i); };
  const Stop stop{bar(kSlotStop), p.error_word};

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // launched as a dependent of whatever precedes it in the stream
  // The item is on its way into the L1 cache while the barriers and the tensor memory are being set up; each role then reads
  // it for itself (kept in registers from here on it cost the roles' loops a spill and 5 % of the time).
  const uint32_t found = load_again(p.serial_at);
  touch_unit(p);
  if (warp == 0) {   // the barriers, two a lane; what arrives on each: one instruction or copy, or the 128 threads of a group
    for (int i = lane; i < kNumBars; i += 32) {
      const bool by_group = (kFp8 && i < kBarEmpty) || (i >= kBarRawEmpty && i < kBarS) || (i >= kBarP && i < kBarO) ||
                            i == kBarMergeFree || i == kBarMergeFull;
      mbar_init(bar(i), by_group ? 128 : 1);
    }
    if (lane == 0) *reinterpret_cast<volatile uint32_t*>(smem + Shape::kBars + 8 * kSlotStop) = 0;
    fence_mbar_init();
  }
  if (warp == 9) tmem_alloc(bar(kSlotTmem), kTmemColumns);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + Shape::kBars + 8 * kSlotTmem);
  // another plan in the workspace than the one this launch was made for: nothing is computed
  const bool run = found == p.serial && blockIdx.y + blockIdx.z * 65535u < uint32_t(p.num_items);
  if (found != p.serial && threadIdx.x == 0) atomicOr(p.error_word, uint32_t(LIBRA_ERR_PLAN_CHANGED));
  const bool solo = load_unit(p).solo;
  const int n_stages = solo ? Shape::kSoloStages : Shape::kStages;
  const uint32_t ring = base + Shape::kRing - uint32_t(n_stages - Shape::kStages) * Shape::kTileBytes;
  int next_copy = -1;         // a copying warp's next tile when it left; -1: it has asked for none
  bool tail_copy = false;     // its newest one signals kBarTail and not the tile's own barrier

  if (run && warp < 8) {
    // ------------------------------------------------------------------ softmax group t: row tile t (both: tile 0 if solo)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Shape::kSoftmaxRegs));
    const int t = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    const uint32_t s_tmem = tmem + lanes + t * 128, o_tmem = tmem + lanes + 256 + t * 128;
    float* const row_factor = reinterpret_cast<float*>(smem + Shape::kFloats);   // [2][128]
    float* const merge_ml = row_factor + 256;                                    // [2][128]
    do {   // left by break when a wait has run out
      ChunkUnit x = load_unit(p);
      const RowMap rows(p, x.row0);
      const int steps = x.steps_of(t), all_steps = x.steps;
      const int kv_pitch = solo ? 2 * kChunkKvTile : kChunkKvTile;
      int kv0 = x.kv_begin + (solo ? t * kChunkKvTile : 0), sees;
      {
        const int tile_row = (solo ? 0 : t * kChunkTileRows) + row;   // row within the item
        int token, head;
        rows.at(p, tile_row, token, head);
        sees = tile_row < x.n_rows ? min(x.kv_end, x.ctx + token + 1) : 0;   // cached tokens this row sees
      }
      // ---- Q: 16 threads (8 at D = 64) bring a row
      if (all_steps > 0 && !(solo && t == 1)) {
        constexpr int kLanes = D / 8, kRowsAtOnce = 128 / kLanes, kVecs = kChunkTileRows / kRowsAtOnce;
        uint4 v[kVecs];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          const int ir = t * kChunkTileRows + row / kLanes + i * kRowsAtOnce;
          v[i] = make_uint4(0, 0, 0, 0);
          if (ir < x.n_rows) {
            int token, head;
            rows.at(p, ir, token, head);
            v[i] = __ldg(reinterpret_cast<const uint4*>(p.q + (int64_t(x.q_start) + token) * p.q_stride +
                                                        int64_t(x.head * p.group + head) * D) + row % kLanes);
          }
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          const int r = row / kLanes + i * kRowsAtOnce;
          if constexpr (kFp8) {
            float down;
            v[i] = scaled_half_row<kLanes>(v[i], down);
            if (row % kLanes == 0) row_factor[t * 128 + r] = down;
          }
          st_shared(q_tiles + t * Shape::kTileBytes + swizzled(r, row % kLanes), v[i]);
        }
      }
      fence_proxy_async();
      arrive(bar(kBarQ + t));
      if constexpr (kFp8) {
        // the row factors come from the group that loaded the tile
        if (!wait_warp(bar(kBarQ + (solo ? 0 : t)), 0, stop)) break;
      }
      auto row_scale = [&] {   // score -> base-2 exponent
        if constexpr (kFp8) {
          // The product with the factor of a row of zeros, or nearly so, may lie below the smallest normal number and be flushed to
          // zero, and -inf * 0 is no masked score.  At that number scores of up to 2^27 weigh all tokens alike, as they should.
          if (all_steps > 0) return fmaxf(p.scale_log2 * row_factor[(solo ? 0 : t) * 128 + row], 0x1p-126f);
        }
        return p.scale_log2;
      };
      float rs = row_scale();
      const bool idle = (solo ? 0 : t * kChunkTileRows) + 32 * (warp & 3) >= x.n_rows;   // a warp without a row
      // ---- the steps
      float m = -INFINITY, l = 0.f;
      bool ok = true;
#pragma unroll 1
      for (int j = 0; j < steps; ++j, kv0 += kv_pitch) {
        ok = wait_warp(bar(kBarS + t), j & 1, stop);
        if (!ok) break;
        fence_after();
        if (idle) {   // its rows of P may hold anything: they reach its rows of O alone, which nobody reads
          arrive(bar(kBarP + t));
          arrive(bar(kBarPTail + t));
          continue;
        }
        float s[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(s + 32 * c, s_tmem + 32 * c);
        wait_ld();
#pragma unroll
        for (int c = 0; c < 4; ++c) settle<32>(s + 32 * c);
        const int limit = sees - kv0;
        if (__any_sync(0xffffffffu, limit < kChunkKvTile)) {
#pragma unroll
          for (int c = 0; c < 128; ++c) s[c] = c < limit ? s[c] : -INFINITY;
        }
        auto row_max = [&] {
          float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
          for (int c = 4; c < 124; c += 8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mx[i] = max3(mx[i], s[c + 2 * i], s[c + 2 * i + 1]);
          }
          return max3(max3(mx[0], mx[1], s[124]), max3(mx[2], mx[3], s[125]), fmaxf(s[126], s[127]));
        };
        float2 sum[2], shift2, rs2;
        uint32_t pk[16];
        auto probabilities = [&](int part) {   // of 32 columns
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            float2 e = fma2(make_float2(s[32 * part + 2 * c], s[32 * part + 2 * c + 1]), rs2, shift2);
            e.x = ex2(e.x);
            e.y = ex2(e.y);
            sum[c & 1] = part == 0 && c < 2 ? e : add2(sum[c & 1], e);
            pk[c] = pack<kBf16>(e.x, e.y);
          }
        };
        auto set_shift = [&] {
          const float x = m == -INFINITY ? 0.f : -m * rs;
          shift2 = make_float2(x, x);
          rs2 = make_float2(rs, rs);
        };
        // The first quarter goes by the running maximum as it stands, while this tile's maximum is being found: the
        // exponentials keep their unit busy meanwhile.  It is done again where the maximum turns out to be too low, as
        // it does in the first step.
        set_shift();
        probabilities(0);
        const float tile_max = row_max();
        if (__any_sync(0xffffffffu, (tile_max - m) * rs > kMaxSlack)) {
          // the product of the step before has finished: its completion comes before that of this step's scores
          const float to = fmaxf(m, tile_max);
          const float alpha = to == -INFINITY ? 1.f : ex2((m - to) * rs);
          m = to;
          l *= alpha;
          // Rounding m * rs multiplies all of the row's probabilities by a power of two whose exponent is the rounding error.  Below
          // 2^24 that is at most a half, and cancels in the result; beyond, it could exceed what a float32 holds.  Scores are whole
          // units apart there: a power of two takes the place of rs, and the product is exact.
          if (m != -INFINITY && fabsf(m * rs) >= 0x1p24f) rs = __uint_as_float(__float_as_uint(rs) & 0x7f800000u);
          if (j > 0) {
#pragma unroll
            for (int c = 0; c < D; c += 16) {
              float o[16];
              tmem_ld16(o, o_tmem + c);
              wait_ld();
              settle<16>(o);
              uint32_t scaled[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) scaled[i] = __float_as_uint(o[i] * alpha);
              tmem_st16(o_tmem + c, scaled);
            }
          }
          set_shift();
          probabilities(0);
        }
        tmem_st16(s_tmem, pk);
#pragma unroll
        for (int part = 1; part < 4; ++part) {
          probabilities(part);
          tmem_st16(s_tmem + 16 * part, pk);
          if (part == Shape::kPEarly - 1) {   // the product starts on these while the rest is being worked out
            wait_st();
            fence_before();
            arrive(bar(kBarP + t));
          }
        }
        sum[0] = add2(sum[0], sum[1]);
        l += sum[0].x + sum[0].y;
        wait_st();
        fence_before();
        arrive(bar(kBarPTail + t));
      }
      if (!ok) break;
      // ---- the result.  Of the item only what the steps need was kept; it is read again while the last product ends.
      x = load_unit(p);
      rs = row_scale();
      if (all_steps > 0) {
        if (!wait_warp(bar(kBarO + t), 0, stop)) break;
        fence_after();
      }
      float w = 1.f;     // weight of this group's part
      if (solo && all_steps > 0) {
        // group 1 hands its part over in the Q tiles (they are free once group 0's products are done too); group 0 merges
        float* const part = reinterpret_cast<float*>(smem);   // [D][128]
        if (t == 0) {
          arrive(bar(kBarMergeFree));
          if (!wait_warp(bar(kBarMergeFull), 0, stop)) break;
        } else {
          if (!wait_warp(bar(kBarMergeFree), 0, stop)) break;
          if (idle) {
          } else if (steps > 0) {
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              float o[32];
              tmem_ld32(o, o_tmem + c);
              wait_ld();
              settle<32>(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) part[(c + i) * 128 + row] = o[i];
            }
          } else {
            for (int c = 0; c < D; ++c) part[c * 128 + row] = 0.f;
          }
          merge_ml[row] = m;
          merge_ml[128 + row] = l;
          arrive(bar(kBarMergeFull));
        }
      }
      if (solo && t == 1) break;   // group 0 writes the result
      float w1 = 0.f;
      if (solo && all_steps > 0) {
        const float m1 = merge_ml[row], l1 = merge_ml[128 + row];
        const float to = fmaxf(m, m1);
        w = to == -INFINITY ? 0.f : ex2((m - to) * rs);
        w1 = to == -INFINITY ? 0.f : ex2((m1 - to) * rs);
        l = l * w + l1 * w1;
        m = to;
      }
      const float inv = p.v_scale / l;
      const float lse = l > 0.f ? (m * rs + lg2(l)) * 0.6931471805599453f : (l == 0.f ? -INFINITY : l);
      const int warp_row = (solo ? 0 : t * kChunkTileRows) + 32 * (warp & 3);
      if (warp_row >= x.n_rows) break;   // no row of this warp's
      const int tile_row = warp_row + lane;
      const bool valid = tile_row < x.n_rows;
      const RowMap rows_out(p, x.row0);
      int token, head;
      rows_out.at(p, valid ? tile_row : 0, token, head);
      const int64_t out_row = (int64_t(x.q_start) + token) * p.num_q_heads + x.head * p.group + head;
      const int64_t part_row = (int64_t(x.slot) + tile_row) * p.num_kv_heads + x.head;
      if (valid) {
        if (x.slot >= 0) p.partial_lse[part_row] = lse;
        else if (p.lse != nullptr) p.lse[out_row] = lse;
      }
      // The loops from here on are not unrolled: this code runs once a block, and in a block's first run on a multiprocessor
      // fetching it takes longer than running it (6300 cycles unrolled, 1900 as it is).
      // Through shared memory, so that the warp writes whole rows: its 32 rows of 2 D bytes (the fp32 partial results in two
      // halves) lie, 16-byte vectors permuted by row, in the Q tile that nobody reads any more (solo: the ring's).
      constexpr int kRowBytes = 2 * D, kRowLanes = kRowBytes / 16, kHalves = 2;
      const uint32_t out_stage = (solo ? base + Shape::kRing : q_tiles + t * Shape::kTileBytes) + uint32_t(warp & 3) * (32 * kRowBytes);
      const uint32_t my_row = out_stage + uint32_t(lane) * kRowBytes;
      auto result = [&](float* o, int c) {   // columns c .. c + 31 of this thread's row
        if (all_steps > 0) {
          tmem_ld32(o, o_tmem + c);
          wait_ld();
          settle<32>(o);
          if (solo) {
            const float* const part = reinterpret_cast<const float*>(smem);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = o[i] * w + part[(c + i) * 128 + row] * w1;
          }
        }
        // a row that has seen nothing is zero whatever the accumulator holds
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = l == 0.f ? 0.f : o[i] * inv;
      };
      auto write_rows = [&](auto address) {   // address(token, head, row): where the row's kRowBytes go
        __syncwarp();
#pragma unroll 2
        for (int i = 0; i < kRowLanes; ++i) {
          const int r = i * (32 / kRowLanes) + lane / kRowLanes, vec = lane % kRowLanes;
          const int r_item = warp_row + r;
          if (r_item < x.n_rows) {
            int token_r, head_r;
            rows_out.at(p, r_item, token_r, head_r);
            reinterpret_cast<uint4*>(address(token_r, head_r, r_item))[vec] =
                ld_shared(out_stage + uint32_t(r) * kRowBytes + uint32_t((vec ^ (r & 7)) << 4));
          }
        }
        __syncwarp();
      };
      if (x.slot < 0) {
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float o[32];
          result(o, c);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            st_shared(my_row + uint32_t(((c / 8 + i) ^ (lane & 7)) << 4),
                      make_uint4(pack<true>(o[8 * i], o[8 * i + 1]), pack<true>(o[8 * i + 2], o[8 * i + 3]),
                                 pack<true>(o[8 * i + 4], o[8 * i + 5]), pack<true>(o[8 * i + 6], o[8 * i + 7])));
          }
        }
        write_rows([&](int token_r, int head_r, int) {
          return p.out + ((int64_t(x.q_start) + token_r) * p.num_q_heads + x.head * p.group + head_r) * D;
        });
      } else {
#pragma unroll 1
        for (int half = 0; half < kHalves; ++half) {
#pragma unroll 1
          for (int c = half * (D / 2); c < (half + 1) * (D / 2); c += 32) {
            float o[32];
            result(o, c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              st_shared(my_row + uint32_t((((c - half * (D / 2)) / 4 + i) ^ (lane & 7)) << 4),
                        make_uint4(__float_as_uint(o[4 * i]), __float_as_uint(o[4 * i + 1]), __float_as_uint(o[4 * i + 2]),
                                   __float_as_uint(o[4 * i + 3])));
            }
          }
          write_rows([&](int, int, int r_item) {
            return p.partial_o + ((int64_t(x.slot) + r_item) * p.num_kv_heads + x.head) * D + half * (D / 2);
          });
        }
      }
    } while (false);
  } else if (warp >= 8 && warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kIssueRegs));
    if (run && warp != 9) {
      // ------------------------------------------------------------------ copies
      const int loader = warp == 8 ? 0 : warp - 9;
      const int n = kFp8 ? Shape::kRawStages : n_stages;
      constexpr int kFull = kFp8 ? kBarRawFull : kBarFull, kEmpty = kFp8 ? kBarRawEmpty : kBarEmpty;
      constexpr int kStageBytes = kFp8 ? Shape::kRawBytes : Shape::kTileBytes;
      constexpr int kBoxes = kFp8 ? 1 : D / 64;                     // per page
      const uint32_t dst0 = kFp8 ? raw : ring;
      const int tile_pages_shift = 7 - p.page_shift;                // 128 tokens are 8, 4 or 2 pages
      const int my_page = lane & ((1 << tile_pages_shift) - 1), my_box = lane >> tile_pages_shift;
      const int page_tokens = 1 << p.page_shift;
      const ChunkUnit x = load_unit(p);
      uint32_t phase = 0;
      int i = loader, stage = loader;   // the next tile that this warp brings, and its place (a ring has three stages or more)
      bool ok = true;
      if (i < 2 * x.steps) {
        const int32_t* row = p.block_table + int64_t(x.b) * p.block_table_ld;
        // this lane's page of step j (every lane of a page holds its id); -1 past the range
        auto page_of = [&](int j) -> int32_t {
          const int tok = x.kv_begin + j * kChunkKvTile + (my_page << p.page_shift);
          if (j >= x.steps || tok >= x.kv_end) return -1;
          const int32_t id = __ldg(row + (tok >> p.page_shift));
          if (id < 0 || int64_t(id) >= p.num_pages) {
            if (my_box == 0) atomicOr(p.error_word, uint32_t(LIBRA_ERR_BAD_PAGE_ID));
            return int32_t(p.num_pages > 0x7ffffffe ? 0x7ffffffe : p.num_pages);   // past the map's end: reads as zeros
          }
          return id;
        };
        int32_t next = page_of(x.step_of(i));
        for (; i < 2 * x.steps; i += kLoaders) {
          const bool is_v = x.is_v(i);
          const int left = x.kv_end - (x.kv_begin + x.step_of(i) * kChunkKvTile);   // live tokens from the tile's first on
          const int32_t page = next;
          next = page_of(i + kLoaders < 2 * x.steps ? x.step_of(i + kLoaders) : x.steps);
          const int pages = min(kChunkKvTile >> p.page_shift, (left + page_tokens - 1) >> p.page_shift);
          const bool tail = !kFp8 && is_v && left < kChunkKvTile;
          ok = wait_warp(bar(kEmpty + stage), phase ^ 1, stop);
          if (!ok) break;
          const uint32_t signal = tail ? bar(kBarTail + loader) : bar(kFull + stage);
          const uint32_t dst = dst0 + stage * kStageBytes;
          if (lane == 0) mbar_expect_tx(signal, uint32_t(pages) * uint32_t(page_tokens) * uint32_t(D * (kFp8 ? 1 : 2)));
          __syncwarp();
          if (my_page < pages && my_box < kBoxes) {
            const int c1 = p.pos_head == 1 ? x.head : (p.pos_page == 1 ? page : 0);
            const int c2 = p.pos_head == 2 ? x.head : (p.pos_page == 2 ? page : 0);
            const int c3 = p.pos_head == 3 ? x.head : (p.pos_page == 3 ? page : 0);
            const uint32_t to = dst + uint32_t(my_box) * (kChunkKvTile * 128) + uint32_t(my_page * page_tokens) * (kFp8 ? D : 128);
            asm volatile(
                "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(to),
                "l"(reinterpret_cast<uint64_t>(is_v ? &map_v : &map_k)), "r"(signal), "r"(my_box * 64), "r"(c1), "r"(c2), "r"(c3)
                : "memory");
          }
          if (tail) {   // rows behind the range are zeroed before the tile is handed on; a block has one such tile, its last
            ok = wait_warp(signal, 0, stop);
            if (!ok) {
              tail_copy = true;
              i += kLoaders;
              break;
            }
            const int chunks = (kChunkKvTile - left) * (D / 8);
            for (int k = lane; k < chunks; k += 32) {
              st_shared(dst + swizzled(left + k / (D / 8), k % (D / 8)), make_uint4(0, 0, 0, 0));
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) arrive(bar(kFull + stage));
          }
          stage += kLoaders;
          if (stage >= n) {
            stage -= n;
            phase ^= 1;
          }
        }
      }
      next_copy = i;
    } else if (run && warp == 9) {
      // ------------------------------------------------------------------ tensor-core instructions
      // The whole warp walks through the steps and one lane issues: what the instructions take (descriptors, addresses) is then
      // known to be the same for the warp; issuing from a branch that a single lane had taken measured 8 % slower (1.71 against
      // 1.58 ms for 4096 new tokens on 12288, 64 / 8 heads).
      constexpr uint32_t kDescS = instr_desc<kBf16>(kChunkKvTile, false), kDescO = instr_desc<kBf16>(D, true);
      const bool leader = elect_one();
      int stage = 0;
      uint32_t phase = 0, n_p = 0;   // n_p: bit t = parity of row tile t's probabilities
      bool ok = true;
      // What the instructions take is worked out ahead of the waits: between a wait and the instructions behind it nothing is
      // computed, the tensor cores would stand still meanwhile.
      const uint32_t ring_low = uniform(desc_low(ring, 0)), q_low = uniform(desc_low(q_tiles, 0));
      const uint32_t tm = uniform(tmem);
      constexpr uint32_t kTileLow = Shape::kTileBytes >> 4, kVLow = uint32_t((kChunkKvTile * 128) >> 4) << 16;   // lbo of V
      auto next_tile = [&](int& at) {   // the next tile of the ring, once it is there
        at = stage;
        if (!wait_warp(bar(kBarFull + stage), phase, stop)) return false;
        if (++stage == n_stages) {
          stage = 0;
          phase ^= 1;
        }
        return true;
      };
      auto scores = [&](int t, uint32_t a0, uint32_t b0) {   // S_t = Q K^T
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = uint32_t((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4;
          mma_ss(tm + t * 128, smem_desc(a0 + off), smem_desc(b0 + off), kDescS, k > 0);
        }
        commit(bar(kBarS + t));
      };
      auto values = [&](int t, uint32_t b0, bool first, int k0, int k1) {   // O_t += P_t V, 16-token slices k0 .. k1 - 1
#pragma unroll
        for (int k = k0; k < k1; ++k) {
          mma_ts(tm + 256 + t * 128, tm + t * 128 + k * 8, smem_desc(b0 + k * (2048 >> 4)), kDescO, !(first && k == 0));
        }
      };
      int turns;
      {
        const ChunkUnit x = load_unit(p);
        turns = uniform(solo ? x.steps : 2 * x.steps);
      }
      if (turns > 0 && wait_warp(bar(kBarQ + 0), 0, stop) && wait_warp(bar(kBarQ + 1), 0, stop)) {
        // Two kinds of items, two loops: written as one with the difference tested, either ran 3 - 8 % slower (the time between the
        // end of a wait and the next product is what this warp is made of).  No __syncwarp: the votes of the waits suffice.
        int k_stage = 0, v_stage = 0;
        if (!solo) {   // turn i is row tile i & 1 at step i / 2; the two share the tiles of K and V
#pragma unroll 1
          for (int i0 = -2; ok && i0 < turns; i0 += 2) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const int i = i0 + t;
              const bool now = i0 >= 0 && i < turns, more = i + 2 < turns;
              if (t == 0) {
                if (now) ok = ok && next_tile(v_stage);
                if (more) ok = ok && next_tile(k_stage);
              }
              const uint32_t v_low = uniform(ring_low + kVLow + v_stage * kTileLow);
              const uint32_t k_low = uniform(ring_low + k_stage * kTileLow);
              if (now) {
                ok = ok && wait_warp(bar(kBarP + t), (n_p >> t) & 1, stop);
                if (!ok) break;
                fence_after();
                if (leader) values(t, v_low, i0 == 0, 0, 2 * Shape::kPEarly);
                ok = wait_warp(bar(kBarPTail + t), (n_p >> t) & 1, stop);
                n_p ^= 1u << t;
              }
              if (!ok) break;
              fence_after();
              if (leader) {
                if (now) {
                  values(t, v_low, false, 2 * Shape::kPEarly, kChunkKvTile / 16);
                  if (t == 1) commit(bar(kBarEmpty + v_stage));
                  if (!more) commit(bar(kBarO + t));
                }
                if (more) {
                  scores(t, q_low + t * kTileLow, k_low);
                  if (t == 1) commit(bar(kBarEmpty + k_stage));
                }
              }
            }
          }
        } else {   // turn i is step i of row tile 0, taken by group i & 1; bound by the copies: the next K is waited for last
          auto signal = [&](int b) {
            if (leader) commit(bar(b));
          };
#pragma unroll 1
          for (int i0 = -2; ok && i0 < turns; i0 += 2) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const int i = i0 + t;
              if (i0 >= 0 && i < turns) {
                ok = ok && next_tile(v_stage);
                fence_after();
                ok = ok && wait_warp(bar(kBarP + t), (n_p >> t) & 1, stop);
                if (!ok) break;
                fence_after();
                uint32_t v_low = uniform(ring_low + kVLow + v_stage * kTileLow);
                if (leader) values(t, v_low, i0 == 0, 0, 2 * Shape::kPEarly);
                ok = wait_warp(bar(kBarPTail + t), (n_p >> t) & 1, stop);
                if (!ok) break;
                n_p ^= 1u << t;
                fence_after();
                v_low = uniform(ring_low + kVLow + v_stage * kTileLow);
                if (leader) values(t, v_low, false, 2 * Shape::kPEarly, kChunkKvTile / 16);
                signal(kBarEmpty + v_stage);
                if (i + 2 >= turns) signal(kBarO + t);
              }
              if (i + 2 < turns) {
                ok = ok && next_tile(k_stage);
                fence_after();
                if (!ok) break;
                const uint32_t k_low = uniform(ring_low + k_stage * kTileLow);
                if (leader) scores(t, q_low, k_low);
                signal(kBarEmpty + k_stage);
              }
            }
          }
        }
        if (ok && turns == 1 && leader) commit(bar(kBarO + 1));   // group 1 has no turn
      }
    }
  } else if (kFp8 && warp >= 12) {
    if constexpr (kFp8) {
      // ------------------------------------------------------------------ E4M3 codes -> fp16 tiles
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kConvertRegs));
      if (run) {
        const int tid = threadIdx.x - 384;
        int stage = 0, rstage = 0;
        uint32_t phase = 0, rphase = 0;
        const ChunkUnit x = load_unit(p);
        {
          for (int i = 0; i < 2 * x.steps; ++i) {
            const int live = x.is_v(i) ? x.kv_end - (x.kv_begin + x.step_of(i) * kChunkKvTile) : kChunkKvTile;   // K needs no zeroing
            if (!wait_warp(bar(kBarRawFull + rstage), rphase, stop) || !wait_warp(bar(kBarEmpty + stage), phase ^ 1, stop)) break;
            const uint8_t* src = smem + Shape::kRaw + rstage * Shape::kRawBytes;
            const uint32_t dst = ring + stage * Shape::kTileBytes;
            constexpr int kVec = D / 16;   // 16-byte vectors of codes per token
#pragma unroll 4
            for (int v = tid; v < kChunkKvTile * kVec; v += 128) {
              const int r = v / kVec, c = v % kVec;
              uint4 in = *reinterpret_cast<const uint4*>(src + r * D + c * 16);
              if (r >= live) in = make_uint4(0, 0, 0, 0);
              uint4 lo, hi;
              cvt_e4m3x4(in.x, lo.x, lo.y);
              cvt_e4m3x4(in.y, lo.z, lo.w);
              cvt_e4m3x4(in.z, hi.x, hi.y);
              cvt_e4m3x4(in.w, hi.z, hi.w);
              // the two 64-channel halves store their even and odd vectors in opposite order: no bank conflicts
              const bool flip = (c >> 2) & 1;
              st_shared(dst + swizzled(r, 2 * c + (flip ? 1 : 0)), flip ? hi : lo);
              st_shared(dst + swizzled(r, 2 * c + (flip ? 0 : 1)), flip ? lo : hi);
            }
            fence_proxy_async();
            arrive(bar(kBarFull + stage));
            arrive(bar(kBarRawEmpty + rstage));
            if (++stage == n_stages) { stage = 0; phase ^= 1; }
            if (++rstage == Shape::kRawStages) { rstage = 0; rphase ^= 1; }
          }
        }
      }
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  fence_after();
  if (stop.set()) {   // a wait has run out, and no role starts anything more: what is under way ends before the block does
    if (warp == 9) {   // the products
      if (elect_one()) commit(bar(kBarDrain));   // the lane that issued them: the same one is elected every time
      for (int k = 0; k < kDrainTries && !mbar_try_wait(bar(kBarDrain), 0); ++k) {}
      __syncwarp();
    } else if (next_copy >= 0) {   // this warp's copies
      const int n = kFp8 ? Shape::kRawStages : n_stages;
      constexpr int kFull = kFp8 ? kBarRawFull : kBarFull;
      for (int g = ring_newest(next_copy); ring_may_fly(g, next_copy, n); g = ring_before(g)) {
        const bool tail = tail_copy && g == ring_newest(next_copy);
        const uint32_t b = tail ? bar(kBarTail + (warp == 8 ? 0 : warp - 9)) : bar(kFull + g % n), parity = tail ? 0 : (g / n) & 1;
        for (int k = 0; k < kDrainTries && !mbar_try_wait(b, parity); ++k) {}
      }
    }
  }
  if (warp == 9) tmem_dealloc(tmem, kTmemColumns);
}

struct ChunkMergeParams {
  const int4* merges;         // two per ChunkMerge
  const uint32_t* serial_at;
  const float* partial_o;
  const float* partial_lse;
  __nv_bfloat16* out;
  float* lse;
  uint32_t serial;
  int32_t num_q_heads, num_kv_heads, group;
};

constexpr int kChunkMergeWarps = 8;

// Log-sum-exp merge of the chunks of a cut item: one warp per row, chunks added in order (no dependence on scheduling).
// grid = (merges x KV heads, ceil(kChunkItemRows / kChunkMergeWarps))
template <int D>
__global__ void __launch_bounds__(kChunkMergeWarps * 32) chunk_merge_kernel(const ChunkMergeParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");   // every thread: see combine_kernel
  if (*p.serial_at != p.serial) return;   // the attention kernel has said so
  constexpr int V = D / 32;
  const int lane = threadIdx.x & 31;
  const int4 a = p.merges[2 * (blockIdx.x / p.num_kv_heads)], b = p.merges[2 * (blockIdx.x / p.num_kv_heads) + 1];
  const int head = blockIdx.x % p.num_kv_heads, n_rows = a.z, n = b.x;
  const int r = blockIdx.y * kChunkMergeWarps + (threadIdx.x >> 5);
  if (r >= n_rows) return;
  const int64_t first = (int64_t(a.w) + r) * p.num_kv_heads + head, pitch = int64_t(n_rows) * p.num_kv_heads;
  const float l0 = lane < n ? p.partial_lse[first + lane * pitch] : -INFINITY;
  const float l1 = lane + 32 < n ? p.partial_lse[first + (lane + 32) * pitch] : -INFINITY;
  float m = fmaxf(l0, l1);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
  if (m == -INFINITY) m = 0.f;
  const float w0 = __expf(l0 - m), w1 = __expf(l1 - m);
  float den = 0.f, num[V];
#pragma unroll
  for (int v = 0; v < V; ++v) num[v] = 0.f;
  const float* src = p.partial_o + first * D + lane * V;
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const float w = __shfl_sync(0xffffffffu, i < 32 ? w0 : w1, i & 31);
    den += w;
#pragma unroll
    for (int v = 0; v < V; ++v) num[v] += w * src[int64_t(i) * pitch * D + v];
  }
  const float inv = den == 0.f ? 0.f : 1.f / den;   // 0: a row that sees nothing; NaN stays NaN
  const int flat = a.y + r, token = flat / p.group;
  const int64_t row = (int64_t(a.x) + token) * p.num_q_heads + head * p.group + flat - token * p.group;
  if (p.lse != nullptr && lane == 0) p.lse[row] = den == 0.f ? -INFINITY : m + __logf(den);
#pragma unroll
  for (int v = 0; v < V; v += 2) {
    *reinterpret_cast<__nv_bfloat162*>(p.out + row * D + lane * V + v) = __floats2bfloat162_rn(num[v] * inv, num[v + 1] * inv);
  }
}

}  // namespace libra
