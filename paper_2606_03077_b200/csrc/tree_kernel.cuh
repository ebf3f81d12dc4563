// Trees of drafted tokens: who sees whom, and the rows of the accepted ones moved together.  Both are latency: 64 sequences with trees of
// 8 to 32, mask and one layer's rows, 6 us together.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "libra.h"

namespace libra {

struct TreeMaskParams {
  const int32_t* parents;     // [rows]
  const int32_t* q_offsets;   // [batch + 1]
  const int32_t* seq_lens;    // [batch]
  uint32_t* mask;             // [rows][mask_ld]
  int32_t* positions;         // [rows], or null
  uint32_t* error_word;
  int32_t max_rows, mask_ld;
};

constexpr int kTreeMaskThreads = 128;

// Word w of every row of a sequence: bit j - 32 w for every ancestor j of the row's token and for itself.  A thread walks from its
// token towards the root, and stops where the ancestors leave its word; the threads of word 0 get to the root and count the depth.
// Bound by latency: a step is one read of shared memory.  grid = (batch, mask_ld), dynamic shared memory: 32 * mask_ld int32
__global__ void __launch_bounds__(kTreeMaskThreads) tree_mask_kernel(const TreeMaskParams p) {
  extern __shared__ int32_t parent[];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int b = blockIdx.x, first_of_word = 32 * int(blockIdx.y);
  const int32_t first = p.q_offsets[b], end = p.q_offsets[b + 1];
  uint32_t bad = 0;
  if (first < 0 || end < first) bad = LIBRA_ERR_BAD_LENGTH;
  else if (end > p.max_rows || end - first > 32 * p.mask_ld) bad = LIBRA_ERR_PLAN_OVERFLOW;
  if (bad) {   // nothing of this sequence is written
    if (threadIdx.x == 0) atomicOr(p.error_word, bad);
    return;
  }
  const int n = end - first;
  for (int i = threadIdx.x; i < n; i += kTreeMaskThreads) {
    int32_t up = p.parents[first + i];
    if (up < -1 || up >= i) {
      atomicOr(p.error_word, uint32_t(LIBRA_ERR_BAD_TREE));
      up = -1;
    }
    parent[i] = up;
  }
  __syncthreads();
  const int32_t cached = p.seq_lens[b] - n;
  for (int i = threadIdx.x; i < n; i += kTreeMaskThreads) {
    uint32_t bits = 0;
    int depth = -1;
    for (int at = i; at >= first_of_word; at = parent[at]) {
      if (at < first_of_word + 32) bits |= 1u << (at & 31);
      ++depth;
    }
    p.mask[int64_t(first + i) * p.mask_ld + blockIdx.y] = bits;
    if (blockIdx.y == 0 && p.positions) p.positions[first + i] = cached + depth;
  }
}

struct TreeKeepParams {
  const int32_t* kept;        // [batch][kept_ld]
  const int32_t* n_kept;      // [batch]
  const int32_t* q_offsets;
  const int32_t* seq_lens;
  const int32_t* block_table;
  uint8_t* k_pool;
  uint8_t* v_pool;
  int32_t* new_lens;          // [batch], or null
  uint32_t* error_word;
  int64_t stride_page, stride_head, stride_token;   // of the pools, in bytes
  int64_t num_pages;
  int32_t kept_ld, block_table_ld, page_shift;
  int32_t num_kv_heads, vectors;                    // 16-byte vectors of a row of one head
};

constexpr int kTreeKeepThreads = 256;
constexpr int kTreeKeepRows = 64;    // whose addresses are worked out together
constexpr int kTreeKeepAtOnce = 8;   // rows whose loads are in flight together

// Row i of the kept ones goes from slot cached + kept[i] to slot cached + i.  A thread moves one 16-byte column of all of them, in
// ascending order: kept[i] >= i, so that a row is read before a later one is put in its place, and needs no other thread's moves.
// grid = (batch, ceil(columns / kTreeKeepThreads)), columns = 2 pools x heads x vectors
__global__ void __launch_bounds__(kTreeKeepThreads) tree_keep_kernel(const TreeKeepParams p) {
  __shared__ int64_t from[kTreeKeepRows], to[kTreeKeepRows];   // from < 0: not moved
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int b = blockIdx.x;
  const int32_t len = p.seq_lens[b], n = p.q_offsets[b + 1] - p.q_offsets[b], m = p.n_kept[b];
  const int32_t cached = len - n;
  const int32_t* const kept = p.kept + int64_t(b) * p.kept_ld;
  uint32_t bad = 0;
  if (n < 0 || len < 0 || cached < 0) bad = LIBRA_ERR_BAD_LENGTH;
  else if ((int64_t(len) - 1) >> p.page_shift >= p.block_table_ld) bad = LIBRA_ERR_PLAN_OVERFLOW;
  else if (m < 0 || m > n || m > p.kept_ld) bad = LIBRA_ERR_BAD_TREE;
  else {
    for (int i = threadIdx.x; i < m; i += kTreeKeepThreads) {
      if (kept[i] >= n || kept[i] <= (i > 0 ? kept[i - 1] : -1)) bad = LIBRA_ERR_BAD_TREE;
    }
  }
  const bool refused = __syncthreads_or(int(bad)) != 0;
  if (blockIdx.y == 0) {
    if (bad) atomicOr(p.error_word, bad);
    if (threadIdx.x == 0 && p.new_lens) p.new_lens[b] = refused ? len : cached + m;
  }
  if (refused) return;
  const int per_pool = p.num_kv_heads * p.vectors;
  const int col = int(blockIdx.y) * kTreeKeepThreads + threadIdx.x;
  const bool is_v = col >= per_pool, mine = col < 2 * per_pool;
  const int in_pool = is_v ? col - per_pool : col, head = in_pool / p.vectors;
  uint8_t* const base = (is_v ? p.v_pool : p.k_pool) + head * p.stride_head + (in_pool - head * p.vectors) * 16;
  for (int i0 = 0; i0 < m; i0 += kTreeKeepRows) {
    const int rows = min(m - i0, kTreeKeepRows);
    __syncthreads();   // the rows before have been moved
    for (int i = threadIdx.x; i < rows; i += kTreeKeepThreads) {
      int64_t at[2];
      bool move = kept[i0 + i] != i0 + i;
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        const int32_t t = cached + (side ? i0 + i : kept[i0 + i]);
        const int32_t page = p.block_table[int64_t(b) * p.block_table_ld + (t >> p.page_shift)];
        if (move && (page < 0 || page >= p.num_pages)) {
          if (blockIdx.y == 0) atomicOr(p.error_word, uint32_t(LIBRA_ERR_BAD_PAGE_ID));
          move = false;
        }
        at[side] = int64_t(page) * p.stride_page + int64_t(t & ((1 << p.page_shift) - 1)) * p.stride_token;
      }
      from[i] = move ? at[0] : -1;
      to[i] = at[1];
    }
    __syncthreads();
    if (mine) {
      for (int i = 0; i < rows; i += kTreeKeepAtOnce) {
        uint4 row[kTreeKeepAtOnce];
#pragma unroll
        for (int u = 0; u < kTreeKeepAtOnce; ++u) {
          if (i + u < rows && from[i + u] >= 0) row[u] = *reinterpret_cast<const uint4*>(base + from[i + u]);
        }
#pragma unroll
        for (int u = 0; u < kTreeKeepAtOnce; ++u) {
          if (i + u < rows && from[i + u] >= 0) *reinterpret_cast<uint4*>(base + to[i + u]) = row[u];
        }
      }
    }
  }
}

}  // namespace libra
