// Block tables and slot maps made on the GPU: pages handed out to sequences that grow and taken back from those that shrink.
//
//   extend  sequence b of L_b tokens gets n_b more:  w_b = ceil((L_b + n_b) / P) - ceil(L_b / P) pages, in the order of the batch
//           and of the pages; the k-th of them all is free[count - 1 - k].  Row q_offsets[b] + i is token t = L_b + i, in slot
//           page(t / P) * P + t % P; a page whose id is outside the pool has numbers below -1 for slots, which whoever uses them reports.
//   trim    sequence b keeps its first m_b tokens: pages from ceil(m_b / P) on go back; the k-th of the F of them is
//           free[count + F - 1 - k], so that what extend has taken trim puts back in the order it was.
//
// Integers only.  A token's page index follows from its position, and a page is new exactly where its first token is, so that one
// pass over the rows writes positions, slots and block table; what it needs is the two prefix sums (rows and pages).
//
// One cluster of up to 8 blocks.  Every block computes the prefix sums of the whole batch for itself (up to 4096 sequences, four a
// thread) into its shared memory - that is cheaper than handing them round - and the rows, or the pages that go back, are shared out
// between the blocks.  All checks are made on the sums before anything is written.  seq_lens and the
// count change in place: the first block writes them once all have read them (cluster barrier).
//
// What bounds it: latency; in long batches the instructions of eight multiprocessors.  A step of 64 sequences, extend and trim: 6 us
// together; 256 sequences with 115K new tokens: 13 us together.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "libra.h"

namespace libra {

constexpr int kTablePerThread = 4;
constexpr int kTableMaxThreads = 1024;
constexpr int kTableMaxBatch = kTablePerThread * kTableMaxThreads;
constexpr int kTableMaxBlocks = 8;   // of the cluster
constexpr int kTableRows = 8;        // of a thread and turn in long batches; no more than a page has tokens

struct TableParams {
  const int32_t* change;   // extend: new tokens of each sequence; trim: tokens that it keeps
  int32_t* seq_lens;
  int32_t* block_table;
  int32_t* free_pages;
  int32_t* free_count;
  int32_t* q_offsets;      // extend only, as the next two, which may be null
  int32_t* positions;
  int32_t* slots;
  uint32_t* error_word;
  int64_t num_pages;
  int32_t batch, block_table_ld, page_shift, max_rows;
};

namespace table {

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t n;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

struct Sums {
  int64_t rows;    // may pass 32 bits where a call is refused
  int32_t pages;   // as many as rows at most
};

// Exclusive prefix sums over the threads of the block, and the totals.  Of the warps the first `busy` have something.
__device__ __forceinline__ Sums block_scan(Sums mine, int busy, Sums& total) {
  __shared__ Sums warp_sums[kTableMaxThreads / 32 + 1];   // the total behind the last
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sums in = mine;
  if (warp < busy) {
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int64_t r = __shfl_up_sync(0xffffffffu, in.rows, off);
      const int32_t g = __shfl_up_sync(0xffffffffu, in.pages, off);
      if (lane >= off) {
        in.rows += r;
        in.pages += g;
      }
    }
    if (lane == 31) warp_sums[warp] = in;
  }
  __syncthreads();
  if (warp == 0) {   // the warps' sums become what lies before each
    const Sums own = lane < busy ? warp_sums[lane] : Sums{0, 0};
    Sums upto = own;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int64_t r = __shfl_up_sync(0xffffffffu, upto.rows, off);
      const int32_t g = __shfl_up_sync(0xffffffffu, upto.pages, off);
      if (lane >= off) {
        upto.rows += r;
        upto.pages += g;
      }
    }
    __syncwarp();
    warp_sums[lane] = {upto.rows - own.rows, upto.pages - own.pages};
    if (lane == 31) warp_sums[32] = upto;
  }
  __syncthreads();
  total = warp_sums[32];
  const Sums before = warp_sums[warp];
  return {before.rows + in.rows - mine.rows, before.pages + in.pages - mine.pages};
}

// ceil(len / page size) of a length that is not negative
__device__ __forceinline__ int32_t pages_of(int32_t len, int page_shift) {
  return int32_t((uint32_t(len) + (1u << page_shift) - 1) >> page_shift);
}

// A page's first slot.  That of an id outside the pool: such that all of the page's are negative and none is -1, which asks for a row
// not to be stored.  (The id times the page size may be a good slot in 32 bits, and for id -1 the page's last slot is -1.)
__device__ __forceinline__ int32_t first_slot(int32_t id, const TableParams& p) {
  return uint32_t(id) < uint32_t(p.num_pages) ? id << p.page_shift : -(1 << p.page_shift) - 1;   // there are fewer than 2^27 pages
}

// The last i in [0, n) with begins[i] <= x; begins[0] <= x.
__device__ __forceinline__ int owner_of(const int32_t* begins, int n, int32_t x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begins[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

}  // namespace table

// grid = one cluster; dynamic shared memory: 3 * batch + 1 int32 (extend), 2 * batch (trim)
__global__ void __launch_bounds__(kTableMaxThreads) cache_extend_kernel(const TableParams p) {
  using namespace table;
  extern __shared__ int32_t sh[];
  int32_t* const row_begin = sh;                       // [batch + 1]
  int32_t* const page_begin = sh + p.batch + 1;        // [batch]
  int32_t* const length = page_begin + p.batch;        // [batch], before
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t rank = cluster_rank(), ranks = cluster_size();
  const int b0 = threadIdx.x * kTablePerThread, P = 1 << p.page_shift;
  const int64_t most = min(int64_t(p.block_table_ld) << p.page_shift, int64_t(0x7fffffff));   // that a row describes
  const int32_t count = *p.free_count;
  const bool counted = count >= 0 && count <= p.num_pages;
  uint32_t bad = counted ? 0u : LIBRA_ERR_BAD_LENGTH;
  int32_t len[kTablePerThread], add[kTablePerThread], want[kTablePerThread];
  Sums mine = {0, 0};
#pragma unroll
  for (int i = 0; i < kTablePerThread; ++i) {
    const bool live = b0 + i < p.batch;
    len[i] = live ? p.seq_lens[b0 + i] : 0;
    add[i] = live ? p.change[b0 + i] : 0;
    if (len[i] < 0 || add[i] < 0) {
      bad |= LIBRA_ERR_BAD_LENGTH;
      len[i] = add[i] = 0;
    }
    if (int64_t(len[i]) + add[i] > most) {   // a sum that is left fits 31 bits
      bad |= LIBRA_ERR_PLAN_OVERFLOW;
      add[i] = 0;
    }
    want[i] = pages_of(len[i] + add[i], p.page_shift) - pages_of(len[i], p.page_shift);
    mine.rows += add[i];
    mine.pages += want[i];
  }
  Sums total;
  Sums at = block_scan(mine, (p.batch + 32 * kTablePerThread - 1) / (32 * kTablePerThread), total);
  if (total.rows > p.max_rows) bad |= LIBRA_ERR_PLAN_OVERFLOW;
  else if (counted && total.pages > count) bad |= LIBRA_ERR_NO_PAGES;
  // every block comes to the same verdict
  const bool refused = __syncthreads_or(int(bad)) != 0;
  if (refused) {   // nothing changes, and the batch has no new rows
    if (rank == 0) {
      if (bad) atomicOr(p.error_word, bad);
      for (int b = threadIdx.x; b <= p.batch; b += blockDim.x) p.q_offsets[b] = 0;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kTablePerThread; ++i) {
    const int b = b0 + i;
    if (b < p.batch) {
      row_begin[b] = int32_t(at.rows);
      page_begin[b] = at.pages;
      length[b] = len[i];
    }
    at.rows += add[i];
    at.pages += want[i];
  }
  const int32_t rows = int32_t(total.rows);
  if (threadIdx.x == 0) row_begin[p.batch] = rows;
  __syncthreads();
  if (ranks > 1) cluster_arrive();   // this block has read the lengths and the count
  // A row a thread while there are threads enough (64 sequences, extend and trim: 6.0 us, with kTableRows 9.0), else kTableRows (115K rows: 13.0
  // us, with one 32), with whole vectors written where the arrays lie on them.
  const int64_t threads = int64_t(ranks) * blockDim.x;
  const int per = rows > threads ? kTableRows : 1;
  const bool vectors = per > 1 && ((reinterpret_cast<uintptr_t>(p.positions) | reinterpret_cast<uintptr_t>(p.slots)) & 15) == 0;
  for (int64_t r0 = (int64_t(rank) * blockDim.x + threadIdx.x) * per; r0 < rows; r0 += threads * per) {
    const int n = int(min(int64_t(per), rows - r0));
    int b = owner_of(row_begin, p.batch, int32_t(r0));
    int32_t pos[kTableRows], slot[kTableRows];
    for (int i = 0; i < n; ++b) {   // the rows of one sequence, in two pages at most; sequences without new tokens have none
      const int m = min(n - i, row_begin[b + 1] - (int32_t(r0) + i));
      if (m == 0) continue;
      const int32_t L = length[b], first = L + (int32_t(r0) + i - row_begin[b]);
      const int32_t page0 = first >> p.page_shift, page1 = (first + m - 1) >> p.page_shift, had = pages_of(L, p.page_shift);
      int32_t* const row = p.block_table + int64_t(b) * p.block_table_ld;
      // a page's id comes from the stack where the page is new, and is entered by the thread that has the page's first token
      const int32_t* const stack = p.free_pages + (count - 1 - page_begin[b] + had);
      const int32_t id0 = page0 >= had ? stack[-page0] : row[page0];
      const int32_t id1 = page1 == page0 ? id0 : (page1 >= had ? stack[-page1] : row[page1]);
      if (page0 >= had && (first & (P - 1)) == 0) row[page0] = id0;
      if (page1 != page0 && page1 >= had) row[page1] = id1;
      const int32_t slots0 = first_slot(id0, p), slots1 = first_slot(id1, p);
#pragma unroll
      for (int k = 0; k < kTableRows; ++k) {
        if (k >= i && k < i + m) {
          pos[k] = first + (k - i);
          slot[k] = (pos[k] >> p.page_shift == page0 ? slots0 : slots1) + (pos[k] & (P - 1));
        }
      }
      i += m;
    }
    if (vectors && n == kTableRows) {
#pragma unroll
      for (int k = 0; k < kTableRows; k += 4) {
        if (p.positions) *reinterpret_cast<int4*>(p.positions + r0 + k) = make_int4(pos[k], pos[k + 1], pos[k + 2], pos[k + 3]);
        if (p.slots) *reinterpret_cast<int4*>(p.slots + r0 + k) = make_int4(slot[k], slot[k + 1], slot[k + 2], slot[k + 3]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kTableRows; ++k) {
        if (k < n && p.positions) p.positions[r0 + k] = pos[k];
        if (k < n && p.slots) p.slots[r0 + k] = slot[k];
      }
    }
  }
  __syncwarp();   // the lanes' loops differ in length, and the barrier is one instruction of whole warps
  if (ranks > 1) cluster_wait();
  if (rank == 0) {
#pragma unroll
    for (int i = 0; i < kTablePerThread; ++i) {
      if (b0 + i < p.batch && add[i] > 0) p.seq_lens[b0 + i] = len[i] + add[i];
    }
    for (int b = threadIdx.x; b <= p.batch; b += blockDim.x) p.q_offsets[b] = row_begin[b];
    if (threadIdx.x == 0) *p.free_count = count - total.pages;
  }
}

__global__ void __launch_bounds__(kTableMaxThreads) cache_trim_kernel(const TableParams p) {
  using namespace table;
  extern __shared__ int32_t sh[];
  int32_t* const page_begin = sh;              // [batch]
  int32_t* const left = sh + p.batch;          // [batch]: pages that stay
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t rank = cluster_rank(), ranks = cluster_size();
  const int b0 = threadIdx.x * kTablePerThread;
  const int64_t most = int64_t(p.block_table_ld) << p.page_shift;
  const int32_t count = *p.free_count;
  uint32_t bad = count < 0 || count > p.num_pages ? LIBRA_ERR_BAD_LENGTH : 0u;
  int32_t len[kTablePerThread], keep[kTablePerThread], stay[kTablePerThread], gone[kTablePerThread];
  Sums mine = {0, 0};   // rows: the pages once more, in 64 bits
#pragma unroll
  for (int i = 0; i < kTablePerThread; ++i) {
    const bool live = b0 + i < p.batch;
    len[i] = live ? p.seq_lens[b0 + i] : 0;
    keep[i] = live ? p.change[b0 + i] : 0;
    if (len[i] > most) bad |= LIBRA_ERR_PLAN_OVERFLOW;
    if (keep[i] < 0 || keep[i] > len[i]) bad |= LIBRA_ERR_BAD_LENGTH;
    if (bad) len[i] = keep[i] = 0;
    stay[i] = pages_of(keep[i], p.page_shift);
    gone[i] = pages_of(len[i], p.page_shift) - stay[i];
    mine.rows += gone[i];
    mine.pages += gone[i];
  }
  Sums total;
  Sums at = block_scan(mine, (p.batch + 32 * kTablePerThread - 1) / (32 * kTablePerThread), total);
  if (count + total.rows > p.num_pages) bad |= LIBRA_ERR_BAD_LENGTH;   // more pages than there are
  const bool refused = __syncthreads_or(int(bad)) != 0;
  if (refused) {
    if (rank == 0 && bad) atomicOr(p.error_word, bad);
    return;
  }
#pragma unroll
  for (int i = 0; i < kTablePerThread; ++i) {
    if (b0 + i < p.batch) {
      page_begin[b0 + i] = at.pages;
      left[b0 + i] = stay[i];
    }
    at.pages += gone[i];
  }
  __syncthreads();
  if (ranks > 1) cluster_arrive();
  const int64_t step = int64_t(ranks) * blockDim.x;
  for (int64_t k = int64_t(rank) * blockDim.x + threadIdx.x; k < total.pages; k += step) {
    const int b = owner_of(page_begin, p.batch, int32_t(k));
    p.free_pages[count + total.pages - 1 - k] = p.block_table[int64_t(b) * p.block_table_ld + left[b] + (k - page_begin[b])];
  }
  __syncwarp();   // the lanes' loops differ in length, and the barrier is one instruction of whole warps
  if (ranks > 1) cluster_wait();
  if (rank == 0) {
#pragma unroll
    for (int i = 0; i < kTablePerThread; ++i) {
      if (b0 + i < p.batch && keep[i] != len[i]) p.seq_lens[b0 + i] = keep[i];
    }
    if (threadIdx.x == 0) *p.free_count = count + total.pages;
  }
}

}  // namespace libra
