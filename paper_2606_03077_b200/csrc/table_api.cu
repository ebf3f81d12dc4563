// Entry points that hand pages out and take them back on the GPU.  See include/libra.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "handle.hpp"
#include "launch.hpp"
#include "libra.h"
#include "table_kernel.cuh"

namespace {

using libra::DeviceGuard;
using libra::fail_cuda;

bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// What both calls check, and the parameters they share.
int common(libra_handle_t h, const int32_t* change, int32_t* seq_lens, int32_t* block_table, int32_t batch, int32_t* free_pages,
           int32_t* free_count, void* error_word_dev, libra::TableParams* p) {
  if (!h || !free_pages || !free_count || !error_word_dev) return LIBRA_INVALID_ARGUMENT;
  if (batch < 0 || batch > h->cfg.max_batch) return LIBRA_INVALID_ARGUMENT;
  if (batch > 0 && (!change || !seq_lens || !block_table)) return LIBRA_INVALID_ARGUMENT;   // not read where there are no sequences
  if (off(change, 4) || off(seq_lens, 4) || off(block_table, 4) || off(free_pages, 4) || off(free_count, 4) || off(error_word_dev, 4)) {
    return LIBRA_INVALID_ARGUMENT;
  }
  if (batch > 0 && change == seq_lens) return LIBRA_INVALID_ARGUMENT;   // other blocks may still be reading the one while the other is written
  if (batch > libra::kTableMaxBatch) return LIBRA_UNSUPPORTED_SHAPE;
  if (h->cfg.num_pages > 0x7fffffff / h->cfg.page_size) return LIBRA_UNSUPPORTED_SHAPE;   // a slot's number
  *p = {};
  p->change = change;
  p->seq_lens = seq_lens;
  p->block_table = block_table;
  p->free_pages = free_pages;
  p->free_count = free_count;
  p->error_word = static_cast<uint32_t*>(error_word_dev);
  p->num_pages = h->cfg.num_pages;
  p->batch = batch;
  p->block_table_ld = h->cfg.block_table_ld;
  p->page_shift = h->cfg.page_size == 16 ? 4 : (h->cfg.page_size == 32 ? 5 : 6);
  return LIBRA_OK;
}

// `work`: rows, or pages at most, that the threads share out
int launch_table(libra_handle_t h, void (*fn)(libra::TableParams), const libra::TableParams& p, int64_t work, size_t smem, void* stream) {
  DeviceGuard guard(h->cfg.device);
  if (guard.err != cudaSuccess) return fail_cuda(h, guard.err);
  if (smem > 40 * 1024) {   // beside the static part
    // not this call's bytes but the most: the limit is the process's, and a call on another thread must not find it below its own
    constexpr size_t most = (3 * size_t(libra::kTableMaxBatch) + 1) * sizeof(int32_t);
    LIBRA_CUDA_TRY(h, cudaFuncSetAttribute(reinterpret_cast<const void*>(fn), cudaFuncAttributeMaxDynamicSharedMemorySize, int(most)));
  }
  int64_t threads = std::max(1, (p.batch + libra::kTablePerThread - 1) / libra::kTablePerThread);
  threads = std::max<int64_t>(threads, std::min<int64_t>(work, libra::kTableMaxThreads));
  threads = std::min<int64_t>((threads + 31) / 32 * 32, libra::kTableMaxThreads);
  unsigned blocks = 1;
  while (blocks < unsigned(libra::kTableMaxBlocks) && int64_t(blocks) * threads < work) blocks *= 2;
  LIBRA_CUDA_TRY(h, libra::launch(h->pdl, blocks, fn, dim3(blocks), unsigned(threads), smem, static_cast<cudaStream_t>(stream), p));
  ++h->launches;
  return LIBRA_OK;
}

}  // namespace

extern "C" {

int libra_cache_extend(libra_handle_t h, const int32_t* new_tokens, int32_t* seq_lens, int32_t* block_table, int32_t batch,
                       int32_t* free_pages, int32_t* free_count, int32_t* q_offsets, int32_t* positions, int32_t* slots,
                       int32_t max_rows, void* error_word_dev, void* stream) {
  libra::TableParams p;
  const int rc = common(h, new_tokens, seq_lens, block_table, batch, free_pages, free_count, error_word_dev, &p);
  if (rc != LIBRA_OK) return rc;
  if (!q_offsets || off(q_offsets, 4) || off(positions, 4) || off(slots, 4) || max_rows < 0) return LIBRA_INVALID_ARGUMENT;
  if (q_offsets == new_tokens || q_offsets == seq_lens) return LIBRA_INVALID_ARGUMENT;
  p.q_offsets = q_offsets;
  p.positions = positions;
  p.slots = slots;
  p.max_rows = max_rows;
  return launch_table(h, libra::cache_extend_kernel, p, max_rows, (3 * size_t(batch) + 1) * sizeof(int32_t), stream);
}

int libra_cache_trim(libra_handle_t h, const int32_t* keep_lens, int32_t* seq_lens, int32_t* block_table, int32_t batch,
                     int32_t* free_pages, int32_t* free_count, void* error_word_dev, void* stream) {
  libra::TableParams p;
  const int rc = common(h, keep_lens, seq_lens, block_table, batch, free_pages, free_count, error_word_dev, &p);
  if (rc != LIBRA_OK) return rc;
  if (batch == 0) return LIBRA_OK;
  const int64_t pages = std::min(int64_t(batch) * h->cfg.block_table_ld, h->cfg.num_pages);
  return launch_table(h, libra::cache_trim_kernel, p, (pages + 15) / 16, 2 * size_t(batch) * sizeof(int32_t), stream);
}

}  // extern "C"
