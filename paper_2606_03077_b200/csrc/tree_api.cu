// Entry points for trees of drafted tokens, but the attention (chunk_api.cu).  See include/libra.h.
#include <cuda_runtime.h>

#include <cstdint>

#include "handle.hpp"
#include "launch.hpp"
#include "libra.h"
#include "tree_kernel.cuh"

namespace {

using libra::DeviceGuard;
using libra::fail_cuda;

bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

}  // namespace

extern "C" {

int libra_tree_mask(libra_handle_t h, const int32_t* parents, const int32_t* q_offsets, const int32_t* seq_lens, int32_t batch,
                    int32_t max_rows, uint32_t* mask, int32_t mask_ld, int32_t* positions, void* error_word_dev, void* stream) {
  if (!h || !q_offsets || !error_word_dev) return LIBRA_INVALID_ARGUMENT;
  if (batch < 0 || batch > h->cfg.max_batch || max_rows < 0 || mask_ld <= 0) return LIBRA_INVALID_ARGUMENT;
  if ((batch > 0 && !seq_lens) || (max_rows > 0 && (!parents || !mask))) return LIBRA_INVALID_ARGUMENT;
  if (off(parents, 4) || off(q_offsets, 4) || off(seq_lens, 4) || off(mask, 4) || off(positions, 4) || off(error_word_dev, 4)) {
    return LIBRA_INVALID_ARGUMENT;
  }
  if (mask_ld > LIBRA_TREE_MAX_TOKENS / 32) return LIBRA_UNSUPPORTED_SHAPE;
  if (batch == 0 || max_rows == 0) return LIBRA_OK;
  DeviceGuard guard(h->cfg.device);
  if (guard.err != cudaSuccess) return fail_cuda(h, guard.err);
  libra::TreeMaskParams p;
  p.parents = parents;
  p.q_offsets = q_offsets;
  p.seq_lens = seq_lens;
  p.mask = mask;
  p.positions = positions;
  p.error_word = static_cast<uint32_t*>(error_word_dev);
  p.max_rows = max_rows;
  p.mask_ld = mask_ld;
  LIBRA_CUDA_TRY(h, libra::launch(h->pdl, 1, libra::tree_mask_kernel, dim3(unsigned(batch), unsigned(mask_ld)), libra::kTreeMaskThreads,
                                  size_t(mask_ld) * 32 * sizeof(int32_t), static_cast<cudaStream_t>(stream), p));
  ++h->launches;
  return LIBRA_OK;
}

int libra_tree_keep(libra_handle_t h, const int32_t* kept, int32_t kept_ld, const int32_t* n_kept, const int32_t* q_offsets,
                    const int32_t* seq_lens, const int32_t* block_table, int32_t batch, void* k_pages, void* v_pages,
                    int32_t* new_lens, void* error_word_dev, void* stream) {
  if (!h || !q_offsets || !k_pages || !v_pages || !error_word_dev) return LIBRA_INVALID_ARGUMENT;
  if (batch < 0 || batch > h->cfg.max_batch || kept_ld <= 0) return LIBRA_INVALID_ARGUMENT;
  if (batch > 0 && (!kept || !n_kept || !seq_lens || !block_table)) return LIBRA_INVALID_ARGUMENT;
  if (off(kept, 4) || off(n_kept, 4) || off(q_offsets, 4) || off(seq_lens, 4) || off(block_table, 4) || off(k_pages, 16) ||
      off(v_pages, 16) || off(new_lens, 4) || off(error_word_dev, 4)) {
    return LIBRA_INVALID_ARGUMENT;
  }
  if (batch > 0 && new_lens == seq_lens) return LIBRA_INVALID_ARGUMENT;   // other blocks of the sequence may not have read its length yet
  if (batch == 0) return LIBRA_OK;
  DeviceGuard guard(h->cfg.device);
  if (guard.err != cudaSuccess) return fail_cuda(h, guard.err);
  const int eb = h->fp8 ? 1 : 2;
  libra::TreeKeepParams p;
  p.kept = kept;
  p.n_kept = n_kept;
  p.q_offsets = q_offsets;
  p.seq_lens = seq_lens;
  p.block_table = block_table;
  p.k_pool = static_cast<uint8_t*>(k_pages);
  p.v_pool = static_cast<uint8_t*>(v_pages);
  p.new_lens = new_lens;
  p.error_word = static_cast<uint32_t*>(error_word_dev);
  p.stride_page = h->stride_page * eb;
  p.stride_head = h->stride_head * eb;
  p.stride_token = h->stride_token * eb;
  p.num_pages = h->cfg.num_pages;
  p.kept_ld = kept_ld;
  p.block_table_ld = h->cfg.block_table_ld;
  p.page_shift = h->cfg.page_size == 16 ? 4 : (h->cfg.page_size == 32 ? 5 : 6);
  p.num_kv_heads = h->cfg.num_kv_heads;
  p.vectors = h->cfg.head_dim * eb / 16;
  const int64_t columns = int64_t(2) * p.num_kv_heads * p.vectors;
  const int64_t blocks = (columns + libra::kTreeKeepThreads - 1) / libra::kTreeKeepThreads;
  if (blocks > 65535) return LIBRA_UNSUPPORTED_SHAPE;   // grid
  LIBRA_CUDA_TRY(h, libra::launch(h->pdl, 1, libra::tree_keep_kernel, dim3(unsigned(batch), unsigned(blocks)), libra::kTreeKeepThreads, 0,
                                  static_cast<cudaStream_t>(stream), p));
  ++h->launches;
  return LIBRA_OK;
}

}  // extern "C"
