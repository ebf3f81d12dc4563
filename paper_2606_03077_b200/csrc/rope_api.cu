// Entry points of the rotary positions and of the append with rotation.  See include/libra.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "handle.hpp"
#include "libra.h"
#include "rope_kernel.cuh"

namespace {

using libra::DeviceGuard;
using libra::fail_cuda;

bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

bool valid_rope(const libra_rope_t* r) {   // a struct that libra_rope_init filled
  return r->rotary_dim >= 2 && r->rotary_dim % 2 == 0 && r->rotary_dim <= 2 * LIBRA_ROPE_MAX_PAIRS &&
         (r->layout == LIBRA_ROPE_HALF || r->layout == LIBRA_ROPE_INTERLEAVED);
}

constexpr int kMaxHeads = 16384;   // a block's rows are divided by the heads with one 32-bit multiplication

uint32_t inverse(int heads) { return uint32_t(((uint64_t(1) << 32) + heads - 1) / heads); }

// Tokens per block: as many as share the block's threads in the sine and cosine pass (one evaluation per thread), fewer
// when that would leave multiprocessors without a block.
int tokens_per_block(int64_t tokens, int pairs, int n_sm) {
  int64_t t = pairs > 0 ? libra::kRopeThreads / pairs : libra::kRopeMaxTokens;
  t = std::min<int64_t>(t, tokens / (4 * int64_t(n_sm)));
  return int(std::max<int64_t>(1, std::min<int64_t>(t, libra::kRopeMaxTokens)));
}

template <typename T, int kWide>
cudaError_t launch_apply(const libra::RopeApplyParams& p, bool wide, unsigned grid, size_t smem, cudaStream_t st) {
  const bool half = p.rope.layout == LIBRA_ROPE_HALF;
  void (*fn)(libra::RopeApplyParams) =
      wide ? (half ? libra::rope_apply_kernel<T, kWide, true, true> : libra::rope_apply_kernel<T, kWide, true, false>)
           : (half ? libra::rope_apply_kernel<T, 1, false, true> : libra::rope_apply_kernel<T, 2, false, false>);
  fn<<<grid, libra::kRopeThreads, smem, st>>>(p);
  return cudaGetLastError();
}

}  // namespace

extern "C" {

int libra_rope_apply(int32_t device, const libra_rope_t* rope, const void* x, void* out, int32_t dtype,
                     const int32_t* positions, int64_t n_tokens, int32_t n_heads, int32_t head_dim,
                     int64_t x_stride_token, int64_t x_stride_head, int64_t out_stride_token, int64_t out_stride_head,
                     int32_t direction, void* stream) {
  if (device < 0 || !rope || !x || !out || !positions || n_tokens < 0 || n_heads <= 0 || head_dim <= 0) {
    return LIBRA_INVALID_ARGUMENT;
  }
  if (!valid_rope(rope) || dtype < LIBRA_ROPE_BF16 || dtype > LIBRA_ROPE_F32) return LIBRA_INVALID_ARGUMENT;
  if (direction != LIBRA_ROPE_FORWARD && direction != LIBRA_ROPE_GRADIENT) return LIBRA_INVALID_ARGUMENT;
  if (x_stride_token < 0 || x_stride_head < 0 || out_stride_token < 0 || out_stride_head < 0) return LIBRA_INVALID_ARGUMENT;
  // rows of the output must not overlap one another: all heads of a token before the next token, or all tokens of a head before
  // the next head
  if ((n_tokens > 1 && out_stride_token < head_dim) || (n_heads > 1 && out_stride_head < head_dim)) return LIBRA_INVALID_ARGUMENT;
  if (n_tokens > 1 && n_heads > 1) {
    const __int128 heads_span = __int128(n_heads - 1) * out_stride_head + head_dim;
    const __int128 tokens_span = __int128(n_tokens - 1) * out_stride_token + head_dim;
    if (out_stride_token < heads_span && out_stride_head < tokens_span) return LIBRA_INVALID_ARGUMENT;
  }
  if (x == out && (x_stride_token != out_stride_token || x_stride_head != out_stride_head)) return LIBRA_INVALID_ARGUMENT;
  if (head_dim % 2 != 0 || head_dim > 1024 || rope->rotary_dim > head_dim) return LIBRA_UNSUPPORTED_SHAPE;
  if (n_heads > kMaxHeads || n_tokens > 0x7fffffff) return LIBRA_UNSUPPORTED_SHAPE;
  const int eb = dtype == LIBRA_ROPE_F32 ? 4 : 2;
  if (!aligned(x, eb) || !aligned(out, eb) || !aligned(positions, 4)) return LIBRA_INVALID_ARGUMENT;
  if (n_tokens == 0) return LIBRA_OK;
  DeviceGuard guard(device);
  if (guard.err != cudaSuccess) return fail_cuda(nullptr, guard.err);
  int n_sm = 0;
  const cudaError_t e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, device);
  if (e != cudaSuccess) return fail_cuda(nullptr, e);

  libra::RopeApplyParams p;
  p.x = x;
  p.out = out;
  p.positions = positions;
  p.x_stride_token = x_stride_token;
  p.x_stride_head = x_stride_head;
  p.out_stride_token = out_stride_token;
  p.out_stride_head = out_stride_head;
  p.n_tokens = n_tokens;
  p.n_heads = n_heads;
  p.head_dim = head_dim;
  p.heads_inverse = inverse(n_heads);
  p.gradient = direction == LIBRA_ROPE_GRADIENT;
  p.rope = *rope;
  const int pairs = rope->rotary_dim / 2;
  p.tokens_per_block = tokens_per_block(n_tokens, pairs, n_sm);
  const unsigned grid = unsigned((n_tokens + p.tokens_per_block - 1) / p.tokens_per_block);
  const size_t smem = size_t(p.tokens_per_block) * pairs * sizeof(float2);
  // 16-byte vectors where every row, the rotated part (each half of it, in the half layout) and what passes through start
  // and end on one
  const int v = 16 / eb, part = rope->layout == LIBRA_ROPE_HALF ? pairs : rope->rotary_dim;
  const bool wide = aligned(x, 16) && aligned(out, 16) && part % v == 0 && head_dim % v == 0 && x_stride_token % v == 0 &&
                    x_stride_head % v == 0 && out_stride_token % v == 0 && out_stride_head % v == 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t r;
  if (dtype == LIBRA_ROPE_BF16) r = launch_apply<__nv_bfloat16, 8>(p, wide, grid, smem, st);
  else if (dtype == LIBRA_ROPE_F16) r = launch_apply<__half, 8>(p, wide, grid, smem, st);
  else r = launch_apply<float, 4>(p, wide, grid, smem, st);
  return r == cudaSuccess ? LIBRA_OK : fail_cuda(nullptr, r);
}

int libra_rope_append(libra_handle_t h, const libra_rope_t* rope, const void* q, int64_t q_stride, void* q_out,
                      int64_t q_out_stride, const void* k_new, const void* v_new, int64_t kv_stride,
                      const int32_t* q_offsets, const int32_t* seq_lens, const int32_t* block_table, int32_t batch,
                      int32_t max_rows, void* k_pages, void* v_pages, void* error_word_dev, void* stream) {
  if (!h || !k_new || !v_new || !q_offsets || !seq_lens || !block_table || !k_pages || !v_pages || !error_word_dev) {
    return LIBRA_INVALID_ARGUMENT;
  }
  if ((q == nullptr) != (q_out == nullptr) || batch < 0 || batch > h->cfg.max_batch || max_rows < 0) return LIBRA_INVALID_ARGUMENT;
  if (rope && !valid_rope(rope)) return LIBRA_INVALID_ARGUMENT;
  const int D = h->cfg.head_dim;
  const int64_t q_row = int64_t(h->cfg.num_q_heads) * D, kv_row = int64_t(h->cfg.num_kv_heads) * D;
  if (kv_stride < kv_row || kv_stride % 8) return LIBRA_INVALID_ARGUMENT;
  if (q && (q_stride < q_row || q_stride % 8 || q_out_stride < q_row || q_out_stride % 8)) return LIBRA_INVALID_ARGUMENT;
  if (q && q == q_out && q_stride != q_out_stride) return LIBRA_INVALID_ARGUMENT;
  if (!aligned(q, 16) || !aligned(q_out, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(k_pages, 16) ||
      !aligned(v_pages, 16) || !aligned(q_offsets, 4) || !aligned(seq_lens, 4) || !aligned(block_table, 4) ||
      !aligned(error_word_dev, 4)) {
    return LIBRA_INVALID_ARGUMENT;
  }
  // the kernel flushes what is not normal to zero
  if (h->fp8 && (!std::isnormal(1.f / h->k_scale) || !std::isnormal(1.f / h->v_scale))) return LIBRA_INVALID_ARGUMENT;
  if (rope && rope->rotary_dim > D) return LIBRA_UNSUPPORTED_SHAPE;
  const int heads = (q ? h->cfg.num_q_heads : 0) + 2 * h->cfg.num_kv_heads;
  if (heads > kMaxHeads) return LIBRA_UNSUPPORTED_SHAPE;
  if (batch == 0 || max_rows == 0) return LIBRA_OK;
  DeviceGuard guard(h->cfg.device);
  if (guard.err != cudaSuccess) return fail_cuda(h, guard.err);

  libra::RopeAppendParams p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.k_new = static_cast<const __nv_bfloat16*>(k_new);
  p.v_new = static_cast<const __nv_bfloat16*>(v_new);
  p.q_stride = q_stride;
  p.q_out_stride = q_out_stride;
  p.kv_stride = kv_stride;
  p.q_offsets = q_offsets;
  p.seq_lens = seq_lens;
  p.block_table = block_table;
  p.k_pool = k_pages;
  p.v_pool = v_pages;
  p.error_word = static_cast<uint32_t*>(error_word_dev);
  p.stride_page = h->stride_page;
  p.stride_head = h->stride_head;
  p.stride_token = h->stride_token;
  p.num_pages = h->cfg.num_pages;
  p.k_inv_scale = 1.f / h->k_scale;
  p.v_inv_scale = 1.f / h->v_scale;
  p.batch = batch;
  p.max_tokens = max_rows;
  p.block_table_ld = h->cfg.block_table_ld;
  p.page_shift = h->cfg.page_size == 16 ? 4 : (h->cfg.page_size == 32 ? 5 : 6);
  p.num_q_heads = h->cfg.num_q_heads;
  p.num_kv_heads = h->cfg.num_kv_heads;
  p.head_dim = D;
  p.heads = heads;
  p.heads_inverse = inverse(heads);
  if (rope) p.rope = *rope;
  else p.rope = libra_rope_t{};   // rotary_dim 0: every channel passes through
  const int pairs = p.rope.rotary_dim / 2;
  p.tokens_per_block = tokens_per_block(max_rows, pairs, h->n_sm_dev);
  const unsigned grid = unsigned((int64_t(max_rows) + p.tokens_per_block - 1) / p.tokens_per_block);
  const size_t smem = size_t(p.tokens_per_block) * pairs * sizeof(float2);
  const bool half = p.rope.layout == LIBRA_ROPE_HALF;
  const bool wide = (half ? pairs : p.rope.rotary_dim) % 8 == 0;
  void (*fn)(libra::RopeAppendParams);
  if (h->fp8) {
    fn = wide ? (half ? libra::rope_append_kernel<uint8_t, 8, true, true> : libra::rope_append_kernel<uint8_t, 8, true, false>)
              : (half ? libra::rope_append_kernel<uint8_t, 1, false, true> : libra::rope_append_kernel<uint8_t, 2, false, false>);
  } else {
    fn = wide ? (half ? libra::rope_append_kernel<__nv_bfloat16, 8, true, true>
                      : libra::rope_append_kernel<__nv_bfloat16, 8, true, false>)
              : (half ? libra::rope_append_kernel<__nv_bfloat16, 1, false, true>
                      : libra::rope_append_kernel<__nv_bfloat16, 2, false, false>);
  }
  fn<<<grid, libra::kRopeThreads, smem, static_cast<cudaStream_t>(stream)>>>(p);
  LIBRA_CUDA_TRY(h, cudaGetLastError());
  ++h->launches;
  return LIBRA_OK;
}

}  // extern "C"
