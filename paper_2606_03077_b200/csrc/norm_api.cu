// Entry points of the norms of q and k with rotation.  See include/libra.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "handle.hpp"
#include "launch.hpp"
#include "libra.h"
#include "norm_kernel.cuh"

namespace {

using libra::DeviceGuard;
using libra::fail_cuda;
using libra::NormKind;
using libra::NormParams;

constexpr int kMaxHeads = 16384;
constexpr int kMaxDim = 1024;
constexpr int kMostBlocks = 8;       // a multiprocessor, of the gradient's sums: sizes its workspace

bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

bool valid_rope(const libra_rope_t* r) {   // a struct that libra_rope_init filled
  return r->rotary_dim >= 2 && r->rotary_dim % 2 == 0 && r->rotary_dim <= 2 * LIBRA_ROPE_MAX_PAIRS &&
         (r->layout == LIBRA_ROPE_HALF || r->layout == LIBRA_ROPE_INTERLEAVED);
}

// Rows of an output that do not overlap one another: all heads of a token before the next token, or all tokens of a head before
// the next head.
bool rows_apart(int64_t n_tokens, int32_t n_heads, int32_t head_dim, int64_t token, int64_t head) {
  if ((n_tokens > 1 && token < head_dim) || (n_heads > 1 && head < head_dim)) return false;
  if (n_tokens > 1 && n_heads > 1) {
    const __int128 heads_span = __int128(n_heads - 1) * head + head_dim, tokens_span = __int128(n_tokens - 1) * token + head_dim;
    if (token < heads_span && head < tokens_span) return false;
  }
  return true;
}

bool wide_rows(const void* p, int64_t token, int64_t head, int v) { return aligned(p, 16) && token % v == 0 && head % v == 0; }

// How a row is held by a group of lanes: the elements of a vector (0: the row goes through shared memory).  v: those of 16 bytes.
// Vectors of 8 bytes where R / 2 is an odd multiple of four 16-bit elements: 8192 tokens of 16 + 4 heads of 80, 40 of them turned, 27 us and
// 38 for the gradient, against 165 and 204 through shared memory.  Vectors of 16 where both would do: half the instructions a byte.
int lay_out(NormParams* p, bool wide, int v) {
  const int R = p->rope.rotary_dim, D = p->head_dim;
  const bool half = p->rope.layout == LIBRA_ROPE_HALF;
  if (!wide) return 0;
  if (v == 8 && half && R % 16 == 8) v = 4;   // 8 bytes: R / 2 is an odd multiple of four elements
  if (D % v != 0 || R % (half ? 2 * v : v) != 0) return 0;
  p->items = half ? R / (2 * v) + ((D - R) / v + 1) / 2 : (D / v + 1) / 2;
  if (p->items > 32) return 0;
  for (p->lanes_shift = 0; 1 << p->lanes_shift < p->items; ++p->lanes_shift) {}
  return v;
}

// Steps of every kind and of a token: the rows that a warp holds at once, or one
void count_steps(NormParams* p, bool by_lanes) {
  const int rows = by_lanes ? 32 >> p->lanes_shift : 1;
  p->steps = 0;
  for (NormKind& k : p->kind) p->steps += k.steps = (k.n_heads + rows - 1) / rows;
}

unsigned blocks_for(int64_t steps, int warps, int64_t most) {
  return unsigned(std::max<int64_t>(1, std::min<int64_t>((steps + warps - 1) / warps, most)));
}

typedef void (*NormFn)(NormParams);

// v: the elements of a vector where a group of lanes holds a row, else 0
template <typename T, int V>
NormFn apply_fn(int v, bool wide, bool half) {
  if constexpr (V == 8) {
    if (v == 4) return libra::norm_rope_kernel<T, T, 4, true, false>;
  }
  if (v) return half ? libra::norm_rope_kernel<T, T, V, true, false> : libra::norm_rope_kernel<T, T, V, false, false>;
  if (wide) return half ? libra::norm_rope_any_kernel<T, T, V, true, true, false> : libra::norm_rope_any_kernel<T, T, V, true, false, false>;
  return half ? libra::norm_rope_any_kernel<T, T, 1, false, true, false> : libra::norm_rope_any_kernel<T, T, 1, false, false, false>;
}
template <typename T, int V>
NormFn gradient_fn(int v, bool wide, bool half) {
  if constexpr (V == 8) {
    if (v == 4) return libra::norm_rope_gradient_kernel<T, 4, true>;
  }
  if (v) return half ? libra::norm_rope_gradient_kernel<T, V, true> : libra::norm_rope_gradient_kernel<T, V, false>;
  if (wide) return half ? libra::norm_rope_gradient_any_kernel<T, V, true, true> : libra::norm_rope_gradient_any_kernel<T, V, true, false>;
  return half ? libra::norm_rope_gradient_any_kernel<T, 1, false, true> : libra::norm_rope_gradient_any_kernel<T, 1, false, false>;
}
template <typename P>
NormFn append_fn(int v, bool half) {   // the handle's strides and addresses are multiples of 16 bytes
  typedef __nv_bfloat16 T;
  if (v == 4) return libra::norm_rope_kernel<T, P, 4, true, true>;
  if (v) return half ? libra::norm_rope_kernel<T, P, 8, true, true> : libra::norm_rope_kernel<T, P, 8, false, true>;
  return half ? libra::norm_rope_any_kernel<T, P, 8, true, true, true> : libra::norm_rope_any_kernel<T, P, 8, true, false, true>;
}

int check_call(int32_t device, const libra_rope_t* rope, int32_t dtype, const int32_t* positions, int64_t n_tokens, int32_t head_dim,
               float eps) {
  if (device < 0 || n_tokens < 0 || head_dim <= 0 || dtype < LIBRA_ROPE_BF16 || dtype > LIBRA_ROPE_F32) return LIBRA_INVALID_ARGUMENT;
  if (rope && (!valid_rope(rope) || (!positions && n_tokens > 0))) return LIBRA_INVALID_ARGUMENT;
  if (!aligned(positions, 4) || !std::isnormal(eps) || eps < 0.f) return LIBRA_INVALID_ARGUMENT;
  if (head_dim % 2 != 0 || head_dim > kMaxDim || (rope && rope->rotary_dim > head_dim) || n_tokens > 0x7fffffff) return LIBRA_UNSUPPORTED_SHAPE;
  return LIBRA_OK;
}

int sm_count(int device, int* n) {
  const cudaError_t e = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, device);
  return e == cudaSuccess ? LIBRA_OK : fail_cuda(nullptr, e);
}

void set_common(NormParams* p, const libra_rope_t* rope, const int32_t* positions, int64_t n_tokens, int32_t head_dim, float eps) {
  p->positions = positions;
  p->n_tokens = n_tokens;
  p->head_dim = head_dim;
  p->eps = eps;
  p->inv_dim = 1.f / float(head_dim);
  if (rope) p->rope = *rope;   // else rotary_dim 0: nothing turns
}

}  // namespace

extern "C" {

int libra_norm_rope_apply(int32_t device, const libra_rope_t* rope, const libra_norm_rows_t* q, const libra_norm_rows_t* k,
                          int32_t dtype, const int32_t* positions, int64_t n_tokens, int32_t head_dim, float eps, void* stream) {
  if (!q) return LIBRA_INVALID_ARGUMENT;
  const int rc = check_call(device, rope, dtype, positions, n_tokens, head_dim, eps);
  if (rc != LIBRA_OK) return rc;
  const int eb = dtype == LIBRA_ROPE_F32 ? 4 : 2, v = 16 / eb;
  NormParams p = {};
  bool wide = true;
  for (int i = 0; i < 2; ++i) {
    const libra_norm_rows_t* t = i ? k : q;
    if (!t) continue;
    if (!t->weight || t->n_heads <= 0 || (n_tokens > 0 && (!t->x || !t->out))) return LIBRA_INVALID_ARGUMENT;
    if (t->x_stride_token < 0 || t->x_stride_head < 0 || t->out_stride_token < 0 || t->out_stride_head < 0) return LIBRA_INVALID_ARGUMENT;
    if (!aligned(t->x, eb) || !aligned(t->out, eb) || !aligned(t->weight, eb)) return LIBRA_INVALID_ARGUMENT;
    if (!rows_apart(n_tokens, t->n_heads, head_dim, t->out_stride_token, t->out_stride_head)) return LIBRA_INVALID_ARGUMENT;
    if (t->x && t->x == t->out && (t->x_stride_token != t->out_stride_token || t->x_stride_head != t->out_stride_head)) return LIBRA_INVALID_ARGUMENT;
    if (t->n_heads > kMaxHeads) return LIBRA_UNSUPPORTED_SHAPE;
    NormKind& kind = p.kind[i];
    kind.x = t->x;
    kind.out = t->out;
    kind.weight = t->weight;
    kind.x_token = t->x_stride_token;
    kind.x_head = t->x_stride_head;
    kind.out_token = t->out_stride_token;
    kind.out_head = t->out_stride_head;
    kind.n_heads = t->n_heads;
    wide = wide && wide_rows(t->x, t->x_stride_token, t->x_stride_head, v) && wide_rows(t->out, t->out_stride_token, t->out_stride_head, v) &&
           aligned(t->weight, 16);
  }
  if (n_tokens == 0) return LIBRA_OK;
  if (k && k->out == q->out) return LIBRA_INVALID_ARGUMENT;
  DeviceGuard guard(device);
  if (guard.err != cudaSuccess) return fail_cuda(nullptr, guard.err);
  int n_sm = 0;
  if (sm_count(device, &n_sm) != LIBRA_OK) return LIBRA_CUDA_ERROR;
  set_common(&p, rope, positions, n_tokens, head_dim, eps);
  wide = wide && head_dim % v == 0;
  const int vec = lay_out(&p, wide, v);
  const bool by_lanes = vec != 0, half = p.rope.layout == LIBRA_ROPE_HALF;
  count_steps(&p, by_lanes);
  const NormFn fn = dtype == LIBRA_ROPE_BF16  ? apply_fn<__nv_bfloat16, 8>(vec, wide, half)
                    : dtype == LIBRA_ROPE_F16 ? apply_fn<__half, 8>(vec, wide, half)
                                              : apply_fn<float, 4>(vec, wide, half);
  const int warps = by_lanes ? libra::kNormWarps : libra::kNormAnyWarps;
  const unsigned grid = blocks_for(n_tokens * p.steps, warps, int64_t(n_sm) * (by_lanes ? libra::kNormBlocks : 16));
  const size_t smem = by_lanes ? 0 : size_t(warps) * head_dim * sizeof(float);
  const cudaError_t e = libra::launch(true, 1, fn, dim3(grid), unsigned(warps * 32), smem, static_cast<cudaStream_t>(stream), p);
  return e == cudaSuccess ? LIBRA_OK : fail_cuda(nullptr, e);
}

int libra_norm_rope_workspace_size(int32_t device, int32_t head_dim, size_t* bytes) {
  if (device < 0 || head_dim <= 0 || !bytes) return LIBRA_INVALID_ARGUMENT;
  if (head_dim % 2 != 0 || head_dim > kMaxDim) return LIBRA_UNSUPPORTED_SHAPE;
  int n_sm = 0;
  if (sm_count(device, &n_sm) != LIBRA_OK) return LIBRA_CUDA_ERROR;
  *bytes = size_t(n_sm) * kMostBlocks * 2 * head_dim * sizeof(float);
  return LIBRA_OK;
}

int libra_norm_rope_gradient(int32_t device, const libra_rope_t* rope, const libra_norm_grads_t* q, const libra_norm_grads_t* k,
                             int32_t dtype, const int32_t* positions, int64_t n_tokens, int32_t head_dim, float eps,
                             void* workspace_dev, size_t workspace_bytes, void* stream) {
  if (!q || !workspace_dev || !aligned(workspace_dev, 16)) return LIBRA_INVALID_ARGUMENT;
  const int rc = check_call(device, rope, dtype, positions, n_tokens, head_dim, eps);
  if (rc != LIBRA_OK) return rc;
  const int eb = dtype == LIBRA_ROPE_F32 ? 4 : 2, v = 16 / eb;
  NormParams p = {};
  libra::NormSumParams s = {};
  bool wide = true;
  for (int i = 0; i < 2; ++i) {
    const libra_norm_grads_t* t = i ? k : q;
    if (!t) continue;
    if (!t->weight || !t->grad_weight || t->n_heads <= 0) return LIBRA_INVALID_ARGUMENT;
    if (n_tokens > 0 && (!t->x || !t->grad_out || !t->grad_x)) return LIBRA_INVALID_ARGUMENT;   // no row is read without tokens
    if (t->x_stride_token < 0 || t->x_stride_head < 0 || t->grad_out_stride_token < 0 || t->grad_out_stride_head < 0 ||
        t->grad_x_stride_token < 0 || t->grad_x_stride_head < 0) {
      return LIBRA_INVALID_ARGUMENT;
    }
    if (!aligned(t->x, eb) || !aligned(t->grad_out, eb) || !aligned(t->weight, eb) || !aligned(t->grad_x, eb) || !aligned(t->grad_weight, 4)) {
      return LIBRA_INVALID_ARGUMENT;
    }
    if (!rows_apart(n_tokens, t->n_heads, head_dim, t->grad_x_stride_token, t->grad_x_stride_head)) return LIBRA_INVALID_ARGUMENT;
    if (t->x && t->grad_x == t->x && (t->x_stride_token != t->grad_x_stride_token || t->x_stride_head != t->grad_x_stride_head)) return LIBRA_INVALID_ARGUMENT;
    if (t->grad_x && t->grad_x == t->grad_out &&
        (t->grad_out_stride_token != t->grad_x_stride_token || t->grad_out_stride_head != t->grad_x_stride_head)) {
      return LIBRA_INVALID_ARGUMENT;
    }
    if (t->n_heads > kMaxHeads) return LIBRA_UNSUPPORTED_SHAPE;
    NormKind& kind = p.kind[i];
    kind.x = t->x;
    kind.grad = t->grad_out;
    kind.out = t->grad_x;
    kind.weight = t->weight;
    kind.x_token = t->x_stride_token;
    kind.x_head = t->x_stride_head;
    kind.grad_token = t->grad_out_stride_token;
    kind.grad_head = t->grad_out_stride_head;
    kind.out_token = t->grad_x_stride_token;
    kind.out_head = t->grad_x_stride_head;
    kind.n_heads = t->n_heads;
    s.out[i] = t->grad_weight;
    wide = wide && wide_rows(t->x, t->x_stride_token, t->x_stride_head, v) &&
           wide_rows(t->grad_out, t->grad_out_stride_token, t->grad_out_stride_head, v) &&
           wide_rows(t->grad_x, t->grad_x_stride_token, t->grad_x_stride_head, v) && aligned(t->weight, 16);
  }
  if (k && (k->grad_weight == q->grad_weight || (n_tokens > 0 && k->grad_x == q->grad_x))) return LIBRA_INVALID_ARGUMENT;   // neither adds to the other
  DeviceGuard guard(device);
  if (guard.err != cudaSuccess) return fail_cuda(nullptr, guard.err);
  int n_sm = 0;
  if (sm_count(device, &n_sm) != LIBRA_OK) return LIBRA_CUDA_ERROR;
  if (workspace_bytes < size_t(n_sm) * kMostBlocks * 2 * head_dim * sizeof(float)) return LIBRA_WORKSPACE_TOO_SMALL;
  set_common(&p, rope, positions, n_tokens, head_dim, eps);
  p.partial = static_cast<float*>(workspace_dev);
  wide = wide && head_dim % v == 0;
  const int vec = lay_out(&p, wide, v);
  const bool by_lanes = vec != 0, half = p.rope.layout == LIBRA_ROPE_HALF;
  count_steps(&p, by_lanes);
  const int warps = !by_lanes ? libra::kNormAnyWarps
                              : (dtype == LIBRA_ROPE_F32 ? libra::kNormGradThreads<float> : libra::kNormGradThreads<__half>) / 32;
  const unsigned blocks = blocks_for(n_tokens * p.steps, warps, int64_t(n_sm) * (by_lanes ? 1 : kMostBlocks));
  const NormFn fn = dtype == LIBRA_ROPE_BF16  ? gradient_fn<__nv_bfloat16, 8>(vec, wide, half)
                    : dtype == LIBRA_ROPE_F16 ? gradient_fn<__half, 8>(vec, wide, half)
                                              : gradient_fn<float, 4>(vec, wide, half);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int kinds = k ? 2 : 1;
  // a warp's: the ring, which also holds the sums of both kinds at the end, or rows of float32 (x, the gradient, each kind's sums)
  constexpr size_t ring = libra::kNormGradAhead * libra::kNormGradStepBytes, row = kMaxDim * sizeof(float);
  static_assert(2 * 32 * 16 * sizeof(float) <= ring, "the sums of two kinds: rows of 32 items of two vectors of eight channels at most");
  const size_t smem = size_t(warps) * (by_lanes ? ring : (2 + kinds) * size_t(head_dim) * sizeof(float));
  if (smem > 40 * 1024) {   // beside the static part
    // not this call's bytes but the most of the kernel: the limit is the process's, and a call on another thread must not find it below its own
    const size_t most = size_t(warps) * (by_lanes ? ring : 4 * row);
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(fn), cudaFuncAttributeMaxDynamicSharedMemorySize, int(most));
    if (e != cudaSuccess) return fail_cuda(nullptr, e);
  }
  cudaError_t e = libra::launch(true, 1, fn, dim3(blocks), unsigned(warps * 32), smem, st, p);
  if (e != cudaSuccess) return fail_cuda(nullptr, e);
  s.partial = p.partial;
  s.head_dim = head_dim;
  s.channels = kinds * head_dim;
  s.blocks = int32_t(blocks);
  e = libra::launch(true, 1, libra::norm_sum_kernel, dim3(unsigned(s.channels + 31) / 32), 32 * libra::kNormSumSlices, 0, st, s);
  return e == cudaSuccess ? LIBRA_OK : fail_cuda(nullptr, e);
}

int libra_norm_rope_append(libra_handle_t h, const libra_rope_t* rope, const void* q_weight, const void* k_weight, float eps,
                           const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k_new, const void* v_new,
                           int64_t kv_stride, const int32_t* positions, const int32_t* slots, const int32_t* n_rows, int32_t max_rows,
                           void* k_pages, void* v_pages, void* error_word_dev, void* stream) {
  if (!h || !k_pages || !v_pages || !error_word_dev || max_rows < 0) return LIBRA_INVALID_ARGUMENT;
  if (max_rows > 0 && (!k_new || !v_new || !slots || (rope && !positions))) return LIBRA_INVALID_ARGUMENT;   // no row is read where there is none
  if ((max_rows > 0 && (q == nullptr) != (q_out == nullptr)) || (rope && !valid_rope(rope))) return LIBRA_INVALID_ARGUMENT;
  if (!std::isnormal(eps) || eps < 0.f) return LIBRA_INVALID_ARGUMENT;
  const int D = h->cfg.head_dim;
  const int64_t q_row = int64_t(h->cfg.num_q_heads) * D, kv_row = int64_t(h->cfg.num_kv_heads) * D;
  if (kv_stride < kv_row || kv_stride % 8) return LIBRA_INVALID_ARGUMENT;
  if (q && (q_stride < q_row || q_stride % 8 || q_out_stride < q_row || q_out_stride % 8)) return LIBRA_INVALID_ARGUMENT;
  if (q && q == q_out && q_stride != q_out_stride) return LIBRA_INVALID_ARGUMENT;
  if (!aligned(q, 16) || !aligned(q_out, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(k_pages, 16) ||
      !aligned(v_pages, 16) || !aligned(q_weight, 16) || !aligned(k_weight, 16) || !aligned(positions, 4) || !aligned(slots, 4) ||
      !aligned(n_rows, 4) || !aligned(error_word_dev, 4)) {
    return LIBRA_INVALID_ARGUMENT;
  }
  // the kernel flushes what is not normal to zero
  if (h->fp8 && (!std::isnormal(1.f / h->k_scale) || !std::isnormal(1.f / h->v_scale))) return LIBRA_INVALID_ARGUMENT;
  if (rope && rope->rotary_dim > D) return LIBRA_UNSUPPORTED_SHAPE;
  if (h->cfg.num_pages > 0x7fffffff / h->cfg.page_size) return LIBRA_UNSUPPORTED_SHAPE;   // a slot's number
  if (h->cfg.num_q_heads > kMaxHeads || h->cfg.num_kv_heads > kMaxHeads) return LIBRA_UNSUPPORTED_SHAPE;
  if (max_rows == 0) return LIBRA_OK;
  DeviceGuard guard(h->cfg.device);
  if (guard.err != cudaSuccess) return fail_cuda(h, guard.err);

  NormParams p = {};
  const void* x[3] = {q, k_new, v_new};
  void* out[3] = {q_out, k_pages, v_pages};
  const void* weight[3] = {q_weight, k_weight, nullptr};
  for (int i = 0; i < 3; ++i) {
    NormKind& kind = p.kind[i];
    kind.x = x[i];
    kind.out = out[i];
    kind.weight = weight[i];
    kind.x_token = i == 0 ? q_stride : kv_stride;
    kind.x_head = kind.out_head = D;
    kind.out_token = q_out_stride;
    kind.n_heads = i == 0 ? (q ? h->cfg.num_q_heads : 0) : h->cfg.num_kv_heads;
  }
  set_common(&p, rope, positions, max_rows, D, eps);
  p.slots = slots;
  p.n_rows = n_rows;
  p.error_word = static_cast<uint32_t*>(error_word_dev);
  p.num_slots = h->cfg.num_pages * h->cfg.page_size;
  p.stride_page = h->stride_page;
  p.stride_head = h->stride_head;
  p.stride_token = h->stride_token;
  p.k_inv_scale = 1.f / h->k_scale;
  p.v_inv_scale = 1.f / h->v_scale;
  p.page_shift = h->cfg.page_size == 16 ? 4 : (h->cfg.page_size == 32 ? 5 : 6);
  const int vec = lay_out(&p, true, 8);
  const bool by_lanes = vec != 0, half = p.rope.layout == LIBRA_ROPE_HALF;
  count_steps(&p, by_lanes);
  const NormFn fn = h->fp8 ? append_fn<uint8_t>(vec, half) : append_fn<__nv_bfloat16>(vec, half);
  const int warps = by_lanes ? libra::kNormWarps : libra::kNormAnyWarps;
  const unsigned grid = blocks_for(int64_t(max_rows) * p.steps, warps, int64_t(h->n_sm_dev) * (by_lanes ? libra::kNormBlocks : 16));
  LIBRA_CUDA_TRY(h, libra::launch(h->pdl, 1, fn, dim3(grid), unsigned(warps * 32), by_lanes ? 0 : size_t(warps) * D * sizeof(float),
                                  static_cast<cudaStream_t>(stream), p));
  ++h->launches;
  return LIBRA_OK;
}

}  // extern "C"
