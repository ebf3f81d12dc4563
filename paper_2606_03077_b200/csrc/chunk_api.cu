// Entry points of the chunk attention.  See include/libra.h.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "chunk_kernel.cuh"
#include "chunk_plan.hpp"
#include "handle.hpp"
#include "libra.h"

namespace {

using libra::DeviceGuard;
using libra::fail_cuda;

typedef void (*ChunkKernelFn)(const CUtensorMap, const CUtensorMap, const libra::ChunkParams);

struct ChunkBuild {
  ChunkKernelFn fn;
  int threads, smem;
  int registers;   // that the roles' setmaxnreg counts on
};
template <int D, bool kFp8>
ChunkBuild build_of() {
  using S = libra::ChunkShape<D, kFp8>;
  return {libra::chunk_kernel<D, kFp8>, S::kThreads, S::kDynamicBytes, S::kLaunchRegs};
}
const ChunkBuild kBuilds[2][2] = {{build_of<64, false>(), build_of<64, true>()}, {build_of<128, false>(), build_of<128, true>()}};

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
constexpr size_t kHeaderBytes = 256;   // the plan's serial number

// A number for every plan of the process, so that a launch can tell whether the workspace still holds its own.
uint32_t next_serial() {
  static std::atomic<uint32_t> counter{0};
  uint32_t n = ++counter;
  while (n == 0) n = ++counter;
  return n;
}

// As a programmatic dependent of its predecessor where the handle allows it; the kernels wait for that one inside.
template <typename... P, typename... A>
cudaError_t launch(bool dependent, void (*fn)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t lc = {};
  lc.gridDim = grid;
  lc.blockDim = dim3(threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = attr;
  lc.numAttrs = dependent ? 1 : 0;
  return cudaLaunchKernelEx(&lc, fn, args...);
}

int set_attributes(libra_handle_t h) {
  if (h->chunk.attributes_set) return LIBRA_OK;
  for (const auto& row : kBuilds) {
    for (const ChunkBuild& b : row) {
      cudaFuncAttributes a;
      LIBRA_CUDA_TRY(h, cudaFuncGetAttributes(&a, reinterpret_cast<const void*>(b.fn)));
      // setmaxnreg waits for registers that the launch did not bring: never start such a build
      if (int64_t(a.numRegs) * b.threads < b.registers) return fail_cuda(h, cudaErrorInvalidConfiguration);
      LIBRA_CUDA_TRY(h, cudaFuncSetAttribute(reinterpret_cast<const void*>(b.fn), cudaFuncAttributeMaxDynamicSharedMemorySize, b.smem));
    }
  }
  h->chunk.attributes_set = true;
  return LIBRA_OK;
}

}  // namespace

extern "C" {

int libra_chunk_plan_host(int32_t n_sm, int32_t num_q_heads, int32_t num_kv_heads, const int32_t* q_lens,
                          const int32_t* seq_lens, int32_t batch, int32_t* items, int32_t items_capacity,
                          int32_t* num_items, int32_t* merges, int32_t merges_capacity, int32_t* num_merges,
                          int64_t* partial_rows) {
  if (n_sm <= 0 || num_kv_heads <= 0 || num_q_heads <= 0 || num_q_heads % num_kv_heads != 0 || batch < 0) return LIBRA_INVALID_ARGUMENT;
  if ((batch > 0 && (!q_lens || !seq_lens)) || items_capacity < 0 || merges_capacity < 0) return LIBRA_INVALID_ARGUMENT;
  if (!num_items || !num_merges || !partial_rows || (items_capacity > 0 && !items) || (merges_capacity > 0 && !merges)) {
    return LIBRA_INVALID_ARGUMENT;
  }
  for (int32_t b = 0; b < batch; ++b) {
    if (q_lens[b] < 0 || seq_lens[b] < 0) return LIBRA_INVALID_ARGUMENT;
  }
  try {
    libra::ChunkPlan plan;
    if (!libra::make_chunk_plan(n_sm, num_q_heads, num_kv_heads, q_lens, seq_lens, batch, &plan)) return LIBRA_UNSUPPORTED_SHAPE;
    *num_items = int32_t(plan.items.size());
    *num_merges = int32_t(plan.merges.size());
    *partial_rows = plan.partial_rows;
    if (int64_t(plan.items.size()) > items_capacity || int64_t(plan.merges.size()) > merges_capacity) return LIBRA_WORKSPACE_TOO_SMALL;
    if (!plan.items.empty()) std::memcpy(items, plan.items.data(), plan.items.size() * sizeof(libra::ChunkItem));
    if (!plan.merges.empty()) std::memcpy(merges, plan.merges.data(), plan.merges.size() * sizeof(libra::ChunkMerge));
  } catch (...) {   // out of host memory
    return LIBRA_INVALID_ARGUMENT;
  }
  return LIBRA_OK;
}

int libra_chunk_workspace_size(libra_handle_t h, int64_t max_tokens, size_t* bytes) {
  if (!h || !bytes || max_tokens < 0) return LIBRA_INVALID_ARGUMENT;
  if (max_tokens > 0x7fffffff) return LIBRA_UNSUPPORTED_SHAPE;
  const int64_t items = libra::chunk_max_items(h->n_sm_dev, h->group, max_tokens, h->cfg.max_batch);
  // partial rows times KV heads: the planner's limit, or every row cut as often as one can be
  const int64_t rows = std::min(libra::chunk_max_partial_rows(h->n_sm_dev),
                                max_tokens * h->cfg.num_q_heads * libra::kChunkMaxSplits);
  size_t n = kHeaderBytes;
  n += align_up(size_t(items) * sizeof(libra::ChunkItem), 256);
  n += align_up(size_t(items) * sizeof(libra::ChunkMerge), 256);
  n += align_up(size_t(rows) * sizeof(float), 256);
  n += size_t(rows) * h->cfg.head_dim * sizeof(float);
  *bytes = align_up(n, 256);
  return LIBRA_OK;
}

int libra_chunk_plan(libra_handle_t h, const int32_t* q_lens_host, const int32_t* seq_lens_host, int32_t batch,
                     void* workspace_dev, size_t workspace_bytes, void* stream) {
  if (!h || batch < 0 || batch > h->cfg.max_batch || (batch > 0 && (!q_lens_host || !seq_lens_host)) || !workspace_dev) {
    return LIBRA_INVALID_ARGUMENT;
  }
  if (reinterpret_cast<uintptr_t>(workspace_dev) % 256 != 0) return LIBRA_INVALID_ARGUMENT;
  const int64_t max_len = int64_t(h->cfg.block_table_ld) * h->cfg.page_size;
  for (int32_t b = 0; b < batch; ++b) {
    if (q_lens_host[b] < 0 || seq_lens_host[b] < 0 || seq_lens_host[b] > max_len) return LIBRA_INVALID_ARGUMENT;
  }
  libra_handle_s::Chunk& c = h->chunk;
  libra::ChunkPlan plan;
  try {
    if (!libra::make_chunk_plan(h->n_sm_dev, h->cfg.num_q_heads, h->cfg.num_kv_heads, q_lens_host, seq_lens_host, batch, &plan)) {
      return LIBRA_UNSUPPORTED_SHAPE;
    }
  } catch (...) {   // out of host memory
    return LIBRA_INVALID_ARGUMENT;
  }
  const size_t items_bytes = plan.items.size() * sizeof(libra::ChunkItem);
  const size_t merges_bytes = plan.merges.size() * sizeof(libra::ChunkMerge);
  const size_t rows = size_t(plan.partial_rows) * h->cfg.num_kv_heads;
  const size_t merges_off = kHeaderBytes + align_up(items_bytes, 256);
  const size_t lse_off = merges_off + align_up(merges_bytes, 256);
  const size_t o_off = lse_off + align_up(rows * sizeof(float), 256);
  if (workspace_bytes < o_off + rows * h->cfg.head_dim * sizeof(float)) return LIBRA_WORKSPACE_TOO_SMALL;
  if (int64_t(plan.items.size()) > int64_t(65535) * 65535) return LIBRA_UNSUPPORTED_SHAPE;   // grid

  DeviceGuard guard(h->cfg.device);
  if (guard.err != cudaSuccess) return fail_cuda(h, guard.err);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  LIBRA_CUDA_TRY(h, cudaStreamIsCapturing(st, &capture));
  if (capture != cudaStreamCaptureStatusNone) return LIBRA_INVALID_ARGUMENT;
  const int rc = set_attributes(h);
  if (rc != LIBRA_OK) return rc;

  c.planned = false;
  // pinned staging: two buffers by turns, each reused once its copy is done, grown when it is too small
  const int k = c.next_staging;
  const size_t bytes = merges_off + merges_bytes;
  if (!c.staging_done[k]) LIBRA_CUDA_TRY(h, cudaEventCreateWithFlags(&c.staging_done[k], cudaEventDisableTiming));
  else LIBRA_CUDA_TRY(h, cudaEventSynchronize(c.staging_done[k]));
  if (c.staging_bytes[k] < bytes) {
    if (c.staging[k]) cudaFreeHost(c.staging[k]);
    c.staging[k] = nullptr;
    c.staging_bytes[k] = 0;
    const size_t want = align_up(bytes + bytes / 2, 4096);
    LIBRA_CUDA_TRY(h, cudaHostAlloc(&c.staging[k], want, cudaHostAllocDefault));
    c.staging_bytes[k] = want;
  }
  uint8_t* to = static_cast<uint8_t*>(c.staging[k]);
  const uint32_t serial = next_serial();
  std::memset(to, 0, kHeaderBytes);
  std::memcpy(to, &serial, sizeof(serial));
  if (items_bytes) std::memcpy(to + kHeaderBytes, plan.items.data(), items_bytes);
  if (merges_bytes) std::memcpy(to + merges_off, plan.merges.data(), merges_bytes);
  LIBRA_CUDA_TRY(h, cudaMemcpyAsync(workspace_dev, to, bytes, cudaMemcpyHostToDevice, st));
  LIBRA_CUDA_TRY(h, cudaEventRecord(c.staging_done[k], st));
  c.next_staging = k ^ 1;
  c.serial = serial;
  c.workspace = workspace_dev;
  c.n_items = int32_t(plan.items.size());
  c.n_merges = int32_t(plan.merges.size());
  c.merges_off = merges_off;
  c.lse_off = lse_off;
  c.o_off = o_off;
  c.planned = true;
  return LIBRA_OK;
}

int libra_chunk_attn(libra_handle_t h, const void* q, int64_t q_stride, const void* k_pages, const void* v_pages,
                     const int32_t* block_table, void* out, float* lse, void* error_word_dev, void* stream) {
  if (!h || !q || !k_pages || !v_pages || !block_table || !out || !error_word_dev) return LIBRA_INVALID_ARGUMENT;
  if (q_stride < int64_t(h->cfg.num_q_heads) * h->cfg.head_dim || q_stride % 8 != 0) return LIBRA_INVALID_ARGUMENT;
  auto off = [](const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; };
  if (off(q, 16) || off(k_pages, 16) || off(v_pages, 16) || off(out, 16) || off(block_table, 4) || off(lse, 4) || off(error_word_dev, 4)) {
    return LIBRA_INVALID_ARGUMENT;
  }
  // the kernels flush what is not normal to zero
  if (!std::isnormal(h->scale_log2 * h->k_scale) || !std::isnormal(h->v_scale)) return LIBRA_INVALID_ARGUMENT;
  libra_handle_s::Chunk& c = h->chunk;
  if (!c.planned) return LIBRA_NOT_PLANNED;
  if (c.n_items == 0) return LIBRA_OK;
  DeviceGuard guard(h->cfg.device);
  if (guard.err != cudaSuccess) return fail_cuda(h, guard.err);
  cudaStream_t st = static_cast<cudaStream_t>(stream);

  // whole pages: 64 channels with 128-byte swizzle as the tensor cores read them, or an 8-bit row as it is
  const int row_bytes = h->fp8 ? h->cfg.head_dim : 128;
  const CUtensorMapSwizzle swizzle = h->fp8 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B;
  CUtensorMap map_k, map_v;
  int pos_head = 0, pos_page = 0, pos_token = 0;
  int rc = libra::encode_pool_map(h, k_pages, row_bytes, h->cfg.page_size, swizzle, &map_k, &pos_head, &pos_page, &pos_token);
  if (rc == LIBRA_OK) {
    rc = libra::encode_pool_map(h, v_pages, row_bytes, h->cfg.page_size, swizzle, &map_v, &pos_head, &pos_page, &pos_token);
  }
  if (rc != LIBRA_OK) return rc;

  uint8_t* ws = static_cast<uint8_t*>(c.workspace);
  libra::ChunkParams p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.q_stride = q_stride;
  p.block_table = block_table;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.serial_at = reinterpret_cast<const uint32_t*>(ws);
  p.items = reinterpret_cast<const int4*>(ws + kHeaderBytes);
  p.partial_o = reinterpret_cast<float*>(ws + c.o_off);
  p.partial_lse = reinterpret_cast<float*>(ws + c.lse_off);
  p.error_word = static_cast<uint32_t*>(error_word_dev);
  p.num_pages = h->cfg.num_pages;
  p.serial = c.serial;
  p.num_items = c.n_items;
  p.num_q_heads = h->cfg.num_q_heads;
  p.num_kv_heads = h->cfg.num_kv_heads;
  p.group = h->group;
  p.group_inverse = uint32_t((65536 + h->group - 1) / h->group);
  p.block_table_ld = h->cfg.block_table_ld;
  p.page_shift = h->cfg.page_size == 16 ? 4 : (h->cfg.page_size == 32 ? 5 : 6);
  p.pos_head = pos_head;
  p.pos_page = pos_page;
  p.pos_token = pos_token;
  p.scale_log2 = h->scale_log2 * h->k_scale;
  p.v_scale = h->v_scale;
  const int di = h->cfg.head_dim == 128 ? 1 : 0;
  const ChunkBuild& b = kBuilds[di][h->fp8 ? 1 : 0];
  const dim3 blocks(unsigned(p.num_kv_heads), unsigned(std::min(c.n_items, 65535)), unsigned((c.n_items + 65534) / 65535));
  LIBRA_CUDA_TRY(h, launch(h->pdl, b.fn, blocks, unsigned(b.threads), size_t(b.smem), st, map_k, map_v, p));
  ++h->launches;
  if (c.n_merges > 0) {
    libra::ChunkMergeParams m;
    m.merges = reinterpret_cast<const int4*>(ws + c.merges_off);
    m.serial_at = p.serial_at;
    m.partial_o = p.partial_o;
    m.partial_lse = p.partial_lse;
    m.out = p.out;
    m.lse = lse;
    m.serial = c.serial;
    m.num_q_heads = p.num_q_heads;
    m.num_kv_heads = p.num_kv_heads;
    m.group = p.group;
    const dim3 grid(unsigned(c.n_merges * p.num_kv_heads), unsigned(libra::kChunkItemRows / libra::kChunkMergeWarps));
    LIBRA_CUDA_TRY(h, launch(h->pdl, di ? libra::chunk_merge_kernel<128> : libra::chunk_merge_kernel<64>, grid,
                             unsigned(libra::kChunkMergeWarps * 32), 0, st, m));
    ++h->launches;
  }
  return LIBRA_OK;
}

}  // extern "C"
