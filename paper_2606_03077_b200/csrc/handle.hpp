// The handle behind the C ABI and the small helpers that every file of entry points uses.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <vector>

#include "libra.h"
#include "plan_layout.hpp"
#include "planner.hpp"

namespace libra {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct DeviceGuard {
  int prev = -1;
  bool switched = false;
  cudaError_t err = cudaSuccess;
  explicit DeviceGuard(int dev) {
    err = cudaGetDevice(&prev);
    if (err == cudaSuccess && prev != dev) {
      err = cudaSetDevice(dev);
      switched = (err == cudaSuccess);
    }
  }
  ~DeviceGuard() {
    if (switched) cudaSetDevice(prev);
  }
};

}  // namespace libra

struct libra_handle_s {
  libra_config_t cfg;
  libra::PlanParams params;          // the planner's parameters in force (defaults resolved)
  libra_plan_params_t params_in{};   // as given at creation (0 = default)
  int n_sm_dev = 0;
  bool two_slot_auto = false;        // the default of two slots per SM is in force (see kVariantPair)
  int group = 0;
  float scale_log2 = 0.f;
  int64_t stride_page = 0, stride_head = 0, stride_token = 0;
  int64_t pool_elems = 0;
  int last_cuda_error = 0;
  int variant = -1;         // -1: chosen by the number of column tiles
  int max_q_len = 1;        // query tokens per sequence the workspace is laid out for
  bool fp8 = false;         // the pools hold E4M3 codes; keys and values are code * k_scale / v_scale
  float k_scale = 1.f, v_scale = 1.f;
  int fp8_variant = -1;     // -1: chosen by the number of column tiles
  libra::EncodeTiledFn encode = nullptr;

  // workspace layout: control words | arrival counters | partial LSE | partial O | oversized plans
  int64_t max_items = 0;
  size_t cnt_off = 0, cnt_bytes = 0, lse_off = 0, o_off = 0, plan_off = 0, plan_bytes = 0, workspace_bytes = 0;
  void* clean_workspace = nullptr;  // workspace whose control words and counters are known to be zero
  int combine_mode = 1;     // 0: separate kernel, 1: inside the decode kernel
  bool pdl = true;          // programmatic dependent launches (decode after its predecessor, combine after decode)
  float* lse_out = nullptr;     // optional second output of the step (libra_set_lse_output)
  bool early_prefetch = false;  // the caller's promise about the preceding kernel (libra_set_early_prefetch)
  bool l2_warmup = true;        // libra_set_cache_warmup

  // pinned staging for uploads of plans too large for the kernel parameters
  int32_t* staging[2] = {nullptr, nullptr};
  cudaEvent_t staging_done[2] = {nullptr, nullptr};
  bool staging_used[2] = {false, false};
  int next_staging = 0;

  // last plan
  bool planned = false;
  libra::HostPlan plan;
  std::vector<int32_t> items_flat;
  void* workspace = nullptr;
  int32_t num_items = 0;
  void* last_stream = nullptr;
  bool device_planned = false;  // the last plan was made by the device-side planner: counts live in the workspace
  int64_t decodes_on_plan = 0;  // decode launches enqueued since the last plan call
  int32_t length_hint = 0;      // libra_set_length_hint: the caller's bound on the lengths of device-planned batches (0 = none)
  int32_t dev_item_bound = 0;   // device-side plan: the most work items the planned batch can have (sizes the grids)
  int32_t planned_batch = 0;
  size_t dev_counts_off = 0, dev_per_seq_off = 0, dev_entries_off = 0, dev_fixes_off = 0;
  std::vector<int32_t> export_scratch;
  bool plan_in_params = true;   // the usual case: the plan travels with every launch
  libra::ParamPlan pp;          // work items, then one entry per empty sequence
  libra::ParamFix pf;           // merges for the combine kernel

  // tensor maps of the pools seen most recently (callers often rotate between a few pools)
  struct PoolMaps {
    const void* k_ptr = nullptr;
    const void* v_ptr = nullptr;
    CUtensorMap map_k, map_v;
  };
  static constexpr int kMapCache = 8;
  PoolMaps maps[kMapCache];
  int next_map = 0;
  int pos_head = 0, pos_page = 0, pos_token = 0;

  // chunk attention: its own plan and workspace
  struct Chunk {
    bool planned = false;
    uint32_t serial = 0;              // of the plan, also in the workspace
    void* workspace = nullptr;
    int32_t n_items = 0, n_merges = 0;
    int32_t most_new = 0;             // new tokens of a sequence
    size_t merges_off = 0, lse_off = 0, o_off = 0;
    void* staging[2] = {nullptr, nullptr};   // pinned, grown when a plan needs more
    size_t staging_bytes[2] = {0, 0};
    cudaEvent_t staging_done[2] = {nullptr, nullptr};
    int next_staging = 0;
    bool attributes_set = false;
  } chunk;

  // profiling
  bool profiling = false;
  std::vector<cudaEvent_t> events;  // 3 per call
  int profiled_calls = 0;
  int64_t launches = 0;
};

namespace libra {

inline int fail_cuda(libra_handle_t h, cudaError_t e) {
  if (h) h->last_cuda_error = int(e);
  (void)cudaGetLastError();
  return LIBRA_CUDA_ERROR;
}

// Tiled tensor map of one pool: dimension 0 is head_dim (contiguous); the other three (token, head, page) are ordered by
// increasing stride.  Box = row_bytes of a row x box_tokens tokens of one head and page; pos_* receive the coordinate slots.
inline int encode_pool_map(libra_handle_t h, const void* base, int row_bytes, int box_tokens, CUtensorMapSwizzle swizzle,
                           CUtensorMap* map, int* pos_head, int* pos_page, int* pos_token) {
  struct Dim {
    int64_t stride, size;
    uint32_t box;
    int kind;
  };
  Dim dims[3] = {{h->stride_token, h->cfg.page_size, uint32_t(box_tokens), 0},
                 {h->stride_head, h->cfg.num_kv_heads, 1u, 1},
                 {h->stride_page, h->cfg.num_pages, 1u, 2}};
  std::stable_sort(dims, dims + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  const int eb = h->fp8 ? 1 : 2;   // bytes per element
  cuuint64_t gdim[4] = {cuuint64_t(h->cfg.head_dim), 0, 0, 0};
  cuuint64_t gstride[3];
  cuuint32_t box[4] = {cuuint32_t(row_bytes / eb), 0, 0, 0};
  cuuint32_t estride[4] = {1, 1, 1, 1};
  for (int i = 0; i < 3; ++i) {
    gdim[i + 1] = cuuint64_t(dims[i].size);
    gstride[i] = cuuint64_t(dims[i].stride) * eb;
    box[i + 1] = dims[i].box;
    if (dims[i].kind == 0) *pos_token = i + 1;
    if (dims[i].kind == 1) *pos_head = i + 1;
    if (dims[i].kind == 2) *pos_page = i + 1;
  }
  const CUresult r = h->encode(map, h->fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                               const_cast<void*>(base), gdim, gstride, box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    h->last_cuda_error = int(cudaErrorInvalidValue);
    return LIBRA_CUDA_ERROR;
  }
  return LIBRA_OK;
}

#define LIBRA_CUDA_TRY(h, expr)                       \
  do {                                                \
    cudaError_t e__ = (expr);                         \
    if (e__ != cudaSuccess) return fail_cuda(h, e__); \
  } while (0)

}  // namespace libra
