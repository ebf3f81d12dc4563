// The handle behind the C ABI and the small helpers that every file of entry points uses.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

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

#define LIBRA_CUDA_TRY(h, expr)                       \
  do {                                                \
    cudaError_t e__ = (expr);                         \
    if (e__ != cudaSuccess) return fail_cuda(h, e__); \
  } while (0)

}  // namespace libra
