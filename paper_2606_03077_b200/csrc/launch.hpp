// Launches shared by the files of entry points.
#pragma once
#include <cuda_runtime.h>

namespace libra {

// As a programmatic dependent of its predecessor where the handle allows it; the kernels wait for that one inside.
// cluster > 1: blocks of a cluster along x.
template <typename... P, typename... A>
cudaError_t launch(bool dependent, unsigned cluster, void (*fn)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st,
                   const A&... args) {
  cudaLaunchConfig_t lc = {};
  lc.gridDim = grid;
  lc.blockDim = dim3(threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  cudaLaunchAttribute attr[2];
  if (dependent) {
    attr[lc.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[lc.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[lc.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[lc.numAttrs].val.clusterDim.x = cluster;
    attr[lc.numAttrs].val.clusterDim.y = 1;
    attr[lc.numAttrs++].val.clusterDim.z = 1;
  }
  lc.attrs = attr;
  return cudaLaunchKernelEx(&lc, fn, args...);
}

}  // namespace libra
