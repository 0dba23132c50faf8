// Host side of the tensor-core kernels: tensor maps, and launches as a chain of programmatic dependents.
#pragma once

#include <cudaTypedefs.h>

#include "gc_internal.cuh"

namespace gc {

enum MapType { MAP_BF16, MAP_F16, MAP_F32 };

// Map of `rank` dimensions (up to 4), innermost first; ld[i]: elements between neighbours of dimension i + 1.  Box 128
// bytes x box_rows x box_planes, 128-byte swizzle; narrow: 64 bytes, 64-byte swizzle.
int map_nd(CUtensorMap* map, const void* base, int rank, const long long* dims, const long long* ld, int box_rows,
           int box_planes = 1, MapType type = MAP_BF16, bool narrow = false);

// A launch with clusters of `cl` CTAs (1: none); `chained`: as a dependent of the call's kernel before it.
template <typename... P, typename... A>
int launch_chain(void (*kern)(P...), const char* name, unsigned grid, int block, size_t smem, int cl, bool chained,
                 cudaStream_t s, A... args) {
  cudaLaunchAttribute at[2];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = at;
  if (cl > 1) {
    at[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    at[cfg.numAttrs].val.clusterDim.x = (unsigned)cl;
    at[cfg.numAttrs].val.clusterDim.y = at[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  if (chained) {
    at[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
  }
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
  count_launches(1);
  return cuda_check(e, name);
}

}  // namespace gc
