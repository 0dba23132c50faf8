// Tensor maps of the tensor-core kernels.
#include "tc_host.cuh"

namespace gc {
namespace {

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &q) ==
            cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr);
    return PFN_cuTensorMapEncodeTiled_v12000(nullptr);
  }();
  return fn;
}

}  // namespace

int map_nd(CUtensorMap* map, const void* base, int rank, const long long* dims, const long long* ld, int box_rows,
           int box_planes, MapType type, bool narrow) {
  auto fn = encode_fn();
  if (!fn) return fail(GC_ERR_CUDA, "cuTensorMapEncodeTiled entry point unavailable");
  const bool f32 = type == MAP_F32;
  cuuint64_t d[4], st[3];
  cuuint32_t box[4] = {(f32 ? 32u : 64u) >> narrow, (cuuint32_t)box_rows, (cuuint32_t)box_planes, 1}, one[4] = {1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) d[i] = (cuuint64_t)dims[i];
  for (int i = 0; i + 1 < rank; ++i) st[i] = (cuuint64_t)ld[i] * (f32 ? 4 : 2);
  const CUresult r = fn(map,
                        f32               ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                        : type == MAP_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                          : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                        (cuuint32_t)rank, const_cast<void*>(base), d, st, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        narrow ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? GC_OK : fail(GC_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

}  // namespace gc
