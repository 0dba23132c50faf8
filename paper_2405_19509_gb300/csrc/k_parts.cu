// Rows of a matrix as 16-bit parts for the tensor cores: x = x0 + x1 + ..., part q the bf16 of what the parts before
// left.  Each keeps 8 bits, whatever the size of x.
//
// Bound: HBM (a copy).  A warp takes segments of 256 columns, several an SM in flight.
#include "linear.cuh"
#include "tc_host.cuh"

namespace gc {
namespace {

using namespace rowwise;

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_parts(const T* __restrict__ x, long long ld, long long rows, int C, int Cp,
                                               int parts, __nv_bfloat16* __restrict__ out) {
  const int lane = threadIdx.x & 31;
  const int segs = (Cp + kSeg - 1) / kSeg;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const long long n = rows * segs, step = (long long)gridDim.x * 8;
  for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < n; i += step) {
    const long long row = i / segs;
    const int col0 = (int)(i - row * segs) * kSeg;
    float v[8];
    load_seg<VEC>(x + row * ld, col0, lane, C, v);
    uint32_t far = 0;
    for (int q = 0; q < parts; ++q) {
      uint32_t w[4];
      linear::next_part(v, q == 0, q + 1 == parts, far, w);
      linear::store_part<VEC>(out + ((size_t)q * rows + row) * Cp, col0, lane, Cp, w);
    }
  }
}

}  // namespace

int launch_parts(const void* x, int dtype, int64_t ld, long long rows, int C, int Cp, int parts, __nv_bfloat16* out,
                 bool chained, cudaStream_t s) {
  const bool bf = dtype == GC_BF16;
  const bool vec = C % 8 == 0 && rows_16(x, ld, bf ? 2 : 4);
  const long long blocks = (rows * ((Cp + kSeg - 1) / kSeg) + 7) / 8;
  const unsigned grid = (unsigned)std::min<long long>(blocks, 16LL * device_sm_count());
  if (bf)
    return launch_chain(vec ? k_parts<__nv_bfloat16, true> : k_parts<__nv_bfloat16, false>, "k_parts", grid, 256, 0, 1,
                        chained, s, (const __nv_bfloat16*)x, (long long)ld, rows, C, Cp, parts, out);
  return launch_chain(vec ? k_parts<float, true> : k_parts<float, false>, "k_parts", grid, 256, 0, 1, chained, s,
                      (const float*)x, (long long)ld, rows, C, Cp, parts, out);
}

}  // namespace gc
