// Rows as bf16 parts for the tensor cores (PartsJob): each part keeps 8 bits, whatever the size of the value.
//
// Bound: HBM (a copy), and its launch, which two matrices share.
#include "linear.cuh"
#include "tc_host.cuh"

namespace gc {
namespace {

__global__ void __launch_bounds__(256) k_parts(const PartsJob a, const PartsJob b) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int i = blockIdx.x;
  linear::form_parts(i < a.blocks ? a : b, i < a.blocks ? i : i - a.blocks);
}

}  // namespace

int launch_parts(const PartsJob& a, const PartsJob& b, cudaStream_t s) {
  return launch_chain(k_parts, "k_parts", (unsigned)(a.blocks + b.blocks), 256, 0, 1, false, s, a, b);
}

}  // namespace gc
