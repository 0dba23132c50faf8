// Dropout with an optional residual, out = residual + D(x), D(x) = x * keep / (1 - p), the mask
// drawn from counters (rowwise.cuh) and never stored: the gradient of D is the same call on the
// gradient.
//
// Bound: HBM (x and the residual read once, out written once) for fp32, and nearly the integer pipe
// for bf16: ten rounds of two wide multiplications give eight 16-bit numbers, about ten
// instructions an element against four to six bytes of it.  A 32-bit number an element would double
// that; 2^-16 is the resolution of p instead, and the scale is that of the p that is drawn, so that
// the expectation of D(x) is x.  A warp takes 256 columns of a row at a time.  32,768 rows of 4096 bf16
// with residual, 805 MB: 126 us, 6.4 TB/s (136 with the rounds' keys formed in the kernel and eight blocks an
// SM).
#include <algorithm>

#include "rowwise.cuh"

namespace gc {
namespace {

using namespace rowwise;

constexpr int kThreadsD = 256;

template <typename T, bool VEC, bool RES>
__global__ void __launch_bounds__(kThreadsD)
    k_dropout(const T* x, long long ldx, const T* res, long long ldr, T* out, long long ldo,
              long long rows, int cols, int nseg, long long step_rows, int step_seg, Mask m) {
  const int lane = threadIdx.x & 31;
  const long long w = ((long long)blockIdx.x * kThreadsD + threadIdx.x) >> 5;
  long long row = w / nseg;
  int seg = (int)(w - row * nseg);
  while (row < rows) {
    const int col0 = seg * kSeg;
    float v[8], r[8];
    load_seg<VEC>(x + row * ldx, col0, lane, cols, v);
    if (RES) load_seg<VEC>(res + row * ldr, col0, lane, cols, r);
    if (m.t) drop_seg<VEC>(m, row, col0, lane, v);
    if (RES) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += r[j];
    }
    store_seg<VEC>(out + row * ldo, col0, lane, cols, v);
    row += step_rows;
    seg += step_seg;
    if (seg >= nseg) {
      seg -= nseg;
      ++row;
    }
  }
}

template <typename T, bool VEC, bool RES>
int go(const void* x, int64_t ldx, const void* res, int64_t ldr, void* out, int64_t ldo, int64_t rows,
       int cols, const Mask& m, cudaStream_t s) {
  const int nseg = (cols + kSeg - 1) / kSeg;
  const long long warps = rows * nseg;
  // blocks an SM, each warp with several segments to follow: bf16 with residual (805 MB) 139, 130, 126, 132 us by
  // 4, 5, 6, 8, fp32 (773 MB) 121, 126, 129, 136
  const long long grid = std::min<long long>((warps * 32 + kThreadsD - 1) / kThreadsD,
                                             (long long)device_sm_count() * (sizeof(T) == 2 ? 6 : 4));
  const long long W = grid * (kThreadsD / 32);
  k_dropout<T, VEC, RES><<<(unsigned)grid, kThreadsD, 0, s>>>(
      (const T*)x, ldx, (const T*)res, ldr, (T*)out, ldo, rows, cols, nseg, W / nseg, (int)(W % nseg), m);
  count_launches(1);
  return cuda_check(cudaGetLastError(), "k_dropout");
}

template <typename T>
int by_layout(const void* x, int64_t ldx, const void* res, int64_t ldr, void* out, int64_t ldo,
              int64_t rows, int cols, const Mask& m, cudaStream_t s) {
  const int e = sizeof(T);
  const bool vec = cols % 8 == 0 && rows_16(x, ldx, e) && rows_16(res, ldr, e) && rows_16(out, ldo, e);
  if (vec) return res ? go<T, true, true>(x, ldx, res, ldr, out, ldo, rows, cols, m, s)
                      : go<T, true, false>(x, ldx, res, ldr, out, ldo, rows, cols, m, s);
  return res ? go<T, false, true>(x, ldx, res, ldr, out, ldo, rows, cols, m, s)
             : go<T, false, false>(x, ldx, res, ldr, out, ldo, rows, cols, m, s);
}

}  // namespace

int launch_dropout(const void* x, int64_t ldx, const void* res, int64_t ldr, int dtype, int64_t rows,
                   int cols, const DropArgs& d, void* out, int64_t ldo, cudaStream_t s) {
  const Mask m = make_mask(d.p, d.seed, d.offset, d.row0, cols);
  return dtype == GC_BF16 ? by_layout<__nv_bfloat16>(x, ldx, res, ldr, out, ldo, rows, cols, m, s)
                          : by_layout<float>(x, ldx, res, ldr, out, ldo, rows, cols, m, s);
}

}  // namespace gc
