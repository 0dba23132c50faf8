// What the kernels of orthogonalised matrices share: the norm, from its squares to the factors that divide by it.
#pragma once

#include "gc_internal.cuh"

namespace gc {

// Small matrices, a cluster each (k_newton_small.cu).
bool ns_small(const NsShape& s);
int launch_ns_small(const NsShape& s, const NsIO& io, cudaStream_t st);

// sum += the squares of v, whose sum in 32 bits is q: that, where 32 bits hold it.
template <int K>
__device__ __forceinline__ void add_squares(float q, const float (&v)[K], double& sum) {
  if (q > 1e-24f && q < 1e37f) {
    sum += q;
    return;
  }
#pragma unroll
  for (int j = 0; j < K; ++j) sum += (double)v[j] * v[j];
}

// scale / max(sqrt(sum), eps) as three factors, none of which leaves fp32's range: the norm is f 2^e.  down: a norm below eps
// that the steps, which enlarge nothing more than `amp` times, leave below 2^-down is taken 2^down times as large.
__device__ __forceinline__ void norm_factors(double sum, float eps, float amp, float scale, float* factor, int* down) {
  double norm = sqrt(sum);
  *down = 0;
  if (norm < (double)eps) {
    const double t = norm / (double)eps * (double)amp;
    if (t < 1) *down = t > 0x1p-125 ? -ilogb(t) - 1 : 125;  // t <= 2^-down < 2 t
    norm = eps;
  }
  if (isinf(norm) || isnan(norm)) {
    factor[0] = factor[1] = 1.f;
    factor[2] = isinf(norm) ? 0.f : (float)norm;
    return;
  }
  int e = 0;
  const double f = frexp(norm, &e);
  e -= *down;
  factor[0] = ldexpf(1.f, -(e / 2));
  factor[1] = ldexpf(1.f, -(e - e / 2));
  factor[2] = (float)((double)scale / f);
}

}  // namespace gc
