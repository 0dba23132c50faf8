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

// |u| / max(|u|, eps) of a norm's square, 1 of one that is not finite.
__device__ __forceinline__ float norm_ratio(double sum, float eps) {
  const double norm = sqrt(sum);
  return norm < (double)eps ? (float)(norm / (double)eps) : 1.f;
}
// The least power of two that is no less than x, between 2^-125 and 1.
__device__ __forceinline__ float power_above(float x) {
  int e = 0;
  if (!(x < 1.f)) return 1.f;
  frexpf(x, &e);
  return x < 0x1p-125f ? 0x1p-125f : ldexpf(1.f, e);
}
// scale / (lam max(sqrt(sum), eps)), lam a power of two, as three factors, none of which leaves fp32's range: the norm is f 2^e.
__device__ __forceinline__ void norm_factors(double sum, float eps, float lam, float scale, float* factor) {
  double norm = sqrt(sum);
  if (norm < (double)eps) norm = eps;
  if (isinf(norm) || isnan(norm)) {
    factor[0] = factor[1] = 1.f;
    factor[2] = isinf(norm) ? 0.f : (float)norm;
    return;
  }
  int e = 0;
  const double f = frexp(norm, &e);
  e += ilogbf(lam);
  factor[0] = ldexpf(1.f, -(e / 2));
  factor[1] = ldexpf(1.f, -(e - e / 2));
  factor[2] = (float)((double)scale / f);
}

}  // namespace gc
