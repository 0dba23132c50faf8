// What the linear layer and its gradient share: activations, and rows as parts for the tensor cores.
#pragma once

#include <algorithm>

#include "rowwise.cuh"

namespace gc {

// 16-bit parts [parts][rows][Cp] of a matrix (k_parts.cu), zero from C to Cp, a multiple of 8.
int launch_parts(const void* x, int dtype, int64_t ld, long long rows, int C, int Cp, int parts, __nv_bfloat16* out,
                 bool chained, cudaStream_t s);

namespace linear {

constexpr float kBf16Max = 0x1.fep+127f;

// The next bf16 part of eight values, which keep their rest; far: bits of those past bf16's largest value, where fp32 goes
// on for another 2^-8 of it.  Their parts are cut off, not rounded, so that sums of them do not leave the range either.
// Of a value that is not finite the parts after the first are 0.
__device__ __forceinline__ void next_part(float (&v)[8], uint32_t& far, float (&h)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (fabsf(v[j]) > kBf16Max) far |= 1u << j;
    const bool cut = far >> j & 1 && isfinite(v[j]);
    h[j] = cut ? __uint_as_float(__float_as_uint(v[j]) & 0xffff0000u) : __bfloat162float(__float2bfloat16_rn(v[j]));
    v[j] = isfinite(h[j]) ? v[j] - h[j] : 0.f;
  }
}

constexpr float kRoot2 = 1.4142135623730951f, kInvRoot2Pi = 0.3989422804014327f;
constexpr float kTanh0 = 0.7978845608028654f, kTanh1 = 0.044715f;  // sqrt(2 / pi); Hendrycks and Gimpel's cubic

// 1 / (1 + exp(-x)).  exp overflows to infinity, whose quotient is 0.
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + expf(-x)); }

// act(z).  gelu by the error function, gelu_tanh by the tanh of a cubic u: (1 + tanh u) / 2 = sigmoid(2 u).
__device__ __forceinline__ float activate(int act, float z) {
  switch (act) {
    case GC_ACT_RELU:
      return z < 0.f ? 0.f : z;  // NaN stays
    case GC_ACT_GELU:
      return 0.5f * z * (1.f + erff(z * (1.f / kRoot2)));
    case GC_ACT_GELU_TANH:
      return z * sigmoid(2.f * kTanh0 * z * fmaf(kTanh1, z * z, 1.f));
    case GC_ACT_SILU:
      return z * sigmoid(z);
    default:
      return z;
  }
}

// act'(z): of relu 0 at 0.  Past 100 the others' slopes are 0 or 1, and a product of an infinity there would be none.
__device__ __forceinline__ float slope(int act, float z) {
  if (fabsf(z) > 100.f) z = copysignf(100.f, z);  // NaN stays
  switch (act) {
    case GC_ACT_RELU:
      return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    case GC_ACT_GELU:
      return fmaf(z * kInvRoot2Pi, expf(-0.5f * z * z), 0.5f * (1.f + erff(z * (1.f / kRoot2))));
    case GC_ACT_GELU_TANH: {
      const float s = sigmoid(2.f * kTanh0 * z * fmaf(kTanh1, z * z, 1.f));
      return fmaf(z * s * (1.f - s), 2.f * kTanh0 * fmaf(3.f * kTanh1, z * z, 1.f), s);
    }
    case GC_ACT_SILU: {
      const float s = sigmoid(z);
      return s * fmaf(z, 1.f - s, 1.f);
    }
    default:
      return 1.f;
  }
}

}  // namespace linear
}  // namespace gc
