// What the linear layer and its gradient share: activations, and rows as parts for the tensor cores.
#pragma once

#include <algorithm>

#include "rowwise.cuh"

namespace gc {

// bf16 parts [parts][rows][Cp] of a matrix, zero from C to Cp, a multiple of 8: x = x0 + x1 + ..., part q the bf16 of what the
// parts before left.  `blocks` blocks of 256 threads form them, none of an empty job.
struct PartsJob {
  const void* x;
  long long ld, rows;
  int C, Cp, parts, bf16, vec, blocks;
  __nv_bfloat16* out;
};
inline PartsJob parts_job(const void* x, int dtype, int64_t ld, long long rows, int C, int Cp, int parts, __nv_bfloat16* out) {
  const long long blocks = (rows * ((Cp + rowwise::kSeg - 1) / rowwise::kSeg) + 7) / 8;
  const int bf = dtype == GC_BF16;
  return PartsJob{x, (long long)ld, rows, C, Cp, parts, bf, C % 8 == 0 && rowwise::rows_16(x, ld, bf ? 2 : 4),
                  (int)std::min<long long>(blocks, 16LL * device_sm_count()), out};
}
// Two matrices' in one launch (k_parts.cu).
int launch_parts(const PartsJob& a, const PartsJob& b, cudaStream_t s);

namespace linear {

constexpr float kBf16Max = 0x1.fep+127f;
constexpr float kInvRoot2Pi = 0.3989422804014327f;
constexpr float kTanh0 = 0.7978845608028654f, kTanh1 = 0.044715f;  // sqrt(2 / pi); Hendrycks and Gimpel's cubic

// The next bf16 part of eight values as packed pairs; the values keep their rest (of no use after the last).  far: bits of those past bf16's largest
// value, where fp32 goes on for another 2^-8 of it.  Their parts are cut off, not rounded, so that sums of them do not leave the
// range either.  Of a value that is not finite the parts after the first are 0.
__device__ __forceinline__ void next_part(float (&v)[8], bool first, bool last, uint32_t& far, uint32_t (&w)[4]) {
  uint32_t ones = far;  // whether the first part's exponent is all ones, or was where that is felt later
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
    w[j] = *reinterpret_cast<const uint32_t*>(&t);
    if (first) ones |= ((w[j] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  }
  if (ones == 0) {
    if (last) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] -= __uint_as_float(w[j] << 16);
      v[2 * j + 1] -= __uint_as_float(w[j] & 0xffff0000u);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t b = __float_as_uint(v[j]);
    const bool finite = isfinite(v[j]);
    if (fabsf(v[j]) > kBf16Max) far |= 1u << j;
    if (far >> j & 1 && finite) w[j / 2] = (w[j / 2] & (j % 2 ? 0x0000ffffu : 0xffff0000u)) | (j % 2 ? b & 0xffff0000u : b >> 16);
    v[j] = finite ? v[j] - __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16) : 0.f;
  }
}

// ... and stored, as rowwise.cuh's segments lie: rows of Cp values.
template <bool VEC>
__device__ __forceinline__ void store_part(__nv_bfloat16* row, int col0, int lane, int Cp, const uint32_t (&w)[4]) {
  if (VEC) {
    const int c = col0 + lane * 8;
    if (c < Cp) *reinterpret_cast<uint4*>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
  uint16_t* to = reinterpret_cast<uint16_t*>(row);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = col0 + j * 32 + lane;
    if (c < Cp) to[c] = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
  }
}

// Block `block` of a job: a warp takes segments of 256 columns, several an SM in flight.
template <typename T, bool VEC>
__device__ __forceinline__ void form_parts(const PartsJob& p, int block) {
  const int lane = threadIdx.x & 31;
  const int segs = (p.Cp + rowwise::kSeg - 1) / rowwise::kSeg;
  const long long n = p.rows * segs, step = (long long)p.blocks * 8;
  for (long long i = (long long)block * 8 + (threadIdx.x >> 5); i < n; i += step) {
    const long long row = i / segs;
    const int col0 = (int)(i - row * segs) * rowwise::kSeg;
    float v[8];
    rowwise::load_seg<VEC>(reinterpret_cast<const T*>(p.x) + row * p.ld, col0, lane, p.C, v);
    uint32_t far = 0;
    for (int q = 0; q < p.parts; ++q) {
      uint32_t w[4];
      next_part(v, q == 0, q + 1 == p.parts, far, w);
      store_part<VEC>(p.out + ((size_t)q * p.rows + row) * p.Cp, col0, lane, p.Cp, w);
    }
  }
}
__device__ __forceinline__ void form_parts(const PartsJob& p, int block) {
  if (p.bf16)
    p.vec ? form_parts<__nv_bfloat16, true>(p, block) : form_parts<__nv_bfloat16, false>(p, block);
  else
    p.vec ? form_parts<float, true>(p, block) : form_parts<float, false>(p, block);
}

// 2^x and 1 / x by the special function unit, 2 and 1 units in the last place off; 2^x of x below -126 is 0.
__device__ __forceinline__ float power2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f;

// 1 / (1 + exp(-x)), of x / log2(e).  2^-x overflows to infinity, whose reciprocal is 0.
__device__ __forceinline__ float sigmoid2(float x) { return reciprocal(1.f + power2(-x)); }

// The normal distribution's tail and density (times sqrt(2 pi)): Phi(-|z|) = exp(-z^2 / 2) t q(t), t = 1 / (1 + 0.35 |z|),
// with q of degree 8 fitted to the least relative error, 3.2e-8, over |z| <= 14.5.  In fp32 it is 1e-6 off for |z| < 3 and 1e-5
// at 13, where 1 + erf has lost all digits.
__device__ __forceinline__ float tail(float z, float* density) {
  const float t = reciprocal(fmaf(0.35f, fabsf(z), 1.f));
  float q = -0x1.ddba88p-6f;
  q = fmaf(q, t, 0x1.26fa9ap-3f);
  q = fmaf(q, t, -0x1.05fb9ep-2f);
  q = fmaf(q, t, 0x1.464b9ap-3f);
  q = fmaf(q, t, -0x1.7c5bdep-6f);
  q = fmaf(q, t, 0x1.b05920p-4f);
  q = fmaf(q, t, 0x1.eac964p-4f);
  q = fmaf(q, t, 0x1.1e70cap-3f);
  q = fmaf(q, t, 0x1.1df1c6p-3f);
  *density = power2(-0.5f * kLog2e * z * z);
  return *density * (t * q);
}

// ... of two |z| by the two-wide instructions, with the same bits.
__device__ __forceinline__ float2 tail(float2 z, float2* density) {
  using rowwise::both;
  const float2 u = __ffma2_rn(both(0.35f), z, both(1.f));
  const float2 t = make_float2(reciprocal(u.x), reciprocal(u.y));
  float2 q = both(-0x1.ddba88p-6f);
  q = __ffma2_rn(q, t, both(0x1.26fa9ap-3f));
  q = __ffma2_rn(q, t, both(-0x1.05fb9ep-2f));
  q = __ffma2_rn(q, t, both(0x1.464b9ap-3f));
  q = __ffma2_rn(q, t, both(-0x1.7c5bdep-6f));
  q = __ffma2_rn(q, t, both(0x1.b05920p-4f));
  q = __ffma2_rn(q, t, both(0x1.eac964p-4f));
  q = __ffma2_rn(q, t, both(0x1.1e70cap-3f));
  q = __ffma2_rn(q, t, both(0x1.1df1c6p-3f));
  const float2 e = __fmul2_rn(__fmul2_rn(both(-0.5f * kLog2e), z), z);
  *density = make_float2(power2(e.x), power2(e.y));
  return __fmul2_rn(*density, __fmul2_rn(t, q));
}

// act(z).  gelu = z Phi(z), which keeps the tail's digits and of +inf is that; gelu_tanh by the tanh of a cubic u:
// (1 + tanh u) / 2 = sigmoid(2 u).
__device__ __forceinline__ float activate(int act, float z) {
  switch (act) {
    case GC_ACT_RELU:
      return z < 0.f ? 0.f : z;  // NaN stays
    case GC_ACT_GELU: {
      float e;
      const float p = tail(z, &e);
      return z * (z > 0.f ? 1.f - p : p);
    }
    case GC_ACT_GELU_TANH:
      return z * sigmoid2(z * fmaf(2.f * kLog2e * kTanh0 * kTanh1, z * z, 2.f * kLog2e * kTanh0));
    case GC_ACT_SILU:
      return z * sigmoid2(kLog2e * z);
    default:
      return z;
  }
}

// act'(z): of relu 0 at 0.  Past 100 the others' slopes are 0 or 1, and a product of an infinity there would be none.
__device__ __forceinline__ float slope(int act, float z) {
  if (act == GC_ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
  if (fabsf(z) > 100.f) z = copysignf(100.f, z);  // NaN stays
  switch (act) {
    case GC_ACT_GELU: {
      float e;
      const float p = tail(z, &e);
      return fmaf(z * kInvRoot2Pi, e, z > 0.f ? 1.f - p : p);
    }
    case GC_ACT_GELU_TANH: {
      const float s = sigmoid2(z * fmaf(2.f * kLog2e * kTanh0 * kTanh1, z * z, 2.f * kLog2e * kTanh0));
      return fmaf(z * s * (1.f - s), fmaf(6.f * kTanh0 * kTanh1, z * z, 2.f * kTanh0), s);
    }
    case GC_ACT_SILU: {
      const float s = sigmoid2(kLog2e * z);
      return s * fmaf(z, 1.f - s, 1.f);
    }
    default:
      return 1.f;
  }
}

// min(|z|, 100), NaN of NaN.
__device__ __forceinline__ float near(float z) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(z)), "f"(100.f));
  return r;
}
// gelu and v gelu' of two values.
__device__ __forceinline__ void gelu(float& a, float& b) {
  float2 e;
  const float2 p = tail(make_float2(fabsf(a), fabsf(b)), &e);
  const float2 q = __fadd2_rn(rowwise::both(1.f), make_float2(-p.x, -p.y));
  const float2 y = __fmul2_rn(make_float2(a, b), make_float2(a > 0.f ? q.x : p.x, b > 0.f ? q.y : p.y));
  a = y.x;
  b = y.y;
}
__device__ __forceinline__ void times_gelu_slope(float2 z, float& a, float& b) {
  const float2 m = make_float2(near(z.x), near(z.y));
  float2 e;
  const float2 p = tail(m, &e);
  const float2 q = __fadd2_rn(rowwise::both(1.f), make_float2(-p.x, -p.y));
  const float2 zk = __fmul2_rn(make_float2(copysignf(m.x, z.x), copysignf(m.y, z.y)), rowwise::both(kInvRoot2Pi));
  const float2 y = __fmul2_rn(make_float2(a, b), __ffma2_rn(zk, e, make_float2(z.x > 0.f ? q.x : p.x, z.y > 0.f ? q.y : p.y)));
  a = y.x;
  b = y.y;
}

// v *= act'(z), the activation chosen once for eight values.
__device__ __forceinline__ void times_slope(int act, const float (&z)[8], float (&v)[8]) {
#define GC_ALL(A)                                                             \
  case A:                                                                     \
    _Pragma("unroll") for (int j = 0; j < 8; ++j) v[j] *= slope(A, z[j]);     \
    break;
  switch (act) {
    case GC_ACT_GELU:
#pragma unroll
      for (int j = 0; j < 8; j += 2) times_gelu_slope(make_float2(z[j], z[j + 1]), v[j], v[j + 1]);
      break;
    GC_ALL(GC_ACT_RELU)
    GC_ALL(GC_ACT_GELU_TANH)
    GC_ALL(GC_ACT_SILU)
  }
#undef GC_ALL
}

}  // namespace linear
}  // namespace gc
