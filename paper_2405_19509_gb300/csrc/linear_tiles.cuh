// The epilogue of the linear layer's tiles and of its gradient's rows, and the join of a sum's ranges.
#pragma once

#include "linear.cuh"
#include "tc_tiles.cuh"

namespace gc {
namespace linear {

using namespace tiles;

// y = residual + act(v + bias) of a sum v, with z = v + bias kept where it is wanted.
struct Finish {
  int F, act, bf16;
  const float* bias;
  const void* res;
  void *y, *z;
  long long ldr, ldy, ldz;
  int vec;  // rows of y, z and residual in groups of four

  template <typename T>
  __device__ __forceinline__ void one(long long row, int c, float v) const {
    using rowwise::to_f;
    if (bias) v += __ldg(bias + c);
    if (z) reinterpret_cast<T*>(z)[row * ldz + c] = rowwise::from_f<T>(v);
    v = linear::activate(act, v);
    if (res) v += to_f(reinterpret_cast<const T*>(res)[row * ldr + c]);
    reinterpret_cast<T*>(y)[row * ldy + c] = rowwise::from_f<T>(v);
  }
  static __device__ __forceinline__ void put4(__nv_bfloat16* p, const float (&v)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
  static __device__ __forceinline__ void put4(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
  static __device__ __forceinline__ void add4(const __nv_bfloat16* p, float (&v)[4]) {
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    v[0] += __uint_as_float(q.x << 16);
    v[1] += __uint_as_float(q.x & 0xffff0000u);
    v[2] += __uint_as_float(q.y << 16);
    v[3] += __uint_as_float(q.y & 0xffff0000u);
  }
  static __device__ __forceinline__ void add4(const float* p, float (&v)[4]) {
    const float4 q = *reinterpret_cast<const float4*>(p);
    v[0] += q.x;
    v[1] += q.y;
    v[2] += q.z;
    v[3] += q.w;
  }
  // Columns c .. c + 3 of a row, c a multiple of 4; bias4: of these columns.
  template <typename T>
  __device__ __forceinline__ void four(long long row, int c, float4 s, float4 bias4) const {
    if (c + 4 > F) {
      const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (c + e < F) one<T>(row, c + e, v[e]);
      return;
    }
    float v[4] = {s.x + bias4.x, s.y + bias4.y, s.z + bias4.z, s.w + bias4.w};
    if (z) put4(reinterpret_cast<T*>(z) + row * ldz + c, v);
    if (act != GC_ACT_NONE) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = linear::activate(act, v[e]);
    }
    if (res) add4(reinterpret_cast<const T*>(res) + row * ldr + c, v);
    put4(reinterpret_cast<T*>(y) + row * ldy + c, v);
  }
  __device__ __forceinline__ float4 bias_of(int c) const {
    if (!bias || c + 4 > F) return make_float4(0.f, 0.f, 0.f, 0.f);
    return make_float4(__ldg(bias + c), __ldg(bias + c + 1), __ldg(bias + c + 2), __ldg(bias + c + 3));
  }
};

// A warp's part of a tile: rows row0 .. of T, columns col0 ..; to `part` (rows of fp32 sums, ld apart) where the sum
// is one of several ranges, else through the epilogue.
template <int NC, int U, typename Get>
__device__ __forceinline__ void store_rows(const Finish& f, long long T, float* part, int ld_part, int row0, int col0,
                                           uint8_t* box, Get get) {
  const int lane = threadIdx.x & 31;
  const int rows = (int)min(T - row0, 32LL);
#pragma unroll(U)
  for (int c = 0; c < NC; ++c) {
    float v[32];
    __syncwarp();
    get(c, v);
    const int col = col0 + c * 32;
    if (rows <= 0 || col >= f.F) continue;
    box_put(box, lane, v);
    __syncwarp();
    if (part) {
      float* to = part + (size_t)row0 * ld_part + col;
      by_fours(box, lane, [&](int r, int j, float4 s) {
        if (r < rows && col + j < f.F) *reinterpret_cast<float4*>(to + (size_t)r * ld_part + j) = s;
      });
    } else if (f.vec) {
      const float4 b = f.bias_of(col + (lane & 7) * 4);
      by_fours(box, lane, [&](int r, int j, float4 s) {
        if (r >= rows || col + j >= f.F) return;
        if (f.bf16)
          f.four<__nv_bfloat16>(row0 + r, col + j, s, b);
        else
          f.four<float>(row0 + r, col + j, s, b);
      });
    } else {
      by_rows<4>(box, lane, col + lane < f.F ? rows : 0, [&](int r, float s) {
        if (f.bf16)
          f.one<__nv_bfloat16>(row0 + r, col + lane, s);
        else
          f.one<float>(row0 + r, col + lane, s);
      });
    }
  }
}

// Four columns a thread: the ranges' sums in their order, and the epilogue.
template <typename T>
static __global__ void __launch_bounds__(256) k_linear_join(const float* __restrict__ part, int ks, long long rows, int ld,
                                                     Finish f) {
  start_next();
  wait_prior();
  const int per = ld / 4;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i / per;
  if (row >= rows) return;
  const int c = (int)(i - row * per) * 4;
  const float* at = part + (size_t)row * ld + c;
  float4 s = __ldcg(reinterpret_cast<const float4*>(at));
#pragma unroll 8
  for (int k = 1; k < ks; ++k) {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(at + (size_t)k * rows * ld));
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  }
  if (f.vec) {
    f.four<T>(row, c, s, f.bias_of(c));
  } else {
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < f.F) f.one<T>(row, c + e, v[e]);
  }
}

inline int launch_join(const float* part, int ks, long long rows, int ld, const Finish& f, cudaStream_t st) {
  const unsigned grid = (unsigned)((rows * (ld / 4) + 255) / 256);
  return f.bf16 ? launch_chain(k_linear_join<__nv_bfloat16>, "k_linear_join", grid, 256, 0, 1, true, st, part, ks, rows,
                               ld, f)
                : launch_chain(k_linear_join<float>, "k_linear_join", grid, 256, 0, 1, true, st, part, ks, rows, ld, f);
}

}  // namespace linear
}  // namespace gc
