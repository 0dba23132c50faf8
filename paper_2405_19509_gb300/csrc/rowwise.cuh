// What the row-wise operators (dropout, layer norm) share: segments of 256 columns that a warp
// holds in registers, and the counter-based dropout mask.
//
// A segment is 256 columns of a row, eight values a lane.  VEC: eight neighbouring columns a lane
// (rows on 16-byte boundaries, a multiple of eight columns), else columns a warp width apart, one
// element a load, so that rows of any width and alignment are read in whole sectors.
#pragma once

#include "gc_internal.cuh"

namespace gc {
namespace rowwise {

constexpr int kSeg = 256;  // columns of a segment

template <bool VEC>
__device__ __forceinline__ int seg_col(int col0, int lane, int j) {
  return VEC ? col0 + lane * 8 + j : col0 + j * 32 + lane;
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// The segment at col0 of a row as it lies in memory, and its values (zeros past the row's end): a load
// may be issued long before its values are wanted.
template <bool VEC, typename T>
struct RawSeg;
template <>
struct RawSeg<true, __nv_bfloat16> {
  uint4 q;
  __device__ __forceinline__ void load(const __nv_bfloat16* row, int col0, int lane, int cols) {
    const int c = col0 + lane * 8;
    q = c < cols ? *reinterpret_cast<const uint4*>(row + c) : make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(w[j] << 16);
      v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
};
template <>
struct RawSeg<true, float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* row, int col0, int lane, int cols) {
    const int c = col0 + lane * 8;
    a = b = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < cols) {
      a = *reinterpret_cast<const float4*>(row + c);
      b = *reinterpret_cast<const float4*>(row + c + 4);
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};
template <typename T>
struct RawSeg<false, T> {
  T x[8];
  __device__ __forceinline__ void load(const T* row, int col0, int lane, int cols) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = col0 + j * 32 + lane;
      x[j] = c < cols ? row[c] : from_f<T>(0.f);
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f(x[j]);
  }
};
template <bool VEC, typename T>
__device__ __forceinline__ void load_seg(const T* row, int col0, int lane, int cols, float (&v)[8]) {
  RawSeg<VEC, T> r;
  r.load(row, col0, lane, cols);
  r.values(v);
}
// Values 2j, 2j + 1 of a segment for the two-wide instructions.
__device__ __forceinline__ float2 two(const float (&v)[8], int j) { return make_float2(v[2 * j], v[2 * j + 1]); }
__device__ __forceinline__ void put(float (&v)[8], int j, float2 x) {
  v[2 * j] = x.x;
  v[2 * j + 1] = x.y;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Whether value j of the segment is a column of the row: all of a lane's eight are, or none, when VEC.
template <bool VEC>
__device__ __forceinline__ bool in_row(int col0, int lane, int j, int cols) {
  return VEC ? col0 + lane * 8 < cols : col0 + j * 32 + lane < cols;
}

template <bool VEC, typename T>
__device__ __forceinline__ void store_seg(T* row, int col0, int lane, int cols, const float (&v)[8]) {
  if (VEC) {
    const int c = col0 + lane * 8;
    if (c >= cols) return;
    if (sizeof(T) == 2) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&t);
      }
      *reinterpret_cast<uint4*>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = col0 + j * 32 + lane;
      if (c < cols) row[c] = from_f<T>(v[j]);
    }
  }
}

// The mask: element (row, column c) is dropped when its 16-bit number is below t.  The eight numbers
// of columns 8g .. 8g + 7 are the halves (low first) of the four words of Philox4x32-10 (Salmon et
// al., "Parallel random numbers: as easy as 1, 2, 3", SC 2011) at counter (row * ceil(cols / 8) + g,
// offset) under the key `seed`: a function of the point and the column alone, so that every worker
// that holds a point draws the same mask, whatever rows it works on.
struct Mask {
  uint32_t k[20];   // the rounds' keys
  uint32_t c2, c3;
  uint32_t t;       // drop below, of 2^16; 0: nothing is dropped
  float scale;      // 2^16 / (2^16 - t)
  long long row0;   // point of the first row
  int groups;       // ceil(cols / 8)
};

__device__ __forceinline__ void philox(const Mask& m, unsigned long long e, uint32_t (&x)[4]) {
  x[0] = (uint32_t)e;
  x[1] = (uint32_t)(e >> 32);
  x[2] = m.c2;
  x[3] = m.c3;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long a = (unsigned long long)x[0] * 0xD2511F53u;
    const unsigned long long b = (unsigned long long)x[2] * 0xCD9E8D57u;
    x[0] = (uint32_t)(b >> 32) ^ x[1] ^ m.k[2 * r];
    x[1] = (uint32_t)b;
    x[2] = (uint32_t)(a >> 32) ^ x[3] ^ m.k[2 * r + 1];
    x[3] = (uint32_t)a;
  }
}

// Applies the mask to a segment of row `row` (of the call).  Warp-collective when not VEC: a lane
// draws one group, and its neighbours fetch their bit of it.
template <bool VEC>
__device__ __forceinline__ void drop_seg(const Mask& m, long long row, int col0, int lane, float (&v)[8]) {
  const unsigned long long e =
      (unsigned long long)(m.row0 + row) * (unsigned)m.groups + (unsigned)(col0 / 8 + lane);
  uint32_t x[4];
  philox(m, e, x);
  const uint32_t th = m.t << 16;
  if (VEC) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 y = __fmul2_rn(two(v, j), both(m.scale));
      v[2 * j] = x[j] << 16 >= th ? y.x : 0.f;  // th's low half is zero
      v[2 * j + 1] = x[j] >= th ? y.y : 0.f;
    }
  } else {
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t u = j % 2 ? x[j / 2] : x[j / 2] << 16;
      bits |= (u >= th ? 1u : 0u) << j;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t b = __shfl_sync(0xffffffffu, bits, j * 4 + lane / 8);
      v[j] = (b >> (lane & 7)) & 1 ? v[j] * m.scale : 0.f;
    }
  }
}

inline Mask make_mask(double p, uint64_t seed, uint64_t offset, int64_t row0, int cols) {
  Mask m;
  int t = (int)(p * 65536 + 0.5);
  if (t > 65535) t = 65535;
  m.t = (uint32_t)t;
  m.scale = 65536.f / (float)(65536 - t);
  for (int r = 0; r < 10; ++r) {
    m.k[2 * r] = (uint32_t)seed + (uint32_t)r * 0x9E3779B9u;
    m.k[2 * r + 1] = (uint32_t)(seed >> 32) + (uint32_t)r * 0xBB67AE85u;
  }
  m.c2 = (uint32_t)offset;
  m.c3 = (uint32_t)(offset >> 32);
  m.row0 = row0;
  m.groups = (cols + 7) / 8;
  return m;
}

// Whether rows at p, ld elements apart, may be read in 16-byte pieces (NULL: not there).
inline bool rows_16(const void* p, int64_t ld, int elt) {
  return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * elt % 16 == 0);
}

}  // namespace rowwise
}  // namespace gc
