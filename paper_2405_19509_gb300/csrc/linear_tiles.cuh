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
  int box;  // ... and whole 16-byte pieces

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

__device__ __forceinline__ void activate32(int act, float (&v)[32]) {
  switch (act) {  // outside the loop: one activation's code at a time
#define GC_ALL(A)                                                  \
  case A:                                                          \
    _Pragma("unroll") for (int j = 0; j < 32; ++j) v[j] = linear::activate(A, v[j]); \
    break;
    case GC_ACT_GELU:
#pragma unroll
      for (int j = 0; j < 32; j += 2) linear::gelu(v[j], v[j + 1]);
      break;
    GC_ALL(GC_ACT_RELU)
    GC_ALL(GC_ACT_GELU_TANH)
    GC_ALL(GC_ACT_SILU)
#undef GC_ALL
  }
}

// 32 x 32 sums, a lane a row, through the epilogue and out by way of the box.  Rows of y, z and residual are whole 16-byte
// pieces; what is past their ends is not stored.
template <typename T, typename Get>
__device__ __forceinline__ void store_box(const Finish& f, int rows, int row0, int col, int c, uint8_t* box,
                                          const CUtensorMap* out, Get get) {
  const int lane = threadIdx.x & 31;
  const int n = f.F - col;
  constexpr int N = sizeof(T) == 2 ? 1 : 2;  // boxes
  const float own = f.bias && lane < n ? __ldg(f.bias + col + lane) : 0.f;
  Rows32 res[N];
  if (f.res) {
    const char* from = reinterpret_cast<const char*>(reinterpret_cast<const T*>(f.res) + (long long)row0 * f.ldr + col);
#pragma unroll
    for (int h = 0; h < N; ++h)
      res[h].load(from + 64 * h, f.ldr * (long long)sizeof(T), rows, n * (int)sizeof(T) - 64 * h, lane);
  }
  float v[32];
  get(c, v);
  if (f.bias) {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xffffffffu, own, j);
  }
  auto put = [&](const CUtensorMap* map) {
    if (sizeof(T) == 4) {
      store_32(map, box, lane, v, n, col, row0, 0);
      return;
    }
    box_free(lane);
    box_put_16(box, lane, [&](int j) { return pack_bf16(v[j], v[j + 1]); });
    box_store(map, box, lane, col, row0, 0);
  };
  if (f.z) put(&out[1]);
  activate32(f.act, v);
  if (f.res) {
    box_free(lane);
#pragma unroll
    for (int h = 0; h < N; ++h) {
      res[h].turn(box, lane);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w[4] = {res[h].q[j].x, res[h].q[j].y, res[h].q[j].z, res[h].q[j].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (sizeof(T) == 2) {
            v[8 * j + 2 * e] += __uint_as_float(w[e] << 16);
            v[8 * j + 2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u);
          } else {
            v[16 * h + 4 * j + e] += __uint_as_float(w[e]);
          }
        }
      }
    }
  }
  put(&out[0]);
}

// A warp's part of a tile: rows row0 .. of T, columns col0 ..; to plane `range` of the fp32 sums that `part` maps where the sum is
// one of several ranges (range >= 0), else through the epilogue.
template <int NC, typename Get>
__device__ __forceinline__ void store_rows(const Finish& f, long long T, int range, const CUtensorMap* part, int row0, int col0,
                                           uint8_t* box, const CUtensorMap* out, Get get) {
  const int lane = threadIdx.x & 31;
  const int rows = (int)min(T - row0, 32LL);
#pragma unroll 1
  for (int c = 0; c < NC; ++c) {
    const int col = col0 + c * 32;
    __syncwarp();
    const bool any = rows > 0 && col < f.F;
    if (f.box && range < 0 && any) {
      if (f.bf16)
        store_box<__nv_bfloat16>(f, rows, row0, col, c, box, out, get);
      else
        store_box<float>(f, rows, row0, col, c, box, out, get);
      continue;
    }
    float v[32];
    get(c, v);
    if (!any) continue;
    if (range >= 0) {
      store_32(part, box, lane, v, f.F - col, col, row0, range);
    } else {
      by_rows(box, lane, v, rows, f.F - col, [&](int r, int j, float s) {
        if (f.bf16)
          f.one<__nv_bfloat16>(row0 + r, col + j, s);
        else
          f.one<float>(row0 + r, col + j, s);
      });
    }
  }
}

// Maps of y and z, where their rows and the residual's are whole 16-byte pieces (a store by TMA writes no less), and in the
// place of y's of `ks` ranges' sums.
inline int finish_maps(Finish* f, long long T, float* part, int ks, int ld_part, Maps* m) {
  const int e = f->bf16 ? 2 : 4;
  f->box = f->F * e % 16 == 0 && rowwise::rows_16(f->y, f->ldy, e) && rowwise::rows_16(f->z, f->ldz, e) && rowwise::rows_16(f->res, f->ldr, e);
  m->out[0] = m->out[1] = m->a_turned = m->b_turned = m->a[0];
  if (ks > 1) return box_map(&m->out[0], part, MAP_F32, ld_part, T, ks, ld_part, T * ld_part);
  if (!f->box) return GC_OK;
  const MapType t = f->bf16 ? MAP_BF16 : MAP_F32;
  int rc = box_map(&m->out[0], f->y, t, f->F, T, 1, f->ldy, T * f->ldy);
  if (!rc && f->z) rc = box_map(&m->out[1], f->z, t, f->F, T, 1, f->ldz, T * f->ldz);
  return rc;
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

inline bool fours(const void* q, int64_t ld, int elt) {
  return !q || (reinterpret_cast<uintptr_t>(q) % (4 * elt) == 0 && ld % 4 == 0);
}
// The epilogue of a call; its box is for finish_maps to say.
inline Finish finish_of(const LinearShape& s, const LinearIO& io) {
  const int e = s.x_dtype == GC_BF16 ? 2 : 4;
  return Finish{s.F, s.act, e == 2, io.bias, io.res, io.y, io.z, (long long)io.ldr, (long long)io.ldy, (long long)io.ldz,
                fours(io.res, io.ldr, e) && fours(io.y, io.ldy, e) && fours(io.z, io.ldz, e), 0};
}
inline Finish finish_of(const LinearGradShape& s, const LinearGradIO& io) {
  const int e = s.x_dtype == GC_BF16 ? 2 : 4;
  return Finish{s.C, GC_ACT_NONE, e == 2, nullptr, nullptr, io.dX, nullptr, 0, (long long)io.lddx, 0, fours(io.dX, io.lddx, e), 0};
}

inline int launch_join(const float* part, int ks, long long rows, int ld, const Finish& f, cudaStream_t st) {
  const unsigned grid = (unsigned)((rows * (ld / 4) + 255) / 256);
  return f.bf16 ? launch_chain(k_linear_join<__nv_bfloat16>, "k_linear_join", grid, 256, 0, 1, true, st, part, ks, rows,
                               ld, f)
                : launch_chain(k_linear_join<float>, "k_linear_join", grid, 256, 0, 1, true, st, part, ks, rows, ld, f);
}

}  // namespace linear

// Small layers, in fp32 products (k_linear_small.cu).  G and Gb of a chunk have the same bits whatever chunks a call has, so
// their choice looks at a chunk's work alone.
// Measured as graph replays, kernels here against tiles (us): 256 x 256 x 256 in bf16 6.1 against 8.5, x 512, 2^25 products, 6.4 against
// 8.7, where 2^26 took 10.8 here and take 8.7 on tiles; in fp32 6.8 against 13.1 for 2^25, 18.5 against 13.4 for 2^27.  Rows of 2048
// by 8192 in bf16: one 5.7, two 7.6, four 17, eight 27, against 12.7; with an fp32 W, which tiles copy in parts, 10, 14, 21, 36 against
// 40.  dx of 256 x 256 x 160, 2^23.3, 6.7 against 16.8, of 2^24.6 15.4 against 16.8; six chunks' G of 2^21 each 5.4 against 11.9, of 2^24
// 21 against 17.4.  (A repeated call finds up to some 100 MB of operands in L2.)
// A sum runs alone in a block there, some 2 us for 64 of its products: 16 x 5632 x 64 took 184 us.
constexpr int kLinearRows = 8, kLinearSum = 256;
constexpr double kLinearSmall = 1 << 25, kLinearSmallDx = 1 << 24, kLinearSmallChunk = 1 << 21;
inline bool linear_small(const LinearShape& s) {
  const bool copies = s.x_dtype != GC_BF16 || s.w_dtype != GC_BF16 || !s.x_16 || !s.w_16;
  if (s.T > kLinearRows && s.C > kLinearSum) return false;
  return s.T <= 2 || (double)s.T * s.C * s.F <= (s.T <= kLinearRows && copies ? 2 : 1) * kLinearSmall;
}
inline bool linear_small_dx(const LinearGradShape& s) {
  return s.F <= kLinearSum && (double)s.N * s.n_c * s.C * s.F <= kLinearSmallDx;
}
inline bool linear_small_g(const LinearGradShape& s) {
  return s.n_c <= kLinearSum && (double)s.n_c * s.C * s.F <= kLinearSmallChunk;
}
int launch_linear_small(const LinearShape& s, const LinearIO& io, const linear::Finish& f, cudaStream_t st);
int launch_linear_grad_small(const LinearGradShape& s, const LinearGradIO& io, const linear::Finish& f, cudaStream_t st);

}  // namespace gc
