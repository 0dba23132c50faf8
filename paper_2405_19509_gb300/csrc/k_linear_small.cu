// Linear layers too small for tiles on the tensor cores, in fp32 products of the values as they are, one launch each.
//   k_linear_rows   up to eight rows of x: a pass over W, a warp two rows of it at a time
//   k_linear_small  tiles of 32 x 32 of y, of dx and of the chunks' G
//
// Bound: k_linear_rows the latency of two rounds of loads (1 x 2048 x 8192 in bf16, 34 MB of W: 11 us from HBM, 3.0 TB/s, 5.7 where W
// lies in L2); the others latency: one launch, one or two rounds of
// loads and some 10^3 to 10^4 products a thread.
#include <algorithm>

#include "linear_tiles.cuh"

namespace gc {
namespace {

using namespace linear;
using rowwise::kSeg;
using rowwise::load_seg;
using rowwise::RawSeg;
using rowwise::to_f;

constexpr int kW = 2;        // rows of W that a warp takes at a time
constexpr int kAhead = 4;    // segments of them in flight

// `split` warps of a block share the segments of kW rows of W; their sums are added in the warps' order.
template <typename TX, typename TW, bool VEC, int R>
__global__ void __launch_bounds__(256) k_linear_rows(const TX* __restrict__ X, long long ldx, const TW* __restrict__ W, long long ldw,
                                                     int T, int C, int split, const Finish f) {
  __shared__ float red[8][kW * R];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = warp % split, f0 = (blockIdx.x * (8 / split) + warp / split) * kW;
  float acc[kW][R];
#pragma unroll
  for (int i = 0; i < kW; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) acc[i][r] = 0.f;
  if (f0 < f.F) {
    const TW* w[kW];
#pragma unroll
    for (int i = 0; i < kW; ++i) w[i] = W + (long long)min(f0 + i, f.F - 1) * ldw;
    for (int c0 = part * kSeg; c0 < C; c0 += kAhead * split * kSeg) {
      RawSeg<VEC, TW> raw[kAhead][kW];
#pragma unroll
      for (int a = 0; a < kAhead; ++a)
#pragma unroll
        for (int i = 0; i < kW; ++i) raw[a][i].load(w[i], c0 + a * split * kSeg, lane, C);
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const int c = c0 + a * split * kSeg;
        if (c >= C) break;
        float v[kW][8];
#pragma unroll
        for (int i = 0; i < kW; ++i) raw[a][i].values(v[i]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (r < T) {
            float x[8];
            load_seg<VEC>(X + r * ldx, c, lane, C, x);
#pragma unroll
            for (int i = 0; i < kW; ++i)
#pragma unroll
              for (int j = 0; j < 8; ++j) acc[i][r] = fmaf(x[j], v[i][j], acc[i][r]);
          }
        }
      }
    }
  }
  float own = 0.f;  // lane i * R + r: the sum of row r and of w[i]
#pragma unroll
  for (int i = 0; i < kW; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[i][r] += __shfl_xor_sync(0xffffffffu, acc[i][r], o);
      if (lane == i * R + r) own = acc[i][r];
    }
  const int i = lane / R, r = lane % R;
  if (split > 1) {
    if (lane < kW * R) red[warp][lane] = own;
    __syncthreads();
    if (part != 0) return;
    if (lane < kW * R)
      for (int s = 1; s < split; ++s) own += red[warp + s][lane];
  }
  if (lane < kW * R && r < T && f0 + i < f.F) f.one<TX>(r, f0 + i, own);
}

// ---- 32 x 32 tiles ---------------------------------------------------------------------------------
constexpr int kT = 32, kK = 64, kLd = kT + 4;  // K in steps of 64; operands lie [k][32] in shared memory
constexpr int kGroups = 4;                     // groups of 64 threads, each a quarter of a step, 4 x 4 sums a thread

struct Steps {
  float a[kK][kLd], b[kK][kLd];
};

// Eight of 32 x 64 values of rows with K innermost: a warp eight of K, a lane a row.
template <bool VEC, typename T>
__device__ __forceinline__ void take_in(float (&v)[8], const T* from, long long ld, int rows, int k) {
  const int lane = threadIdx.x & 31, k0 = (threadIdx.x >> 5) * 8;
  const T* at = from + lane * ld + k0;
  if (VEC && lane < rows && k0 + 8 <= k) {
    RawSeg<true, T> raw;
    raw.load(at, 0, 0, 8);
    raw.values(v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = lane < rows && k0 + j < k ? to_f(at[j]) : 0.f;
}
// Eight of 64 x 32 values of rows that are K's: a warp eight of K, a lane a column.
template <typename T>
__device__ __forceinline__ void take_out(float (&v)[8], const T* from, long long ld, int cols, int k) {
  const int lane = threadIdx.x & 31, k0 = (threadIdx.x >> 5) * 8;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = k0 + j < k && lane < cols ? to_f(from[(k0 + j) * ld + lane]) : 0.f;
}

// What a thread holds of the next step while the products of this one run.
struct Next {
  float a[8], b[8], z[8];
};

// A tile's sums: thread t has row t / 8 and columns 4 (t mod 8) ..  load takes a step's values, turn(a, z) makes the first
// operand's of them.
template <typename Load, typename Turn>
__device__ __forceinline__ float4 tile_32(Steps (&s)[2], int K, Load load, Turn turn) {
  const int t = threadIdx.x & 63, g = threadIdx.x >> 6, lane = threadIdx.x & 31, k8 = (threadIdx.x >> 5) * 8;
  const int r = t / 8 * 4, c = t % 8 * 4;
  float acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
  Next n;
  load(n, 0, min(K, kK));
  for (int k0 = 0, at = 0; k0 < K; k0 += kK, at ^= 1) {
    turn(n.a, n.z, min(K - k0, kK) - k8);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[at].a[k8 + j][lane] = n.a[j];
      s[at].b[k8 + j][lane] = n.b[j];
    }
    __syncthreads();
    if (k0 + kK < K) load(n, k0 + kK, min(K - k0 - kK, kK));
#pragma unroll
    for (int k = 0; k < kK / kGroups; ++k) {
      const float4 a = *reinterpret_cast<const float4*>(&s[at].a[g * (kK / kGroups) + k][r]);
      const float4 b = *reinterpret_cast<const float4*>(&s[at].b[g * (kK / kGroups) + k][c]);
      const float x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
    }
  }
  // the groups' sums, in their order
  __syncthreads();
  float(*red)[kT][kLd] = reinterpret_cast<float(*)[kT][kLd]>(&s[0]);
  static_assert(kGroups * kT <= 2 * kK, "the groups' sums fit a step's place");
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<float4*>(&red[g][r + i][c]) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
  __syncthreads();
  const int row = threadIdx.x / 8, col = threadIdx.x % 8 * 4;
  float4 v = *reinterpret_cast<const float4*>(&red[0][row][col]);
#pragma unroll
  for (int q = 1; q < kGroups; ++q) {
    const float4 x = *reinterpret_cast<const float4*>(&red[q][row][col]);
    v.x += x.x;
    v.y += x.y;
    v.z += x.z;
    v.w += x.w;
  }
  return v;
}

template <typename T>
__device__ __forceinline__ void leave(const Finish& f, long long r0, int c0, int rows, int cols, float4 v) {
  const int row = threadIdx.x / 8, col = threadIdx.x % 8 * 4;
  if (row >= rows || col >= cols) return;
  if (f.vec) {
    f.four<T>(r0 + row, c0 + col, v, f.bias_of(c0 + col));
    return;
  }
  const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (col + j < cols) f.one<T>(r0 + row, c0 + col + j, e[j]);
}

template <typename TX, typename TW, bool VEC>
__global__ void __launch_bounds__(256) k_linear_small(const TX* __restrict__ X, long long ldx, const TW* __restrict__ W,
                                                      long long ldw, long long T, int C, const Finish f) {
  __shared__ __align__(16) Steps s[2];
  const int nt = (f.F + kT - 1) / kT;
  const long long r0 = (long long)(blockIdx.x / nt) * kT;
  const int c0 = (blockIdx.x % nt) * kT;
  const int rows = (int)min(T - r0, (long long)kT), cols = min(f.F - c0, kT);
  const float4 v = tile_32(
      s, C,
      [&](Next& n, int k0, int k) {
        take_in<VEC>(n.a, X + r0 * ldx + k0, ldx, rows, k);
        take_in<VEC>(n.b, W + c0 * ldw + k0, ldw, cols, k);
      },
      [](float(&)[8], const float(&)[8], int) {});
  leave<TX>(f, r0, c0, rows, cols, v);
}

// Blocks: the tiles of dx, then those of every chunk's G; the blocks of its first columns sum Gb, alone where G is not wanted.
template <typename TX, typename TW, bool VEC>
__global__ void __launch_bounds__(256)
    k_linear_grad_small(const TX* __restrict__ dy, long long lddy, const TX* __restrict__ z, long long ldz,
                        const TX* __restrict__ X, long long ldx, const TW* __restrict__ W, long long ldw, int act, int n_c,
                        long long T, int C, int ndx, const Finish f, int F, float* __restrict__ G, long long ldg,
                        float* __restrict__ Gb, long long ldgb) {
  __shared__ __align__(16) Steps s[2];
  const int ct = (C + kT - 1) / kT;
  // d of the step's values; past K they are zeros, which the slope of no z may touch
  auto slopes = [&](float(&d)[8], const float(&u)[8], int k) {
    if (act == GC_ACT_NONE) return;
    times_slope(act, u, d);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= k) d[j] = 0.f;
  };
  if ((int)blockIdx.x < ndx) {
    const long long r0 = (long long)(blockIdx.x / ct) * kT;
    const int c0 = (blockIdx.x % ct) * kT;
    const int rows = (int)min(T - r0, (long long)kT), cols = min(C - c0, kT);
    const float4 v = tile_32(
        s, F,
        [&](Next& n, int k0, int k) {
          take_in<VEC>(n.a, dy + r0 * lddy + k0, lddy, rows, k);
          if (act != GC_ACT_NONE) take_in<VEC>(n.z, z + r0 * ldz + k0, ldz, rows, k);
          take_out(n.b, W + k0 * ldw + c0, ldw, cols, k);
        },
        slopes);
    leave<TX>(f, r0, c0, rows, cols, v);
    return;
  }
  const int wide = G ? ct : 1, ft = (F + kT - 1) / kT;
  const int i = blockIdx.x - ndx, chunk = i / (ft * wide), at = i - chunk * ft * wide;
  const int f0 = at / wide * kT, c0 = at % wide * kT;
  const int rows = min(F - f0, kT), cols = G ? min(C - c0, kT) : 0;
  const long long t0 = (long long)chunk * n_c;
  float sum = 0.f;  // of d over the warp's points, a lane a column of d
  const float4 v = tile_32(
      s, n_c,
      [&](Next& n, int k0, int k) {
        take_out(n.a, dy + (t0 + k0) * lddy + f0, lddy, rows, k);
        if (act != GC_ACT_NONE) take_out(n.z, z + (t0 + k0) * ldz + f0, ldz, rows, k);
        take_out(n.b, G ? X + (t0 + k0) * ldx + c0 : X, ldx, cols, k);
      },
      [&](float(&d)[8], const float(&u)[8], int k) {
        slopes(d, u, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += d[j];
      });
  if (Gb && c0 == 0) {
    __syncthreads();
    s[0].a[threadIdx.x >> 5][threadIdx.x & 31] = sum;
    __syncthreads();
    if (threadIdx.x < 32 && (int)threadIdx.x < rows) {
      for (int w = 1; w < 8; ++w) sum += s[0].a[w][threadIdx.x];
      Gb[chunk * ldgb + f0 + threadIdx.x] = sum;
    }
  }
  const int row = threadIdx.x / 8, col = threadIdx.x % 8 * 4;
  if (!G || row >= rows) return;
  float* g = G + chunk * ldg + (long long)(f0 + row) * C + c0 + col;
  if (col + 4 <= cols && reinterpret_cast<uintptr_t>(g) % 16 == 0) {
    *reinterpret_cast<float4*>(g) = v;
    return;
  }
  const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (col + j < cols) g[j] = e[j];
}

template <typename TX, typename TW, bool VEC>
int launch_rows(const LinearShape& s, const LinearIO& io, const Finish& f, cudaStream_t st) {
  // warps that share a pair of rows, so that a few rows of W still fill the device
  const int segs = (s.C + kSeg - 1) / kSeg;
  int split = 1;
  while (split < 8 && split < segs && (long long)(s.F + kW - 1) / kW * split < 16LL * device_sm_count()) split *= 2;
  const int per = 8 / split * kW;
  const unsigned grid = (unsigned)((s.F + per - 1) / per);
  auto go = [&](auto kern) {
    return launch_chain(kern, "k_linear_rows", grid, 256, 0, 1, false, st, (const TX*)io.X, (long long)io.ldx, (const TW*)io.W,
                        (long long)io.ldw, (int)s.T, s.C, split, f);
  };
  return s.T == 1   ? go(k_linear_rows<TX, TW, VEC, 1>)
         : s.T == 2 ? go(k_linear_rows<TX, TW, VEC, 2>)
         : s.T <= 4 ? go(k_linear_rows<TX, TW, VEC, 4>)
                    : go(k_linear_rows<TX, TW, VEC, 8>);
}

template <typename TX, typename TW>
int launch_typed(const LinearShape& s, const LinearIO& io, const Finish& f, cudaStream_t st) {
  const bool vec = rowwise::rows_16(io.X, io.ldx, sizeof(TX)) && rowwise::rows_16(io.W, io.ldw, sizeof(TW));
  if (s.T <= kLinearRows)
    return vec && s.C % 8 == 0 ? launch_rows<TX, TW, true>(s, io, f, st) : launch_rows<TX, TW, false>(s, io, f, st);
  const unsigned grid = (unsigned)(((s.T + kT - 1) / kT) * ((s.F + kT - 1) / kT));
  return launch_chain(vec ? k_linear_small<TX, TW, true> : k_linear_small<TX, TW, false>, "k_linear_small", grid, 256, 0, 1, false,
                      st, (const TX*)io.X, (long long)io.ldx, (const TW*)io.W, (long long)io.ldw, s.T, s.C, f);
}

template <typename TX, typename TW>
int launch_grad_typed(const LinearGradShape& s, const LinearGradIO& io, const Finish& f, cudaStream_t st) {
  const bool vec = rowwise::rows_16(io.dy, io.lddy, sizeof(TX)) && rowwise::rows_16(s.act == GC_ACT_NONE ? nullptr : io.z, io.ldz, sizeof(TX));
  const int ct = (s.C + kT - 1) / kT, ft = (s.F + kT - 1) / kT;
  const long long T = (long long)s.N * s.n_c;
  const int ndx = io.dX ? (int)((T + kT - 1) / kT) * ct : 0;
  const int ng = io.G ? s.N * ft * ct : io.Gb ? s.N * ft : 0;
  return launch_chain(vec ? k_linear_grad_small<TX, TW, true> : k_linear_grad_small<TX, TW, false>, "k_linear_grad_small",
                      (unsigned)(ndx + ng), 256, 0, 1, false, st, (const TX*)io.dy, (long long)io.lddy, (const TX*)io.z,
                      (long long)io.ldz, (const TX*)io.X, (long long)io.ldx, (const TW*)io.W, (long long)io.ldw, s.act, s.n_c,
                      T, s.C, ndx, f, s.F, io.G, (long long)io.ldg, io.Gb, (long long)io.ldgb);
}

}  // namespace

int launch_linear_small(const LinearShape& s, const LinearIO& io, const linear::Finish& f, cudaStream_t st) {
  const bool wb = s.w_dtype == GC_BF16;
  if (s.x_dtype == GC_BF16)
    return wb ? launch_typed<__nv_bfloat16, __nv_bfloat16>(s, io, f, st) : launch_typed<__nv_bfloat16, float>(s, io, f, st);
  return wb ? launch_typed<float, __nv_bfloat16>(s, io, f, st) : launch_typed<float, float>(s, io, f, st);
}

int launch_linear_grad_small(const LinearGradShape& s, const LinearGradIO& io, const linear::Finish& f, cudaStream_t st) {
  const bool wb = s.w_dtype == GC_BF16;
  if (s.x_dtype == GC_BF16)
    return wb ? launch_grad_typed<__nv_bfloat16, __nv_bfloat16>(s, io, f, st)
              : launch_grad_typed<__nv_bfloat16, float>(s, io, f, st);
  return wb ? launch_grad_typed<float, __nv_bfloat16>(s, io, f, st)
            : launch_grad_typed<float, float>(s, io, f, st);
}

}  // namespace gc
