// Newton-Schulz orthogonalisation of small matrices (k_newton.cu's steps), in fp32 products and one launch: a cluster a matrix,
// whose CTAs hold a slice of the longer side each in shared memory.  A step is
//   A = X X^T,  Y = A X,  X <- a X + b Y + c A Y
// of which the last two need the CTA's own slice alone.  A CTA sends its part of A, by rows, to the CTAs that add them up,
// and those send the sums to all: two barriers of the cluster a step, and no load waits for another SM.
//
// Bound: latency, the barriers and some 10^3 products a thread and step.
#include <cooperative_groups.h>

#include <algorithm>

#include "newton.cuh"
#include "tc_host.cuh"

namespace gc {
namespace {

namespace cg = cooperative_groups;

constexpr int kSide = 64;         // the shorter side at most
constexpr int kSlice = 256;       // a CTA's part of the longer side at most
constexpr int kMostCtas = 8;
constexpr int kLd = kSide + 4;    // the slice lies [k][kLd], the m x m matrices [i][kLd]
constexpr int kPartRows = kSide + 4 * kMostCtas;  // rows of all CTAs' parts, each CTA's a multiple of four
constexpr int kThreads = 256;
constexpr size_t smem_bytes(int slice) { return (size_t)(2 * slice + kPartRows + kSide) * kLd * sizeof(float); }
static_assert(smem_bytes(kSlice) + 256 <= kSmemMax, "shared memory");

struct Cut {
  int ctas, slice;
  double us;  // a step's time, all waves of matrices
};
// The cluster whose estimated time is least: barriers and phases some 2 us, three products of 4 x 4 sums a thread.
Cut cut_of(const NsShape& s) {
  const int m = std::min(s.rows, s.cols), n = std::max(s.rows, s.cols);
  Cut best{0, 0, 1e30};
  for (int c = 1; c <= kMostCtas; c *= 2) {
    const int slice = ((n + c - 1) / c + 3) / 4 * 4;
    if (slice > kSlice) continue;
    const double waves = (double)(((long long)s.batch * c + device_sm_count() - 1) / device_sm_count());
    const double us = waves * (2 + 3.0 * m * m * slice / 120000);
    if (us < best.us) best = Cut{c, slice, us};
  }
  return best;
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T, bool MOM>
__global__ void __launch_bounds__(kThreads) k_ns_small(const NsShape s, const NsIO io, int slice) {
  extern __shared__ __align__(16) float sm[];
  __shared__ double red[kThreads / 32], total;
  __shared__ float factor[3];
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int mat = blockIdx.x / ctas, tid = threadIdx.x, lane = tid & 31;
  const bool wide = s.rows <= s.cols;
  const int m = min(s.rows, s.cols), n = max(s.rows, s.cols), mp = (m + 3) / 4 * 4;
  const int first = rank * slice, kn = max(0, min(n - first, slice));
  float *X = sm, *Y = X + slice * kLd, *parts = Y + slice * kLd, *A = parts + kPartRows * kLd;
  auto sync = [&] {
    if (ctas > 1)
      cluster.sync();
    else
      __syncthreads();
  };
  for (int i = tid; i < slice * kLd; i += kThreads) X[i] = 0.f;
  __syncthreads();

  // the slice of u, and the sum of its squares; neighbouring threads neighbouring columns of u
  const T* u = reinterpret_cast<const T*>(io.u) + mat * io.su;
  float* mom = MOM ? io.m + mat * io.sm : nullptr;
  const int inner = wide ? kn : m, count = kn * m;
  auto place = [&](int e, long long* row, int* col) {  // element e's place in u; returns its place in X
    const int o = e / inner, i = e - o * inner;
    *row = wide ? o : first + o;
    *col = wide ? first + i : i;
    return wide ? i * kLd + o : o * kLd + i;
  };
  double sum = 0;
  for (int e0 = tid; e0 < count; e0 += 4 * kThreads) {
    float v[4], q = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = e0 + j * kThreads;
      v[j] = 0.f;
      if (e >= count) continue;
      long long row;
      int col;
      const int at = place(e, &row, &col);
      if (MOM) {
        const float g = __fdiv_rn(to_f(u[row * io.ldu + col]), io.points);
        float* to = mom + row * io.ldm + col;
        v[j] = __fmaf_rn(io.mu, *to, g);
        *to = v[j];
        if (io.nesterov) v[j] = __fmaf_rn(io.mu, v[j], g);
      } else {
        v[j] = to_f(u[row * io.ldu + col]);
      }
      X[at] = v[j];
      q = fmaf(v[j], v[j], q);
    }
    add_squares(q, v, sum);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) red[tid >> 5] = sum;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kThreads / 32; ++w) sum += red[w];
    total = sum;
  }
  sync();
  if (tid == 0) {
    sum = 0;
    for (int r = 0; r < ctas; ++r) sum += *cluster.map_shared_rank(&total, r);
    norm_factors(sum, io.eps, 1.f, 1.f, factor);  // fp32 needs no other scale for a small norm
  }
  __syncthreads();
  const float p0 = factor[0], p1 = factor[1], r1 = factor[2];
  for (int i = tid; i < slice * kLd; i += kThreads) X[i] = X[i] * p0 * p1 * r1;

  const int side = mp / 4, tiles = side * side;
  const int each = ((mp + ctas - 1) / ctas + 3) / 4 * 4, row0 = min(rank * each, mp), rows = min(each, mp - row0);
  int share = 1;  // threads of a tile of A, which split its sum; 16 x 2000 has 16 tiles
  while (share < 32 && tiles * share * 2 <= kThreads) share *= 2;
  const int groups = (kn + 3) / 4;  // of the slice's columns, which are padded to a multiple of four
  const float a = s.coeffs[0], b = s.coeffs[1], c = s.coeffs[2];
  // f(k, i, sums): M S for columns k .. k + 3 of the slice S and rows i .. i + 3, a thread 4 x 4.  M is symmetric to the
  // last bit: the products and sums of its halves are the same.
  auto product = [&](const float* M, const float* S, auto f) {
    for (int t = tid; t < side * groups; t += kThreads) {
      const int i = t % side * 4, k = t / side * 4;
      float acc[4][4] = {};
#pragma unroll 2
      for (int j = 0; j < mp; j += 4) {
        float p[4][4], x[4][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 v = *reinterpret_cast<const float4*>(M + (j + e) * kLd + i);
          const float4 w = *reinterpret_cast<const float4*>(S + (k + e) * kLd + j);
          p[e][0] = v.x, p[e][1] = v.y, p[e][2] = v.z, p[e][3] = v.w;
          x[e][0] = w.x, x[e][1] = w.y, x[e][2] = w.z, x[e][3] = w.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int g = 0; g < 4; ++g) acc[e][h] = fmaf(x[e][g], p[g][h], acc[e][h]);
      }
      f(k, i, acc);
    }
  };
  for (int step = 0; step < s.steps; ++step) {
    __syncthreads();
    // the slice's part of A, 4 x 4 a thread or `share` neighbouring ones, to the CTA of its rows
    for (int t = tid; t - tid < tiles * share; t += kThreads) {
      const int tile = min(t / share, tiles - 1), g = t % share;
      const int i = tile / side * 4, j = tile % side * 4, o = i / each;
      float acc[4][4] = {};
#pragma unroll 4
      for (int k = g; k < kn; k += share) {
        const float4 p = *reinterpret_cast<const float4*>(X + k * kLd + i), q = *reinterpret_cast<const float4*>(X + k * kLd + j);
        const float x[4] = {p.x, p.y, p.z, p.w}, y[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int f = 0; f < 4; ++f) acc[e][f] = fmaf(x[e], y[f], acc[e][f]);
      }
      for (int w = 1; w < share; w *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int f = 0; f < 4; ++f) acc[e][f] += __shfl_xor_sync(0xffffffffu, acc[e][f], w);
      if (t >= tiles * share) break;
      float* to = ctas == 1 ? A + i * kLd : cluster.map_shared_rank(parts, o) + (rank * each + i - o * each) * kLd;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((e & (share - 1)) == g)
          *reinterpret_cast<float4*>(to + e * kLd + j) = make_float4(acc[e][0], acc[e][1], acc[e][2], acc[e][3]);
    }
    sync();
    if (ctas > 1) {
      for (int t = tid; t < rows * side; t += kThreads) {
        const int r = t / side, q = t % side * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int o = 0; o < ctas; ++o) {
          const float4 x = *reinterpret_cast<const float4*>(parts + (o * each + r) * kLd + q);
          v.x += x.x;
          v.y += x.y;
          v.z += x.z;
          v.w += x.w;
        }
#pragma unroll 8
        for (int o = 0; o < ctas; ++o)
          *reinterpret_cast<float4*>(cluster.map_shared_rank(A, o) + (row0 + r) * kLd + q) = v;
      }
      cluster.sync();
    }
    product(A, X, [&](int k, int i, const float(&acc)[4][4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<float4*>(Y + (k + e) * kLd + i) = make_float4(acc[e][0], acc[e][1], acc[e][2], acc[e][3]);
    });
    __syncthreads();
    product(A, Y, [&](int k, int i, const float(&acc)[4][4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float4* at = reinterpret_cast<float4*>(X + (k + e) * kLd + i);
        const float4 x = *at, y = *reinterpret_cast<const float4*>(Y + (k + e) * kLd + i);
        *at = make_float4(fmaf(c, acc[e][0], fmaf(b, y.x, a * x.x)), fmaf(c, acc[e][1], fmaf(b, y.y, a * x.y)),
                          fmaf(c, acc[e][2], fmaf(b, y.z, a * x.z)), fmaf(c, acc[e][3], fmaf(b, y.w, a * x.w)));
      }
    });
  }
  __syncthreads();
  for (int e = tid; e < count; e += kThreads) {
    long long row;
    int col;
    const float v = X[place(e, &row, &col)];
    T* to = reinterpret_cast<T*>(io.out) + mat * io.so + row * io.ldo + col;
    if (MOM)
      *reinterpret_cast<float*>(to) = fmaf(io.step, v, io.keep * *reinterpret_cast<float*>(to));
    else if (sizeof(T) == 2)
      *reinterpret_cast<__nv_bfloat16*>(to) = __float2bfloat16_rn(v);
    else
      *reinterpret_cast<float*>(to) = v;
  }
  // A CTA leaves after the last barrier of the last step, when nothing of its memory is read or written from elsewhere.
}

template <typename T, bool MOM>
int launch(const NsShape& s, const NsIO& io, cudaStream_t st) {
  static SmemOptIn allow;
  GC_CUDA(allow(k_ns_small<T, MOM>, smem_bytes(kSlice)));
  const Cut cut = cut_of(s);
  return launch_chain(k_ns_small<T, MOM>, "k_ns_small", (unsigned)(s.batch * cut.ctas), kThreads, smem_bytes(cut.slice), cut.ctas,
                      false, st, s, io, cut.slice);
}

}  // namespace

// Tiles take some 24 us a step, however small the matrices.
bool ns_small(const NsShape& s) { return std::min(s.rows, s.cols) <= kSide && cut_of(s).us <= 20; }

int launch_ns_small(const NsShape& s, const NsIO& io, cudaStream_t st) {
  if (io.m) return launch<float, true>(s, io, st);
  return s.dtype == GC_BF16 ? launch<__nv_bfloat16, false>(s, io, st) : launch<float, false>(s, io, st);
}

}  // namespace gc
