// Layer norm with an optional residual branch and dropout before it, and its gradient.
//   forward   h = residual + D(x);  mu, rstd of each row of h;  y = (h - mu) rstd gamma + beta
//   backward  n = (h - mu) rstd, a = dy gamma;
//             dresidual = rstd (a - mean(a) - n mean(a n)) + dh;  dx = D(dresidual);
//             per chunk of rows  G_i = [sum dy n, sum dy]
//
// Bound: HBM.  A row stays in registers between the statistics and the output, so each input is read
// once.  The row's sums go through one exchange: a warp forms the sum of its values and their squares
// about its own mean, and the warps' parts are merged exactly,
//   M2 = sum_w M2_w + n_w (mu_w - mu)^2,
// with no loss where the mean is large against the spread (all in fp32).  The statistics are those
// of h before it is rounded for the store.
//
// Backward: a block takes a range of rows of one chunk and keeps the column sums in registers, so
// that dy and h are read once for dx and G together; the blocks' sums of a chunk are added in a fixed
// order by a second kernel.  Rows wider than kFusedCols do not leave room for the sums: their column
// sums come from a pass of their own, before dx may be written over dy.
#include <algorithm>

#include "rowwise.cuh"

namespace gc {
namespace {

using namespace rowwise;

constexpr int kFusedCols = 8192;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// s / n to the last digit or so where 1 / n is at hand: s * (1 / n) and one correction.
__device__ __forceinline__ float div_by(float s, float n, float inv) {
  const float q = s * inv;
  return fmaf(fmaf(-q, n, s), inv, q);
}
// The sum over the first W lanes (a power of two; the others hold zeros), in every lane of them.
template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = W / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return W < 32 ? __shfl_sync(0xffffffffu, v, 0) : v;
}

// The eight values at the segment's columns of a per-column vector, `dflt` where there is none.
template <bool VEC>
__device__ __forceinline__ void load_cols(const float* p, float dflt, bool vec, int col0, int lane,
                                          int cols, float (&v)[8]) {
  if (p && VEC && vec) {
    load_seg<true>(p, col0, lane, cols, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = seg_col<VEC>(col0, lane, j);
      v[j] = p && c < cols ? __ldg(p + c) : dflt;
    }
  }
}

struct NormArgs {
  const void *x, *res;
  const float *gamma, *beta;
  void *y, *h;
  float *mean, *rstd;
  long long ldx, ldr, ldy, ldh, rows;
  int cols, vec_cols;  // vec_cols: gamma and beta on 16-byte boundaries
  float eps;
  Mask m;
};

// TPR threads a row, VPT segments a warp of them.  A warp a row: four rows a block, no barrier.  Up to two
// segments a warp the next row is on its way while this one is worked on.  What bounds it then is the
// instructions: a row's exchange is the same hundred a lane for one segment or for two.  (16,384 rows of
// 4096 bf16 with dropout and residual, 537 MB: four segments and no row ahead 155 us, one and a row ahead 105, two 102,
// and 92 with two-wide arithmetic; 65,536 rows of 1024: one 110, two 100, two-wide 91.)
template <typename T, bool VEC, int TPR, int VPT>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR, TPR == 32 ? 8 : 1024 / TPR)
    k_norm(NormArgs a) {
  constexpr int WPR = TPR / 32;                       // warps a row
  constexpr int RPB = TPR == 32 ? 4 : 1;              // rows a block
  constexpr bool AHEAD = VPT <= 2;
  __shared__ float2 part[2][WPR];
  const int lane = threadIdx.x & 31;
  const int warp = TPR == 32 ? 0 : threadIdx.x >> 5;
  const long long step = (long long)gridDim.x * RPB;
  long long row = (long long)blockIdx.x * RPB + (TPR == 32 ? threadIdx.x >> 5 : 0);
  RawSeg<VEC, T> x[VPT], r[VPT];
  int n_w = 0, n_l = 0;  // columns of this warp, and of warp `lane`
#pragma unroll
  for (int q = 0; q < VPT; ++q) {
    n_w += max(0, min(kSeg, a.cols - (q * WPR + warp) * kSeg));
    if (lane < WPR) n_l += max(0, min(kSeg, a.cols - (q * WPR + lane) * kSeg));
  }
  const float fn_w = (float)n_w, fn_l = (float)n_l, fn = (float)a.cols;
  const float inv_w = n_w ? 1.f / fn_w : 0.f, inv_l = n_l ? 1.f / fn_l : 0.f, inv = 1.f / fn;
  auto fetch = [&](long long at) {
#pragma unroll
    for (int q = 0; q < VPT; ++q) x[q].load((const T*)a.x + at * a.ldx, (q * WPR + warp) * kSeg, lane, a.cols);
    if (a.res) {
#pragma unroll
      for (int q = 0; q < VPT; ++q) r[q].load((const T*)a.res + at * a.ldr, (q * WPR + warp) * kSeg, lane, a.cols);
    }
  };
  if (AHEAD && row < a.rows) fetch(row);
  int flip = 0;
  for (; row < a.rows; row += step, flip ^= 1) {
    float v[VPT][8];
    if (!AHEAD) fetch(row);
#pragma unroll
    for (int q = 0; q < VPT; ++q) {
      x[q].values(v[q]);
      if (a.m.t) drop_seg<VEC>(a.m, row, (q * WPR + warp) * kSeg, lane, v[q]);
      if (a.res) {
        float t[8];
        r[q].values(t);
#pragma unroll
        for (int j = 0; j < 4; ++j) put(v[q], j, __fadd2_rn(two(v[q], j), two(t, j)));
      }
    }
    if (AHEAD && row + step < a.rows) fetch(row + step);
    if (a.h) {
#pragma unroll
      for (int q = 0; q < VPT; ++q)
        store_seg<VEC>((T*)a.h + row * a.ldh, (q * WPR + warp) * kSeg, lane, a.cols, v[q]);
    }
    // the warp's sum, and its squares about its own mean
    float2 pair = both(0.f);
#pragma unroll
    for (int q = 0; q < VPT; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) pair = __fadd2_rn(pair, two(v[q], j));
    const float s = warp_sum(pair.x + pair.y);
    const float mu_w = div_by(s, fn_w, inv_w);
    pair = both(0.f);
#pragma unroll
    for (int q = 0; q < VPT; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float2 d = __fadd2_rn(two(v[q], j), both(-mu_w));
        const int col0 = (q * WPR + warp) * kSeg;
        if (!in_row<VEC>(col0, lane, 2 * j, a.cols)) d.x = 0.f;
        if (!in_row<VEC>(col0, lane, 2 * j + 1, a.cols)) d.y = 0.f;
        pair = __ffma2_rn(d, d, pair);
      }
    const float m2 = warp_sum(pair.x + pair.y);
    float mu = mu_w, M2 = m2;
    if (WPR > 1) {
      if (lane == 0) part[flip][warp] = make_float2(s, m2);
      __syncthreads();  // the two buffers alternate: one barrier a row
      // lane w merges warp w's part
      const float2 p = lane < WPR ? part[flip][lane] : make_float2(0.f, 0.f);
      mu = div_by(lanes_sum<WPR>(p.x), fn, inv);
      const float d = div_by(p.x, fn_l, inv_l) - mu;
      M2 = lanes_sum<WPR>(fmaf(fn_l * d, d, p.y));
    }
    const float rstd = rsqrtf(M2 * inv + a.eps);
    if (warp == 0 && lane == 0) {
      if (a.mean) a.mean[row] = mu;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int q = 0; q < VPT; ++q) {
      const int col0 = (q * WPR + warp) * kSeg;
      float g[8], b[8];
      load_cols<VEC>(a.gamma, 1.f, a.vec_cols, col0, lane, a.cols, g);
      load_cols<VEC>(a.beta, 0.f, a.vec_cols, col0, lane, a.cols, b);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        put(v[q], j, __ffma2_rn(__fmul2_rn(__fadd2_rn(two(v[q], j), both(-mu)), both(rstd)), two(g, j), two(b, j)));
      store_seg<VEC>((T*)a.y + row * a.ldy, col0, lane, a.cols, v[q]);
    }
  }
}

template <typename T, bool VEC, int TPR, int VPT>
int go_norm(const NormArgs& a, cudaStream_t s) {
  constexpr int RPB = TPR == 32 ? 4 : 1;
  constexpr int threads = TPR == 32 ? 128 : TPR;
  const long long blocks = (a.rows + RPB - 1) / RPB;
  // bf16 rows without dropout leave the SMs idle half the time, and fewer rows at once suit the memory better:
  // 2^26 values with residual by 768 and 1024 threads an SM, rows of 1024 columns 88 and 98 us, of 2048 84 and 96, of
  // 4096 83 and 94; of 256 95 and 86, and without residual 60 and 57.  With dropout 95 and 91 (4096); fp32 with
  // residual 177 and 169, without 112 and 102.
  const int per_sm = sizeof(T) == 2 && !a.m.t && threads <= 256 ? 768 : 1024;
  const long long grid = std::min<long long>(blocks, (long long)device_sm_count() * (per_sm / threads));
  k_norm<T, VEC, TPR, VPT><<<(unsigned)grid, threads, 0, s>>>(a);
  count_launches(1);
  return cuda_check(cudaGetLastError(), "k_norm");
}

// Two segments a warp up to 16384 columns (but for one that fills a block), 1024 threads an SM; wider rows
// by four.
template <typename T, bool VEC>
int norm_by_width(const NormArgs& a, cudaStream_t s) {
  const int c = a.cols;
  if (c <= 256) return go_norm<T, VEC, 32, 1>(a, s);
  if (c <= 512) return go_norm<T, VEC, 32, 2>(a, s);
  if (c <= 1024) return go_norm<T, VEC, 64, 2>(a, s);
  if (c <= 2048) return go_norm<T, VEC, 128, 2>(a, s);
  if (c <= 4096) return go_norm<T, VEC, 256, 2>(a, s);
  if (c <= 8192) return go_norm<T, VEC, 1024, 1>(a, s);  // 210 us for 16,384 rows of 8192, 225 by two segments
  if (c <= 16384) return go_norm<T, VEC, 1024, 2>(a, s);
  return go_norm<T, VEC, 1024, 4>(a, s);
}

// ------------------------------------------------------------------------------------ backward
struct NormGradArgs {
  const void *dy, *h, *dh;
  const float *mean, *rstd, *gamma;
  void *dx, *dres;
  float* sums;         // per (chunk, slice) 2 * cols column sums: G itself or partial ones
  long long sums_ld;   // between slices
  long long lddy, ldh, lddh, lddx, lddr;
  int slices;
  uint32_t n_c, rows_per_slice;  // a slice's end, and the row after a chunk's last, may be past 2^31
  int cols, vec_cols;
  Mask m;
};

// TPR threads a row, two segments a warp; a block takes a slice of a chunk's rows, the next one on its way
// while one is worked on.  SUMS: the column sums for G as well.  512 threads an SM have registers for
// all that.  (16,384 rows of 4096 bf16 with residual, 671 MB, with dropout and without it: no row ahead 168 us;
// one segment a warp, 1024 threads 144 and 123; two 133 and 125; two, 768 threads, which spill, 179 and 165;
// two with two-wide arithmetic 129 and 122.)
constexpr int kGradSegs = 2;
constexpr int kGradThreads = 512;  // an SM
template <typename T, bool VEC, int TPR, bool SUMS>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR, TPR == 32 ? kGradThreads / 128 : kGradThreads / TPR)
    k_norm_grad(NormGradArgs a) {
  constexpr int WPR = TPR / 32, RPB = TPR == 32 ? 4 : 1, Q = kGradSegs;
  __shared__ float2 part[2][WPR];
  const int lane = threadIdx.x & 31;
  const int warp = TPR == 32 ? 0 : threadIdx.x >> 5;
  const int chunk = blockIdx.x / a.slices, slice = blockIdx.x - chunk * a.slices;
  const uint32_t r_end = min(a.n_c, (slice + 1) * a.rows_per_slice);
  uint32_t r = slice * a.rows_per_slice + (TPR == 32 ? threadIdx.x >> 5 : 0);
  const long long first = (long long)chunk * a.n_c;
  float sg[Q][8], sb[Q][8];
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int j = 0; j < 8; ++j) sg[q][j] = sb[q][j] = 0.f;
  const float inv = 1.f / (float)a.cols;
  RawSeg<VEC, T> xd[Q], xh[Q], xa[Q];
  float mu, rstd;
  auto fetch = [&](long long row) {
    mu = __ldg(a.mean + row);
    rstd = __ldg(a.rstd + row);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int col0 = (q * WPR + warp) * kSeg;
      xd[q].load((const T*)a.dy + row * a.lddy, col0, lane, a.cols);
      xh[q].load((const T*)a.h + row * a.ldh, col0, lane, a.cols);
      if (a.dh) xa[q].load((const T*)a.dh + row * a.lddh, col0, lane, a.cols);
    }
  };
  if (r < r_end) fetch(first + r);
  int flip = 0;
  for (; r < r_end; r += RPB, flip ^= 1) {
    const long long row = first + r;
    float d[Q][8], n[Q][8];
    float2 p1 = both(0.f), p2 = both(0.f);
    RawSeg<VEC, T> ya[Q];
    const float scale = rstd;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int col0 = (q * WPR + warp) * kSeg;
      float g[8];
      load_cols<VEC>(a.gamma, 1.f, a.vec_cols, col0, lane, a.cols, g);
      xd[q].values(d[q]);
      xh[q].values(n[q]);
      ya[q] = xa[q];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // h - mean; rstd is left to y and to the row's sum.  Past the row's end that is -mean, and dy zero:
        // n, which need not be finite there, is not formed
        const float2 y = two(d[q], j), x = __fadd2_rn(two(n[q], j), both(-mu));
        if (SUMS) {
          put(sg[q], j, __ffma2_rn(__fmul2_rn(y, both(scale)), x, two(sg[q], j)));
          put(sb[q], j, __fadd2_rn(y, two(sb[q], j)));
        }
        const float2 e = __fmul2_rn(y, two(g, j));
        p1 = __fadd2_rn(p1, e);
        p2 = __ffma2_rn(e, x, p2);
        put(n[q], j, x);
        put(d[q], j, e);
      }
    }
    if (r + RPB < r_end) fetch(row + RPB);
    float c1 = warp_sum(p1.x + p1.y), c2 = warp_sum(p2.x + p2.y);
    if (WPR > 1) {
      if (lane == 0) part[flip][warp] = make_float2(c1, c2);
      __syncthreads();
      const float2 p = lane < WPR ? part[flip][lane] : make_float2(0.f, 0.f);
      c1 = lanes_sum<WPR>(p.x);
      c2 = lanes_sum<WPR>(p.y);
    }
    c1 *= inv;
    c2 = c2 * inv * scale * scale;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int col0 = (q * WPR + warp) * kSeg;
      float t[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (a.dh) ya[q].values(t);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 e = __ffma2_rn(two(n[q], j), both(-c2), __fadd2_rn(two(d[q], j), both(-c1)));
        put(d[q], j, __ffma2_rn(e, both(scale), two(t, j)));
      }
      if (a.dres) store_seg<VEC>((T*)a.dres + row * a.lddr, col0, lane, a.cols, d[q]);
      if (a.dx) {
        if (a.m.t) drop_seg<VEC>(a.m, row, col0, lane, d[q]);
        store_seg<VEC>((T*)a.dx + row * a.lddx, col0, lane, a.cols, d[q]);
      }
    }
  }
  if (!SUMS) return;
  // the block's column sums; where a warp takes a row, the four warps' in order
  float* out = a.sums + (size_t)blockIdx.x * a.sums_ld;
  if constexpr (TPR == 32) {
    __shared__ float acc[4][Q * kSeg];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          acc[threadIdx.x >> 5][seg_col<VEC>(q * kSeg, lane, j)] = which ? sb[q][j] : sg[q][j];
      __syncthreads();
      for (int c = threadIdx.x; c < a.cols; c += 128)
        out[(size_t)which * a.cols + c] = acc[0][c] + acc[1][c] + acc[2][c] + acc[3][c];
    }
  } else {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = seg_col<VEC>((q * WPR + warp) * kSeg, lane, j);
        if (c < a.cols) {
          out[c] = sg[q][j];
          out[(size_t)a.cols + c] = sb[q][j];
        }
      }
  }
}

// dx and dresidual of rows too wide for k_norm_grad's registers: a block a row, read twice (the
// second time from the cache).
template <typename T, bool VEC>
__global__ void __launch_bounds__(1024) k_norm_grad_wide(NormGradArgs a, long long rows) {
  __shared__ float2 part[2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float inv = 1.f / (float)a.cols;
  int flip = 0;
  for (long long row = blockIdx.x; row < rows; row += gridDim.x, flip ^= 1) {
    const float mu = __ldg(a.mean + row), rstd = __ldg(a.rstd + row);
    const T* dyr = (const T*)a.dy + row * a.lddy;
    const T* hr = (const T*)a.h + row * a.ldh;
    float c1 = 0.f, c2 = 0.f;
    for (int col0 = warp * kSeg; col0 < a.cols; col0 += 32 * kSeg) {
      float d[8], n[8], g[8];
      load_seg<VEC>(dyr, col0, lane, a.cols, d);
      load_seg<VEC>(hr, col0, lane, a.cols, n);
      load_cols<VEC>(a.gamma, 1.f, a.vec_cols, col0, lane, a.cols, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (seg_col<VEC>(col0, lane, j) < a.cols) {
          c1 = fmaf(d[j], g[j], c1);
          c2 = fmaf(d[j] * g[j], (n[j] - mu) * rstd, c2);
        }
      }
    }
    c1 = warp_sum(c1);
    c2 = warp_sum(c2);
    if (lane == 0) part[flip][warp] = make_float2(c1, c2);
    __syncthreads();
    c1 = warp_sum(part[flip][lane].x) * inv;
    c2 = warp_sum(part[flip][lane].y) * inv;
    for (int col0 = warp * kSeg; col0 < a.cols; col0 += 32 * kSeg) {
      float d[8], n[8], g[8], t[8];
      load_seg<VEC>(dyr, col0, lane, a.cols, d);
      load_seg<VEC>(hr, col0, lane, a.cols, n);
      load_cols<VEC>(a.gamma, 1.f, a.vec_cols, col0, lane, a.cols, g);
      if (a.dh) load_seg<VEC>((const T*)a.dh + row * a.lddh, col0, lane, a.cols, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = rstd * (d[j] * g[j] - c1 - (n[j] - mu) * rstd * c2);
        d[j] = a.dh ? v + t[j] : v;
      }
      if (a.dres) store_seg<VEC>((T*)a.dres + row * a.lddr, col0, lane, a.cols, d);
      if (a.dx) {
        if (a.m.t) drop_seg<VEC>(a.m, row, col0, lane, d);
        store_seg<VEC>((T*)a.dx + row * a.lddx, col0, lane, a.cols, d);
      }
    }
  }
}

// Column sums of rows too wide for k_norm_grad's: a thread a column, a block a range of rows.
template <typename T>
__global__ void __launch_bounds__(256) k_norm_cols(NormGradArgs a) {
  const int c = blockIdx.y * 256 + threadIdx.x;
  const int chunk = blockIdx.x / a.slices, slice = blockIdx.x - chunk * a.slices;
  const uint32_t r_end = min(a.n_c, (slice + 1) * a.rows_per_slice);
  if (c >= a.cols) return;
  float sg = 0.f, sb = 0.f;
#pragma unroll 4
  for (uint32_t r = slice * a.rows_per_slice; r < r_end; ++r) {
    const long long row = (long long)chunk * a.n_c + r;
    const float d = to_f(((const T*)a.dy)[row * a.lddy + c]);
    const float n = (to_f(((const T*)a.h)[row * a.ldh + c]) - __ldg(a.mean + row)) * __ldg(a.rstd + row);
    sg = fmaf(d, n, sg);
    sb += d;
  }
  float* out = a.sums + (size_t)blockIdx.x * a.sums_ld;
  out[c] = sg;
  out[(size_t)a.cols + c] = sb;
}

// G_i = the slices' sums in a fixed order: eight interleaved groups, then the groups.
__global__ void __launch_bounds__(256) k_norm_grad_reduce(const float* __restrict__ part, int slices,
                                                          int cols2, float* __restrict__ G, long long ldg) {
  __shared__ float acc[8][32];
  const int x = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + x;
  const float* p = part + (size_t)blockIdx.y * slices * cols2;
  float s = 0.f;
  if (c < cols2) {
#pragma unroll 4
    for (int k = g; k < slices; k += 8) s += p[(size_t)k * cols2 + c];
  }
  acc[g][x] = s;
  __syncthreads();
  if (g == 0 && c < cols2) {
#pragma unroll
    for (int k = 1; k < 8; ++k) s += acc[k][x];
    G[(long long)blockIdx.y * ldg + c] = s;
  }
}

// Threads a row of the fused form.
int grad_tpr(int cols) {
  int t = 32;
  while (t * 8 * kGradSegs < cols) t *= 2;
  return t;
}

struct Slices {
  int count, rows;
};
// Row ranges of a chunk: enough blocks of `threads` for every SM to hold kGradThreads, at least four or
// eight rows a warp (the sums of a range are written and read once more).
Slices slices_of(int N, int n_c, int threads, int min_rows) {
  const long long blocks = (long long)device_sm_count() * std::max(1, kGradThreads / threads);
  long long want = std::max<long long>(1, blocks / N);
  want = std::min<long long>(want, ((long long)n_c + min_rows - 1) / min_rows);
  const long long rows = (n_c + want - 1) / want;
  return {(int)((n_c + rows - 1) / rows), (int)rows};
}
Slices grad_slices(int N, int n_c, int cols) {
  if (cols > kFusedCols) return slices_of(N, n_c, 256, 32);
  const int tpr = grad_tpr(cols);
  return slices_of(N, n_c, tpr == 32 ? 128 : tpr, tpr == 32 ? 32 : 4);
}

template <typename T, bool VEC, int TPR, bool SUMS>
int go_grad(const NormGradArgs& a, int N, cudaStream_t s) {
  k_norm_grad<T, VEC, TPR, SUMS><<<(unsigned)(N * a.slices), TPR == 32 ? 128 : TPR, 0, s>>>(a);
  count_launches(1);
  return cuda_check(cudaGetLastError(), "k_norm_grad");
}

template <typename T, bool VEC, bool SUMS>
int grad_by_width(const NormGradArgs& a, int N, cudaStream_t s) {
  switch (grad_tpr(a.cols)) {
    case 32: return go_grad<T, VEC, 32, SUMS>(a, N, s);
    case 64: return go_grad<T, VEC, 64, SUMS>(a, N, s);
    case 128: return go_grad<T, VEC, 128, SUMS>(a, N, s);
    case 256: return go_grad<T, VEC, 256, SUMS>(a, N, s);
    default: return go_grad<T, VEC, 512, SUMS>(a, N, s);
  }
}

template <typename T>
int grad_run(NormGradArgs a, int N, float* G, long long ldg, float* part, bool vec, cudaStream_t s) {
  const Slices sl = grad_slices(N, a.n_c, a.cols);
  a.slices = sl.count;
  a.rows_per_slice = sl.rows;
  const bool direct = sl.count == 1;
  a.sums = direct ? G : part;
  a.sums_ld = direct ? ldg : 2LL * a.cols;
  int rc = GC_OK;
  if (a.cols > kFusedCols) {
    if (G) {
      const dim3 grid((unsigned)(N * sl.count), (unsigned)((a.cols + 255) / 256));
      k_norm_cols<T><<<grid, 256, 0, s>>>(a);
      count_launches(1);
      rc = cuda_check(cudaGetLastError(), "k_norm_cols");
    }
    if (rc == GC_OK && (a.dx || a.dres)) {
      const long long rows = (long long)N * a.n_c;
      const unsigned grid = (unsigned)std::min<long long>(rows, 2LL * device_sm_count());
      if (vec)
        k_norm_grad_wide<T, true><<<grid, 1024, 0, s>>>(a, rows);
      else
        k_norm_grad_wide<T, false><<<grid, 1024, 0, s>>>(a, rows);
      count_launches(1);
      rc = cuda_check(cudaGetLastError(), "k_norm_grad_wide");
    }
  } else if (G) {
    rc = vec ? grad_by_width<T, true, true>(a, N, s) : grad_by_width<T, false, true>(a, N, s);
  } else {
    rc = vec ? grad_by_width<T, true, false>(a, N, s) : grad_by_width<T, false, false>(a, N, s);
  }
  if (rc != GC_OK || !G || direct) return rc;
  k_norm_grad_reduce<<<dim3((unsigned)((2 * a.cols + 31) / 32), (unsigned)N), 256, 0, s>>>(
      part, sl.count, 2 * a.cols, G, ldg);
  count_launches(1);
  return cuda_check(cudaGetLastError(), "k_norm_grad_reduce");
}

}  // namespace

int launch_norm(const NormIO& io, int dtype, int64_t rows, int cols, float eps, const DropArgs& d,
                cudaStream_t s) {
  NormArgs a{};
  a.x = io.x;
  a.res = io.res;
  a.gamma = io.gamma;
  a.beta = io.beta;
  a.y = io.y;
  a.h = io.h;
  a.mean = io.mean;
  a.rstd = io.rstd;
  a.ldx = io.ldx;
  a.ldr = io.ldr;
  a.ldy = io.ldy;
  a.ldh = io.ldh;
  a.rows = rows;
  a.cols = cols;
  a.eps = eps;
  a.m = make_mask(d.p, d.seed, d.offset, d.row0, cols);
  a.vec_cols = rows_16(io.gamma, 0, 4) && rows_16(io.beta, 0, 4);
  const int e = dtype == GC_BF16 ? 2 : 4;
  const bool vec = cols % 8 == 0 && rows_16(io.x, io.ldx, e) && rows_16(io.res, io.ldr, e) &&
                   rows_16(io.y, io.ldy, e) && rows_16(io.h, io.ldh, e);
  if (dtype == GC_BF16)
    return vec ? norm_by_width<__nv_bfloat16, true>(a, s) : norm_by_width<__nv_bfloat16, false>(a, s);
  return vec ? norm_by_width<float, true>(a, s) : norm_by_width<float, false>(a, s);
}

size_t norm_grad_ws_bytes(int N, int n_c, int cols) {
  const Slices sl = grad_slices(N, n_c, cols);
  return sl.count == 1 ? 0 : align_up((size_t)N * sl.count * 2 * cols * sizeof(float), 256);
}

int launch_norm_grad(const NormGradIO& io, int dtype, int N, int n_c, int cols, const DropArgs& d,
                     Carve& ws, cudaStream_t s) {
  NormGradArgs a{};
  a.dy = io.dy;
  a.h = io.h;
  a.dh = io.dh;
  a.mean = io.mean;
  a.rstd = io.rstd;
  a.gamma = io.gamma;
  a.dx = io.dx;
  a.dres = io.dres;
  a.lddy = io.lddy;
  a.ldh = io.ldh;
  a.lddh = io.lddh;
  a.lddx = io.lddx;
  a.lddr = io.lddr;
  a.n_c = n_c;
  a.cols = cols;
  a.m = make_mask(d.p, d.seed, d.offset, d.row0, cols);
  a.vec_cols = rows_16(io.gamma, 0, 4);
  const int e = dtype == GC_BF16 ? 2 : 4;
  const bool vec = cols % 8 == 0 && rows_16(io.dy, io.lddy, e) && rows_16(io.h, io.ldh, e) &&
                   rows_16(io.dh, io.lddh, e) && rows_16(io.dx, io.lddx, e) && rows_16(io.dres, io.lddr, e);
  float* part = ws.take<float>(norm_grad_ws_bytes(N, n_c, cols) / sizeof(float));
  return dtype == GC_BF16 ? grad_run<__nv_bfloat16>(a, N, io.G, io.ldg, part, vec, s)
                          : grad_run<float>(a, N, io.G, io.ldg, part, vec, s);
}

}  // namespace gc
