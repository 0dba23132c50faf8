// Newton-Schulz orthogonalisation of matrices, and the momentum step that uses it:
//   X <- u / max(|u|_F, eps),  then `steps` times  A = X X^T,  P = a I + b A + c A^2,  X <- P X
// an odd polynomial of the singular values, X X^T taken on the shorter side (m of m x n).
//   k_ns_norm       momentum = mu momentum + g / Ntil (where there is one), and the sum of u's squares
//   k_ns_scale      X as 16-bit parts
//   k_tiles<NsOp>   the three products of a step, each with its epilogue: A, then P, then the next X; of the last step
//                   the output, or w = keep w - step O
//   k_ns_join       the same epilogues where a tile's sum runs in ranges
//
// X stays as u lies, wide or tall: of a tall u the products are X^T X and X P, whose operands are read MN-major, and
// nothing is transposed.  A and P are symmetric: tiles above the diagonal are not formed, and where an operand's K blocks
// would be theirs, those below are read in their place, MN-major for K-major.
//
// Parts are fp16 of values times a power of two.  Singular values stay below kMost (the entry point checks the
// polynomial), so entries of X, A and P fit, and the parts of an entry end at 2^-24 / scale, 2^-37 for X: what is lost is
// absolute, beside singular values of 1, or of lam where a step's X has none above that (k_ns_scale).
// X, A and P take two parts everywhere, 22 bits, three products each, whose sums leave tensor memory every two K blocks: 0.4 to
// 7.8e-6 from 64 bits in the 2-norm over 130 shapes up to 4100 wide, dense and sparse ones, where torch's fp32 products have 0.3 to
// 4.3e-6 (one part: 2e-3 to 2e-2).  Of rank 20 or less up to 1.4e-4, torch's 2.2e-4: what rounding leaves of singular values of 0 is
// enlarged as any small one.  A bf16 u, whose result is rounded to 1.66e-3, takes the same parts, and sums of four K blocks, which take
// 3% less than of two: with X in A and P in one part each the result was 1.75 to 1.95e-3 off.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "newton.cuh"
#include "tc_tiles.cuh"

namespace gc {
namespace {

using namespace tiles;
using namespace rowwise;

constexpr float kMost = 4.f;    // bound of the singular values
constexpr float kTerms = 60.f;  // ... and of |a| + |b| s^2 + |c| s^4 over them
constexpr float kSX = 8192.f, kSA = 2048.f, kSP = 1024.f;  // kSX kMost, kSA kMost^2 and kSP kTerms are below 65504

constexpr int kMostSteps = 64;
constexpr int kParts = 2, kProd = 3;  // of a value; products of two values' parts i + j < 2

// Parts [kParts][batch][rows][ld] of matrices.
struct Parts {
  __half* p;
  long long plane, mat;
  int ld;
};

enum { NS_A, NS_P, NS_X, NS_OUT, NS_STEP };
struct Epilogue {
  int kind, rows, cols, batch;
  float s;             // scale of a sum
  Parts out;           // its rows may be written past their ends up to 16 bytes
  Parts A;             // NS_P: a I + b A + s sum
  float a, b;
  void* w;             // NS_OUT, NS_STEP: rows of results
  long long ldw, sw;
  int bf16, box;       // box: rows are whole 16-byte pieces
  float keep;          // NS_STEP: w = keep w + s sum
  const float* lam;    // [batch], and the next X's behind them: X is lam times what its parts hold

  __device__ __forceinline__ void one(int mat, float l, long long r, int c, float x) const {
    x *= l;
    if (bf16) {
      reinterpret_cast<__nv_bfloat16*>(w)[mat * sw + r * ldw + c] = __float2bfloat16_rn(s * x);
    } else {
      float* to = reinterpret_cast<float*>(w) + mat * sw + r * ldw + c;
      *to = kind == NS_STEP ? fmaf(s, x, keep * *to) : s * x;
    }
  }
  // 32 x 32 sums at (row0, col0), a lane a row, of which m rows and n columns exist, to w.
  __device__ __forceinline__ void finish_w(float (&v)[32], uint8_t* buf, const CUtensorMap* map, int mat, int row0, int col0,
                                           int m, int n) const {
    const int lane = threadIdx.x & 31;
    const float l = lam[mat];
    if (!box) {
      by_rows(buf, lane, v, m, n, [&](int r, int j, float x) { one(mat, l, row0 + r, col0 + j, x); });
      return;
    }
    Rows32 old[2];
    if (kind == NS_STEP) {
      const float* from = reinterpret_cast<const float*>(w) + mat * sw + (long long)row0 * ldw + col0;
      old[0].load(from, ldw * 4, m, n * 4, lane);
      old[1].load(from + 16, ldw * 4, m, n * 4 - 64, lane);
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = s * (l * v[j]);
    box_free(lane);
    if (bf16) {
      box_put_16(buf, lane, [&](int j) { return pack_bf16(v[j], v[j + 1]); });
      box_store(map, buf, lane, col0, row0, mat);
      return;
    }
    if (kind == NS_STEP) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        old[h].turn(buf, lane);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float* x = v + 16 * h + 4 * j;
          x[0] = fmaf(keep, __uint_as_float(old[h].q[j].x), x[0]);
          x[1] = fmaf(keep, __uint_as_float(old[h].q[j].y), x[1]);
          x[2] = fmaf(keep, __uint_as_float(old[h].q[j].z), x[2]);
          x[3] = fmaf(keep, __uint_as_float(old[h].q[j].w), x[3]);
        }
      }
    }
    store_32(map, buf, lane, v, n, col0, row0, mat);
  }
  // ... or as parts.
  __device__ __forceinline__ void finish_parts(float (&v)[32], uint8_t* buf, const CUtensorMap* map, int mat, int row0, int col0,
                                               int m, int n) const {
    const int lane = threadIdx.x & 31;
    if (kind == NS_P) {
      const float l2 = lam[mat] * lam[mat], sum = s * l2 * l2, b2 = b * l2;
      box_free(lane);
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = fmaf(sum, v[j], row0 + lane == col0 + j ? a : 0.f);
      for (int q = 0; q < kParts; ++q) {
        Rows32 part;  // rows of A end past a multiple of eight
        part.load(A.p + q * A.plane + mat * A.mat + (long long)row0 * A.ld + col0, A.ld * 2LL, m, (n + 7) / 8 * 16, lane);
        part.turn(buf, lane);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w4[4] = {part.q[j].x, part.q[j].y, part.q[j].z, part.q[j].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w4[e]));
            v[8 * j + 2 * e] = fmaf(b2, t.x, v[8 * j + 2 * e]);
            v[8 * j + 2 * e + 1] = fmaf(b2, t.y, v[8 * j + 2 * e + 1]);
          }
        }
      }
    } else {
      const float f = kind == NS_X ? s * (lam[mat] / lam[batch + mat]) : s;
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] *= f;
    }
    for (int q = 0; q < kParts; ++q) {
      uint32_t h[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const __half2 t = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
        const float2 f = __half22float2(t);
        h[j] = *reinterpret_cast<const uint32_t*>(&t);
        v[2 * j] -= f.x;
        v[2 * j + 1] -= f.y;
      }
      box_free(lane);
      box_put_16(buf, lane, [&](int j) { return h[j / 2]; });
      box_store(map, buf, lane, col0, row0, q * batch + mat);
    }
  }
  __device__ __forceinline__ void finish(float (&v)[32], uint8_t* buf, const CUtensorMap* map, int mat, int row0, int col0) const {
    const int m = min(rows - row0, 32), n = cols - col0;
    if (kind >= NS_OUT)
      finish_w(v, buf, map, mat, row0, col0, m, n);
    else
      finish_parts(v, buf, map, mat, row0, col0, m, n);
  }
};

// A tile's place: of a symmetric result the tiles of row tile i are those that begin at or before its last row.
__host__ __device__ inline int sym_tiles(int rows, int tn) {
  const int mt = (rows + TM - 1) / TM, nt = (rows + tn - 1) / tn, per = TM / tn;
  return per * mt * (mt - 1) / 2 + nt;  // the last row tile has all of them
}

struct NsOp {
  static constexpr bool kTurns = true;
  struct Params {
    Common q;
    Epilogue e;
    int batch, mt, nt, per, tn, sym;  // tiles of rows, of columns, of a matrix
    Ranges k;
    Divisor by_per, by_nt;
    int seg;
    int a_mn, b_mn;
    int a_sym, b_sym;                 // operands of which what is above the diagonal's blocks is not there
  };
  static __device__ __forceinline__ void before(const Params&, int, int) {}
  static __device__ __forceinline__ int jobs(const Params& p, int unit) {
    return (int)(((long long)p.batch * p.per * p.k.ks - unit + p.q.units - 1) / p.q.units);
  }
  static __device__ __forceinline__ Job job(const Params& p, int unit, int k) {
    const int i = unit + k * p.q.units, at = p.k.by.of(i);
    Job t;
    t.kind = 0;
    t.range = i - at * p.k.ks;
    t.b = p.by_per.of(at);
    const int tile = at - t.b * p.per;
    if (p.sym) {
      const int w = TM / p.tn;  // row tile r begins at w r (r + 1) / 2
      int r = (int)((sqrtf(8.f / (float)w * (float)tile + 1.f) - 1.f) * 0.5f);
      while (w * r * (r + 1) / 2 > tile) --r;
      while (r + 1 < p.mt && w * (r + 1) * (r + 2) / 2 <= tile) ++r;
      t.m0 = r * TM;
      t.n0 = (tile - w * r * (r + 1) / 2) * p.tn;
    } else {
      const int m = p.by_nt.of(tile);
      t.m0 = m * TM;
      t.n0 = (tile - m * p.nt) * p.tn;
    }
    t.kb0 = p.k.first(t.range);
    t.nkb = p.k.count(t.range);
    t.na = t.nb = t.lim = kParts;
    t.seg = p.seg;
    t.a_mn = p.a_mn;
    t.b_mn = p.b_mn;
    t.a_turn = p.a_sym ? turn_of(t.m0) : kNever;
    t.b_turn = p.b_sym ? turn_of(t.n0) : kNever;
    return t;
  }
  template <int NC, typename Get>
  static __device__ __forceinline__ void store(const Params& p, const Job& t, int row0, int col0, uint8_t* box,
                                               const CUtensorMap* out, Get get) {
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int c = 0; c < NC; ++c) {
      float v[32];
      __syncwarp();
      get(c, v);
      const int col = col0 + c * 32;
      if (row0 >= p.e.rows || col >= p.e.cols) continue;
      if (p.k.ks > 1)  // sums of the ranges [ks][batch][rows][cols, up to a multiple of four]
        store_32(&out[1], box, lane, v, p.e.cols - col, col, row0, t.range * p.batch + t.b);
      else
        p.e.finish(v, box, out, t.b, row0, col);
    }
  }
};

// A warp a block of 32 x 32: the ranges' sums in their order, and the epilogue.
__global__ void __launch_bounds__(128) k_ns_join(const __grid_constant__ CUtensorMap out, const float* __restrict__ part,
                                                 int ks, int ld, int sym, int tn, const __grid_constant__ Epilogue e) {
  __shared__ __align__(1024) uint8_t boxes[4 * BOX];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint8_t* box = boxes + warp * BOX;
  start_next();
  wait_prior();
  const int br = (e.rows + 31) / 32, bc = (e.cols + 31) / 32;
  const long long i = (long long)blockIdx.x * 4 + warp;
  if (i >= (long long)e.batch * br * bc) return;
  const int mat = (int)(i / (br * bc)), at = (int)(i - (long long)mat * br * bc);
  const int row0 = at / bc * 32, col0 = at % bc * 32;
  const int m0 = row0 / TM * TM, n0 = col0 / tn * tn;
  if (sym && n0 >= m0 + TM) return;
  const size_t range = (size_t)e.batch * e.rows * ld;
  const float* from = part + ((size_t)mat * e.rows + row0) * ld + col0;
  const int m = min(e.rows - row0, 32), n = (ld - col0) * 4;  // ld: a multiple of 4
  float v[32];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    Rows32 sum;
    sum.load(from + 16 * h, ld * 4LL, m, n - 64 * h, lane);
    for (int k = 1; k < ks; ++k) {
      Rows32 x;
      x.load(from + 16 * h + k * range, ld * 4LL, m, n - 64 * h, lane);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sum.q[j].x = __float_as_uint(__uint_as_float(sum.q[j].x) + __uint_as_float(x.q[j].x));
        sum.q[j].y = __float_as_uint(__uint_as_float(sum.q[j].y) + __uint_as_float(x.q[j].y));
        sum.q[j].z = __float_as_uint(__uint_as_float(sum.q[j].z) + __uint_as_float(x.q[j].z));
        sum.q[j].w = __float_as_uint(__uint_as_float(sum.q[j].w) + __uint_as_float(x.q[j].w));
      }
    }
    sum.turn(box, lane);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[16 * h + 4 * j] = __uint_as_float(sum.q[j].x);
      v[16 * h + 4 * j + 1] = __uint_as_float(sum.q[j].y);
      v[16 * h + 4 * j + 2] = __uint_as_float(sum.q[j].z);
      v[16 * h + 4 * j + 3] = __uint_as_float(sum.q[j].w);
    }
  }
  e.finish(v, box, &out, mat, row0, col0);
  if (lane == 0) bulk_wait_all();
}

// What u is: the matrix itself, or the momentum of a gradient (and, looking ahead, the gradient once more).
struct Source {
  const void* u;   // MOM: the gradient
  float* m;        // MOM: the momentum
  long long ldu, su, ldm, sm;
  int rows, cols, batch, blocks, nesterov;
  float mu, points;
};

template <typename T, bool VEC, bool MOM, bool UPDATE>
__device__ __forceinline__ void load_u(const Source& s, int mat, int row, int col0, int lane, float (&v)[8]) {
  const T* u = reinterpret_cast<const T*>(s.u) + mat * s.su + row * s.ldu;
  if (!MOM) {
    load_seg<VEC>(u, col0, lane, s.cols, v);
    return;
  }
  float* m = s.m + mat * s.sm + row * s.ldm;
  float g[8];
  load_seg<VEC>(m, col0, lane, s.cols, v);
  if (UPDATE || s.nesterov) {
    load_seg<VEC>(u, col0, lane, s.cols, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = __fdiv_rn(g[j], s.points);
  }
  if (UPDATE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __fmaf_rn(s.mu, v[j], g[j]);
    store_seg<VEC>(m, col0, lane, s.cols, v);
  }
  if (s.nesterov) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __fmaf_rn(s.mu, v[j], g[j]);
  }
}

// Sums of squares [batch][blocks], in 64 bits; eight values at a time in 32 where these hold them.
template <typename T, bool VEC, bool MOM>
__global__ void __launch_bounds__(256) k_ns_norm(const Source s, double* __restrict__ sums) {
  __shared__ double red[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int mat = blockIdx.x / s.blocks, block = blockIdx.x - mat * s.blocks;
  const int segs = (s.cols + kSeg - 1) / kSeg;
  start_next();
  wait_prior();
  double sum = 0;
  const long long n = (long long)s.rows * segs;
#pragma unroll 2
  for (long long i = (long long)block * 8 + warp; i < n; i += (long long)s.blocks * 8) {
    const int row = (int)(i / segs), col0 = (int)(i - (long long)row * segs) * kSeg;
    float v[8];
    load_u<T, VEC, MOM, MOM>(s, mat, row, col0, lane, v);
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) q = fmaf(v[j], v[j], q);
    add_squares(q, v, sum);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) red[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) sum += red[w];
    sums[blockIdx.x] = sum;
  }
}

// The polynomial f(s) = a s + b s^3 + c s^5, and |f| at the s^2 > 0 where its slope is 0 (infinite where there is none).
struct Poly {
  float a, b, c;
  float at[2], value[2];
  int steps;
  // The largest |f(s)| of s in [0, most], and what rounding may add.
  __device__ __forceinline__ float bound(float most) const {
    const float q = most * most;
    float v = most * fabsf(fmaf(fmaf(c, q, b), q, a));
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (at[i] < q) v = fmaxf(v, value[i]);
    return v * (1.f + 1e-5f);
  }
};

// X / lam as parts, and lam of every step's X: the power of two above the bound of its singular values, at most 1, so that an X that
// starts far below 1, from a |u| below eps, keeps its parts' digits wherever the steps take it.  The powers of A are taken
// times lam^2.
template <typename T, bool VEC, bool MOM>
__global__ void __launch_bounds__(256) k_ns_scale(const Source s, const double* __restrict__ sums, float eps, Poly poly, Parts X,
                                                  float* __restrict__ lam) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int mat = blockIdx.x / s.blocks, block = blockIdx.x - mat * s.blocks;
  const int segs = (s.cols + kSeg - 1) / kSeg;
  start_next();
  wait_prior();
  __shared__ double red[8];
  __shared__ float factor[3];
  double sum = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < s.blocks; i += 256) sum += __ldcg(sums + (size_t)mat * s.blocks + i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) red[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) sum += red[w];
    const float ratio = norm_ratio(sum, eps);
    norm_factors(sum, eps, power_above(ratio), kSX, factor);
    if (block == 0) {
      float most = ratio;
      for (int i = 0; i < poly.steps; ++i, most = poly.bound(most)) lam[(size_t)i * s.batch + mat] = power_above(most);
    }
  }
  __syncthreads();
  const float p0 = factor[0], p1 = factor[1], r = factor[2];
  const long long n = (long long)s.rows * segs;
#pragma unroll 2
  for (long long i = (long long)block * 8 + warp; i < n; i += (long long)s.blocks * 8) {
    const int row = (int)(i / segs), col0 = (int)(i - (long long)row * segs) * kSeg;
    float v[8];
    load_u<T, VEC, MOM, false>(s, mat, row, col0, lane, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = v[j] * p0 * p1 * r;
    __half* to = X.p + mat * X.mat + (long long)row * X.ld;
    for (int q = 0; q < kParts; ++q, to += X.plane) {
      float h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const __half x = __float2half_rn(v[j]);
        h[j] = __half2float(x);
        v[j] -= h[j];
      }
      if (VEC) {
        const int c = col0 + lane * 8;
        if (c < X.ld) {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __half2 t = __floats2half2_rn(h[2 * j], h[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t*>(&t);
          }
          *reinterpret_cast<uint4*>(to + c) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = col0 + j * 32 + lane;
          if (c < s.cols) to[c] = __float2half_rn(h[j]);
        }
      }
    }
  }
}

// One of a step's products: result rows x cols over K.
struct Product {
  int rows, cols, K, sym;
  int a_mn, b_mn;
  int a_sym, b_sym;
};

Split cut_of(const Product& g, int batch) {
  return split_of([&](int tn) { return (long long)batch * (g.sym ? sym_tiles(g.rows, tn) : tiles_of(g.rows, TM) * tiles_of(g.cols, tn)); },
                  (double)batch * g.rows * g.cols, (g.K + BK - 1) / BK, kProd, device_sm_count() / 2);
}

struct Scratch {
  bool wide;
  int m, n, blocks;
  Parts X[2], A, P;
  double* sums;
  float *lam, *part;
  Product pa, pp2, px;
  Split ca, cp, cx;
};

Parts take_parts(Carve& c, int batch, int rows, int cols) {
  Parts t;
  t.ld = (cols + 7) / 8 * 8;
  t.mat = (long long)rows * t.ld;
  t.plane = batch * t.mat;
  t.p = c.take<__half>((size_t)kParts * t.plane);
  return t;
}

Scratch carve_ns(Carve& c, const NsShape& s) {
  Scratch w{};
  w.wide = s.rows <= s.cols;
  w.m = std::min(s.rows, s.cols);
  w.n = std::max(s.rows, s.cols);
  const long long segs = (long long)s.rows * ((s.cols + kSeg - 1) / kSeg);
  // at most four blocks an SM over all matrices, each of which adds up all blocks' sums: a step of 2048 x 2048 takes 117 us, with
  // eight 123
  w.blocks = (int)std::max(1LL, std::min((segs + 15) / 16, 4LL * device_sm_count() / std::min(s.batch, 4 * device_sm_count())));
  w.X[0] = take_parts(c, s.batch, s.rows, s.cols);
  w.X[1] = take_parts(c, s.batch, s.rows, s.cols);
  w.A = take_parts(c, s.batch, w.m, w.m);
  w.P = take_parts(c, s.batch, w.m, w.m);
  w.sums = c.take<double>((size_t)s.batch * w.blocks);
  w.lam = c.take<float>((size_t)kMostSteps * s.batch);
  w.pa = Product{w.m, w.m, w.n, 1, !w.wide, !w.wide, 0, 0};
  w.pp2 = Product{w.m, w.m, w.m, 1, 0, 0, 1, 1};
  w.px = w.wide ? Product{w.m, w.n, w.m, 0, 0, 1, 1, 0} : Product{w.n, w.m, w.m, 0, 0, 0, 0, 1};
  w.ca = cut_of(w.pa, s.batch);
  w.cp = cut_of(w.pp2, s.batch);
  w.cx = cut_of(w.px, s.batch);
  size_t part = 0;
  auto need = [&](const Product& g, const Split& t) {
    if (t.ks > 1) part = std::max(part, (size_t)t.ks * s.batch * g.rows * ((g.cols + 3) / 4 * 4));
  };
  need(w.pa, w.ca);
  need(w.pp2, w.cp);
  need(w.px, w.cx);
  if (part) w.part = c.take<float>(part);
  return w;
}

int launch_product(const NsShape& s, const Product& g, const Split& cut, const Parts& A, const Parts& B, const Epilogue& e,
                   bool bits16, float* part, uint32_t* status, bool stall, const char* name, cudaStream_t st) {
  NsOp::Params p{};
  p.e = e;
  p.batch = s.batch;
  p.tn = cut.tn;
  p.sym = g.sym;
  p.mt = tiles_of(g.rows, TM);
  p.nt = tiles_of(g.cols, cut.tn);
  p.per = g.sym ? sym_tiles(g.rows, cut.tn) : p.mt * p.nt;
  const int nkb = (g.K + BK - 1) / BK;
  p.k = Ranges(nkb, cut.ks);
  p.by_per = Divisor((uint32_t)p.per);
  p.by_nt = Divisor((uint32_t)p.nt);
  p.seg = bits16 ? std::min(nkb, 4) : segment(false, kProd, nkb);
  p.a_mn = g.a_mn;
  p.b_mn = g.b_mn;
  p.a_sym = g.a_sym;
  p.b_sym = g.b_sym;
  const int ld_part = (g.cols + 3) / 4 * 4;
  p.q.f16 = 1;
  p.q.a_both = g.rows > 128;
  p.q.a_rows = g.rows > 128 ? 128 : (g.rows + 7) / 8 * 8;
  p.q.spin_limit = wait_limit(kSpin);
  p.q.stall = stall;
  p.q.status = status;
  Maps m;
  int rc;
  auto map = [&](CUtensorMap* t, const Parts& x, int mn, int extent, int box) {
    return mn ? operand_map(t, x.p, true, extent, g.K, s.batch, kParts, x.ld, x.mat, x.plane, BK)
              : operand_map(t, x.p, true, g.K, extent, s.batch, kParts, x.ld, x.mat, x.plane, box);
  };
  if ((rc = map(&m.a[0], A, g.a_mn, g.rows, p.q.a_rows)) || (rc = map(&m.b[0], B, g.b_mn, g.cols, cut.tn / 2)))
    return rc;
  m.a[1] = m.out[0] = m.out[1] = m.a_turned = m.a[0];
  m.b[1] = m.b_turned = m.b[0];
  if (g.a_sym && (rc = map(&m.a_turned, A, 1, g.rows, 0))) return rc;
  if (g.b_sym && (rc = map(&m.b_turned, B, 1, g.cols, 0))) return rc;
  if (cut.ks > 1 && (rc = box_map(&m.out[1], part, MAP_F32, ld_part, g.rows, (long long)cut.ks * s.batch, ld_part, (long long)g.rows * ld_part)))
    return rc;
  if (e.kind < NS_OUT)
    rc = box_map(&m.out[0], e.out.p, MAP_F16, g.cols, g.rows, (long long)kParts * s.batch, e.out.ld, e.out.mat);
  else if (e.box)
    rc = box_map(&m.out[0], e.w, e.bf16 ? MAP_BF16 : MAP_F32, g.cols, g.rows, s.batch, e.ldw, e.sw);
  if (rc) return rc;
  const long long jobs = (long long)s.batch * p.per * cut.ks;
  rc = cut.tn == 256 ? launch_tiles<NsOp, 256>(m, p, jobs, kParts, kParts, name, true, st)
                     : launch_tiles<NsOp, 128>(m, p, jobs, kParts, kParts, name, true, st);
  if (rc || cut.ks == 1) return rc;
  const long long blocks = (long long)s.batch * ((g.rows + 31) / 32) * ((g.cols + 31) / 32);
  return launch_chain(k_ns_join, "k_ns_join", (unsigned)((blocks + 3) / 4), 128, 0, 1, true, st, m.out[0], (const float*)part, cut.ks,
                      ld_part, g.sym, cut.tn, e);
}

template <typename T, bool MOM>
int launch_start(const Source& src, const Scratch& w, bool vec, float eps, const Poly& poly, cudaStream_t st) {
  const unsigned grid = (unsigned)(src.batch * src.blocks);
  int rc = launch_chain(vec ? k_ns_norm<T, true, MOM> : k_ns_norm<T, false, MOM>, "k_ns_norm", grid, 256, 0, 1, false, st, src,
                        w.sums);
  if (rc) return rc;
  return launch_chain(vec ? k_ns_scale<T, true, MOM> : k_ns_scale<T, false, MOM>, "k_ns_scale", grid, 256, 0, 1, true, st, src,
                      (const double*)w.sums, eps, poly, w.X[0], w.lam);
}

// s^2 where the slope a + 3 b s^2 + 5 c s^4 of f(s) = a s + b s^3 + c s^5 is zero; what is not above 0 is none.
struct Turns {
  double at[2] = {-1, -1};
  explicit Turns(const float* k) {
    const double a = k[0], b = k[1], c = k[2], d = 9 * b * b - 20 * a * c;
    if (c != 0 && d >= 0) {
      at[0] = (-3 * b + sqrt(d)) / (10 * c);
      at[1] = (-3 * b - sqrt(d)) / (10 * c);
    } else if (c == 0 && b != 0) {
      at[0] = -a / (3 * b);
    }
  }
};
double value_of(const float* k, double s) { return fabs(s * (k[0] + s * s * (k[1] + s * s * (double)k[2]))); }

Poly poly_of(const NsShape& s) {
  const Turns t(s.coeffs);
  Poly p{s.coeffs[0], s.coeffs[1], s.coeffs[2], {INFINITY, INFINITY}, {0.f, 0.f}, s.steps};
  for (int i = 0; i < 2; ++i)
    if (t.at[i] > 0) {
      p.at[i] = (float)t.at[i];
      p.value[i] = (float)value_of(s.coeffs, sqrt(t.at[i]));
    }
  return p;
}

}  // namespace

// From singular values of at most 1, the largest after each step, at the end of the range or where the slope is zero, and the
// largest factor |a| + |b| s^2 + |c| s^4 that one may have come by.
bool ns_coefficients_bounded(const float* k, int steps) {
  const Turns turns(k);
  double most = 1;
  for (int i = 0; i < steps; ++i) {
    const double q = most * most, terms = fabs((double)k[0]) + q * (fabs((double)k[1]) + q * fabs((double)k[2]));
    double next = value_of(k, most);
    for (double t : turns.at)
      if (t > 0 && t < q) next = std::max(next, value_of(k, sqrt(t)));
    if (!(next <= kMost && terms <= kTerms)) return false;
    most = std::max(next, 1e-30);
  }
  return true;
}

size_t ns_ws_bytes(const NsShape& s) {
  Carve c(nullptr);
  if (!ns_small(s)) carve_ns(c, s);
  return c.bytes();
}

int launch_ns(const NsShape& s, const NsIO& io, Carve& ws, uint32_t* status, cudaStream_t st) {
  if (ns_small(s)) return launch_ns_small(s, io, st);
  const Scratch w = carve_ns(ws, s);
  const bool bf = s.dtype == GC_BF16, mom = io.m != nullptr;
  const int e = bf ? 2 : 4;
  Source src{io.u, io.m, (long long)io.ldu, (long long)io.su, (long long)io.ldm, (long long)io.sm,
             s.rows, s.cols, s.batch, w.blocks, io.nesterov, io.mu, io.points};
  const bool vec = s.cols % 8 == 0 && rows_16(io.u, io.ldu, e) && (s.batch == 1 || io.su * e % 16 == 0) &&
                   (!mom || (rows_16(io.m, io.ldm, 4) && (s.batch == 1 || io.sm % 4 == 0)));
  const Poly poly = poly_of(s);
  int rc = mom  ? launch_start<float, true>(src, w, vec, io.eps, poly, st)
           : bf ? launch_start<__nv_bfloat16, false>(src, w, vec, io.eps, poly, st)
                : launch_start<float, false>(src, w, vec, io.eps, poly, st);
  if (rc) return rc;
  bool stall = take_stall(GC_STALL_MUON);
  for (int i = 0; i < s.steps; ++i) {
    const Parts &X = w.X[i & 1], &Y = w.X[1 - (i & 1)];
    Epilogue ea{};
    ea.kind = NS_A;
    ea.rows = ea.cols = w.m;
    ea.batch = s.batch;
    ea.s = kSA / (kSX * kSX);
    ea.out = w.A;
    ea.lam = w.lam + (size_t)i * s.batch;
    if ((rc = launch_product(s, w.pa, w.ca, X, X, ea, bf, w.part, status, stall, "k_ns_a", st))) return rc;
    stall = false;
    Epilogue ep = ea;
    ep.kind = NS_P;
    ep.s = s.coeffs[2] * (kSP / (kSA * kSA));
    ep.out = w.P;
    ep.A = w.A;
    ep.a = s.coeffs[0] * kSP;
    ep.b = s.coeffs[1] * (kSP / kSA);
    if ((rc = launch_product(s, w.pp2, w.cp, w.A, w.A, ep, bf, w.part, status, false, "k_ns_p", st))) return rc;
    Epilogue ex{};
    ex.lam = ea.lam;
    ex.rows = s.rows;
    ex.cols = s.cols;
    ex.batch = s.batch;
    if (i + 1 < s.steps) {
      ex.kind = NS_X;
      ex.s = 1.f / kSP;
      ex.out = Y;
    } else {
      ex.kind = mom ? NS_STEP : NS_OUT;
      ex.s = (mom ? io.step : 1.f) / (kSP * kSX);
      ex.keep = io.keep;
      ex.w = io.out;
      ex.ldw = io.ldo;
      ex.sw = io.so;
      ex.bf16 = bf;
      // one row, or one matrix, needs no stride, but a map has one
      if (s.rows == 1) ex.ldw = (s.cols + 7) / 8 * 8;
      if (s.batch == 1) ex.sw = s.rows * ex.ldw;
      ex.box = s.cols * e % 16 == 0 && rows_16(io.out, ex.ldw, e) && ex.sw * e % 16 == 0;
    }
    if ((rc = launch_product(s, w.px, w.cx, w.wide ? w.P : X, w.wide ? X : w.P, ex, bf, w.part, status, false, "k_ns_x", st)))
      return rc;
  }
  return GC_OK;
}

}  // namespace gc
