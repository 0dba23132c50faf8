// Softmax cross entropy over a large vocabulary, in pieces of it, with its gradient per chunk:
//   z = X W^T,  lse_t = log sum_v exp z_tv,  loss_t = lse_t - z_{t, y_t}
//   P = exp(z - lse) - onehot(y)  (rows without a label: 0),  dX = P W,  G_i = P_i^T X_i
// for T = N n_c rows of C values and V rows of W.  Neither z nor P exists as a whole:
//   k_xent_parts   X (and W where it is fp32, or does not lie on 16-byte boundaries) as bf16 parts; losses
//                  alone read bf16 rows where they lie
//   k_xent<STAT>   z tile by tile in tensor memory; per row and 128 columns the largest and the sum of
//                  the exponentials about it go to scratch; k_xent_lse joins them
//   k_xent<PROB>   z again for one piece of the vocabulary, written as P's bf16 parts
//   k_xent<GRAD>   dX += P W and G_i = P_i^T X_i of that piece, in one launch (k_xent_dx where the sum of dX
//                  runs in ranges)
// The loss of a single point is a pass over W (k_xent_one); its gradient is formed like those of more points, with
// the lse of the tiles, so that a chunk of one point has the same G in a call of its own and beside others.
//
// Bound: the tensor pipe.  Per row, column and value of C: one product for lse, one for P, one for
// dX, and two for G, whose 32-bit result wants P to 2^-17, as bf16 hi + lo; a bf16 dX is rounded to 2^-8,
// and takes P so too, the hi alone.  fp32 X and W enter as hi + lo too, W in a bf16 dX as well (X_hi W_hi +
// X_hi W_lo + X_lo W_hi; the dropped term is 2^-16 at most).  All sums are fp32.  z is not kept: T V values of it are gigabytes,
// while a piece of P is kPieceElems values.
//
// One persistent kernel shape: a pair of CTAs (cta_group::2) per 256 x 256 tile, each CTA holding
// 128 rows of A and of B for a 64-wide K block (warp 0, TMA), the leader's warp 1 issuing the MMAs,
// eight warps per CTA draining one of two accumulators while the other is filled.  Each CTA loads its own
// rows: no copy goes to another SM.  MMAs and copies are issued by an elected lane of a
// warp that stays together: from a branch on the lane a 64-wide K block took 900 clocks to issue where
// its MMAs take 512.  Operands that lie with K outermost (W in dX, P and X in G) are read MN-major: boxes of
// 64 columns x 64 K rows.  Rows past a chunk's end, columns past V and past C are zero-filled by TMA.  P, G
// and the fp32 dX leave by way of 32-row boxes in shared memory (1,540 points, C = 1000, V = 10007: 575 -> 371
// us).  Every wait is bounded (GC_ERR_TIMEOUT).
//
// 8,192 points, C = 2048, V = 65536, bf16: losses alone 1.11 ms, 1.97 PFLOP/s, the rate of the library's bf16
// product (the tensor pipe is active 90% of the clocks), 1.65 ms with MMAs issued from a branch; with the
// gradient in eight chunks 7.0 ms, 11.0 TFLOP issued at 1.57 PFLOP/s, near what the power limit allows (1.7).
#include <algorithm>

#include "rowwise.cuh"
#include "tc_host.cuh"
#include "tc_pair.cuh"

namespace gc {
namespace {

using namespace tcp;

constexpr int TILE = 256, HALF = 128, BK = 64;
constexpr int OP_BYTES = HALF * BK * 2;  // a CTA's 128 x 64 share of an operand tile
constexpr int kMaxStages = 6;
constexpr int kEpi = 8;
constexpr int BOX = 32 * 128;  // a store box: 32 rows of 128 bytes, 128-byte swizzle
constexpr long long kSpinX = 1LL << 32;
// Values of a piece of P: 512 MB as two bf16 parts.  Larger pieces mean fewer waves that are not full and fewer
// sums of dX to add to (8,192 points, V = 65536, C = 2048, 2^24 to 2^27: 7.9, 7.3, 7.1, 7.0 ms; 4,096 points,
// V = 32768, C = 256: 743, 536, 422, 393 us), though from 2^25 on they leave L2.
constexpr long long kPieceElems = 1LL << 27;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kBf16Max = 0x1.fep+127f;

constexpr int kNone = -1, kNoneBad = -2;  // labels that are none, the latter of a row that is not finite
// K blocks of a product for a 32-bit result that are summed in tensor memory before the sum goes to
// registers: an addition there is cut off, not rounded, and all errors have one sign (5,569 points, C = 384,
// fp32: G was 1.9e-5 off in one sum, 2e-8 a step).  Four blocks leave bf16's G as exact as fp32 products are:
// 8,192 points in eight chunks, C = 2048, V = 65536 by 8, 4, 2 blocks: 1.2e-6, 6.9e-7, 4.7e-7 off in the 2-norm
// (5.6e-7 in fp32) at 6.7, 7.0, 7.4 ms.  bf16 results do without.
constexpr int kSegment = 4;
// ... and the K blocks of z, times its products, likewise: 128 steps, C = 2048 in bf16.  Losses of bf16 rows of
// 1024, 2048, 4096, 8192: 3.5, 7.3, 7.1, 7.0e-7 off; in one sum 3.4, 7.0, 15, 30e-7, at the same times.
constexpr int kSegmentZ = 32;
enum { STAT = 0, PROB = 1, GRAD = 2 };
constexpr int kThreadsX = 64 + 32 * kEpi;
// The ring of operand stages and the store boxes of each epilogue warp.
constexpr int ring_bytes(int mode) { return (mode == PROB ? 10 : 12) * OP_BYTES; }
constexpr int boxes(int mode) { return mode == PROB ? 2 : mode == GRAD ? 1 : 0; }
constexpr size_t smem_bytes(int mode) { return ring_bytes(mode) + kEpi * boxes(mode) * BOX + 1024 + 256; }
static_assert(smem_bytes(PROB) <= kSmemMax && smem_bytes(GRAD) <= kSmemMax, "shared memory");

// A point's label: from the array that k_xent_parts leaves, or where X needs no copy as the caller gave it.
struct Labels {
  const int* lab;  // negative: none
  const void* y;   // used where lab is NULL
  int y64, V;
  __device__ __forceinline__ long long given(long long row) const {
    return y64 ? __ldg(reinterpret_cast<const long long*>(y) + row) : __ldg(reinterpret_cast<const int*>(y) + row);
  }
  __device__ __forceinline__ int at(long long row) const {
    if (lab) return __ldg(lab + row);
    const long long l = given(row);
    return l >= 0 && l < V ? (int)l : kNone;
  }
};

struct XentParams {
  long long T;
  int C, V, N, n_c;
  int nx, nw;          // bf16 parts of X and of W
  int z_seg;           // K blocks of z that are summed in tensor memory at a time
  int v0, w;           // PROB, GRAD: the piece is columns [v0, v0 + w)
  int np, np_dx;       // parts of P: kept, and that enter dX
  int mt, nt, group;   // tiles of T and of the columns; row tiles that share a sweep of the columns
  int units;           // clusters, one tile each at a time
  // rows of A that a CTA loads of X's and P's rows, and whether the second half of a tile has any: of a few
  // points no more than there are (the rows of the accumulator past them hold anything, and are not read)
  int a_rows, a_both;
  // GRAD: dX tiles, round robin; then G's, `extra` each for the units past the first `r`, which
  // have one dX tile less, and the rest round robin
  int ndx, ct, vt, ndw, r, extra;
  int ks, split;       // K ranges of a dX tile (ndx counts each); split: they leave their sums in `acc` as
                       // [ks][T][ld_acc], for k_xent_dx to add
  int stage_ops, stages;
  int first_piece, last_piece;
  Labels lab;
  const float* lse;
  float* target;       // STAT: z at the label
  float2* part;        // STAT: [slots][T], 128 columns a slot
  __nv_bfloat16* P;    // [np][T][Pp]
  int Pp;
  float* acc;          // fp32 dX of the pieces so far
  long long ld_acc;
  void* dX;
  long long ld_dx;
  int dx_bf16;
  float* G;
  long long ldg;
  int g_box, acc_box;  // G and the fp32 dX in whole boxes: rows on 16-byte boundaries
  long long spin_limit;
  int stall;
  uint32_t* status;
};

struct TileAt {
  int kind;            // 0: z, 1: dX, 2: G
  int m0, n0, chunk;
  int nkb, na, nb;
  int kb0, range;      // dX: the first K block, the K range
  int seg;             // K blocks that are summed in tensor memory at a time
};

template <int MODE>
__device__ __forceinline__ int tiles_of(const XentParams& p, int unit) {
  if (MODE != GRAD) return (int)(((long long)p.mt * p.nt - unit + p.units - 1) / p.units);
  const int nb = p.units - p.r;
  const int ndx = (p.ndx - unit + p.units - 1) / p.units;
  const int rest = p.ndw - p.extra * nb;
  return ndx + (unit >= p.r ? p.extra : 0) + (rest - unit + p.units - 1) / p.units;
}

// The k-th tile of a unit.
template <int MODE>
__device__ __forceinline__ TileAt tile_at(const XentParams& p, int unit, int k) {
  TileAt t;
  if (MODE != GRAD) {
    const int i = unit + k * p.units;
    const int per = p.group * p.nt, g = i / per, rem = i - g * per;
    const int gm = min(p.group, p.mt - g * p.group);
    const int n = rem / gm;
    t.kind = 0;
    t.m0 = (g * p.group + rem - n * gm) * TILE;
    t.n0 = n * TILE;
    t.chunk = t.kb0 = t.range = 0;
    t.nkb = (p.C + BK - 1) / BK;
    t.na = p.nx;
    t.nb = p.nw;
    t.seg = p.z_seg;
    return t;
  }
  const int ndx = (p.ndx - unit + p.units - 1) / p.units;
  if (k < ndx) {
    const int i = unit + k * p.units, at = i / p.ks, nkb = (p.w + BK - 1) / BK;
    t.kind = 1;
    t.range = i - at * p.ks;
    t.m0 = at / p.ct * TILE;
    t.n0 = at % p.ct * TILE;
    t.chunk = 0;
    t.kb0 = (int)((long long)t.range * nkb / p.ks);
    t.nkb = (int)((long long)(t.range + 1) * nkb / p.ks) - t.kb0;
    t.na = p.np_dx;
    t.nb = p.nw;
    t.seg = p.dx_bf16 ? t.nkb : kSegment;
    return t;
  }
  k -= ndx;
  const int nb = p.units - p.r, mine = unit >= p.r ? p.extra : 0;
  const int i = k < mine ? k * nb + unit - p.r : p.extra * nb + (k - mine) * p.units + unit;
  const int per = p.vt * p.ct, c = i / per, rem = i - c * per;
  t.kind = 2;
  t.kb0 = t.range = 0;
  t.chunk = c;
  t.m0 = rem / p.ct * TILE;
  t.n0 = rem % p.ct * TILE;
  t.nkb = (p.n_c + BK - 1) / BK;
  t.na = p.np;
  t.nb = p.nx;
  t.seg = kSegment;
  return t;
}

// The kernels of a call are a chain, each launched while the one before it runs (programmatic dependent
// launches): a kernel lets the next one start, and touches nothing that another wrote before wait_prior().
__device__ __forceinline__ void start_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_prior() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// v[at] for an index that is not known beforehand: a tree of selections (an indexed array of registers
// would go through local memory with all its values).
__device__ __forceinline__ float pick(const float (&v)[64], int at) {
  float w[32];
#pragma unroll
  for (int j = 0; j < 32; ++j) w[j] = at & 32 ? v[j + 32] : v[j];
#pragma unroll
  for (int h = 16; h; h >>= 1)
#pragma unroll
    for (int j = 0; j < h; ++j) w[j] = at & h ? w[j + h] : w[j];
  return w[0];
}

// 32 consecutive values of a row of an output on a 16-byte boundary.
template <typename T>
__device__ __forceinline__ void store_row(T* dst, const float (&v)[32]) {
  if (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 32; j += 4)
      *reinterpret_cast<float4*>(dst + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
  } else {
#pragma unroll
    for (int j = 0; j < 32; j += 8) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(v[j + 2 * e], v[j + 2 * e + 1]);
        w[e] = *reinterpret_cast<const uint32_t*>(&t);
      }
      *reinterpret_cast<uint4*>(dst + j) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// Row `lane` of a box: 16-byte piece j lies at j ^ (row mod 8), which makes both the rows' and the
// columns' accesses free of bank conflicts.
__device__ __forceinline__ void box_row(uint8_t* box, int lane, const float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    *reinterpret_cast<float4*>(box + lane * 128 + ((j ^ (lane & 7)) * 16)) =
        make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}
__device__ __forceinline__ void box_row_half(uint8_t* box, int lane, int first, const float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(v[8 * j + 2 * e], v[8 * j + 2 * e + 1]);
      w[e] = *reinterpret_cast<const uint32_t*>(&t);
    }
    *reinterpret_cast<uint4*>(box + lane * 128 + (((first + j) ^ (lane & 7)) * 16)) =
        make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// The box may be written again: its last store has read it.
__device__ __forceinline__ void box_free(int lane) {
  if (lane == 0) bulk_wait_read<0>();
  __syncwarp();
}
// The box's rows in turn, a lane a column, U at a time: f(row, value) for outputs whose rows lie on no 16-byte
// boundary.
template <int U, typename F>
__device__ __forceinline__ void by_rows(const uint8_t* box, int lane, int rows, F f) {
#pragma unroll U
  for (int r = 0; r < 32; ++r) {
    const float x = *reinterpret_cast<const float*>(box + r * 128 + (((lane / 4) ^ (r & 7)) * 16) + lane % 4 * 4);
    if (r < rows) f(r, x);
  }
}
// What the warp wrote to its box is there for a store, which lane 0 issues.
__device__ __forceinline__ void box_ready() {
  fence_async_smem();
  __syncwarp();
}

// The epilogue of STAT and PROB: `get` gives 64 (STAT) or 32 columns of a lane's row, in turn; U of those in a
// loop's body.
template <int MODE, int U, typename Get>
__device__ __forceinline__ void epilogue(const XentParams& p, const TileAt& t, long long row_in, int half, int lab,
                                         float l2, uint8_t* box, const CUtensorMap* mOut, Get get) {
  const int lane = threadIdx.x & 31;
  if (MODE == STAT) {
    float m = -INFINITY, s = 0.f;
#pragma unroll(U)
    for (int c = 0; c < HALF / 64; ++c) {
      float v[64];
      __syncwarp();
      get(c, v);
      const int col = t.n0 + half * HALF + c * 64;
      const int n = p.V - col;
      if (n < 64) {
#pragma unroll
        for (int j = 0; j < 64; ++j)
          if (j >= n) v[j] = -INFINITY;
      }
      if (lab >= col && lab < col + 64) p.target[row_in] = pick(v, lab - col);
      float top[4] = {m, v[0], v[1], v[2]};
#pragma unroll
      for (int j = 3; j < 64; ++j) top[j % 4] = fmaxf(top[j % 4], v[j]);
      const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
      const float ref = most == -INFINITY ? 0.f : most * kLog2e;
      float2 e[2] = {make_float2(s * ex2(fmaf(m, kLog2e, -ref)), 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int j = 0; j < 64; j += 2) {
        const float2 a = __ffma2_rn(make_float2(v[j], v[j + 1]), make_float2(kLog2e, kLog2e), make_float2(-ref, -ref));
        e[j / 2 % 2] = __fadd2_rn(e[j / 2 % 2], make_float2(ex2(a.x), ex2(a.y)));
      }
      s = (e[0].x + e[0].y) + (e[1].x + e[1].y);
      m = most;
    }
    if (row_in < p.T && t.n0 < p.V) p.part[(long long)(t.n0 / HALF + half) * p.T + row_in] = make_float2(m, s);
  } else {
#pragma unroll(U)
    for (int c = 0; c < HALF / 32; ++c) {
      float v[32];
      __syncwarp();
      get(c, v);
      if (t.n0 >= p.w || row_in - lane >= p.T) continue;  // nothing of the warp's rows or columns exists
      const int at = lab - (p.v0 + t.n0 + half * HALF + c * 32);  // the label's place here
#pragma unroll
      for (int j = 0; j < 32; j += 2) {
        const float2 a = __ffma2_rn(make_float2(v[j], v[j + 1]), make_float2(kLog2e, kLog2e), make_float2(-l2, -l2));
        v[j] = lab >= 0 ? ex2(a.x) : 0.f;
        v[j + 1] = lab >= 0 ? ex2(a.y) : 0.f;
      }
      if (at >= 0 && at < 32) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (j == at) v[j] -= 1.f;
      }
      if (c % 2 == 0) box_free(lane);
      box_row_half(box, lane, c % 2 * 4, v);
      if (p.np == 2) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] -= __bfloat162float(__float2bfloat16_rn(v[j]));
        box_row_half(box + BOX, lane, c % 2 * 4, v);
      }
      if (c % 2) {  // 64 columns, all parts in one store
        box_ready();
        if (lane == 0) {
          store_3d(mOut, box, t.n0 + half * HALF + (c - 1) * 32, (int)row_in, 0);
          bulk_commit();
        }
      }
    }
  }
}

// The epilogue of GRAD: `get` gives 32 columns of a lane's row, in turn.
template <typename Get>
__device__ __forceinline__ void store_grad(const XentParams& p, const TileAt& t, long long row_in, int half, uint8_t* box,
                                           const CUtensorMap* mOut, const CUtensorMap* mAcc, Get get) {
  const int lane = threadIdx.x & 31;
  if (t.kind == 1) {
    const bool out = p.last_piece && p.dx_bf16 && !p.split;  // the sum is complete and leaves in bf16
    const bool first = p.first_piece || p.split;
    float* acc = p.acc + (p.split ? (size_t)t.range * p.T * p.ld_acc : 0);
    const bool vec = p.ld_acc % 4 == 0 && reinterpret_cast<uintptr_t>(p.acc) % 16 == 0 &&
                     (!out || (p.ld_dx % 8 == 0 && reinterpret_cast<uintptr_t>(p.dX) % 16 == 0));
#pragma unroll
    for (int c = 0; c < HALF / 32; ++c) {
      float v[32];
      __syncwarp();
      get(c, v);
      const int col = t.n0 + half * HALF + c * 32, n = p.C - col;
      if (n <= 0 || row_in - lane >= p.T) continue;
      if (!out && p.acc_box) {
        box_free(lane);
        box_row(box, lane, v);
        box_ready();
        if (lane == 0) {
          if (first)
            store_3d(mAcc, box, col, (int)row_in, t.range);
          else
            add_3d(mAcc, box, col, (int)row_in, 0);  // one addition an element and piece, in the pieces' order
          bulk_commit();
        }
        continue;
      }
      if (!vec || n < 32) {
        box_free(lane);
        box_row(box, lane, v);
        __syncwarp();
        float* a = acc + (row_in - lane) * p.ld_acc + col + lane;
        __nv_bfloat16* o = (__nv_bfloat16*)p.dX + (row_in - lane) * p.ld_dx + col + lane;
        const long long rows = p.T - (row_in - lane);
        by_rows<2>(box, lane, lane < n ? (int)min(rows, 32LL) : 0, [&](int r, float x) {
          if (!first) x += a[r * p.ld_acc];
          if (out)
            o[r * p.ld_dx] = __float2bfloat16_rn(x);
          else
            a[r * p.ld_acc] = x;
        });
        continue;
      }
      if (row_in >= p.T) continue;
      float* a = acc + row_in * p.ld_acc + col;
      if (!first) {
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float4 q = *reinterpret_cast<const float4*>(a + j);
          v[j] += q.x;
          v[j + 1] += q.y;
          v[j + 2] += q.z;
          v[j + 3] += q.w;
        }
      }
      if (out)
        store_row((__nv_bfloat16*)p.dX + row_in * p.ld_dx + col, v);
      else
        store_row(a, v);
    }
  } else {
    const int lv = (int)row_in;  // row of the piece
#pragma unroll
    for (int c = 0; c < HALF / 32; ++c) {
      float v[32];
      __syncwarp();
      get(c, v);
      const int col = t.n0 + half * HALF + c * 32, n = p.C - col;
      if (n <= 0 || lv - lane >= p.w) continue;
      box_free(lane);
      box_row(box, lane, v);
      if (p.g_box) {
        box_ready();
        if (lane == 0) {
          store_3d(mOut, box, col, p.v0 + lv, t.chunk);
          bulk_commit();
        }
      } else {
        __syncwarp();
        float* g = p.G + t.chunk * p.ldg + (long long)(p.v0 + lv - lane) * p.C + col + lane;
        by_rows<8>(box, lane, lane < n ? min(p.w - (lv - lane), 32) : 0,
                   [&](int r, float x) { g[(long long)r * p.C] = x; });
      }
    }
  }
}

// Tensor maps: mA, mB of the first product (z: X and W rows; GRAD: P rows and W columns for dX), mP4
// and mX4 (GRAD: P and X of a chunk, columns x points); of the stores, mOut (PROB: P; GRAD: G) and
// mAcc (GRAD: the fp32 dX).
template <int MODE>
__global__ void __launch_bounds__(kThreadsX, 1)
    k_xent(const __grid_constant__ CUtensorMap mA, const __grid_constant__ CUtensorMap mB,
           const __grid_constant__ CUtensorMap mP4, const __grid_constant__ CUtensorMap mX4,
           const __grid_constant__ CUtensorMap mOut, const __grid_constant__ CUtensorMap mAcc, XentParams p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t* store_box = smem + ring_bytes(MODE);  // boxes(MODE) an epilogue warp
  // the leader's: the pair's loads landed; each CTA's: the MMAs on the stage are done
  uint64_t* full = reinterpret_cast<uint64_t*>(store_box + kEpi * boxes(MODE) * BOX);
  uint64_t* empty = full + kMaxStages;
  uint64_t* tfull = empty + kMaxStages;  // [2] each CTA's: accumulator filled
  uint64_t* tempty = tfull + 2;          // [2] the leader's: drained by both CTAs
  uint64_t* done = tempty + 2;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int unit = blockIdx.x / 2;
  const int half_m = (int)cta_rank();  // the half of the pair's rows
  const int S = p.stages, stage_bytes = p.stage_ops * OP_BYTES;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&tfull[a], 1);
      mbar_init(&tempty[a], 2 * kEpi);
    }
    mbar_init(done, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(tmem_holder, 512);
  fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  fence_after();
  const uint32_t tmem_base = *tmem_holder;
  start_next();
  wait_prior();
  const int ntiles = tiles_of<MODE>(p, unit);
  if (warp == 0) {
    const bool one = elect_one();
    uint32_t it = 0, ph = 0;
    int s = 0;
    bool ok = !p.stall;
    for (int k = 0; k < ntiles && ok; ++k) {
      const TileAt t = tile_at<MODE>(p, unit, k);
      const int ma = t.m0 + half_m * HALF, nb = t.n0 + half_m * HALF;
      const bool rows_a = t.kind < 2, skip_a = rows_a && half_m == 1 && !p.a_both;
      const uint32_t bytes = 2 * t.nb * OP_BYTES + (rows_a ? t.na * p.a_rows * BK * 2 * (p.a_both ? 2 : 1)
                                                           : 2 * t.na * OP_BYTES);
      for (int kb = t.kb0; kb < t.kb0 + t.nkb; ++kb, ++it) {
        if (!mbar_wait(&empty[s], ph ^ 1, abort_flag, p.status, p.spin_limit)) ok = false;
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        if (one) {
          if (half_m == 0) mbar_expect_tx(&full[s], bytes);
          const uint32_t bar = at_rank(&full[s], 0);
          uint8_t* st = smem + (size_t)s * stage_bytes;
          for (int i = 0; i < t.na; ++i, st += OP_BYTES) {
            if (!rows_a) {
              load_4d(st, &mP4, ma, kb * BK, t.chunk, i, bar);
              load_4d(st + OP_BYTES / 2, &mP4, ma + 64, kb * BK, t.chunk, i, bar);
            } else if (!skip_a) {
              load_3d(st, &mA, kb * BK, ma, i, bar);
            }
          }
          for (int i = 0; i < t.nb; ++i, st += OP_BYTES) {
            if (t.kind == 0) {
              load_3d(st, &mB, kb * BK, p.v0 + nb, i, bar);
            } else if (t.kind == 1) {
              load_3d(st, &mB, nb, p.v0 + kb * BK, i, bar);
              load_3d(st + OP_BYTES / 2, &mB, nb + 64, p.v0 + kb * BK, i, bar);
            } else {
              load_4d(st, &mX4, nb, kb * BK, t.chunk, i, bar);
              load_4d(st + OP_BYTES / 2, &mX4, nb + 64, kb * BK, t.chunk, i, bar);
            }
          }
        }
        __syncwarp();
        if (++s == S) {
          s = 0;
          ph ^= 1;
        }
      }
    }
    // drain: a stage whose MMAs are done has landed everywhere.  After an abort nothing arrives any
    // more; the copies in flight land within the one limit.
    for (uint32_t k = it > (uint32_t)S ? it - S : 0; k < it; ++k) {
      volatile int no_abort = 0;
      const bool in = mbar_wait(&empty[k % S], (k / S) & 1, &no_abort, p.status, 1LL << 28);
      if (!__all_sync(0xffffffffu, in)) break;
    }
  } else if (warp == 1) {
    if (half_m == 0) {
      const bool one = elect_one();
      const uint16_t pair = 3;
      uint32_t ph = 0, use = 0;  // use: accumulators filled so far, in turn the one and the other
      int s = 0;
      bool ok = true;
      for (int k = 0; k < ntiles && ok; ++k) {
        const TileAt t = tile_at<MODE>(p, unit, k);
        const bool a_mn = t.kind == 2, b_mn = t.kind >= 1;
        const uint32_t idesc = idesc_256(a_mn, b_mn);
        const uint32_t a_step = (a_mn ? 2048 : 32) >> 4, b_step = (b_mn ? 2048 : 32) >> 4;
        const uint64_t da0 = sdesc(smem_u32(smem), a_mn ? OP_BYTES / 2 : 16, 1024);
        const uint64_t db0 = sdesc(smem_u32(smem) + t.na * OP_BYTES, b_mn ? OP_BYTES / 2 : 16, 1024);
        for (int kb = 0, left = 0; kb < t.nkb; ++kb) {
          const int ab = use & 1;
          if (left == 0) {
            left = t.seg;
            ok = mbar_wait(&tempty[ab], ((use >> 1) & 1) ^ 1, abort_flag, p.status, p.spin_limit);
          }
          ok = ok && mbar_wait(&full[s], ph, abort_flag, p.status, p.spin_limit);
          if (!__all_sync(0xffffffffu, ok)) {
            ok = false;
            break;
          }
          const bool opens = left == t.seg, closes = --left == 0 || kb == t.nkb - 1;
          if (opens) fence_after();
          if (one) {
            const uint32_t d = tmem_base + (uint32_t)(ab * TILE);
            // the descriptors of the stage: only the address, in 16-byte units, differs
            const uint64_t at = (uint64_t)((uint32_t)s * (uint32_t)stage_bytes >> 4);
            uint64_t da = da0 + at;
            for (int i = 0; i < t.na; ++i, da += OP_BYTES >> 4) {
              uint64_t db = db0 + at;
              for (int j = 0; j < t.nb && i + j < 2; ++j, db += OP_BYTES >> 4) {
#pragma unroll
                for (int ks = 0; ks < BK / 16; ++ks)
                  mma(d, da + (uint64_t)(ks * a_step), db + (uint64_t)(ks * b_step), idesc,
                      (!opens || i + j + ks > 0) ? 1u : 0u);
              }
            }
            commit_to(&empty[s], pair);
            if (closes) commit_to(&tfull[ab], pair);
          }
          __syncwarp();
          if (closes) {
            left = 0;
            ++use;
          }
          if (++s == S) {
            s = 0;
            ph ^= 1;
          }
        }
      }
      if (one) commit_own(done);
      __syncwarp();
      volatile int no_abort = 0;
      mbar_wait(done, 0, &no_abort, p.status, 1LL << 28);
      __syncwarp();
    }
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint32_t use = 0;
    bool ok = true;
    auto filled = [&] {
      ok = mbar_wait(&tfull[use & 1], (use >> 1) & 1, abort_flag, p.status, p.spin_limit);
      ok = __all_sync(0xffffffffu, ok);
      if (ok) fence_after();
      return ok;
    };
    auto release = [&] {
      fence_before();
      __syncwarp();
      if (lane == 0) arrive_remote(at_rank(&tempty[use & 1], 0));
    };
    auto at = [&] {
      return tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)((use & 1) * TILE + half * HALF);
    };
    for (int k = 0; k < ntiles && ok; ++k) {
      const TileAt t = tile_at<MODE>(p, unit, k);
      const long long row = (long long)t.m0 + half_m * HALF + quarter * 32 + lane;
      int lab = kNone;
      float l2 = 0.f;  // the row's lse, in powers of two
      if (MODE != GRAD && row < p.T) {  // on their way while the accumulator fills
        lab = p.lab.at(row);
        if (MODE == PROB) l2 = __ldg(p.lse + row) * kLog2e;
      }
      uint8_t* box = store_box + (warp - 2) * boxes(MODE) * BOX;
      if (t.nkb > t.seg) {
        float sum[HALF];
#pragma unroll
        for (int j = 0; j < HALF; ++j) sum[j] = 0.f;
        for (int left = t.nkb; left > 0 && filled(); left -= t.seg, ++use) {
#pragma unroll
          for (int j = 0; j < HALF; j += 16) tmem_add16(at() + (uint32_t)j, sum + j);
          release();
        }
        if (!ok) break;
        auto get = [&](int c, auto& v) {
          constexpr int n = sizeof(v) / sizeof(float);
#pragma unroll
          for (int j = 0; j < n; ++j) v[j] = sum[c * n + j];
        };
        if constexpr (MODE == GRAD)
          store_grad(p, t, row, half, box, &mOut, &mAcc, get);
        else
          epilogue<MODE, HALF / 32>(p, t, row, half, lab, l2, box, &mOut, get);
        continue;
      }
      if (!filled()) break;
      auto get = [&](int c, auto& v) {  // the accumulator is handed back when the last of it is in registers
        constexpr int n = sizeof(v) / sizeof(float);
        if constexpr (n == 64)
          tmem_ld64(at() + (uint32_t)(c * n), v);
        else
          tmem_ld32(at() + (uint32_t)(c * n), v);
        if (c == HALF / n - 1) release();
      };
      if constexpr (MODE == GRAD)
        store_grad(p, t, row, half, box, &mOut, &mAcc, get);
      else
        epilogue<MODE, MODE == STAT ? 1 : HALF / 32>(p, t, row, half, lab, l2, box, &mOut, get);
      ++use;
    }
    if (boxes(MODE) && lane == 0) bulk_wait_all();
  }
  fence_before();
  __syncthreads();
  // no CTA leaves, or gives its tensor memory back, while another may still reach it
  cluster_arrive();
  cluster_wait();
  if (warp == 1) {
    fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

// bf16 parts [parts][rows][Cp] of a matrix: hi = bf16(x), lo = bf16(x - hi), zero from C to Cp; past bf16's
// largest value, where fp32 goes on for another 2^-8 of it, that is hi.  A block a row at a time, or a warp
// (WPR = 1: short rows).  With labels: lab = the label as an int, kNone where there is none.  The products that
// follow multiply such a row by zeros, so what is not finite in it enters as zero (kNoneBad).
template <typename T, bool VEC, int WPR>
__global__ void __launch_bounds__(256)
    k_xent_parts(const T* __restrict__ x, long long ld, long long rows, int C, int Cp, int parts,
                 const void* __restrict__ y, int y64, int V, int* __restrict__ lab,
                 __nv_bfloat16* __restrict__ out, uint32_t* status) {
  using namespace rowwise;
  const int lane = threadIdx.x & 31, warp = WPR == 1 ? 0 : threadIdx.x >> 5;
  start_next();
  wait_prior();
  constexpr int RPB = 8 / WPR;
  for (long long row = (long long)blockIdx.x * RPB + (WPR == 1 ? threadIdx.x >> 5 : 0); row < rows;
       row += (long long)gridDim.x * RPB) {
    long long l = 0;
    if (y) l = y64 ? reinterpret_cast<const long long*>(y)[row] : reinterpret_cast<const int*>(y)[row];
    const bool live = !y || (l >= 0 && l < V);
    int bad = 0;
    for (int col0 = warp * kSeg; col0 < Cp; col0 += WPR * kSeg) {
      float v[8];
      load_seg<VEC>(x + row * ld, col0, lane, C, v);
      if (!live) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (!isfinite(v[j])) {
            v[j] = 0.f;
            bad = 1;
          }
      }
      for (int q = 0; q < parts; ++q) {
        float h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          h[j] = sizeof(T) == 4 && isfinite(v[j]) ? fminf(fmaxf(v[j], -kBf16Max), kBf16Max) : v[j];
        store_seg<VEC>(out + ((size_t)q * rows + row) * Cp, col0, lane, Cp, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] -= __bfloat162float(__float2bfloat16_rn(h[j]));
      }
    }
    if (y) {
      if (!live) bad = WPR == 1 ? __any_sync(0xffffffffu, bad) : __syncthreads_or(bad);
      if (lane == 0 && warp == 0) {
        lab[row] = live ? (int)l : bad ? kNoneBad : kNone;
        if (l >= V) atomicOr(status, ST_BAD_LABEL);
      }
    }
  }
}

// (m, s) += (m2, s2), the largest value and the sum of exponentials about it.  The same bits wherever it is
// inlined: the product and the sum are not left to the compiler to contract.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
  s = __fmaf_rn(s2, ex2((m2 - ref) * kLog2e), __fmul_rn(s, ex2((m - ref) * kLog2e)));
  m = top;
}

// The loss of one point: the W rows stream once through registers, where a tile of the tensor cores
// would be nearly empty.  Bound: HBM.  A warp takes four neighbouring rows of W at a time, with the next two
// segments of them on their way; x lies in shared memory as fp32 in the order in which lanes read it,
// and the largest value and the sum of exponentials of a warp's rows stay in registers.  The last block
// to finish joins the blocks' sums, in their order.  (C = 2048, V = 65536 bf16, 268 MB: 51 us a call, 5.3
// TB/s; 64 with the loads of a segment issued when it is wanted; the tile kernel takes 59 for any number of
// points up to 256, and two points here 71.)
constexpr int kFewRows = 4;
template <typename TX, typename TW, bool VEC>
__global__ void __launch_bounds__(256)
    k_xent_one(const TX* __restrict__ X, const TW* __restrict__ W, long long ldw, int C, int V,
               const void* __restrict__ y, int y64, float* target, float2* part, float* lse, float* lse_out,
               float* row_loss, double* loss, unsigned int* counter, uint32_t* status) {
  using namespace rowwise;
  extern __shared__ __align__(16) float xs[];  // [segments][2][32][4]
  __shared__ float2 red[8];
  __shared__ int last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int nseg = (C + kSeg - 1) / kSeg;
  start_next();
  wait_prior();
  for (int seg = warp; seg < nseg; seg += 8) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = seg_col<VEC>(seg * kSeg, lane, j);
      v[j] = c < C ? to_f(X[c]) : 0.f;
    }
    float4* d = reinterpret_cast<float4*>(xs + (size_t)seg * kSeg);
    d[lane] = make_float4(v[0], v[1], v[2], v[3]);
    d[32 + lane] = make_float4(v[4], v[5], v[6], v[7]);
  }
  const long long l = y64 ? *reinterpret_cast<const long long*>(y) : *reinterpret_cast<const int*>(y);
  const int label = l >= 0 && l < V ? (int)l : kNone;
  if (blockIdx.x == 0 && threadIdx.x == 0 && l >= V) atomicOr(status, ST_BAD_LABEL);
  __syncthreads();
  float m = -INFINITY, s = 0.f;
  const long long step = (long long)gridDim.x * 8 * kFewRows;
  long long v0 = ((long long)blockIdx.x * 8 + warp) * kFewRows;
  // the next two segments of the rows, over the end of a row to the warp's next ones
  RawSeg<VEC, TW> ahead[2][kFewRows];
  long long fv = v0;
  int fs = 0;
  auto fetch = [&](RawSeg<VEC, TW>(&to)[kFewRows]) {
    if (fv >= V) return;
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) to[r].load(W + min(fv + r, (long long)V - 1) * ldw, fs * kSeg, lane, C);
    if (++fs == nseg) {
      fs = 0;
      fv += step;
    }
  };
  fetch(ahead[0]);
  fetch(ahead[1]);
  for (; v0 < V; v0 += step) {
    float z[kFewRows] = {0.f, 0.f, 0.f, 0.f};
    for (int seg = 0; seg < nseg; ++seg) {
      float w[kFewRows][8];
#pragma unroll
      for (int r = 0; r < kFewRows; ++r) {
        ahead[0][r].values(w[r]);
        ahead[0][r] = ahead[1][r];
      }
      fetch(ahead[1]);
      const float4* d = reinterpret_cast<const float4*>(xs + (size_t)seg * kSeg);
      const float4 a = d[lane], b = d[32 + lane];
      const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int r = 0; r < kFewRows; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[r] = fmaf(w[r][j], x[j], z[r]);
    }
    float top = m;
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
#pragma unroll
      for (int o = 16; o; o >>= 1) z[r] += __shfl_xor_sync(0xffffffffu, z[r], o);
      if (v0 + r >= V) z[r] = -INFINITY;
      if (v0 + r == label && lane == 0) *target = z[r];
      top = fmaxf(top, z[r]);
    }
    const float ref = top == -INFINITY ? 0.f : top * kLog2e;
    s *= ex2(fmaf(m, kLog2e, -ref));
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) s += ex2(fmaf(z[r], kLog2e, -ref));
    m = top;
  }
  if (lane == 0) red[warp] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 8; ++w) join(m, s, red[w].x, red[w].y);
    part[blockIdx.x] = make_float2(m, s);
    __threadfence();
    // the counter is back at zero for the next call
    last = atomicInc(counter, gridDim.x - 1) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  m = -INFINITY;
  s = 0.f;
  for (int k = threadIdx.x; k < (int)gridDim.x; k += 256) {
    const float2 q = __ldcg(part + k);
    join(m, s, q.x, q.y);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
    join(m, s, m2, s2);
  }
  if (lane == 0) red[warp] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 8; ++w) join(m, s, red[w].x, red[w].y);
    const float v = m + logf(s), r = label >= 0 ? v - __ldcg(target) : 0.f;
    *lse = v;
    if (lse_out) *lse_out = v;
    if (row_loss) *row_loss = r;
    if (loss) *loss = (double)r;
  }
}

// dX from the sums of its K ranges, in their order after that of the pieces before; `sum` (fp32) holds it
// until the last piece, whose sum leaves as T.
template <typename T>
__global__ void __launch_bounds__(256) k_xent_dx(const float* __restrict__ part, int ks, long long rows, int C,
                                                 int ld, float* __restrict__ sum, int first, T* __restrict__ dX,
                                                 long long ld_dx) {
  start_next();
  wait_prior();
  const int per = (C + 3) / 4;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i / per;
  if (row >= rows) return;
  const int c = (int)(i - row * per) * 4;
  const size_t at = (size_t)row * ld + c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (!first) s = *reinterpret_cast<const float4*>(sum + at);
#pragma unroll 8
  for (int k = 0; k < ks; ++k) {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(part + (size_t)k * rows * ld + at));
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  }
  if (!dX) {
    *reinterpret_cast<float4*>(sum + at) = s;
    return;
  }
  const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (c + e < C) dX[row * ld_dx + c + e] = rowwise::from_f<T>(v[e]);
}

// lse and loss of the rows from their n partial sums [n][T].  A block takes R rows: a warp's lanes are R
// rows by 32 / R slots (R = 32: whole 256-byte reads; 4: whole sectors, for few rows).  Either way slot k adds to
// sum k mod 64, a warp joins its eight neighbouring sums as a tree and the eight warps' come in turn: a
// point has the same bits in a call of any number of points.
template <int R>
__global__ void __launch_bounds__(256) k_xent_lse(const float2* __restrict__ part, int n, long long T,
                                                  Labels lab, const float* __restrict__ target, uint32_t* status,
                                                  float* __restrict__ lse, float* __restrict__ lse_out,
                                                  float* __restrict__ row_loss) {
  __shared__ float2 sums[8][R];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane % R;
  const long long row = (long long)blockIdx.x * R + r;
  start_next();
  wait_prior();
  constexpr int L = 32 / R, A = 8 / L;  // lanes of a row, sums of a lane: number a L + lane / R of the warp's
  float am[A], as[A];
#pragma unroll
  for (int a = 0; a < A; ++a) {
    am[a] = -INFINITY;
    as[a] = 0.f;
  }
  if (row < T) {
#pragma unroll(8 / A)
    for (int k0 = warp * 8 + lane / R; k0 < n; k0 += 64) {
#pragma unroll
      for (int a = 0; a < A; ++a) {
        if (k0 + a * L < n) {
          const float2 q = __ldcg(part + (k0 + a * L) * T + row);
          join(am[a], as[a], q.x, q.y);
        }
      }
    }
  }
  // sums 0 .. 3 += 4 .. 7, 0, 1 += 2, 3, 0 += 1
#pragma unroll
  for (int h = 4; h; h >>= 1) {
    if (h >= L) {
#pragma unroll
      for (int a = 0; a < h / L; ++a) join(am[a], as[a], am[a + h / L], as[a + h / L]);
    } else {
      const float m2 = __shfl_down_sync(0xffffffffu, am[0], h * R), s2 = __shfl_down_sync(0xffffffffu, as[0], h * R);
      join(am[0], as[0], m2, s2);
    }
  }
  float m = am[0], s = as[0];
  if (lane < R) sums[warp][r] = make_float2(m, s);
  __syncthreads();
  if (warp == 0 && lane < R && row < T) {
#pragma unroll
    for (int w = 1; w < 8; ++w) join(m, s, sums[w][r].x, sums[w][r].y);
    const int at = lab.at(row);
    if (!lab.lab && lab.given(row) >= lab.V) atomicOr(status, ST_BAD_LABEL);
    const float l = at == kNoneBad ? NAN : m + logf(s);
    if (lse) lse[row] = l;
    if (lse_out) lse_out[row] = l;
    if (row_loss) row_loss[row] = at >= 0 ? l - target[row] : 0.f;
  }
}

// (1/T) sum of the rows' losses, in a fixed order.
__global__ void __launch_bounds__(1024) k_xent_loss(const float* __restrict__ row_loss, long long T,
                                                    double* __restrict__ loss) {
  __shared__ double acc[32];
  start_next();
  wait_prior();
  double s = 0.0;
  for (long long i = threadIdx.x; i < T; i += 1024) s += (double)row_loss[i];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) acc[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < 32; ++w) s += acc[w];
    *loss = s / (double)T;
  }
}

// Pairs that the current device holds at once.
template <int MODE>
int resident(int* units) {
  static std::atomic<int> cache[64];
  int dev = 0, n = 0;
  GC_CUDA(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64) n = cache[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    static SmemOptIn allow;
    GC_CUDA(allow(k_xent<MODE>, smem_bytes(MODE)));
    cudaLaunchAttribute at[1];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kThreadsX);
    cfg.dynamicSmemBytes = smem_bytes(MODE);
    cfg.attrs = at;
    cfg.numAttrs = 1;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    GC_CUDA(cudaOccupancyMaxActiveClusters(&n, k_xent<MODE>, &cfg));
    if (n < 1) return fail(GC_ERR_CUDA, "no pair of CTAs fits the device");
    if (dev >= 0 && dev < 64) cache[dev].store(n, std::memory_order_relaxed);
  }
  *units = n;
  return GC_OK;
}

template <int MODE>
int launch_mode(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& c, const CUtensorMap& d,
                const CUtensorMap& out, const CUtensorMap& acc, const XentParams& p, bool chained, cudaStream_t s) {
  return launch_chain(k_xent<MODE>, "k_xent", (unsigned)(2 * p.units), kThreadsX, smem_bytes(MODE), 2, chained, s,
                      a, b, c, d, out, acc, p);
}

template <typename T>
int parts_of(const void* x, int64_t ld, long long rows, int C, int Cp, int parts, const void* y, int y64, int V,
             int* lab, __nv_bfloat16* out, uint32_t* status, bool chained, cudaStream_t s) {
  const bool vec = C % 8 == 0 && rowwise::rows_16(x, ld, sizeof(T)), shorter = Cp <= 4 * rowwise::kSeg;
  const long long blocks = shorter ? (rows + 7) / 8 : rows;
  const unsigned grid = (unsigned)std::min<long long>(blocks, 8LL * device_sm_count());
  auto* kern = shorter ? vec ? k_xent_parts<T, true, 1> : k_xent_parts<T, false, 1>
                       : vec ? k_xent_parts<T, true, 8> : k_xent_parts<T, false, 8>;
  return launch_chain(kern, "k_xent_parts", grid, 256, 0, 1, chained, s, (const T*)x, (long long)ld, rows, C, Cp, parts,
                      y, y64, V, lab, out, status);
}

int tiles(long long n) { return (int)((n + TILE - 1) / TILE); }

// The form for one point, and its blocks (each a slot of `part`): three an SM for bf16 rows (the registers' limit;
// 268 MB: 56, 51, 57 us by 2, 3, 4), two for fp32 ones (131 MB: 28, 30, 30).  It counts finished blocks in a word
// of the workspace header, zero between calls.
constexpr int kOneCounter = 7;
constexpr size_t kOneSmem = 64 * 1024;
size_t one_smem(int C) { return (size_t)(C + rowwise::kSeg - 1) / rowwise::kSeg * rowwise::kSeg * sizeof(float); }
bool one_point(long long T, int C) { return T == 1 && one_smem(C) <= kOneSmem; }
int one_blocks(const XentShape& s) {
  return std::min((s.V + 8 * kFewRows - 1) / (8 * kFewRows), (s.w_dtype == GC_BF16 ? 3 : 2) * device_sm_count());
}

template <typename TX, typename TW>
int launch_one(const XentShape& s, const XentIO& io, float* target, float2* part, float* lse, uint32_t* status,
               cudaStream_t st) {
  const bool vec = s.C % 8 == 0 && rowwise::rows_16(io.W, io.ldw, sizeof(TW));
  auto* kern = vec ? k_xent_one<TX, TW, true> : k_xent_one<TX, TW, false>;
  static SmemOptIn allow[2];
  GC_CUDA(allow[vec](kern, kOneSmem));
  return launch_chain(kern, "k_xent_one", (unsigned)one_blocks(s), 256, one_smem(s.C), 1, false, st,
                      (const TX*)io.X, (const TW*)io.W, (long long)io.ldw, s.C, s.V, io.y, io.y64, target, part, lse,
                      io.lse, io.row_loss, io.loss, status + kOneCounter, status);
}

// Columns of a piece: as many as kPieceElems of P allow, the pieces of one width.
int piece_cols(long long T, int V) {
  const long long most = std::max<long long>(TILE, kPieceElems / T / TILE * TILE);
  const int pieces = (int)((V + most - 1) / most);
  return tiles((V + pieces - 1) / pieces) * TILE;
}

// K ranges of a dX tile: with few tiles (few points, or few columns) the sum over a piece of the
// vocabulary, one 64-wide block after the other, would outlast all else (1,024 points, C = 256, V = 65536:
// four tiles of 1,024 blocks, 276 us at the full rate).  128 tiles in all, sixteen blocks each at least.
int dx_ranges(long long T, int C, int piece) {
  const long long n = (long long)tiles(T) * tiles(C);
  return (int)std::max<long long>(1, std::min<long long>({(128 + n - 1) / n, piece / (16 * BK), 32}));
}

struct XentScratch {
  int Cp, nx, nw, piece, np, ks, ld_acc;
  bool w_in_place, one;
  __nv_bfloat16 *X, *W, *P;
  int* lab;
  float *lse, *target, *row_loss, *acc, *ranges;
  float2* part;
};

XentScratch carve_xent(Carve& c, const XentShape& s) {
  XentScratch w{};
  const long long T = (long long)s.N * s.n_c;
  w.Cp = (s.C + 7) / 8 * 8;
  w.nx = s.x_dtype == GC_BF16 ? 1 : 2;
  w.nw = s.w_dtype == GC_BF16 ? 1 : 2;
  w.w_in_place = s.w_dtype == GC_BF16 && s.w_16;
  w.one = one_point(T, s.C);
  if (!w.one || s.want) {  // one point's loss takes X and W as they are
    w.X = c.take<__nv_bfloat16>((size_t)w.nx * T * w.Cp);
    w.W = w.w_in_place ? nullptr : c.take<__nv_bfloat16>((size_t)w.nw * s.V * w.Cp);
  }
  w.lab = c.take<int>((size_t)T);
  w.lse = c.take<float>((size_t)T);
  w.target = c.take<float>((size_t)T);
  w.row_loss = c.take<float>((size_t)T);
  w.part = c.take<float2>((size_t)T * std::max(w.one ? one_blocks(s) : 0, !w.one || s.want ? 2 * tiles(s.V) : 0));
  if (s.want & (XENT_DX | XENT_G)) {
    w.piece = piece_cols(T, s.V);
    w.np = (s.want & XENT_G) || s.x_dtype == GC_F32 ? 2 : 1;
    w.P = c.take<__nv_bfloat16>((size_t)w.np * T * w.piece);
    if (s.want & XENT_DX) {
      w.ks = dx_ranges(T, s.C, std::min(w.piece, s.V));
      w.ld_acc = (s.C + 3) / 4 * 4;
      if (w.ks > 1) w.ranges = c.take<float>((size_t)w.ks * T * w.ld_acc);
      // the pieces' sum in fp32 (with one range to a tile an fp32 dX holds it itself)
      if (w.piece < s.V && (w.ks > 1 || s.x_dtype == GC_BF16)) w.acc = c.take<float>((size_t)T * w.ld_acc);
    }
  }
  return w;
}

template <int MODE>
int run_z(XentParams p, const CUtensorMap& mX, const CUtensorMap& mW, const CUtensorMap& mOut, bool chained,
          cudaStream_t st) {
  int n = 0;
  const int rc = resident<MODE>(&n);
  if (rc) return rc;
  p.nt = tiles(MODE == STAT ? p.V : p.w);
  p.units = (int)std::min<long long>(n, (long long)p.mt * p.nt);
  p.stage_ops = p.nx + p.nw;
  p.stages = ring_bytes(MODE) / (p.stage_ops * OP_BYTES);
  return launch_mode<MODE>(mX, mW, mX, mX, mOut, mX, p, chained, st);
}

int run_grad(XentParams p, int want, const CUtensorMap& mP, const CUtensorMap& mWt, const CUtensorMap& mP4,
             const CUtensorMap& mX4, const CUtensorMap& mG, const CUtensorMap& mAcc, cudaStream_t st) {
  int n = 0;
  const int rc = resident<GRAD>(&n);
  if (rc) return rc;
  p.ct = tiles(p.C);
  p.vt = tiles(p.w);
  p.ndx = want & XENT_DX ? p.mt * p.ct * p.ks : 0;
  p.ndw = want & XENT_G ? p.N * p.vt * p.ct : 0;
  p.units = (int)std::min<long long>(n, (long long)p.ndx + p.ndw);
  // the units with one dX tile less take that much more of G
  p.r = p.ndx % p.units;
  const int dx_prod = p.np_dx == 1 ? p.nw : 1 + p.nw;
  const double cost_dx = (double)((p.w + BK - 1) / BK) / p.ks * dx_prod;
  const double cost_dw = (double)((p.n_c + BK - 1) / BK) * (1 + p.nx);
  p.extra = p.r == 0 ? 0 : std::min((int)(cost_dx / cost_dw + 0.5), p.ndw / (p.units - p.r));
  p.stage_ops = std::max(p.ndx ? p.np_dx + p.nw : 0, p.ndw ? p.np + p.nx : 0);
  p.stages = ring_bytes(GRAD) / (p.stage_ops * OP_BYTES);
  return launch_mode<GRAD>(mP, mWt, mP4, mX4, mG, mAcc, p, true, st);
}

// Rows' log-sum-exp and losses from their partial sums, and the mean.
int join_rows(const XentScratch& w, int slots, long long T, const Labels& lab, const XentIO& io, uint32_t* status,
              cudaStream_t st) {
  float* row_loss = io.row_loss ? io.row_loss : io.loss ? w.row_loss : nullptr;
  // rows enough for a block an SM: 32 each
  const bool wide = T >= 32LL * device_sm_count();
  const int rc = launch_chain(wide ? k_xent_lse<32> : k_xent_lse<4>, "k_xent_lse",
                              (unsigned)((T + (wide ? 31 : 3)) / (wide ? 32 : 4)), 256, 0, 1, true, st, w.part, slots,
                              T, lab, w.target, status, w.lse, io.lse, row_loss);
  if (rc || !io.loss) return rc;
  return launch_chain(k_xent_loss, "k_xent_loss", 1, 1024, 0, 1, true, st, row_loss, T, io.loss);
}

}  // namespace

size_t xent_ws_bytes(const XentShape& s) {
  Carve c(nullptr);
  carve_xent(c, s);
  return c.bytes();
}

int launch_xent(const XentShape& s, const XentIO& io, Carve& ws, uint32_t* status, cudaStream_t st) {
  const XentScratch w = carve_xent(ws, s);
  const long long T = (long long)s.N * s.n_c;
  const bool xb = s.x_dtype == GC_BF16, wb = s.w_dtype == GC_BF16;
  int rc = GC_OK;
  Labels lab{w.lab, nullptr, 0, s.V};
  const bool one = w.one && (io.loss || io.row_loss || io.lse);
  if (one) {
    rc = xb ? wb ? launch_one<__nv_bfloat16, __nv_bfloat16>(s, io, w.target, w.part, w.lse, status, st)
                 : launch_one<__nv_bfloat16, float>(s, io, w.target, w.part, w.lse, status, st)
            : wb ? launch_one<float, __nv_bfloat16>(s, io, w.target, w.part, w.lse, status, st)
                 : launch_one<float, float>(s, io, w.target, w.part, w.lse, status, st);
    if (rc || !s.want) return rc;
  }
  // losses alone read bf16 rows where they lie; the products of the gradient want a copy that is finite
  const bool x_in_place = !s.want && xb && rowwise::rows_16(io.X, io.ldx, 2);
  bool chained = one;  // whether the call has launched a kernel before
  if (x_in_place) {
    lab = Labels{nullptr, io.y, io.y64, s.V};
  } else {
    rc = xb ? parts_of<__nv_bfloat16>(io.X, io.ldx, T, s.C, w.Cp, 1, io.y, io.y64, s.V, w.lab, w.X, status, chained, st)
            : parts_of<float>(io.X, io.ldx, T, s.C, w.Cp, 2, io.y, io.y64, s.V, w.lab, w.X, status, chained, st);
    if (rc) return rc;
    chained = true;
  }
  if (!w.w_in_place) {
    rc = wb ? parts_of<__nv_bfloat16>(io.W, io.ldw, s.V, s.C, w.Cp, 1, nullptr, 0, 0, nullptr, w.W, status, chained, st)
            : parts_of<float>(io.W, io.ldw, s.V, s.C, w.Cp, 2, nullptr, 0, 0, nullptr, w.W, status, chained, st);
    if (rc) return rc;
    chained = true;
  }
  const void *X = x_in_place ? io.X : w.X, *W = w.w_in_place ? io.W : w.W;
  const long long ldx = x_in_place ? io.ldx : w.Cp, ldw = w.w_in_place ? io.ldw : w.Cp;
  const long long xc = x_in_place ? s.C : w.Cp, wc = w.w_in_place ? s.C : w.Cp;

  XentParams p{};
  p.T = T;
  p.C = s.C;
  p.V = s.V;
  p.N = s.N;
  p.n_c = s.n_c;
  p.nx = w.nx;
  p.nw = w.nw;
  // z in as few sums as the limit allows, of one length
  const int nkb = (s.C + BK - 1) / BK, z_most = kSegmentZ / (w.nx + w.nw - 1), z_sums = (nkb + z_most - 1) / z_most;
  p.z_seg = (nkb + z_sums - 1) / z_sums;
  p.mt = tiles(T);
  p.group = std::min(p.mt, 16);
  p.a_both = T > HALF;
  p.a_rows = T > HALF ? HALF : (int)(T + 7) / 8 * 8;
  p.lab = lab;
  p.lse = w.lse;
  p.target = w.target;
  p.part = w.part;
  p.spin_limit = wait_limit(kSpinX);
  p.stall = take_stall(GC_STALL_XENT) ? 1 : 0;
  p.status = status;

  // z: rows of X and of W, K innermost
  CUtensorMap mX, mW, mP, mWt, mP4, mX4;
  const long long dx[3] = {xc, T, w.nx}, lx[2] = {ldx, T * ldx};
  const long long dw[3] = {wc, s.V, w.nw}, lw[2] = {ldw, (long long)s.V * ldw};
  if ((rc = map_nd(&mX, X, 3, dx, lx, p.a_rows)) || (rc = map_nd(&mW, W, 3, dw, lw, HALF))) return rc;
  XentIO sums = io;
  if (w.one) {  // the lse of P alone: the outputs are there
    sums.loss = nullptr;
    sums.row_loss = sums.lse = nullptr;
  }
  if ((rc = run_z<STAT>(p, mX, mW, mX, chained, st))) return rc;
  if ((rc = join_rows(w, 2 * tiles(s.V), T, lab, sums, status, st))) return rc;
  if (!(s.want & (XENT_DX | XENT_G))) return GC_OK;

  const long long d4x[4] = {w.Cp, s.n_c, s.N, w.nx};
  const long long l4x[3] = {w.Cp, (long long)s.n_c * w.Cp, T * w.Cp};
  if ((rc = map_nd(&mWt, W, 3, dw, lw, BK)) || (rc = map_nd(&mX4, w.X, 4, d4x, l4x, BK))) return rc;
  p.P = w.P;
  p.Pp = w.piece;
  p.np = w.np;
  p.np_dx = xb ? 1 : 2;
  p.dx_bf16 = xb;
  p.dX = io.dX;
  p.ld_dx = io.lddx;
  p.split = w.ks > 1;
  p.acc = p.split ? w.ranges : xb ? w.acc : (float*)io.dX;
  p.ld_acc = p.split || xb ? w.ld_acc : io.lddx;
  p.G = io.G;
  p.ldg = io.ldg;
  p.stall = 0;
  CUtensorMap mPs, mG = mX, mAcc = mX;
  p.g_box = io.G && s.C % 4 == 0 && rowwise::rows_16(io.G, io.ldg, 4);
  if (p.g_box) {
    const long long dg[3] = {s.C, s.V, s.N}, lg[2] = {s.C, io.ldg};
    if ((rc = map_nd(&mG, io.G, 3, dg, lg, 32, 1, MAP_F32))) return rc;
  }
  p.acc_box = p.acc && (s.want & XENT_DX) && rowwise::rows_16(p.acc, p.ld_acc, 4);
  if (p.acc_box) {
    const long long da[3] = {s.C, T, std::max(1, w.ks)}, la[2] = {p.ld_acc, T * p.ld_acc};
    if ((rc = map_nd(&mAcc, p.acc, 3, da, la, 32, 1, MAP_F32))) return rc;
  }
  for (int v0 = 0; v0 < s.V; v0 += w.piece) {
    p.v0 = v0;
    p.w = std::min(w.piece, s.V - v0);
    p.ks = std::max(1, std::min(w.ks, (p.w + BK - 1) / BK));  // a short last piece has no empty range
    p.first_piece = v0 == 0;
    p.last_piece = v0 + w.piece >= s.V;
    const long long lp[2] = {w.piece, T * w.piece}, dps[3] = {w.piece, T, w.np};
    if ((rc = map_nd(&mPs, w.P, 3, dps, lp, 32, w.np))) return rc;
    if ((rc = run_z<PROB>(p, mX, mW, mPs, true, st))) return rc;
    const long long dp[3] = {p.w, T, w.np};
    const long long d4[4] = {p.w, s.n_c, s.N, w.np};
    const long long l4[3] = {w.piece, (long long)s.n_c * w.piece, T * w.piece};
    if ((rc = map_nd(&mP, w.P, 3, dp, lp, p.a_rows)) || (rc = map_nd(&mP4, w.P, 4, d4, l4, BK)))
      return rc;
    if ((rc = run_grad(p, s.want, mP, mWt, mP4, mX4, mG, mAcc, st))) return rc;
    if (p.split && (s.want & XENT_DX)) {
      const unsigned grid = (unsigned)((T * ((s.C + 3) / 4) + 255) / 256);
      void* out = p.last_piece ? io.dX : nullptr;
      rc = xb ? launch_chain(k_xent_dx<__nv_bfloat16>, "k_xent_dx", grid, 256, 0, 1, true, st, w.ranges, p.ks, T, s.C,
                             w.ld_acc, w.acc, p.first_piece, (__nv_bfloat16*)out, (long long)io.lddx)
              : launch_chain(k_xent_dx<float>, "k_xent_dx", grid, 256, 0, 1, true, st, w.ranges, p.ks, T, s.C,
                             w.ld_acc, w.acc, p.first_piece, (float*)out, (long long)io.lddx);
      if (rc) return rc;
    }
  }
  return GC_OK;
}

}  // namespace gc
