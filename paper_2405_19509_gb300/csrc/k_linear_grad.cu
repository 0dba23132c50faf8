// Gradient of a linear layer with its activation: d = dy act'(z), dx = d W, and per chunk of n_c points G_i = d_i^T x_i
// (F x C) and Gb_i = sum_t d_t.
//   k_linear_d       d as bf16 parts, and its column sums over 128 points at a time, which the tiles' warps join, or
//                    k_linear_gb; and x and W as bf16 parts where they are fp32 or do not lie on 16-byte boundaries
//   k_tiles<GradOp>  dx and all chunks' G in one launch
//   k_linear_join    dx where its tiles' sum over F runs in ranges
//
// d has 24 bits and is an operand of 16.  With bf16 rows it enters G, an fp32 result (what the encode takes), as three parts, three
// products: as hi + lo it left 2.5e-6 of G in the 2-norm where fp32 products leave 0.2 to 0.6e-6.  A bf16 dx takes hi + lo
// (2^-17): of the hi alone it was off by 2.35e-3, where its own rounding is 1.66e-3.  Without an activation d is dy, one part,
// read in place.  fp32 rows enter as three parts, six products.  The sums over a chunk depend on its points alone, bit for bit, whatever chunks a call has: the workers that
// hold a chunk form one gradient.
#include "linear_tiles.cuh"

namespace gc {
namespace {

using namespace tiles;
using namespace linear;
using namespace rowwise;

constexpr int kRowsD = 128;    // points of a block of k_linear_d
constexpr int kMostSums = 64;  // blocks of a chunk whose sums the tiles' warps join; more would hold up the first tile

// A block: 256 columns of 128 points of a chunk, a warp every eighth row, the next one's loads ahead.  The blocks past `blocks` form
// the parts of x and of W.  Bound: HBM and instructions (34 a value with gelu'); four blocks an SM, for which whole rows' loads
// have the registers, take 104 us for 8 x 1024 x 8192 in bf16 and two parts where three take 109, and 72 for 71 on rows of no
// alignment; 111 with three parts.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256, VEC ? 4 : 3)
    k_linear_d(const T* __restrict__ dy, long long lddy, const T* __restrict__ z, long long ldz, int act, int N, int n_c,
               int F, int Fp, int np, __nv_bfloat16* __restrict__ d, float* __restrict__ sums, int R, int blocks,
               const PartsJob x_parts, const PartsJob w_parts) {
  __shared__ float red[8][kSeg];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int segs = (Fp + kSeg - 1) / kSeg;
  if ((int)blockIdx.x >= blocks) {
    start_next();
    wait_prior();
    const int i = (int)blockIdx.x - blocks;
    form_parts(i < x_parts.blocks ? x_parts : w_parts, i < x_parts.blocks ? i : i - x_parts.blocks);
    return;
  }
  const long long i = blockIdx.x, block = i / segs;
  const int col0 = (int)(i - block * segs) * kSeg;
  const int chunk = (int)(block / R), r0 = (int)(block - (long long)chunk * R) * kRowsD;
  const int rows = min(kRowsD, n_c - r0);
  const long long T_all = (long long)N * n_c, first = (long long)chunk * n_c + r0;
  start_next();
  wait_prior();
  float sum[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] = 0.f;
  RawSeg<VEC, T> next_d, next_z;  // of the warp's next row
  auto take = [&](int r) {
    next_d.load(dy + (first + r) * lddy, col0, lane, F);
    if (act != GC_ACT_NONE) next_z.load(z + (first + r) * ldz, col0, lane, F);
  };
  if (warp < rows) take(warp);
#pragma unroll 1
  for (int r = warp; r < rows; r += 8) {
    const long long row = first + r;
    float v[8], u[8];
    next_d.values(v);
    if (act != GC_ACT_NONE) next_z.values(u);
    if (r + 8 < rows) take(r + 8);
    if (act != GC_ACT_NONE) times_slope(act, u, v);  // past the row's end of two zeros
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += v[j];
    uint32_t far = 0;
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      if (q == np) break;
      uint32_t w[4];
      next_part(v, q == 0, q + 1 == np, far, w);
      store_part<VEC>(d + ((size_t)q * T_all + row) * Fp, col0, lane, Fp, w);
    }
  }
  if (!sums) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) red[warp][j * 32 + lane] = sum[j];
  __syncthreads();
  const int c = VEC ? (int)(threadIdx.x & 31) * 8 + (int)(threadIdx.x >> 5) : (int)threadIdx.x;
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) s += red[w][threadIdx.x];
  if (col0 + c < F) sums[block * F + col0 + c] = s;
}

// Gb[chunk][c] from R partial sums: a block 32 columns, warp w the sums w, w + 8, ..., then the warps in order.  Where tiles
// follow and R is small their warps do it (GradOp::before).
__global__ void __launch_bounds__(256) k_linear_gb(const float* __restrict__ sums, int R, int F, float* __restrict__ Gb,
                                                   long long ldgb) {
  __shared__ float red[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int blocks = (F + 31) / 32, chunk = blockIdx.x / blocks, c = (blockIdx.x - chunk * blocks) * 32 + lane;
  start_next();
  wait_prior();
  float s = 0.f;
  if (c < F) {
    const float* at = sums + (size_t)chunk * R * F + c;
#pragma unroll 8
    for (int r = warp; r < R; r += 8) s += __ldcg(at + (size_t)r * F);
  }
  red[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < F) {
#pragma unroll
    for (int w = 1; w < 8; ++w) s += red[w][lane];
    Gb[chunk * ldgb + c] = s;
  }
}

struct GradOp {
  static constexpr bool kTurns = false;
  struct Params {
    Common q;
    Finish f;              // of dx
    long long T;
    int C, F, N;
    int tn, mt, ct, ft;    // tiles of T, of C and of F
    int ndx, dx_each, ng, r, extra; // dx tiles, round robin; then G's, `extra` each for the units past the first r, which have
                           // one dx tile less, and the rest round robin
    Ranges dx_k;           // K blocks of dx
    int c_nkb;             // ... and of G
    Divisor by_ct, by_chunk;  // column tiles; tiles of a chunk's G
    int np_dx, np, nx, nw, lim_dx, lim_g, seg_dx, seg_g;
    float* G;
    long long ldg;
    int g_box;
    const float* sums;     // of d, `R` a chunk, and where their own sum goes; NULL: no place
    int R, gb_blocks;      // blocks of 32 columns
    float* Gb;
    long long ldgb;
  };
  // Before a unit's first tile is there, its epilogue warps sum Gb, a warp 32 columns, with k_linear_gb's bits.
  static __device__ __forceinline__ void before(const Params& p, int warp, int warps) {
    if (!p.sums) return;
    const int lane = threadIdx.x & 31;
    for (int i = warp; i < p.N * p.gb_blocks; i += warps) {
      const int chunk = i / p.gb_blocks, c = (i - chunk * p.gb_blocks) * 32 + lane;
      if (c >= p.F) continue;
      const float* at = p.sums + (size_t)chunk * p.R * p.F + c;
      float s[8];
#pragma unroll
      for (int w = 0; w < 8; ++w) s[w] = 0.f;
      for (int r = 0; r < p.R; r += 8)
#pragma unroll
        for (int w = 0; w < 8; ++w)
          if (r + w < p.R) s[w] += __ldcg(at + (size_t)(r + w) * p.F);
#pragma unroll
      for (int w = 1; w < 8; ++w) s[0] += s[w];
      p.Gb[chunk * p.ldgb + c] = s[0];
    }
  }
  static __device__ __forceinline__ int jobs(const Params& p, int unit) {
    const int ndx = (p.ndx - unit + p.q.units - 1) / p.q.units;
    const int rest = p.ng - p.extra * (p.q.units - p.r);
    return ndx + (unit >= p.r ? p.extra : 0) + (rest - unit + p.q.units - 1) / p.q.units;
  }
  static __device__ __forceinline__ Job job(const Params& p, int unit, int k) {
    Job t;
    t.b_mn = true;
    t.a_turn = t.b_turn = kNever;
    const int ndx = p.dx_each + (unit < p.r ? 1 : 0);
    if (k < ndx) {
      const int i = unit + k * p.q.units, at = p.dx_k.by.of(i), m = p.by_ct.of(at);
      t.kind = t.b = 0;
      t.a_mn = false;
      t.range = i - at * p.dx_k.ks;
      t.m0 = m * TM;
      t.n0 = (at - m * p.ct) * p.tn;
      t.kb0 = p.dx_k.first(t.range);
      t.nkb = p.dx_k.count(t.range);
      t.na = p.np_dx;
      t.nb = p.nw;
      t.lim = p.lim_dx;
      t.seg = p.seg_dx;
      return t;
    }
    k -= ndx;
    const int nb = p.q.units - p.r, mine = unit >= p.r ? p.extra : 0;
    const int i = k < mine ? k * nb + unit - p.r : p.extra * nb + (k - mine) * p.q.units + unit;
    const int c = p.by_chunk.of(i), rem = i - c * (int)p.by_chunk.d, m = p.by_ct.of(rem);
    t.kind = 1;
    t.a_mn = true;
    t.range = t.kb0 = 0;
    t.b = c;
    t.m0 = m * TM;
    t.n0 = (rem - m * p.ct) * p.tn;
    t.nkb = p.c_nkb;
    t.na = p.np;
    t.nb = p.nx;
    t.lim = p.lim_g;
    t.seg = p.seg_g;
    return t;
  }
  template <int NC, typename Get>
  static __device__ __forceinline__ void store(const Params& p, const Job& t, int row0, int col0, uint8_t* box,
                                               const CUtensorMap* out, Get get) {
    const int lane = threadIdx.x & 31;
    if (t.kind == 0) {
      store_rows<NC>(p.f, p.T, p.dx_k.ks > 1 ? t.range : -1, out, row0, col0, box, out, get);
      box_free(lane);  // a tile of G may write the box otherwise
      return;
    }
    const int rows = min(p.F - row0, 32);
#pragma unroll 1
    for (int c = 0; c < NC; ++c) {
      float v[32];
      __syncwarp();
      get(c, v);
      const int col = col0 + c * 32;
      if (rows <= 0 || col >= p.C) continue;
      if (p.g_box) {
        store_32(&out[1], box, lane, v, p.C - col, col, row0, t.b);
      } else {
        float* g = p.G + t.b * p.ldg + (long long)row0 * p.C + col;
        by_rows(box, lane, v, rows, p.C - col, [&](int r, int j, float s) { g[(long long)r * p.C + j] = s; });
      }
    }
    if (p.g_box) box_free(lane);  // and a tile of dx
  }
};

struct Scratch {
  int Cp, Fp, np, np_dx, nx, nw, lim_dx, lim_g, tn, ks, ld_part, R;
  bool x_in_place, w_in_place, d_in_place;
  __nv_bfloat16 *X, *W, *D;
  float *part, *sums;
};

// Clocks of a tile.
double tile_clocks(int tn, int nkb, int prod) { return nkb * block_clocks(tn, prod) + 600; }

Scratch carve_grad(Carve& c, const LinearGradShape& s) {
  Scratch w{};
  const long long T = (long long)s.N * s.n_c;
  const bool xb = s.x_dtype == GC_BF16, wb = s.w_dtype == GC_BF16;
  const bool dx = s.want & LINEAR_DX, g = s.want & LINEAR_G;
  w.Cp = (s.C + 7) / 8 * 8;
  w.Fp = (s.F + 7) / 8 * 8;
  w.nx = xb ? 1 : 3;
  w.nw = wb ? 1 : xb ? 2 : 3;
  w.lim_dx = xb ? 2 : 3;
  w.lim_g = 3;
  w.np_dx = !xb ? 3 : s.act != GC_ACT_NONE ? 2 : 1;
  w.np = !dx && !g ? 0 : g && s.act != GC_ACT_NONE ? 3 : w.np_dx;
  w.d_in_place = xb && s.act == GC_ACT_NONE && s.dy_16;
  w.x_in_place = xb && s.x_16;
  w.w_in_place = wb && s.w_16;
  if (w.np && !w.d_in_place) w.D = c.take<__nv_bfloat16>((size_t)w.np * T * w.Fp);
  if (g && !w.x_in_place) w.X = c.take<__nv_bfloat16>((size_t)w.nx * T * w.Cp);
  if (dx && !w.w_in_place) w.W = c.take<__nv_bfloat16>((size_t)w.nw * s.F * w.Cp);
  w.R = (s.n_c + kRowsD - 1) / kRowsD;
  if (s.want & LINEAR_GB) w.sums = c.take<float>((size_t)s.N * w.R * s.F);
  // the cut whose estimated clocks are fewest, as split_of's, over both kinds of tiles
  const int units = device_sm_count() / 2;
  const int f_nkb = (s.F + BK - 1) / BK, c_nkb = (s.n_c + BK - 1) / BK;
  const int p_dx = products(w.np_dx, w.nw, w.lim_dx), p_g = products(w.np, w.nx, w.lim_g);
  double least = 0;
  w.tn = 256;
  w.ks = 1;
  for (int tn = 256; tn >= 128; tn /= 2) {
    const double nd = dx ? (double)tiles_of(T, TM) * tiles_of(s.C, tn) : 0;
    const double ng = g ? (double)s.N * tiles_of(s.F, TM) * tiles_of(s.C, tn) : 0;
    const double one_g = ng > 0 ? tile_clocks(tn, c_nkb, p_g) : 0;
    for (int ks = 1; ks <= (dx ? 32 : 1) && ks * 2 <= std::max(2, f_nkb); ++ks) {
      if (ks > 1 && nd * (ks - 1) >= 2 * units) break;
      const double one_d = nd > 0 ? tile_clocks(tn, (f_nkb + ks - 1) / ks, p_dx) : 0;
      const double longest = std::max(one_d, one_g), share = (nd * ks * one_d + ng * one_g) / units;
      double clk = std::max(longest, share + (nd * ks + ng > units ? std::min(longest, ng > 0 ? one_g : one_d) / 2 : 0));
      if (ks > 1) clk += 3000 + (double)T * s.C * 8 * ks / 3500;
      if (least == 0 || clk < least) {
        least = clk;
        w.tn = tn;
        w.ks = ks;
      }
    }
  }
  w.ld_part = (s.C + 3) / 4 * 4;
  if (w.ks > 1) w.part = c.take<float>((size_t)w.ks * T * w.ld_part);
  return w;
}

template <typename T>
int launch_d(const LinearGradShape& s, const LinearGradIO& io, const Scratch& w, int np, const PartsJob& x, const PartsJob& W,
             cudaStream_t st) {
  const bool vec = s.F % 8 == 0 && rows_16(io.dy, io.lddy, sizeof(T)) && (s.act == GC_ACT_NONE || rows_16(io.z, io.ldz, sizeof(T)));
  const long long grid = (long long)s.N * w.R * ((w.Fp + kSeg - 1) / kSeg);
  return launch_chain(vec ? k_linear_d<T, true> : k_linear_d<T, false>, "k_linear_d", (unsigned)(grid + x.blocks + W.blocks), 256, 0,
                      1, false, st, (const T*)io.dy, (long long)io.lddy, (const T*)io.z, (long long)io.ldz, s.act, s.N, s.n_c,
                      s.F, w.Fp, np, w.D, w.sums, w.R, (int)grid, x, W);
}

// The outputs that k_linear_small.cu forms.
int small_part(const LinearGradShape& s) {
  return s.want & ((linear_small_dx(s) ? LINEAR_DX : 0) | (linear_small_g(s) ? LINEAR_G | LINEAR_GB : 0));
}

int launch_grad_tiles(const LinearGradShape& s, const LinearGradIO& io, Carve& ws, uint32_t* status, cudaStream_t st) {
  const Scratch w = carve_grad(ws, s);
  const long long T = (long long)s.N * s.n_c;
  const bool xb = s.x_dtype == GC_BF16;
  const bool dx = s.want & LINEAR_DX, g = s.want & LINEAR_G;
  int rc = GC_OK;
  bool chained = false;
  const int np = w.d_in_place ? 0 : w.np;
  PartsJob xp{}, wp{};
  if (g && !w.x_in_place) xp = parts_job(io.X, s.x_dtype, io.ldx, T, s.C, w.Cp, w.nx, w.X);
  if (dx && !w.w_in_place) wp = parts_job(io.W, s.w_dtype, io.ldw, s.F, s.C, w.Cp, w.nw, w.W);
  if (np || w.sums) {
    rc = xb ? launch_d<__nv_bfloat16>(s, io, w, np, xp, wp, st) : launch_d<float>(s, io, w, np, xp, wp, st);
    if (rc) return rc;
    chained = true;
  } else if (xp.blocks + wp.blocks) {
    if ((rc = launch_parts(xp, wp, st))) return rc;
    chained = true;
  }
  const bool gb_in_tiles = w.sums && (dx || g) && w.R <= kMostSums;
  if (w.sums && !gb_in_tiles) {
    if ((rc = launch_chain(k_linear_gb, "k_linear_gb", (unsigned)(s.N * ((s.F + 31) / 32)), 256, 0, 1, chained, st, w.sums,
                           w.R, s.F, io.Gb, (long long)io.ldgb)))
      return rc;
  }
  if (!dx && !g) return GC_OK;
  const void *X = w.x_in_place ? io.X : w.X, *W = w.w_in_place ? io.W : w.W, *D = w.d_in_place ? io.dy : w.D;
  const long long ldx = w.x_in_place ? io.ldx : w.Cp, ldw = w.w_in_place ? io.ldw : w.Cp;
  const long long ldd = w.d_in_place ? io.lddy : w.Fp;
  GradOp::Params p{};
  p.f = finish_of(s, io);
  p.T = T;
  p.C = s.C;
  p.F = s.F;
  p.N = s.N;
  p.tn = w.tn;
  p.mt = tiles_of(T, TM);
  p.ct = tiles_of(s.C, w.tn);
  p.ft = tiles_of(s.F, TM);
  const int f_nkb = (s.F + BK - 1) / BK;
  p.dx_k = Ranges(f_nkb, w.ks);
  p.c_nkb = (s.n_c + BK - 1) / BK;
  p.by_ct = Divisor((uint32_t)p.ct);
  p.by_chunk = Divisor((uint32_t)(p.ft * p.ct));
  p.np_dx = w.np_dx;
  p.np = w.np;
  p.nx = w.nx;
  p.nw = w.nw;
  p.lim_dx = w.lim_dx;
  p.lim_g = w.lim_g;
  const int prod_dx = products(w.np_dx, w.nw, w.lim_dx), prod_g = products(w.np, w.nx, w.lim_g);
  p.seg_dx = segment(xb, prod_dx, f_nkb);
  p.seg_g = segment(false, prod_g, p.c_nkb);
  p.G = io.G;
  p.ldg = io.ldg;
  p.sums = gb_in_tiles ? w.sums : nullptr;
  p.R = w.R;
  p.gb_blocks = (s.F + 31) / 32;
  p.Gb = io.Gb;
  p.ldgb = io.ldgb;
  p.ndx = dx ? p.mt * p.ct * w.ks : 0;
  p.ng = g ? s.N * p.ft * p.ct : 0;
  int units = 0;
  if ((rc = w.tn == 256 ? resident<GradOp, 256>(&units) : resident<GradOp, 128>(&units))) return rc;
  units = (int)std::min<long long>(units, (long long)p.ndx + p.ng);
  p.r = p.ndx % units;
  p.dx_each = p.ndx / units;
  // of G with a short sum those of its store, 256 x tn values: at a pair's share of HBM in boxes, at a quarter of it by rows
  p.g_box = g && s.C % 4 == 0 && rows_16(io.G, io.ldg, 4);
  const double cost_dx = tile_clocks(w.tn, (f_nkb + w.ks - 1) / w.ks, prod_dx);
  const double cost_g = std::max(tile_clocks(w.tn, p.c_nkb, prod_g), (p.g_box ? 25.0 : 90.0) * w.tn);
  p.extra = p.r == 0 ? 0 : std::min((int)(cost_dx / cost_g + 0.5), p.ng / (units - p.r));
  p.q.a_both = T > 128;
  p.q.a_rows = T > 128 ? 128 : (int)(T + 7) / 8 * 8;
  p.q.spin_limit = wait_limit(kSpin);
  p.q.stall = take_stall(GC_STALL_LINEAR) ? 1 : 0;
  p.q.status = status;
  Maps m;
  if ((rc = operand_map(&m.a[0], D, false, s.F, T, 1, w.np, ldd, T * ldd, T * ldd, p.q.a_rows)) ||
      (rc = operand_map(&m.a[1], D, false, s.F, s.n_c, s.N, w.np, ldd, s.n_c * ldd, T * ldd, BK)))
    return rc;
  m.b[0] = m.b[1] = m.a[0];
  m.out[0] = m.out[1] = m.a_turned = m.b_turned = m.a[0];
  if (dx && (rc = finish_maps(&p.f, T, w.part, w.ks, w.ld_part, &m))) return rc;
  if (dx && (rc = operand_map(&m.b[0], W, false, s.C, s.F, 1, w.nw, ldw, s.F * ldw, s.F * ldw, BK))) return rc;
  if (g) {
    if ((rc = operand_map(&m.b[1], X, false, s.C, s.n_c, s.N, w.nx, ldx, s.n_c * ldx, T * ldx, BK))) return rc;
    if (p.g_box) {
      if ((rc = box_map(&m.out[1], io.G, MAP_F32, s.C, s.F, s.N, s.C, io.ldg))) return rc;
    }
  }
  const long long jobs = (long long)p.ndx + p.ng;
  const int most_a = std::max(dx ? w.np_dx : 0, g ? w.np : 0), most_b = std::max(dx ? w.nw : 0, g ? w.nx : 0);
  rc = w.tn == 256 ? launch_tiles<GradOp, 256>(m, p, jobs, most_a, most_b, "k_linear_grad", chained, st)
                   : launch_tiles<GradOp, 128>(m, p, jobs, most_a, most_b, "k_linear_grad", chained, st);
  if (rc || !dx || w.ks == 1) return rc;
  return launch_join(w.part, w.ks, T, w.ld_part, p.f, st);
}

}  // namespace

size_t linear_grad_ws_bytes(const LinearGradShape& s) {
  Carve c(nullptr);
  LinearGradShape t = s;
  t.want &= ~small_part(s);
  if (t.want) carve_grad(c, t);
  return c.bytes();
}

int launch_linear_grad(const LinearGradShape& s, const LinearGradIO& io, Carve& ws, uint32_t* status, cudaStream_t st) {
  if (const int few = small_part(s)) {
    LinearGradIO a = io, b = io;
    (few & LINEAR_DX ? b : a).dX = nullptr;
    (few & LINEAR_G ? b : a).G = nullptr;
    (few & LINEAR_GB ? b : a).Gb = nullptr;
    const int rc = launch_linear_grad_small(s, a, finish_of(s, a), st);
    if (rc || few == s.want) return rc;
    LinearGradShape t = s;
    t.want &= ~few;
    return launch_grad_tiles(t, b, ws, status, st);
  }
  return launch_grad_tiles(s, io, ws, status, st);
}

}  // namespace gc
