// A linear layer: z = x W^T + b, y = residual + act(z), for T rows of C values and F rows of W.
//   k_parts         x and W as bf16 parts where they are fp32 or do not lie on 16-byte boundaries
//   k_tiles<FwdOp>  z tile by tile in tensor memory; bias, activation and residual in the epilogue, z kept on request
//   k_linear_join   the same epilogue where a tile's sum over C runs in ranges
//
// A bf16 x with a bf16 W is one product; an fp32 W enters it as hi + lo (2^-17), two products, so that a bf16 result
// is rounded once.  An fp32 x enters as three parts, 24 bits: with an fp32 W six products (parts i + j < 3), off in the 2-norm by 0.8e-7
// for C = 64 and 6e-7 from 128 on, where fp32 products are off by 1.4e-7, 2e-7 and, for 8192, 1.6e-6.
#include "linear_tiles.cuh"

namespace gc {
namespace {

using namespace tiles;
using namespace linear;

struct FwdOp {
  static constexpr bool kTurns = false;
  struct Params {
    Common q;
    Finish f;
    long long T;
    int mt, nt, tn, group;  // tiles of T and of F; row tiles that share a sweep of the columns
    Divisor per, full, rest;  // tiles of a group of rows; its row tiles, and those of the last group
    Ranges k;
    int seg;
    int nx, nw, lim;
  };
  static __device__ __forceinline__ void before(const Params&, int, int) {}
  static __device__ __forceinline__ int jobs(const Params& p, int unit) {
    return (int)(((long long)p.mt * p.nt * p.k.ks - unit + p.q.units - 1) / p.q.units);
  }
  static __device__ __forceinline__ Job job(const Params& p, int unit, int k) {
    const int i = unit + k * p.q.units, at = p.k.by.of(i);
    const int g = p.per.of(at), rem = at - g * (int)p.per.d;
    const bool last = (g + 1) * p.group > p.mt;
    const int n = last ? p.rest.of(rem) : p.full.of(rem);
    Job t;
    t.kind = t.b = 0;
    t.range = i - at * p.k.ks;
    t.m0 = (g * p.group + rem - n * (int)(last ? p.rest.d : p.full.d)) * TM;
    t.n0 = n * p.tn;
    t.kb0 = p.k.first(t.range);
    t.nkb = p.k.count(t.range);
    t.na = p.nx;
    t.nb = p.nw;
    t.lim = p.lim;
    t.seg = p.seg;
    t.a_mn = t.b_mn = false;
    t.a_turn = t.b_turn = kNever;
    return t;
  }
  template <int NC, typename Get>
  static __device__ __forceinline__ void store(const Params& p, const Job& t, int row0, int col0, uint8_t* box,
                                               const CUtensorMap* out, Get get) {
    store_rows<NC>(p.f, p.T, p.k.ks > 1 ? t.range : -1, out, row0, col0, box, out, get);
  }
};

struct Scratch {
  int Cp, nx, nw, lim, tn, ks, ld_part;
  bool x_in_place, w_in_place;
  __nv_bfloat16 *X, *W;
  float* part;
};

Scratch carve_linear(Carve& c, const LinearShape& s) {
  Scratch w{};
  const bool xb = s.x_dtype == GC_BF16, wb = s.w_dtype == GC_BF16;
  w.Cp = (s.C + 7) / 8 * 8;
  w.nx = xb ? 1 : 3;
  w.nw = wb ? 1 : xb ? 2 : 3;
  w.lim = xb ? 2 : 3;
  w.x_in_place = xb && s.x_16;
  w.w_in_place = wb && s.w_16;
  if (!w.x_in_place) w.X = c.take<__nv_bfloat16>((size_t)w.nx * s.T * w.Cp);
  if (!w.w_in_place) w.W = c.take<__nv_bfloat16>((size_t)w.nw * s.F * w.Cp);
  const int prod = products(w.nx, w.nw, w.lim);
  const Split cut = split_of([&](int tn) { return (long long)tiles_of(s.T, TM) * tiles_of(s.F, tn); }, (double)s.T * s.F,
                             (s.C + BK - 1) / BK, prod, device_sm_count() / 2);
  w.tn = cut.tn;
  w.ks = cut.ks;
  w.ld_part = (s.F + 3) / 4 * 4;
  if (w.ks > 1) w.part = c.take<float>((size_t)w.ks * s.T * w.ld_part);
  return w;
}

}  // namespace

size_t linear_ws_bytes(const LinearShape& s) {
  Carve c(nullptr);
  if (!linear_small(s)) carve_linear(c, s);
  return c.bytes();
}

int launch_linear(const LinearShape& s, const LinearIO& io, Carve& ws, uint32_t* status, cudaStream_t st) {
  if (linear_small(s)) return launch_linear_small(s, io, finish_of(s, io), st);
  const Scratch w = carve_linear(ws, s);
  const bool xb = s.x_dtype == GC_BF16;
  int rc = GC_OK;
  bool chained = false;
  if (!w.x_in_place || !w.w_in_place) {
    const PartsJob none{};
    if ((rc = launch_parts(w.x_in_place ? none : parts_job(io.X, s.x_dtype, io.ldx, s.T, s.C, w.Cp, w.nx, w.X),
                           w.w_in_place ? none : parts_job(io.W, s.w_dtype, io.ldw, s.F, s.C, w.Cp, w.nw, w.W), st)))
      return rc;
    chained = true;
  }
  const void *X = w.x_in_place ? io.X : w.X, *W = w.w_in_place ? io.W : w.W;
  const long long ldx = w.x_in_place ? io.ldx : w.Cp, ldw = w.w_in_place ? io.ldw : w.Cp;
  FwdOp::Params p{};
  p.f = finish_of(s, io);
  p.T = s.T;
  p.tn = w.tn;
  p.mt = tiles_of(s.T, TM);
  p.nt = tiles_of(s.F, w.tn);
  p.group = std::min(p.mt, 16);
  p.per = Divisor((uint32_t)(p.group * p.nt));
  p.full = Divisor((uint32_t)p.group);
  p.rest = Divisor((uint32_t)(p.mt % p.group ? p.mt % p.group : p.group));
  const int nkb = (s.C + BK - 1) / BK;
  p.k = Ranges(nkb, w.ks);
  p.nx = w.nx;
  p.nw = w.nw;
  p.lim = w.lim;
  p.seg = segment(xb, products(w.nx, w.nw, w.lim), nkb);
  p.q.a_both = s.T > 128;
  p.q.a_rows = s.T > 128 ? 128 : (int)(s.T + 7) / 8 * 8;
  p.q.spin_limit = wait_limit(kSpin);
  p.q.stall = take_stall(GC_STALL_LINEAR) ? 1 : 0;
  p.q.status = status;
  Maps m;
  if ((rc = operand_map(&m.a[0], X, false, s.C, s.T, 1, w.nx, ldx, s.T * ldx, s.T * ldx, p.q.a_rows)) ||
      (rc = operand_map(&m.b[0], W, false, s.C, s.F, 1, w.nw, ldw, s.F * ldw, s.F * ldw, w.tn / 2)))
    return rc;
  m.a[1] = m.a[0];
  m.b[1] = m.b[0];
  if ((rc = finish_maps(&p.f, s.T, w.part, w.ks, w.ld_part, &m))) return rc;
  const long long jobs = (long long)p.mt * p.nt * w.ks;
  rc = w.tn == 256 ? launch_tiles<FwdOp, 256>(m, p, jobs, w.nx, w.nw, "k_linear", chained, st)
                   : launch_tiles<FwdOp, 128>(m, p, jobs, w.nx, w.nw, "k_linear", chained, st);
  if (rc || w.ks == 1) return rc;
  return launch_join(w.part, w.ks, s.T, w.ld_part, p.f, st);
}

}  // namespace gc
