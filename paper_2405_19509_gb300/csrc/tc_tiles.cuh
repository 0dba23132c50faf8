// Matrix products in tiles on the tensor cores, as one persistent kernel: k_tiles<Op, TN> works through the
// tiles that an operator `Op` lists (which operands, which range of K) and hands each finished tile to its epilogue.
//
// A pair of CTAs (cta_group::2) takes a 256 x TN tile, TN = 256 or 128, each CTA holding 128 rows of A and TN / 2
// of B for a 64-wide K block: warp 0 loads them by TMA, the leader's warp 1 issues the MMAs, sixteen warps per CTA
// drain one of two accumulators while the other is filled.  Operands lie K-major (rows of K, K innermost) or MN-major (K
// outermost: boxes of 64 columns x 64 K rows).  A value enters in up to three 16-bit parts (x = x0 + x1 + ..., each
// the rounded rest of those before), and the products of parts i and j with i + j < lim are summed: bf16 parts of an
// fp32 value keep 8 bits each whatever its size, fp16 parts 11 each of values that are scaled to the middle of the range.
//
// Sums: an addition in tensor memory is cut off, not rounded, about 4e-8 of the sum so far a step and always towards zero.  So the
// products of a K block end with the largest parts', and those before meet no sum of full size where a segment begins (4096 x 2048 ->
// 4096 in fp32: 1.2e-6 off in the 2-norm the other way round, 0.64e-6 so, at the same time), and 32-bit results leave tensor
// memory every `seg` K blocks and are added in registers.
//
// Bound: the tensor pipe (4 x 128 clocks a K block of one product at TN = 256; TN = 128 spreads few tiles) where tiles are many, else the
// latency of a tile: barriers, the first loads and the epilogue, some 3 us.  Every wait is bounded (GC_ERR_TIMEOUT).
#pragma once

#include <algorithm>

#include "rowwise.cuh"
#include "tc_host.cuh"
#include "tc_pair.cuh"

namespace gc {
namespace tiles {

using namespace tcp;

constexpr int TM = 256, BK = 64;
constexpr int A_BYTES = 128 * BK * 2;  // a CTA's share of a part of A's K block
constexpr int kEpi = 16;               // a quarter of the rows and of the columns each
constexpr int kThreads = 64 + 32 * kEpi;
constexpr int BOX = 32 * 64;           // an epilogue warp's box: 32 rows of 64 bytes
constexpr int RING = 12 * A_BYTES;
constexpr int kMaxStages = 8;
constexpr size_t kSmem = RING + kEpi * BOX + 1024 + 256;
static_assert(kSmem <= kSmemMax, "shared memory");
constexpr long long kSpin = 1LL << 32;

// i / d for 0 <= i < 2^31, 1 <= d < 2^31, by a product (Granlund and Montgomery, "Division by invariant integers using
// multiplication", PLDI 1994): tiles are many and short, and each is found by a few divisions in every role.
struct Divisor {
  uint32_t d, mul, shift;
  Divisor() = default;
  __host__ explicit Divisor(uint32_t n) : d(n) {
    shift = 0;
    while ((1ull << shift) < n) ++shift;
    mul = (uint32_t)(((1ull << 31) * (1ull << shift) + n - 1) / n - (1ull << 31));  // ceil(2^(31 + shift) / n), less 2^31
  }
  __device__ __forceinline__ int of(int i) const {
    return (int)(((unsigned long long)mul * (uint32_t)i + ((unsigned long long)(uint32_t)i << 31)) >> (31 + shift));
  }
};
// nkb K blocks in ks ranges, the first `more` of them one longer.
struct Ranges {
  int ks, each, more;
  Divisor by;
  Ranges() = default;
  __host__ Ranges(int nkb, int n) : ks(n), each(nkb / n), more(nkb % n), by((uint32_t)n) {}
  __device__ __forceinline__ int first(int r) const { return r * each + min(r, more); }
  __device__ __forceinline__ int count(int r) const { return each + (r < more ? 1 : 0); }
};

// One tile: rows [m0, m0 + 256) x columns [n0, n0 + TN) of batch b, K blocks [kb0, kb0 + nkb).
struct Job {
  int kind, m0, n0, b, kb0, nkb, range;
  int na, nb, lim;      // parts of A and of B; products of parts i + j < lim
  int seg;              // K blocks that are summed in tensor memory at a time
  bool a_mn, b_mn;
  int a_turn, b_turn;   // K blocks from which a symmetric operand's are read as their mirrors below the diagonal (kNever)
};
constexpr int kNever = 1 << 30;
// Products of parts i + j < lim.
__host__ __device__ inline int products(int na, int nb, int lim) {
  int n = 0;
  for (int i = 0; i < na; ++i) n += max(0, min(nb, lim - i));
  return n;
}
// The K block from which on a symmetric operand's rows `row` .. are read as their mirrors: the blocks of 256 up to the diagonal exist.
__device__ __forceinline__ int turn_of(int row) { return (row / TM + 1) * (TM / BK); }

// What every operator's parameters hold.
struct Common {
  int units, stage_bytes, stages;
  int a_rows, a_both;   // rows that a CTA loads of a K-major A, and whether the second half of a tile has any
  int f16;              // parts are fp16 (else bf16)
  long long spin_limit;
  int stall;
  uint32_t* status;
};

// Tensor maps of (inner, rows, batch, part) by kind, and the epilogue's.
struct Maps {
  CUtensorMap a[2], b[2], out[2], a_turned, b_turned;
};

__device__ __forceinline__ void start_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_prior() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Instruction descriptor, kind::f16: D fp32, M = 256, N = tn over the pair, A and B both bf16 or both fp16.
__device__ __forceinline__ uint32_t idesc_of(int tn, bool f16, bool a_mn, bool b_mn) {
  return (1u << 4) | (f16 ? 0u : (1u << 7) | (1u << 10)) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
         ((uint32_t)(tn >> 3) << 17) | ((256u >> 4) << 24);
}

// An epilogue warp's 32 x 32 values go through its box, a lane a row: 32 columns of 16 bits or 16 of 32 bits at a time.  Piece j
// (16 bytes) of row r lies at j ^ (r / 2 mod 4), TMA's 64-byte swizzle, so that rows and pieces are written and read without
// bank conflicts.
__device__ __forceinline__ int box_place(int r, int j) { return r * 64 + (j ^ ((r >> 1) & 3)) * 16; }

// Before a box is written: the stores that lane 0 issued from it have read it.
__device__ __forceinline__ void box_free(int lane) {
  if (lane == 0) bulk_wait_read<0>();
  __syncwarp();
}
// two(j): values j and j + 1 as a packed pair.
template <typename Pack>
__device__ __forceinline__ void box_put_16(uint8_t* box, int lane, Pack two) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *reinterpret_cast<uint4*>(box + box_place(lane, j)) = make_uint4(two(8 * j), two(8 * j + 2), two(8 * j + 4), two(8 * j + 6));
}
__device__ __forceinline__ void box_put_32(uint8_t* box, int lane, const float* v) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *reinterpret_cast<float4*>(box + box_place(lane, j)) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}
// The box leaves for (col, row, plane).
__device__ __forceinline__ void box_store(const CUtensorMap* map, const uint8_t* box, int lane, int col, int row, int plane) {
  fence_async_smem();
  __syncwarp();
  if (lane == 0) {
    store_3d(map, box, col, row, plane);
    bulk_commit();
  }
}
// 32 x 32 values of 32 bits, of which the first n columns exist.
__device__ __forceinline__ void store_32(const CUtensorMap* map, uint8_t* box, int lane, const float (&v)[32], int n, int col, int row,
                                         int plane) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (16 * h >= n) break;
    box_free(lane);
    box_put_32(box, lane, v + 16 * h);
    box_store(map, box, lane, col + 16 * h, row, plane);
  }
}
// 32 rows of 64 bytes from memory, four neighbouring lanes a row; they reach a lane a row by way of the box.
struct Rows32 {
  uint4 q[4];
  // the first `rows` rows, `ld` bytes apart, of which `bytes` exist, a multiple of 16
  __device__ __forceinline__ void load(const void* from, long long ld, int rows, int bytes, int lane) {
    const int j = lane % 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = i * 8 + lane / 4;
      q[i] = r < rows && j * 16 < bytes ? __ldcg(reinterpret_cast<const uint4*>(static_cast<const char*>(from) + r * ld + j * 16))
                                        : make_uint4(0, 0, 0, 0);
    }
  }
  // ... as the lane's own row.  The box is free before; the lane may write its own row after.
  __device__ __forceinline__ void turn(uint8_t* box, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(box + box_place(i * 8 + lane / 4, lane % 4)) = q[i];
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = *reinterpret_cast<const uint4*>(box + box_place(lane, j));
    __syncwarp();
  }
};
// f(r, c, value) for the first `rows` rows and `n` columns, 16 neighbouring lanes a row: for rows on no boundary.
template <typename F>
__device__ __forceinline__ void by_rows(uint8_t* box, int lane, const float (&v)[32], int rows, int n, F f) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = 16 * h + lane % 16;
    __syncwarp();
    box_put_32(box, lane, v + 16 * h);
    __syncwarp();
    if (c >= n) continue;
    for (int r0 = lane / 16; r0 < rows; r0 += 16) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const float*>(box + box_place(r0 + 2 * i, c % 16 / 4) + c % 4 * 4);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r0 + 2 * i < rows) f(r0 + 2 * i, c, x[i]);
    }
  }
}

// How a K block's operands lie: descriptors of the first stage's, their steps of 16 K, and the instruction's.
template <int TN>
struct Way {
  uint32_t idesc, a_step, b_step;
  uint64_t a, b;
  __device__ __forceinline__ Way(const Common& q, const Job& t, const uint8_t* smem, bool a_mn, bool b_mn) {
    constexpr int B_BYTES = TN / 2 * BK * 2;
    idesc = idesc_of(TN, q.f16, a_mn, b_mn);
    a_step = (a_mn ? 2048 : 32) >> 4;
    b_step = (b_mn ? 2048 : 32) >> 4;
    a = sdesc(smem_u32(smem), a_mn ? A_BYTES / 2 : 16, 1024);
    b = sdesc(smem_u32(smem) + t.na * A_BYTES, b_mn ? (TN == 256 ? B_BYTES / 2 : B_BYTES) : 16, 1024);
  }
};

template <class Op, int TN>
__global__ void __launch_bounds__(kThreads, 1) k_tiles(const __grid_constant__ Maps maps,
                                                        const __grid_constant__ typename Op::Params p) {
  constexpr int HN = TN / 2;             // B rows of a CTA
  constexpr int QN = TN / 4;             // columns of an epilogue warp
  constexpr int B_BYTES = HN * BK * 2;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t* boxes = smem + RING;
  // the leader's: the pair's loads landed; each CTA's: the MMAs on the stage are done
  uint64_t* full = reinterpret_cast<uint64_t*>(boxes + kEpi * BOX);
  uint64_t* empty = full + kMaxStages;
  uint64_t* tfull = empty + kMaxStages;  // [2] each CTA's: accumulator filled
  uint64_t* tempty = tfull + 2;          // [2] the leader's: drained by both CTAs
  uint64_t* done = tempty + 2;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const Common& q = p.q;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int unit = blockIdx.x / 2;
  const int side = (int)cta_rank();      // the half of the pair's rows
  const int S = q.stages;
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
  if (warp == 1) tmem_alloc(tmem_holder, 2 * TN);
  fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  fence_after();
  const uint32_t tmem_base = *tmem_holder;
  start_next();
  wait_prior();
  const int njobs = Op::jobs(p, unit);
  if (warp == 0) {
    const bool one = elect_one();
    uint32_t it = 0, ph = 0;
    int s = 0;
    bool ok = !q.stall;
    for (int k = 0; k < njobs && ok; ++k) {
      const Job t = Op::job(p, unit, k);
      const int ma = t.m0 + side * 128, nb = t.n0 + side * HN;
      for (int kb = t.kb0; kb < t.kb0 + t.nkb; ++kb, ++it) {
        if (!mbar_wait(&empty[s], ph ^ 1, abort_flag, q.status, q.spin_limit)) ok = false;
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        const bool a_turned = Op::kTurns && kb >= t.a_turn, b_turned = Op::kTurns && kb >= t.b_turn;
        const bool a_mn = t.a_mn || a_turned, b_mn = t.b_mn || b_turned;
        const bool skip_a = !a_mn && side == 1 && !q.a_both;
        const CUtensorMap* mA = a_turned ? &maps.a_turned : &maps.a[t.kind];
        const CUtensorMap* mB = b_turned ? &maps.b_turned : &maps.b[t.kind];
        if (one) {
          const uint32_t bytes = 2 * t.nb * B_BYTES +
                                 (a_mn ? 2 * t.na * A_BYTES : t.na * q.a_rows * BK * 2 * (q.a_both ? 2 : 1));
          if (side == 0) mbar_expect_tx(&full[s], bytes);
          const uint32_t bar = at_rank(&full[s], 0);
          uint8_t* st = smem + (size_t)s * q.stage_bytes;
          for (int i = 0; i < t.na; ++i, st += A_BYTES) {
            if (a_mn) {
              load_4d(st, mA, ma, kb * BK, t.b, i, bar);
              load_4d(st + A_BYTES / 2, mA, ma + 64, kb * BK, t.b, i, bar);
            } else if (!skip_a) {
              load_4d(st, mA, kb * BK, ma, t.b, i, bar);
            }
          }
          for (int i = 0; i < t.nb; ++i, st += B_BYTES) {
            if (b_mn) {
              load_4d(st, mB, nb, kb * BK, t.b, i, bar);
              if (TN == 256) load_4d(st + B_BYTES / 2, mB, nb + 64, kb * BK, t.b, i, bar);
            } else {
              load_4d(st, mB, kb * BK, nb, t.b, i, bar);
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
      const bool in = mbar_wait(&empty[k % S], (k / S) & 1, &no_abort, q.status, 1LL << 28);
      if (!__all_sync(0xffffffffu, in)) break;
    }
  } else if (warp == 1) {
    if (side == 0) {
      const bool one = elect_one();
      const uint16_t pair = 3;
      uint32_t ph = 0, use = 0;  // use: accumulators filled so far, in turn the one and the other
      int s = 0;
      bool ok = true;
      for (int k = 0; k < njobs && ok; ++k) {
        const Job t = Op::job(p, unit, k);
        Way<TN> way(q, t, smem, t.a_mn, t.b_mn);
        // from A's smallest part, with those of B that are taken with it, to the largest; found here, since what the issuing
        // warp does between two K blocks of one product shows (8192 x 2048 -> 8192: 3%)
        const int b_parts = min(t.nb, t.lim + 1 - t.na);
        const uint32_t a_end = (uint32_t)((t.na - 1) * (A_BYTES >> 4)), b_end = (uint32_t)((b_parts - 1) * (B_BYTES >> 4));
        for (int kb = 0, left = 0; kb < t.nkb; ++kb) {
          const int ab = use & 1;
          if (left == 0) {
            left = t.seg;
            ok = mbar_wait(&tempty[ab], ((use >> 1) & 1) ^ 1, abort_flag, q.status, q.spin_limit);
          }
          ok = ok && mbar_wait(&full[s], ph, abort_flag, q.status, q.spin_limit);
          if (!__all_sync(0xffffffffu, ok)) {
            ok = false;
            break;
          }
          const bool opens = left == t.seg, closes = --left == 0 || kb == t.nkb - 1;
          if (opens) fence_after();
          if (Op::kTurns)
            way = Way<TN>(q, t, smem, t.a_mn || t.kb0 + kb >= t.a_turn, t.b_mn || t.kb0 + kb >= t.b_turn);
          if (one) {
            const uint32_t d = tmem_base + (uint32_t)(ab * TN);
            // the descriptors of the stage: only the address, in 16-byte units, differs
            const uint64_t at = (uint64_t)((uint32_t)s * (uint32_t)q.stage_bytes >> 4);
            uint64_t da = way.a + at + a_end;
            uint32_t more = opens ? 0u : 1u, end = b_end;
            int i = t.na, n = b_parts;
            do {
              uint64_t db = way.b + at + end;
              int j = n;
              do {
#pragma unroll
                for (int ks = 0; ks < BK / 16; ++ks) {
                  mma(d, da + (uint64_t)(ks * way.a_step), db + (uint64_t)(ks * way.b_step), way.idesc, more);
                  more = 1u;
                }
                db -= B_BYTES >> 4;
              } while (--j > 0);
              da -= A_BYTES >> 4;
              if (n < t.nb) {
                ++n;
                end += B_BYTES >> 4;
              }
            } while (--i > 0);
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
      mbar_wait(done, 0, &no_abort, q.status, 1LL << 28);
      __syncwarp();
    }
  } else {
    const int quarter = warp & 3, part = (warp - 2) >> 2;
    uint8_t* box = boxes + (warp - 2) * BOX;
    Op::before(p, (int)blockIdx.x * kEpi + warp - 2, (int)gridDim.x * kEpi);
    uint32_t use = 0;
    bool ok = true;
    auto filled = [&] {
      ok = mbar_wait(&tfull[use & 1], (use >> 1) & 1, abort_flag, q.status, q.spin_limit);
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
      return tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)((use & 1) * TN + part * QN);
    };
    for (int k = 0; k < njobs && ok; ++k) {
      const Job t = Op::job(p, unit, k);
      const int row0 = t.m0 + side * 128 + quarter * 32, col0 = t.n0 + part * QN;  // the warp's
      if (t.nkb > t.seg) {
        // the sum of the segments, back into the last one's place
        float sum[QN];
#pragma unroll
        for (int j = 0; j < QN; ++j) sum[j] = 0.f;
        for (int left = t.nkb; filled(); left -= t.seg, ++use) {
#pragma unroll
          for (int j = 0; j < QN; j += 16) tmem_add16(at() + (uint32_t)j, sum + j);
          if (left <= t.seg) break;
          release();
        }
        if (!ok) break;
#pragma unroll
        for (int j = 0; j < QN; j += 16) tmem_st16(at() + (uint32_t)j, sum + j);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      } else if (!filled()) {
        break;
      }
      auto get = [&](int c, float (&v)[32]) {  // the accumulator is handed back when the last of it is in registers
        tmem_ld32(at() + (uint32_t)(c * 32), v);
        if (c == QN / 32 - 1) release();
      };
      Op::template store<QN / 32>(p, t, row0, col0, box, maps.out, get);
      ++use;
    }
    if (lane == 0) bulk_wait_all();
  }
  fence_before();
  __syncthreads();
  // no CTA leaves, or gives its tensor memory back, while the other may still reach it
  cluster_arrive();
  cluster_wait();
  if (warp == 1) {
    fence_after();
    tmem_dealloc(tmem_base, 2 * TN);
  }
}

// ---- host ---------------------------------------------------------------------------------------
inline int tiles_of(long long n, int tile) { return (int)((n + tile - 1) / tile); }

// K blocks that are summed in tensor memory at a time.  Of a 32-bit result so few that the additions that meet a sum of full size
// are at most 28 (six products of two K blocks; three of two 16, one of six 24): 0.1 to 0.65e-6 off in the 2-norm whatever K, where
// torch's fp32 products are off by 0.15e-6 for K = 64 and 1.6e-6 for 8192.  Each end of a segment costs some 700 clocks:
// 8 x 1024 x 2048 -> 8192 with G of three products takes 876 us with two K blocks, 814 with four, 0.8e-6 off, and 1105 with one; sums of
// up to four K blocks would be 0.1e-6 off with one, for 13 to 30% of the time.  Of a result of 16 bits 512 steps, which lose 1e-5.
inline int segment(bool bits16, int prod, int nkb) { return std::min(nkb, bits16 ? 128 / prod : std::max(2, 6 / prod)); }

// Clocks of a K block, as measured.  A 256-wide tile keeps the tensor pipe busy, 512 a product, 570 for one; a 128-wide one, whose
// products are 256 each, takes 633 for one and 1,010 for three, for a reason that has not been found.
inline double block_clocks(int tn, int prod) { return tn == 256 ? 60 + 512.0 * prod : 440 + 190.0 * prod; }

// Width of the tiles and ranges of K for a product of `values` in tiles(width) tiles over nkb K blocks: the cut whose
// estimated clocks are fewest.  A tile's first loads and its epilogue are some 3,000 and 12 a column, which nothing hides where a
// unit has one tile; ranges are joined by another launch that reads their sums.
struct Split {
  int tn, ks;
};
template <typename Tiles>
Split split_of(Tiles tiles, double values, int nkb, int prod, int units) {
  Split best{256, 1};
  double least = 0;
  for (int tn = 256; tn >= 128; tn /= 2) {
    const long long n = tiles(tn);
    for (int ks = 1; ks <= 32 && ks * 2 <= std::max(2, nkb); ++ks) {
      if (ks > 1 && n * (ks - 1) >= 2 * units) break;
      const double waves = (double)((n * ks + units - 1) / units);
      double clk = 3000 + 12.0 * tn + waves * ((nkb + ks - 1) / ks) * block_clocks(tn, prod) + (waves - 1) * 300;
      if (ks > 1) clk += 3000 + values * 8 * ks / 3500;
      if (least == 0 || clk < least) {
        least = clk;
        best = Split{tn, ks};
      }
    }
  }
  return best;
}

// Map of an operand: inner x rows x batch x parts of 16-bit values, `ld`, `ld_b`, `ld_p` elements apart; the box is
// 64 wide and `box_rows` high.
inline int operand_map(CUtensorMap* map, const void* base, bool f16, long long inner, long long rows, long long batch,
                       int parts, long long ld, long long ld_b, long long ld_p, int box_rows) {
  const long long d[4] = {inner, rows, batch, parts}, l[3] = {ld, ld_b, ld_p};
  return map_nd(map, base, 4, d, l, box_rows, 1, f16 ? MAP_F16 : MAP_BF16);
}

// Map of a result that leaves in boxes: cols x rows x batch of 16- or 32-bit values.
inline int box_map(CUtensorMap* map, const void* base, MapType type, long long cols, long long rows, long long batch, long long ld,
                   long long ld_b) {
  const long long d[3] = {cols, rows, batch}, l[2] = {ld, ld_b};
  return map_nd(map, base, 3, d, l, 32, 1, type, true);
}

// Pairs that the current device holds at once.
template <class Op, int TN>
int resident(int* units) {
  static std::atomic<int> cache[64];
  int dev = 0, n = 0;
  GC_CUDA(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64) n = cache[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    static SmemOptIn allow;
    GC_CUDA(allow(k_tiles<Op, TN>, kSmem));
    cudaLaunchAttribute at[1];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    GC_CUDA(cudaOccupancyMaxActiveClusters(&n, k_tiles<Op, TN>, &cfg));
    if (n < 1) return fail(GC_ERR_CUDA, "no pair of CTAs fits the device");
    if (dev >= 0 && dev < 64) cache[dev].store(n, std::memory_order_relaxed);
  }
  *units = n;
  return GC_OK;
}

// Launches `njobs` tiles; most_a, most_b: the most parts of an operand that a tile has.
template <class Op, int TN>
int launch_tiles(const Maps& maps, typename Op::Params p, long long njobs, int most_a, int most_b, const char* name,
                 bool chained, cudaStream_t s) {
  int n = 0;
  const int rc = resident<Op, TN>(&n);
  if (rc) return rc;
  p.q.units = (int)std::min<long long>(n, njobs);
  p.q.stage_bytes = most_a * A_BYTES + most_b * (TN / 2 * BK * 2);
  p.q.stages = std::min(kMaxStages, RING / p.q.stage_bytes);
  return launch_chain(k_tiles<Op, TN>, name, (unsigned)(2 * p.q.units), kThreads, kSmem, 2, chained, s, maps, p);
}

}  // namespace tiles
}  // namespace gc
