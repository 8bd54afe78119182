// refadapt_glu and refadapt_glu_backward: the gated feed-forward,
//
//   hidden = act(g) o w,  g = x Wg^T,  w = x Wu^T,   y = hidden Wd^T
//   du = dy Wd;  dg = du o w o act'(g),  dw = du o act(g)
//   dx = dg Wg + dw Wu;  dWg = dg^T x,  dWu = dw^T x,  dWd = dy^T hidden
//
// bf16 operands, fp32 sums in TMEM. One kernel of CTA pairs (tcgen05 cta_group::2,
// a 256-row output tile per pair) runs all of these products; a launch has a
// list of jobs (products), whose tiles the pairs take in turn:
//   GLU    a tile is w columns of g and the same w of the up projection: rank 0
//          stages Wg's rows as its half of the MMA's N = 2 w, rank 1 Wu's, so one
//          MMA forms both and the epilogue has g and w of a column in one thread;
//   GRAD   du = dy Wd; the epilogue takes g and w and gives dg and dw (TMA tiles);
//   STORE  the four gradients, in one launch: dx sums over both pairs of operands
//          in one accumulator (K = 2 F), so its tiles are the long ones and go
//          first; pairs that get one fewer of them take more of the weights'
//          (Schedule). A job of few tiles and a long K is cut into parts, whose
//          fp32 sums a second kernel adds up in order.
// An operand whose K runs along its rows (Wd, Wg, Wu as B, the rows of every
// operand of a weight's gradient) is read as it lies, MN-major: nothing is
// transposed in memory.
//   warp 0      TMA producer: per stage 128 of K (GRAD: 64) of the CTA's 128 A rows
//               and of its half of the B tile, in boxes of 64 columns (128-byte
//               swizzle; what lies past an edge is read as zeros).
//   warp 1      TMEM allocator (two accumulators of 256 columns) and MMA issuer
//               (rank 0's).
//   warps 2..9  epilogue, two warps per TMEM lane quarter, while the next tile's
//               MMAs fill the other accumulator.
// Measured: 4352 rows, 2048 -> 8192: forward 177-182 us, 1.61-1.65 PFLOP/s, 84-86 % of the
// tensor cores' measured rate (14.3 rounds of tiles take 15, and the clock sinks under the
// power cap). Backward, 4333 rows, 564-576 us, 1.51-1.55 PFLOP/s: GRAD 115 us, where the
// MMAs alone are 82 (its epilogue moves four F-wide tensors through the shared memory that
// feeds the MMAs), STORE 445.
// dg and dw are rounded to bf16 on their way to the products of dx and the weights'
// gradients. It is the one rounding beside the results' own, and puts their error at 2.3e-3
// where 32-bit dg and dw give 1.7e-3. The MMAs of bf16 weights and rows take operands of one
// type: 32 bits would mean tf32 at half the rate, with the weights and rows widened too.
// Calls of few rows read (backward: and write) the weights once and little else, and
// have kernels of their own: forward up to 128 rows glu_rows_kernel and
// glu_some_kernel, du and dx of few rows glu_cols_kernel.
// Every mbarrier wait is bounded; on a timeout the CTA drains its own copies and
// MMAs, frees TMEM, flags the error word and returns.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>

#include "api_common.h"
#include "epi_rows.cuh"
#include "launch_plan.h"
#include "tc_ptx.cuh"

namespace ra {
namespace glu {

constexpr int TM = 256;              // output rows of a pair's tile
constexpr int MAX_BN = 256;          // accumulator columns
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 64 + 32 * EPI_WARPS;
constexpr int TMEM_COLS = 512;
constexpr int GROUP_M = 16;  // tile rows per band of the tile order
constexpr int MAX_JOBS = 4;

enum Kind { GLU, GRAD, STORE };

// Shared memory of a kind's kernel. GLU and STORE: three stages of 128 of K (half
// the hand-offs of six of 64) and a staging buffer per epilogue warp. GRAD: five
// stages of 64, which leaves each epilogue warp two sets of two 32 x 32 tiles.
constexpr int TILE_BYTES = 32 * 64;  // 32 rows of 32 columns
template <int KIND>
struct Cfg {
  static constexpr int BK = KIND == GRAD ? 64 : 128;  // K per stage
  static constexpr int STAGES = KIND == GRAD ? 5 : 3;
  static constexpr int BOX = 128 * 64 * 2;     // of a K-major operand: 128 rows x 64 of K
  static constexpr int MN_BOX = BK * 64 * 2;   // of an MN-major operand: BK of K x 64 columns
  static constexpr int OPERAND_BYTES = 128 * BK * 2;
  static constexpr int STAGE_BYTES = 2 * OPERAND_BYTES;
  static constexpr int EPI_BYTES = KIND == GRAD ? 4 * TILE_BYTES : 32 * 128;  // of a warp
  static constexpr int OFF_EPI = STAGES * STAGE_BYTES;
  static constexpr int OFF_BAR = OFF_EPI + EPI_WARPS * EPI_BYTES;
  static constexpr int TILE_BARS = KIND == GRAD ? 2 * EPI_WARPS : 0;          // sets of tiles loaded
  static constexpr int NUM_BARS = 2 * STAGES + 2 + 2 + 1 + TILE_BARS;  // full, empty, tfull[2], tempty[2], drain
  static constexpr int OFF_MISC = OFF_BAR + NUM_BARS * 8;
  static constexpr int SMEM_ALLOC = OFF_MISC + 16 + 1024;
  static_assert(SMEM_ALLOC <= 232448 && OFF_EPI % 1024 == 0 && EPI_BYTES % 1024 == 0, "shared memory budget");
};

struct Rows {
  __nv_bfloat16* ptr;
  int64_t ss, sr;
};

// Division by a number that the host knows, for n and d below 2^31: the high word
// of n * ceil(2^32 / d) is n / d or one more. The roles' threads divide a few times
// per tile.
struct Div {
  uint32_t d, mul;  // mul 0: d is 1
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const {
    if (mul == 0) return n;
    const uint32_t q = __umulhi(n, mul);
    return q * d > n ? q - 1 : q;
  }
};

struct Job {
  int32_t samples, rows, gated;  // output rows per sample
  int32_t m_tiles, cols;         // row and column tiles of a sample
  int32_t N;                     // output columns
  // K is `spans` runs of span_k, each of span_stages stages: one run; dx: one per
  // operand pair; a weight's gradient: one per sample (K runs along the rows).
  int32_t spans, span_k, span_stages;
  int32_t parts;                 // of K, whole stages each
  Div by_band, by_parts;         // tiles of a band of GROUP_M tile rows; parts
  int32_t rows_k;                // K runs along the rows of both operands
  Rows out[3];                   // GLU: out, pre_gate, pre_up; STORE: the result
  float* partial;                // parts > 1: [part][sample][row][N]
};

// Which units a pair takes. Unit c, c + pairs, ... of the `longs` units that come
// first (and take longer); the `rest` pairs that have one more of them than the
// others then wait `early` rounds of the remaining units, which the others share.
struct Schedule {
  int32_t longs, early;
};
struct Turn {  // the units of pair c, one after the other
  int c, pairs, rest, ahead;
  int64_t t, base;  // the next unit; the first that all pairs share
  bool longs;
  __device__ __forceinline__ Turn(const Schedule& s, int c_, int pairs_) : c(c_), pairs(pairs_) {
    rest = s.longs % pairs;
    ahead = c < rest ? 0 : s.early;
    base = s.longs + int64_t(s.early) * (pairs - rest);
    t = c;
    longs = true;
    settle(s);
  }
  __device__ __forceinline__ void next(const Schedule& s) {
    if (longs) {
      t += pairs;
      settle(s);
    } else if (ahead > 1) {
      --ahead;
      t += pairs - rest;
    } else if (ahead == 1) {
      ahead = 0;
      t = base + c;
    } else {
      t += pairs;
    }
  }

 private:
  __device__ __forceinline__ void settle(const Schedule& s) {  // past the long units?
    if (t < s.longs) return;
    longs = false;
    t = ahead > 0 ? s.longs + (c - rest) : base + c;
  }
};

struct Params {
  int32_t n_jobs, bn;
  Schedule order;
  const int32_t* mode;
  int32_t* err_word;
  uint64_t budget_ns;
  Job job[MAX_JOBS];
  // Operand pairs of a job: STORE's two (dx) follow one another in K; GLU's tm_b
  // are Wg and Wu, one per rank.
  CUtensorMap tm_a[MAX_JOBS][2], tm_b[MAX_JOBS][2];
  CUtensorMap tm_tile[4];  // GRAD: 32 x 32 tiles of pre_gate, pre_up, dg, dw
};

struct Unit {
  int job, s, m0, n0, part, k0, k1;  // k0, k1: stages
};

// Walks the units (a tile's part of K) of the live jobs and samples in order;
// unit indices only grow. Bands of GROUP_M tile rows, rows fastest inside a
// band, so that the tiles in flight share few row and column blocks, held in L2.
template <int KIND>
struct Walk {
  int j = 0, s = 0;
  int64_t begin = 0;
  __device__ __forceinline__ int64_t units(const Params& p) const {
    const Job& job = p.job[j];
    if (job.gated && p.mode[s] == RA_MODE_REUSE) return 0;
    return int64_t(job.m_tiles) * job.cols * job.parts;
  }
  __device__ __forceinline__ bool at(const Params& p, int64_t t, Unit& u) {
    int64_t n = units(p);
    while (t - begin >= n) {
      begin += n;
      if (++s == p.job[j].samples) {
        s = 0;
        if (++j == p.n_jobs) return false;
      }
      n = units(p);
    }
    const Job& job = p.job[j];
    const uint32_t idx = uint32_t(t - begin), tile = job.by_parts(idx), band = job.by_band(tile);
    const uint32_t in_band = tile - band * job.by_band.d;
    const int m_first = int(band) * GROUP_M;
    const uint32_t rows = uint32_t(min(GROUP_M, job.m_tiles - m_first));
    const uint32_t col = rows == GROUP_M ? in_band / GROUP_M : in_band / rows;
    u.job = j;
    u.s = s;
    u.m0 = (m_first + int(in_band - col * rows)) * TM;
    u.n0 = int(col) * (KIND == GLU ? p.bn / 2 : p.bn);
    u.part = int(idx - tile * job.by_parts.d);
    const int stages = job.spans * job.span_stages;
    u.k0 = 0, u.k1 = stages;
    if (job.parts > 1) {
      u.k0 = int(int64_t(stages) * u.part / job.parts);
      u.k1 = int(int64_t(stages) * (u.part + 1) / job.parts);
    }
    return true;
  }
};

// Two values at once of act(g) = g s and act'(g) = s + g s (1 - s) z'(g), with
// s = 1 / (1 + e^-z): z = g for SiLU; for GELU's tanh form 0.5 (1 + tanh(v)) =
// 1 / (1 + e^-2v), so z = 2 sqrt(2/pi) (g + 0.044715 g^3). An exponential that
// overflows gives s = 0. The exponential and the reciprocal are the approximate
// instructions, good to about 2^-22, which a bf16 result does not see.
template <int ACT>
__device__ __forceinline__ uint64_t act2(uint64_t g, uint64_t* grad) {
  constexpr float log2e = 1.4426950408889634f, c = 2.f * 0.7978845608028654f, c3 = 0.044715f * c;
  uint64_t z, q;
  if constexpr (ACT == RA_ACT_GELU) {
    q = f2_mul(g, g);
    z = f2_mul(g, f2_fma(q, f2_pack(-log2e * c3, -log2e * c3), f2_pack(-log2e * c, -log2e * c)));
  } else {
    z = f2_mul(g, f2_pack(-log2e, -log2e));
  }
  float z0, z1;
  f2_unpack(z, z0, z1);
  f2_unpack(f2_add(f2_pack(ex2_approx(z0), ex2_approx(z1)), f2_pack(1.f, 1.f)), z0, z1);
  const uint64_t s = f2_pack(rcp_approx(z0), rcp_approx(z1)), a = f2_mul(g, s);
  if (grad) {
    const uint64_t t = f2_fma(f2_mul(a, f2_pack(-1.f, -1.f)), s, a);
    if constexpr (ACT == RA_ACT_GELU)
      *grad = f2_fma(t, f2_fma(q, f2_pack(3.f * c3, 3.f * c3), f2_pack(c, c)), s);
    else
      *grad = f2_add(t, s);
  }
  return a;
}

__device__ __forceinline__ uint32_t f2_bf16(uint64_t v) {
  float a, b;
  f2_unpack(v, a, b);
  return pack_bf16x2(a, b);
}
__device__ __forceinline__ uint64_t f2_regs(const uint32_t (&v)[32], int i) {
  return f2_pack(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
}

// What an epilogue warp works on: its 32 rows (row0 + lane, nrow of them in the
// sample), which of the two warps of its lane quarter it is, its staging buffer
// and the TMEM address of its lanes in the tile's accumulator.
struct EpiWarp {
  int row0, nrow, half;
  uint8_t* stage;
  uint32_t acc;
};

__device__ __forceinline__ char* row_ptr(const Rows& r, int s, int row, int col) {
  return reinterpret_cast<char*>(r.ptr + s * r.ss + row * r.sr + col);
}

// 64 accumulator columns (the last `cols` - 32 of which may be missing) -> bf16.
__device__ __forceinline__ void pack64(uint32_t acc, int cols, uint4 (&own)[8]) {
  uint32_t* o = reinterpret_cast<uint32_t*>(own);
  uint32_t v[32];
  tmem_ld32(acc, v);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (h == 1 && cols <= 32) break;
    tmem_ld_wait_for(v);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[16 * h + i] = f2_bf16(f2_regs(v, i));
    if (h == 0 && cols > 32) tmem_ld32(acc + 32, v);
  }
}

template <int ACT, class Ready>
__device__ __forceinline__ bool epilogue_glu(const Params& p, const Unit& u, const EpiWarp& w, Ready ready) {
  const Job& job = p.job[u.job];
  const int width = p.bn / 2;
  if (!ready()) return false;
  if (w.nrow <= 0) return true;
#pragma unroll 1
  for (int c = 64 * w.half; c < width; c += 128) {
    const int col = u.n0 + c, cols = min(64, width - c), ncol = min(cols, job.N - col);
    if (ncol <= 0) break;
    uint4 own[8];
    if (job.out[1].ptr) {
      pack64(w.acc + c, cols, own);
      rows_put128(w.stage, own, row_ptr(job.out[1], u.s, w.row0, col), 2 * job.out[1].sr, w.nrow, ncol);
      pack64(w.acc + width + c, cols, own);
      rows_put128(w.stage, own, row_ptr(job.out[2], u.s, w.row0, col), 2 * job.out[2].sr, w.nrow, ncol);
    }
    uint32_t* o = reinterpret_cast<uint32_t*>(own);
    uint32_t g[32], v[32];
    tmem_ld32(w.acc + c, g);
    tmem_ld32(w.acc + width + c, v);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 1 && cols <= 32) break;
      tmem_ld_wait_for(g);
      tmem_ld_wait_for(v);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        o[16 * h + i] = f2_bf16(f2_mul(act2<ACT>(f2_regs(g, i), nullptr), f2_regs(v, i)));
      if (h == 0 && cols > 32) {
        tmem_ld32(w.acc + c + 32, g);
        tmem_ld32(w.acc + width + c + 32, v);
      }
    }
    rows_put128(w.stage, own, row_ptr(job.out[0], u.s, w.row0, col), 2 * job.out[0].sr, w.nrow, ncol);
  }
  return true;
}

// GRAD: a warp's tiles (32 rows of 32 columns of g and of w) come by TMA into one of
// its two sets, the next one's while it works; dg and dw take their places, row for
// row, and leave by TMA. Sets are counted over all tiles of the warp: n.
struct TilePipe {
  uint8_t* sets;   // [2][g, w]
  uint64_t* bars;  // [2]
  int n = 0;       // tiles taken
  int issued = 0;  // tiles whose loads were issued

  __device__ __forceinline__ void load(const Params& p, const Unit& u, int row0, int c) {
    if ((threadIdx.x & 31) == 0) {
      bulk_wait_read_all();  // the set's last dg and dw have left it
      uint8_t* set = sets + (issued & 1) * 2 * TILE_BYTES;
      uint64_t* bar = bars + (issued & 1);
      mbar_arrive_expect_tx(bar, 2 * TILE_BYTES);
      tma_load_4d(set, &p.tm_tile[0], bar, u.n0 + c, row0, 0, u.s);
      tma_load_4d(set + TILE_BYTES, &p.tm_tile[1], bar, u.n0 + c, row0, 0, u.s);
    }
    ++issued;
    __syncwarp();
  }
  __device__ __forceinline__ bool wait(const WaitCtl& ctl) {
    return __all_sync(0xffffffffu, mbar_wait(bars + (n & 1), uint32_t((n >> 1) & 1), ctl));
  }
  // Nothing of this warp's is in flight afterwards.
  __device__ __forceinline__ void drain(uint64_t budget_ns) {
    for (int i = n; i < issued; ++i) mbar_wait_drain(bars + (i & 1), uint32_t((i >> 1) & 1), budget_ns);
    if ((threadIdx.x & 31) == 0) bulk_wait_all();
    __syncwarp();
  }
};

// next: the unit after u, or NULL; next_row0: this warp's first row in it.
template <int ACT, class Ready>
__device__ __forceinline__ bool epilogue_grad(const Params& p, const Unit& u, const EpiWarp& w, TilePipe& pipe,
                                              const WaitCtl& ctl, const Unit* next, int next_row0, Ready ready) {
  const Job& job = p.job[u.job];
  const int lane = threadIdx.x & 31;
  auto has = [&](const Unit& v, int row0, int c) { return c < p.bn && v.n0 + c < job.N && row0 < job.rows; };
  int c = 32 * w.half;
  const bool any = has(u, w.row0, c);
  if (any && pipe.issued == pipe.n) pipe.load(p, u, w.row0, c);
  if (!ready()) return false;
#pragma unroll 1
  for (; any && has(u, w.row0, c); c += 64) {
    uint32_t v[32];
    tmem_ld32(w.acc + c, v);
    if (!pipe.wait(ctl)) {
      tmem_ld_wait_for(v);
      return false;
    }
    uint8_t* set = pipe.sets + (pipe.n & 1) * 2 * TILE_BYTES;
    ++pipe.n;
    uint4 g[4], up[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) g[q] = *stage_slot(set, lane, q), up[q] = *stage_slot(set + TILE_BYTES, lane, q);
    if (has(u, w.row0, c + 64))
      pipe.load(p, u, w.row0, c + 64);
    else if (next && has(*next, next_row0, 32 * w.half))
      pipe.load(p, *next, next_row0, 32 * w.half);
    tmem_ld_wait_for(v);
    uint32_t* gp = reinterpret_cast<uint32_t*>(g);
    uint32_t* wp = reinterpret_cast<uint32_t*>(up);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      uint64_t da;
      const uint64_t a = act2<ACT>(bf2_unpack(gp[i]), &da), du = f2_regs(v, i);
      gp[i] = f2_bf16(f2_mul(f2_mul(du, bf2_unpack(wp[i])), da));
      wp[i] = f2_bf16(f2_mul(du, a));
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) *stage_slot(set, lane, q) = g[q], *stage_slot(set + TILE_BYTES, lane, q) = up[q];
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_4d(&p.tm_tile[2], set, u.n0 + c, w.row0, 0, u.s);
      tma_store_4d(&p.tm_tile[3], set + TILE_BYTES, u.n0 + c, w.row0, 0, u.s);
      bulk_commit();
    }
  }
  return true;
}

template <class Ready>
__device__ __forceinline__ bool epilogue_store(const Params& p, const Unit& u, const EpiWarp& w, Ready ready) {
  const Job& job = p.job[u.job];
  if (!ready()) return false;
  if (w.nrow <= 0) return true;
  const int lane = threadIdx.x & 31;
  if (job.parts == 1) {
#pragma unroll 1
    for (int c = 64 * w.half; c < p.bn && u.n0 + c < job.N; c += 128) {
      uint4 own[8];
      pack64(w.acc + c, 64, own);
      rows_put128(w.stage, own, row_ptr(job.out[0], u.s, w.row0, u.n0 + c), 2 * job.out[0].sr, w.nrow,
                  job.N - u.n0 - c);
    }
    return true;
  }
#pragma unroll 1
  for (int c = 32 * w.half; c < p.bn && u.n0 + c < job.N; c += 64) {
    const int ncol = job.N - u.n0 - c;
    uint32_t v[32];
    tmem_ld32(w.acc + c, v);
    tmem_ld_wait_for(v);
    if (lane < w.nrow) {
      const int64_t row = (int64_t(u.part) * job.samples + u.s) * job.rows + w.row0 + lane;
      float4* dst = reinterpret_cast<float4*>(job.partial + row * job.N + u.n0 + c);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (4 * i < ncol)
          dst[i] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]),
                               __uint_as_float(v[4 * i + 3]));
    }
  }
  return true;
}

// ------------------------------------------------------------------ pipeline
// The majorness of a job's operands: A and B of a weight's gradient are MN-major
// (both rows run along K), so is B where a weight is used untransposed.
template <int KIND>
constexpr bool kBRowsK = KIND != GLU;

// Loads of a unit's stages. it: stages issued so far.
struct Producer {
  uint8_t* smem;
  uint64_t *full, *empty;
  uint32_t full0;  // rank 0's full barriers
  int rank;
  int64_t it = 0;

  template <int KIND, bool A_MN>
  __device__ __forceinline__ bool unit(const Params& p, const Unit& u, const WaitCtl& ctl) {
    constexpr bool B_MN = kBRowsK<KIND>;
    using C = Cfg<KIND>;
    constexpr int STAGES = C::STAGES, BK = C::BK;
    const Job& job = p.job[u.job];
    const int half = p.bn / 2;  // columns of B that a CTA stages
    const uint32_t b_box = B_MN ? uint32_t(C::MN_BOX) : uint32_t(half) * 128u;
    const int b_boxes = B_MN ? (half + 63) / 64 : 2;  // the second may reach past the half: not used
    const int m = u.m0 + rank * 128, n = u.n0 + (KIND == GLU ? 0 : rank * half);
    int span = u.k0 > 0 ? u.k0 / job.span_stages : 0, k = (u.k0 - span * job.span_stages) * BK;
    for (int q = u.k0; q < u.k1; ++q, ++it) {
      const int st = int(it % STAGES);
      if (it >= STAGES && !mbar_wait(empty + st, uint32_t((it / STAGES - 1) & 1), ctl)) return false;
      uint8_t* sa = smem + st * C::STAGE_BYTES;
      uint8_t* sb = sa + C::OPERAND_BYTES;
      const uint32_t bar = full0 + 8u * st;
      const int pair = KIND == STORE && !A_MN ? span : 0;  // dx: the operand pair
      const int ks = A_MN ? span : u.s;                    // sample of A
      const bool second = BK > 64 && job.span_k - k > 64;  // K-major: there is a second box, and it lies inside
      const CUtensorMap* ta = &p.tm_a[u.job][pair];
      const CUtensorMap* tb = &p.tm_b[u.job][KIND == GLU ? rank : pair];
      if (rank == 0)
        mbar_arrive_expect_tx(full + st, 2u * ((A_MN ? 2u * C::MN_BOX : (second ? 2u : 1u) * C::BOX) +
                                               (B_MN || second ? uint32_t(b_boxes) : 1u) * b_box));
      if (A_MN) {
        tma_load_4d_pair(sa, ta, bar, m, k, 0, ks);
        tma_load_4d_pair(sa + C::MN_BOX, ta, bar, m + 64, k, 0, ks);
      } else {
        tma_load_4d_pair(sa, ta, bar, k, m, 0, ks);
        if (second) tma_load_4d_pair(sa + C::BOX, ta, bar, k + 64, m, 0, ks);
      }
      if (B_MN) {
        tma_load_4d_pair(sb, tb, bar, n, k, 0, A_MN ? ks : 0);
        if (b_boxes > 1) tma_load_4d_pair(sb + C::MN_BOX, tb, bar, n + 64, k, 0, A_MN ? ks : 0);
      } else {
        tma_load_4d_pair(sb, tb, bar, k, n, 0, 0);
        if (second) tma_load_4d_pair(sb + C::BOX, tb, bar, k + 64, n, 0, 0);
      }
      k += BK;
      if (k >= job.span_k) k = 0, ++span;
    }
    return true;
  }
};

// MMAs of a unit's stages into the accumulator at d_t.
struct Issuer {
  uint32_t s0;
  uint64_t *full, *empty;
  int64_t it = 0;
  bool issued = false;

  template <int KIND, bool A_MN>
  __device__ __forceinline__ bool unit(const Params& p, const Unit& u, uint32_t d_t, const WaitCtl& ctl) {
    constexpr bool B_MN = kBRowsK<KIND>;
    using C = Cfg<KIND>;
    constexpr int STAGES = C::STAGES, BK = C::BK;
    const Job& job = p.job[u.job];
    const uint32_t idesc = idesc_bf16_f32(TM, p.bn, A_MN, B_MN);
    // A step of 16 of K, in descriptor units of 16 bytes: 32 bytes of a K-major
    // row (64 of K, then the next box), 16 rows of 128 bytes of an MN-major box
    // (whose next 64 columns are the next box).
    const uint64_t da = sdesc_sw128(s0, A_MN ? C::MN_BOX : 16, 1024);
    const uint64_t db = sdesc_sw128(s0 + C::OPERAND_BYTES, B_MN ? C::MN_BOX : 16, 1024);
    int k = u.k0 > 0 ? (u.k0 % job.span_stages) * BK : 0;
    for (int q = u.k0; q < u.k1; ++q, ++it) {
      const int st = int(it % STAGES);
      if (!mbar_wait(full + st, uint32_t((it / STAGES) & 1), ctl)) return false;
      tc_fence_after();
      const uint64_t a = da + uint64_t(st * (C::STAGE_BYTES >> 4)), b = db + uint64_t(st * (C::STAGE_BYTES >> 4));
      const int left = job.span_k - k;
      auto step = [&](int kk) {
        const uint32_t oa = A_MN ? kk * 128 : (kk >> 2) * (C::BOX >> 4) + (kk & 3) * 2;
        const uint32_t ob = B_MN ? kk * 128 : (kk >> 2) * (C::BOX >> 4) + (kk & 3) * 2;
        umma_ss_pair(d_t, a + oa, b + ob, idesc, (q > u.k0 || kk > 0) ? 1u : 0u);
      };
      if (left >= BK) {
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) step(kk);
      } else {
#pragma unroll 1
        for (int kk = 0; 16 * kk < left; ++kk) step(kk);
      }
      umma_commit_pair(empty + st, 0x3);
      issued = true;
      k += BK;
      if (k >= job.span_k) k = 0;
    }
    return true;
  }
};

template <int KIND, int ACT>
__global__ void __launch_bounds__(THREADS, 1) glu_kernel(const __grid_constant__ Params p) {
  using C = Cfg<KIND>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint64_t* full = bars;
  uint64_t* empty = bars + STAGES;
  uint64_t* tfull = bars + 2 * STAGES;
  uint64_t* tempty = bars + 2 * STAGES + 2;
  uint64_t* drain = bars + 2 * STAGES + 4;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int cid = int(blockIdx.x >> 1), ncl = int(gridDim.x >> 1);
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull + b, 1);
      mbar_init(tempty + b, 2 * EPI_WARPS);
    }
    mbar_init(drain, 1);
    for (int i = 0; i < C::TILE_BARS; ++i) mbar_init(drain + 1 + i, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc_pair(tmem_slot, TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // both CTAs' barriers and TMEM exist before any cross-CTA use
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const WaitCtl ctl{abort_flag, p.err_word, p.budget_ns};
  pdl_launch();
  if (warp != 0) pdl_wait();

  int64_t loads = 0;    // the producer's: stages that it loaded
  bool issued = false;  // the issuer's: it has issued MMAs
  if (warp == 0) {
    if (lane == 0) {
      // -------------------------------------------------------------- producer (both CTAs)
      for (int j = 0; j < p.n_jobs; ++j)
        if (p.job[j].rows > 0) {
          tma_prefetch_desc(&p.tm_a[j][0]);
          tma_prefetch_desc(&p.tm_b[j][0]);
        }
      pdl_wait();
      Producer pr{smem, full, empty, mapa_shared(smem_u32(full), 0), int(rank)};
      bool ok = true;
      Walk<KIND> walk;
      Unit u;
      for (Turn turn(p.order, cid, ncl); ok && walk.at(p, turn.t, u); turn.next(p.order)) {
        if (KIND == STORE && p.job[u.job].rows_k)
          ok = pr.unit<KIND, KIND == STORE>(p, u, ctl);
        else
          ok = pr.unit<KIND, false>(p, u, ctl);
      }
      loads = pr.it;
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      // -------------------------------------------------------------- MMA issuer (rank 0)
      Issuer mma{smem_u32(smem), full, empty};
      int i = 0;
      bool ok = true;
      Walk<KIND> walk;
      Unit u;
      for (Turn turn(p.order, cid, ncl); walk.at(p, turn.t, u); turn.next(p.order), ++i) {
        const int buf = i & 1, use = i >> 1;
        if (use > 0 && !(ok = mbar_wait_cluster(tempty + buf, uint32_t((use - 1) & 1), ctl))) break;
        tc_fence_after();
        const uint32_t d_t = tmem + uint32_t(buf * MAX_BN);
        if (KIND == STORE && p.job[u.job].rows_k)
          ok = mma.unit<KIND, KIND == STORE>(p, u, d_t, ctl);
        else
          ok = mma.unit<KIND, false>(p, u, d_t, ctl);
        if (!ok) break;
        umma_commit_pair(tfull + buf, 0x3);
      }
      issued = mma.issued;
    }
  } else {
    // ---------------------------------------------------------------- epilogue (both CTAs)
    const int quarter = warp & 3;
    EpiWarp w;
    w.half = (warp - 2) >> 2;
    w.stage = smem + C::OFF_EPI + (warp - 2) * C::EPI_BYTES;
    const uint32_t tempty0 = mapa_shared(smem_u32(tempty), 0);
    int i = 0;
    TilePipe pipe{w.stage, drain + 1 + 2 * (warp - 2)};
    Walk<KIND> walk;
    Turn turn(p.order, cid, ncl);
    Unit u, next;
    bool more = walk.at(p, turn.t, u);
    auto step = [&] {
      turn.next(p.order);
      more = walk.at(p, turn.t, next);
    };
    for (; more; ++i, u = next) {
      if (KIND == GRAD) step();  // its tiles are loaded ahead
      const int buf = i & 1, use = i >> 1, row = int(rank) * 128 + quarter * 32;
      w.row0 = u.m0 + row;
      w.nrow = min(32, p.job[u.job].rows - w.row0);
      w.acc = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(buf * MAX_BN);
      auto ready = [&] {
        const bool ok = __all_sync(0xffffffffu, mbar_wait(tfull + buf, uint32_t(use & 1), ctl));
        tc_fence_after();
        return ok;
      };
      bool ok;
      if constexpr (KIND == GLU)
        ok = epilogue_glu<ACT>(p, u, w, ready);
      else if constexpr (KIND == GRAD)
        ok = epilogue_grad<ACT>(p, u, w, pipe, ctl, more ? &next : nullptr, next.m0 + row, ready);
      else
        ok = epilogue_store(p, u, w, ready);
      if (!ok) break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (rank == 0)
          mbar_arrive(tempty + buf);
        else
          mbar_arrive_remote(tempty0 + 8u * buf);
      }
      if (KIND != GRAD) step();
    }
    if (KIND == GRAD) pipe.drain(p.budget_ns);
  }
  tc_fence_before();
  __syncthreads();
  // No role waits any more, so the flag is final: it may have been raised after the
  // producer and the issuer were through. What a CTA that gave up has on its way lands
  // before the pair's shared memory and TMEM go. (A rank 0 that did not give up has seen
  // every MMA end, and with them the loads of both CTAs.)
  if (*abort_flag && lane == 0) {
    if (warp == 0 && rank == 0) {
      // rank 0's full barriers count both CTAs' bytes of every phase it armed
      for (int st = 0; st < STAGES; ++st) {
        const int64_t n_s = (loads > st) ? (loads - st + STAGES - 1) / STAGES : 0;
        if (n_s > 0) mbar_wait_drain(full + st, uint32_t((n_s - 1) & 1), p.budget_ns);
      }
    }
    if (warp == 1 && issued) {
      umma_commit_pair(drain, 0x1);
      mbar_wait_drain(drain, 0, p.budget_ns);
    }
    pause_ns(kLandNs);  // rank 1's loads, and the commits' arrivals at rank 1
  }
  __syncwarp();
  cluster_sync_all();
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem, TMEM_COLS);
}

// ------------------------------------------------------------------ few rows
// Up to 16 rows per segment of small weights: bound by the weights' bytes (4 F C) and
// the latency of reading them once (1024 -> 2736, 11 MB: 4.7 us up to 8 rows, 6.1 at 16;
// the kernel for some rows below 7.6, the tiles above 10). A CTA takes eight features,
// its warps share K, and a weight goes from memory into the registers of the mma.sync
// that uses it (m16n8k16: the rows of A are the features' gate rows and their up rows,
// the columns of B eight rows of x), so g and w of a feature and a row end in one
// thread. K is permuted alike in A and B, so that a lane's operands are 16 contiguous
// bytes. Deeper rounds of loads, two features' groups a CTA, a prefetch into L2 ahead of
// the previous kernel's end and four warps measured no better.
// Larger weights go to the kernel for some rows. 8 rows: 45 MB 12.6 us here, 12.3 there,
// 67 MB 14.4 and 14.5, 180 MB 34.8 and 31.1; 16 rows: 45 MB 14.6 and 12.3, 180 MB 38.5
// and 31.3.
bool few_rows(int rows, int64_t weight_bytes) {
  return rows <= 8 ? weight_bytes <= (int64_t(64) << 20) : rows <= 16 && weight_bytes <= (int64_t(24) << 20);
}
constexpr int ROWS_WARPS = 8;

struct RowsSeg {
  Rows x;
  const __nv_bfloat16 *w_gate, *w_up;
  Rows out[3];
  int32_t rows, gated;
};
struct RowsParams {
  int32_t B, F, C;
  const int32_t* mode;
  RowsSeg seg[3];
};

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes, or zeros. Volatile: the loads of a round keep their place before its
// products.
__device__ __forceinline__ uint4 load16_if(const void* ptr, bool in) {
  uint4 v;
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t"
      "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
      "@p ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
      : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
      : "l"(ptr), "r"(int(in))
      : "memory");
  return v;
}

// GROUPS: groups of eight rows; DEPTH: K blocks of 64 (a 128-byte line of a
// weight's row) loaded at once by a warp.
template <int ACT, int GROUPS, int DEPTH>
__global__ void __launch_bounds__(32 * ROWS_WARPS) glu_rows_kernel(const __grid_constant__ RowsParams p) {
  __shared__ float red[ROWS_WARPS][GROUPS][4][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const RowsSeg& sg = p.seg[blockIdx.y];
  pdl_launch();
  const int f = int(blockIdx.x) * 8 + g, total = p.B * sg.rows;
  const __nv_bfloat16 *wg = sg.w_gate + int64_t(f) * p.C + 8 * t, *wu = sg.w_up + int64_t(f) * p.C + 8 * t;
  const __nv_bfloat16* x[GROUPS];
  float acc[GROUPS][4];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int row = min(8 * i + g, total - 1), s = row / sg.rows;  // rows past the last repeat it
    x[i] = sg.x.ptr + s * sg.x.ss + (row - s * sg.rows) * sg.x.sr + 8 * t;
#pragma unroll
    for (int z = 0; z < 4; ++z) acc[i][z] = 0.f;
  }
  pdl_wait();
  for (int k0 = 64 * warp; k0 < p.C; k0 += 64 * ROWS_WARPS * DEPTH) {
    uint4 a[2 * DEPTH][2], b[2 * DEPTH][GROUPS];
#pragma unroll
    for (int q = 0; q < 2 * DEPTH; ++q) {
      const int k = k0 + 64 * ROWS_WARPS * (q >> 1) + 32 * (q & 1);
      const bool in = k + 8 * t < p.C;
      a[q][0] = load16_if(wg + k, in);
      a[q][1] = load16_if(wu + k, in);
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) b[q][i] = load16_if(x[i] + k, in);
    }
#pragma unroll
    for (int q = 0; q < 2 * DEPTH; ++q)
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        const uint4 &ga = a[q][0], &up = a[q][1], &xb = b[q][i];
        mma_16816(acc[i], ga.x, up.x, ga.y, up.y, xb.x, xb.y);
        mma_16816(acc[i], ga.z, up.z, ga.w, up.w, xb.z, xb.w);
      }
  }
#pragma unroll
  for (int i = 0; i < GROUPS; ++i)
#pragma unroll
    for (int z = 0; z < 4; ++z) red[warp][i][z][lane] = acc[i][z];
  __syncthreads();
  if (warp >= GROUPS) return;
  float v[4];
#pragma unroll
  for (int z = 0; z < 4; ++z) {
    v[z] = 0.f;
#pragma unroll
    for (int w = 0; w < ROWS_WARPS; ++w) v[z] += red[w][warp][z][lane];
  }
  float h0, h1;
  f2_unpack(f2_mul(act2<ACT>(f2_pack(v[0], v[1]), nullptr), f2_pack(v[2], v[3])), h0, h1);
  const float res[2][3] = {{h0, v[0], v[2]}, {h1, v[1], v[3]}};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int row = 8 * warp + 2 * t + k, s = row / sg.rows;
    if (row >= total || (sg.gated && p.mode[s] == RA_MODE_REUSE)) continue;
#pragma unroll
    for (int z = 0; z < 3; ++z)
      if (sg.out[z].ptr)
        sg.out[z].ptr[s * sg.out[z].ss + (row - s * sg.rows) * sg.out[z].sr + f] = __float2bfloat16_rn(res[k][z]);
  }
}

// ------------------------------------------------------------------ some rows
// Up to 128 rows, bound by the weights' bytes too. The weights are the MMA's M (up to 64
// features' gate rows, then their up rows) and x its N, so a CTA stages no more of x
// than there are rows, and the features are divided evenly over the SMs. Cold weights,
// 2048 -> 5504: 17 rows 12.4 us (3.6 TB/s), 128 rows 15.3 (tiles of 256 rows: 19.5 and
// 16.2); 4096 -> 11,008: 31.9 (5.6 TB/s) and 38.3 (43.4 and 44.6). Where few features
// would leave SMs idle or a CTA few of its own, a cluster shares K and adds up as in
// glu_cols_kernel: 17 rows of 2496 -> 1344 13.6 us without, 8.4; of 3264 -> 4160 17.2
// and 14.0.
//   warp 0      TMA producer: stages of 64 of K.
//   warp 1      TMEM allocator, MMA issuer.
//   warps 2..5  drain the accumulator (a lane is a feature) into shared memory,
//               where all warps meet g and w of a feature and a row.
constexpr int SOME_MAX = 128;  // columns; x then has as many bytes a stage as the weights
constexpr int SOME_THREADS = 192, SOME_RING = 16;
constexpr int SOME_SLACK = 16384 + 1024;  // the MMA reads 128 rows of A, of which 2 f are its own; alignment
struct alignas(64) SomeSeg {
  CUtensorMap x, w[2];
  Rows out[3];
  int32_t B, rows, nb, N, gated;  // nb: columns of the accumulator that a sample has
};
struct SomeParams {
  SomeSeg seg[3];
  int32_t F, f, stages, cs, ring, stage_bytes, tmem_cols;
  const int32_t* mode;
  int32_t* err_word;
  uint64_t budget_ns;
};

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

template <int ACT>
__global__ void __launch_bounds__(SOME_THREADS) glu_some_kernel(const __grid_constant__ SomeParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[SOME_RING], empty[SOME_RING], done, drain;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const SomeSeg& sg = p.seg[blockIdx.y];
  const int cs = p.cs, rank = cs > 1 ? int(cluster_rank()) : 0, f0 = int(blockIdx.x) / cs * p.f, a_box = 2 * p.f * 128;
  const int k0 = p.stages * rank / cs, stages = p.stages * (rank + 1) / cs - k0;  // this CTA's part of K
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.ring; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    mbar_init(&done, 1);
    mbar_init(&drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc(&tmem_slot, p.tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const WaitCtl ctl{abort_flag, p.err_word, p.budget_ns};
  pdl_launch();
  if (warp != 0) pdl_wait();
  if (warp == 0) {
    if (lane == 0) {
      tma_prefetch_desc(&sg.w[0]);
      tma_prefetch_desc(&sg.w[1]);
      tma_prefetch_desc(&sg.x);
      pdl_wait();
      const uint32_t bytes = uint32_t(a_box + sg.B * sg.nb * 128);
      int it = 0, st = 0, phase = 1;
      for (; it < stages; ++it) {
        if (it >= p.ring && !mbar_wait(empty + st, uint32_t(phase), ctl)) break;
        uint8_t* to = smem + st * p.stage_bytes;
        mbar_arrive_expect_tx(full + st, bytes);
        tma_load_4d(to, &sg.w[0], full + st, 64 * (k0 + it), f0, 0, 0);
        tma_load_4d(to + p.f * 128, &sg.w[1], full + st, 64 * (k0 + it), f0, 0, 0);
        to += a_box;
        for (int s = 0; s < sg.B; ++s, to += sg.nb * 128) tma_load_4d(to, &sg.x, full + st, 64 * (k0 + it), 0, 0, s);
        if (++st == p.ring) st = 0, phase ^= 1;
      }
      // The CTA does not go before its loads have landed: the products that read them
      // have ended, or, where a role gave up, each load is waited for.
      if (it > 0 && !mbar_wait(&done, 0, ctl))
        for (st = 0; st < p.ring && st < it; ++st)
          mbar_wait_drain(full + st, uint32_t((it - 1 - st) / p.ring & 1), p.budget_ns);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = idesc_bf16_f32(128, sg.N, 0, 0), s0 = smem_u32(smem);
      bool ok = true;
      int it = 0, st = 0, phase = 0;
      for (; it < stages; ++it) {
        if (!(ok = mbar_wait(full + st, uint32_t(phase), ctl))) break;
        tc_fence_after();
        const uint32_t a = s0 + uint32_t(st * p.stage_bytes), x = a + a_box;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          umma_ss(tmem, sdesc_sw128(a + kk * 32, 16, 1024), sdesc_sw128(x + kk * 32, 16, 1024), idesc, it > 0 || kk > 0);
        umma_commit(empty + st);
        if (++st == p.ring) st = 0, phase ^= 1;
      }
      if (ok) umma_commit(&done);
      if (it > 0 && !(ok && mbar_wait(&done, 0, ctl))) {  // nor before its MMAs have ended
        umma_commit(&drain);
        mbar_wait_drain(&drain, 0, p.budget_ns);
      }
    }
  } else if (__all_sync(0xffffffffu, mbar_wait(&done, 0, ctl))) {
    tc_fence_after();
    // every load has landed and been used: the accumulator goes where the stages were, [column][feature row]
    const int quarter = warp & 3, row = 32 * quarter + lane;
    float* to = reinterpret_cast<float*>(smem) + row;
    if (32 * quarter < 2 * p.f)
      for (int c = 0; c < sg.N; c += 32) {
        uint32_t v[32];
        tmem_ld32(tmem + (uint32_t(32 * quarter) << 16) + uint32_t(c), v);
        tmem_ld_wait_for(v);
        if (row < 2 * p.f)
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (c + i < sg.N) to[(c + i) * 2 * p.f] = __uint_as_float(v[i]);
      }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, p.tmem_cols);
  }
  if (cs > 1) {
    __syncwarp();
    cluster_sync_all();
  }
  // This CTA's share of the columns, each sample's rows among them.
  const int n0 = sg.N * rank / cs, n1 = *abort_flag ? n0 : min(sg.N * (rank + 1) / cs, sg.B * sg.nb), vecs = p.f / 8;
  const uint32_t sums = smem_u32(smem);
  for (int i = n0 * vecs + int(threadIdx.x); i < n1 * vecs; i += SOME_THREADS) {
    const int n = i / vecs, j = 8 * (i - n * vecs), s = n / sg.nb, r = n - s * sg.nb;
    if (r >= sg.rows || f0 + j >= p.F || (sg.gated && p.mode[s] == RA_MODE_REUSE)) continue;
    uint64_t g[4], w[4];
    const uint32_t at = sums + uint32_t(n * 2 * p.f + j) * 4u;
    if (cs == 1) {
      const float* src = reinterpret_cast<const float*>(smem) + n * 2 * p.f + j;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(src + 4 * q);
        const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(src + p.f + 4 * q);
        g[2 * q] = x.x, g[2 * q + 1] = x.y, w[2 * q] = y.x, w[2 * q + 1] = y.y;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) g[q] = w[q] = 0;
      for (int c = 0; c < cs; ++c) {  // in order
        const uint32_t from = mapa_shared(at, uint32_t(c));
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float4 x = ld_cluster_f4(from + 16 * q), y = ld_cluster_f4(from + 4 * p.f + 16 * q);
          g[2 * q] = f2_add(g[2 * q], f2_pack(x.x, x.y)), g[2 * q + 1] = f2_add(g[2 * q + 1], f2_pack(x.z, x.w));
          w[2 * q] = f2_add(w[2 * q], f2_pack(y.x, y.y)), w[2 * q + 1] = f2_add(w[2 * q + 1], f2_pack(y.z, y.w));
        }
      }
    }
    uint32_t o[3][4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      o[0][q] = f2_bf16(f2_mul(act2<ACT>(g[q], nullptr), w[q])), o[1][q] = f2_bf16(g[q]), o[2][q] = f2_bf16(w[q]);
#pragma unroll
    for (int z = 0; z < 3; ++z)
      if (sg.out[z].ptr)
        *reinterpret_cast<uint4*>(row_ptr(sg.out[z], s, r, f0 + j)) = make_uint4(o[z][0], o[z][1], o[z][2], o[z][3]);
  }
  if (cs > 1) {
    __syncwarp();
    cluster_sync_all();  // the others have read this CTA's sums
  }
}

// ------------------------------------------------------------------ backward, some rows
// du (with dg and dw) and dx of few rows: too few tiles of 256 rows for the SMs, and a
// long K. Here 128 columns of a weight are the MMA's M (MN-major, as they
// lie), up to 128 rows its N, and a cluster of up to eight CTAs shares K: each sums its
// part in TMEM and leaves it in its shared memory, then takes its share of the rows from
// all of them, in order. So nothing goes through memory, and no second kernel joins.
// Warps as in glu_some_kernel.
constexpr int COLS_M = 128, COLS_BK = 64, COLS_N = 128;
constexpr int COLS_W_BYTES = COLS_M * COLS_BK * 2, COLS_RING = 6;
constexpr int COLS_SMEM = 112 * 1024;  // two CTAs an SM
struct alignas(64) ColsParams {
  CUtensorMap a[2], w[2];  // STORE: two operand pairs, one after the other in K
  Rows out[2], pre[2];     // GRAD: dg, dw; g, w. STORE: the result
  int32_t rows, cols, blocks, col_tiles, N, spans, span_stages, ring, tmem_cols;  // blocks of N rows of a sample
  int32_t* err_word;
  uint64_t budget_ns;
};

template <int KIND, int ACT>
__global__ void __launch_bounds__(SOME_THREADS) glu_cols_kernel(const __grid_constant__ ColsParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[COLS_RING], empty[COLS_RING], done, drain;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cs = int(cluster_size()), rank = int(cluster_rank()), unit = int(blockIdx.x) / cs;
  const int tile = unit / p.blocks, r0 = (unit - tile * p.blocks) * p.N, s = tile / p.col_tiles;
  const int c0 = (tile - s * p.col_tiles) * COLS_M;
  const int stages = p.spans * p.span_stages, k0 = stages * rank / cs, k1 = stages * (rank + 1) / cs;
  const int stage_bytes = COLS_W_BYTES + p.N * 128;
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.ring; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    mbar_init(&done, 1);
    mbar_init(&drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc(&tmem_slot, p.tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const WaitCtl ctl{abort_flag, p.err_word, p.budget_ns};
  pdl_launch();
  if (warp != 0) pdl_wait();
  if (warp == 0) {
    if (lane == 0) {
      tma_prefetch_desc(&p.w[0]);
      tma_prefetch_desc(&p.a[0]);
      pdl_wait();
      int it = 0, st = 0, phase = 1, span = k0 / p.span_stages, k = (k0 - span * p.span_stages) * COLS_BK;
      for (; it < k1 - k0; ++it) {
        if (it >= p.ring && !mbar_wait(empty + st, uint32_t(phase), ctl)) break;
        uint8_t* to = smem + st * stage_bytes;
        mbar_arrive_expect_tx(full + st, uint32_t(stage_bytes));  // past an edge: zeros
        tma_load_4d(to, &p.w[span], full + st, c0, k, 0, 0);
        tma_load_4d(to + COLS_W_BYTES / 2, &p.w[span], full + st, c0 + 64, k, 0, 0);
        tma_load_4d(to + COLS_W_BYTES, &p.a[span], full + st, k, r0, 0, s);
        k += COLS_BK;
        if (k >= p.span_stages * COLS_BK) k = 0, ++span;
        if (++st == p.ring) st = 0, phase ^= 1;
      }
      // The CTA does not go before its loads have landed: the products that read them
      // have ended, or, where a role gave up, each load is waited for.
      if (it > 0 && !mbar_wait(&done, 0, ctl))
        for (st = 0; st < p.ring && st < it; ++st)
          mbar_wait_drain(full + st, uint32_t((it - 1 - st) / p.ring & 1), p.budget_ns);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = idesc_bf16_f32(COLS_M, p.N, 1, 0), s0 = smem_u32(smem);
      bool ok = true;
      int it = 0, st = 0, phase = 0;
      for (; it < k1 - k0; ++it) {
        if (!(ok = mbar_wait(full + st, uint32_t(phase), ctl))) break;
        tc_fence_after();
        const uint32_t w = s0 + uint32_t(st * stage_bytes), a = w + COLS_W_BYTES;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)  // 16 rows of 128 bytes; 32 bytes of a row
          umma_ss(tmem, sdesc_sw128(w + kk * 2048, COLS_W_BYTES / 2, 1024), sdesc_sw128(a + kk * 32, 16, 1024), idesc,
                  it > 0 || kk > 0);
        umma_commit(empty + st);
        if (++st == p.ring) st = 0, phase ^= 1;
      }
      if (ok) umma_commit(&done);
      if (it > 0 && !(ok && mbar_wait(&done, 0, ctl))) {  // nor before its MMAs have ended
        umma_commit(&drain);
        mbar_wait_drain(&drain, 0, p.budget_ns);
      }
    }
  } else if (__all_sync(0xffffffffu, mbar_wait(&done, 0, ctl))) {
    tc_fence_after();
    // every load has landed and been used: the sums go where the stages were, [row][column]
    const int quarter = warp & 3;
    float* to = reinterpret_cast<float*>(smem) + 32 * quarter + lane;
    for (int c = 0; c < p.N; c += 32) {
      uint32_t v[32];
      tmem_ld32(tmem + (uint32_t(32 * quarter) << 16) + uint32_t(c), v);
      tmem_ld_wait_for(v);
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (c + i < p.N) to[(c + i) * COLS_M] = __uint_as_float(v[i]);
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, p.tmem_cols);
  }
  __syncwarp();
  cluster_sync_all();
  const int n0 = p.N * rank / cs, n1 = p.N * (rank + 1) / cs;
  const uint32_t mine = smem_u32(smem);
  for (int i = n0 * (COLS_M / 8) + int(threadIdx.x); i < n1 * (COLS_M / 8); i += SOME_THREADS) {
    const int n = i / (COLS_M / 8), j = 8 * (i % (COLS_M / 8)), r = r0 + n, c = c0 + j;
    if (r >= p.rows || c >= p.cols) continue;
    uint4 g, w;
    if constexpr (KIND == GRAD) {
      g = *reinterpret_cast<const uint4*>(row_ptr(p.pre[0], s, r, c));
      w = *reinterpret_cast<const uint4*>(row_ptr(p.pre[1], s, r, c));
    }
    float4 lo = make_float4(0.f, 0.f, 0.f, 0.f), hi = lo;
    for (int q = 0; q < cs; ++q) {
      const uint32_t at = mapa_shared(mine + uint32_t(n * COLS_M + j) * 4u, uint32_t(q));
      const float4 x = ld_cluster_f4(at), y = ld_cluster_f4(at + 16);
      lo.x += x.x, lo.y += x.y, lo.z += x.z, lo.w += x.w;
      hi.x += y.x, hi.y += y.y, hi.z += y.z, hi.w += y.w;
    }
    const uint64_t v[4] = {f2_pack(lo.x, lo.y), f2_pack(lo.z, lo.w), f2_pack(hi.x, hi.y), f2_pack(hi.z, hi.w)};
    if constexpr (KIND == GRAD) {
      uint32_t* gp = reinterpret_cast<uint32_t*>(&g);
      uint32_t* wp = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint64_t da;
        const uint64_t a = act2<ACT>(bf2_unpack(gp[q]), &da);
        gp[q] = f2_bf16(f2_mul(f2_mul(v[q], bf2_unpack(wp[q])), da));
        wp[q] = f2_bf16(f2_mul(v[q], a));
      }
      *reinterpret_cast<uint4*>(row_ptr(p.out[0], s, r, c)) = g;
      *reinterpret_cast<uint4*>(row_ptr(p.out[1], s, r, c)) = w;
    } else {
      *reinterpret_cast<uint4*>(row_ptr(p.out[0], s, r, c)) =
          make_uint4(f2_bf16(v[0]), f2_bf16(v[1]), f2_bf16(v[2]), f2_bf16(v[3]));
    }
  }
  __syncwarp();
  cluster_sync_all();  // the others have read this CTA's sums
}

// Adds up the parts of the jobs that were cut, in order.
struct JoinJob {
  const float* partial;
  int64_t plane, vecs;  // elements of a part; eight-column pieces of the output
  int32_t parts, rows, N;
  Rows out;
};
struct JoinParams {
  int32_t n;
  JoinJob job[MAX_JOBS];
};
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinParams p) {
  pdl_launch();
  pdl_wait();
  for (int j = 0; j < p.n; ++j) {
    const JoinJob& job = p.job[j];
    const int row_vecs = job.N / 8;
    for (int64_t v = blockIdx.x * int64_t(256) + threadIdx.x; v < job.vecs; v += int64_t(gridDim.x) * 256) {
      const int64_t row = v / row_vecs;
      const int col = 8 * int(v - row * row_vecs);
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
      const float* src = job.partial + row * job.N + col;
      for (int q = 0; q < job.parts; ++q, src += job.plane) {
        const float4 a = reinterpret_cast<const float4*>(src)[0], b = reinterpret_cast<const float4*>(src)[1];
        x[0] += a.x, x[1] += a.y, x[2] += a.z, x[3] += a.w, x[4] += b.x, x[5] += b.y, x[6] += b.z, x[7] += b.w;
      }
      const int64_t s = row / job.rows;
      *reinterpret_cast<uint4*>(job.out.ptr + s * job.out.ss + (row - s * job.rows) * job.out.sr + col) =
          make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                     pack_bf16x2(x[6], x[7]));
    }
  }
}

// ------------------------------------------------------------------ host
bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

// Row tensor of B samples of n rows of `cols` features; an output of B > 1 samples has a place for each.
struct RowTensor {
  const void* ptr;
  int64_t ss, sr;
  int B, n, cols;
};
bool check_rows(const char* who, const char* what, const RowTensor& t, bool output) {
  if (t.ptr && aligned16(t.ptr) && t.ss % 8 == 0 && t.sr % 8 == 0 && t.sr >= t.cols &&
      t.ss >= (output && t.B > 1 ? t.cols : 0))
    return true;
  set_error("%s: %s must be given, 16-byte aligned, with strides multiples of 8 elements, row stride >= %d", who, what,
            t.cols);
  return false;
}
RowSpan span_of(const RowTensor& t) { return RowSpan{t.ptr, 2 * t.ss, 2 * t.sr, t.B, t.n, int64_t(2) * t.cols}; }
RowSpan span_of(const void* ptr, int64_t bytes) { return RowSpan{ptr, 0, 0, 1, 1, bytes}; }
// The samples' rows follow one another: B samples of n rows are one of B n.
bool joins(const RowTensor& t) { return t.B == 1 || t.ss == t.n * t.sr; }

// Tensor map of a row tensor: boxes of 64 features x box_rows (MN-major: 128 of K).
bool encode(CUtensorMap* tm, const RowTensor& t, int box_rows) {
  const ra_seg s{const_cast<void*>(t.ptr), t.B > 1 ? t.ss : 0, 0, t.sr, t.n, 0};
  return encode_seg(tm, s, t.B, 1, t.cols, 64, box_rows, true);
}
// 32 x 32 tiles, in shared memory as stage_slot() has them.
bool encode_tiles(CUtensorMap* tm, const RowTensor& t) {
  const ra_seg s{const_cast<void*>(t.ptr), t.B > 1 ? t.ss : 0, 0, t.sr, t.n, 0};
  return encode_seg(tm, s, t.B, 1, t.cols, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B);
}

template <int KIND>
void one_span(Job& job, int k) {
  job.spans = job.parts = 1;
  job.span_k = k;
  job.span_stages = (k + Cfg<KIND>::BK - 1) / Cfg<KIND>::BK;
}
constexpr int BK = Cfg<STORE>::BK;
static_assert(BK == Cfg<GLU>::BK, "one stage length in the cost model");

// The job's tiles are known: the numbers that its walk divides by.
void set_divs(Job& job) {
  auto div = [](int64_t d) { return Div{uint32_t(d), d > 1 ? uint32_t(((int64_t(1) << 32) + d - 1) / d) : 0u}; };
  job.by_band = div(int64_t(GROUP_M) * job.cols);
  job.by_parts = div(job.parts);
}
template <int KIND>
ra_status launch(const char* who, void (*fn)(Params), Params& p, int64_t units, cudaStream_t st) {
  for (int j = 0; j < p.n_jobs; ++j) set_divs(p.job[j]);
  const ra_status as = ensure_dynamic_smem(reinterpret_cast<const void*>(fn), Cfg<KIND>::SMEM_ALLOC, who);
  if (as != RA_OK) return as;
  const int64_t pairs = num_sms() / 2 > 0 ? num_sms() / 2 : 1;
  cudaLaunchAttribute attr[2];
  attr[0] = pdl_attribute();
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(2 * (units < pairs ? units : pairs)));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = Cfg<KIND>::SMEM_ALLOC;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, p);
  if (e != cudaSuccess) {
    set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
    cudaGetLastError();
    return RA_ECUDA;
  }
  return launch_status(who);
}

// Microseconds of a round of tiles of bn columns over `stages` of K, and of a
// launch around its rounds, fitted on a GB300: single waves of long K, and tiles of
// one to four stages, where the epilogue (0.01 us a column) is the longer part but
// not all of the time.
double round_us(int bn, double stages) {
  const double mma = stages / 8.0 * (3.11 + 0.00766 * bn), epilogue = 0.0105 * bn;
  return std::sqrt(mma * mma + epilogue * epilogue);
}
double fixed_us(int bn) { return 4.4 + 0.0088 * bn; }

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A product whose result is stored: M x N over `stages` of K.
struct Shape {
  int64_t samples, M, N, stages;
  int64_t tiles(int bn) const { return samples * div_up(M, TM) * div_up(N, bn); }
};
// The products of refadapt_glu_backward after dy Wd: dx, and the weights'
// gradients. Rows of samples that follow one another are those of one sample.
struct Products {
  Shape x, w[3];
  Products(int B, int rows, int C, int F, int O, bool flat_x, bool flat_w) {
    const int64_t all = int64_t(B) * rows, stages = flat_w ? div_up(all, BK) : B * div_up(rows, BK);
    x = Shape{flat_x ? 1 : B, flat_x ? all : rows, C, 2 * div_up(F, BK)};
    w[0] = w[1] = Shape{1, F, C, stages};
    w[2] = Shape{1, O, F, stages};
  }
};

// How a launch of them is cut: accumulator columns, parts of K of dx and of the
// weights' gradients, and the schedule's early rounds.
struct Plan {
  int bn, parts_x, parts_w, early;
};
constexpr int MAX_PARTS = 16;
// The cheapest by the time of the pair that ends last. More than two rounds of
// tiles are not cut (a part costs a round trip of its fp32 sums).
Plan make_plan(const Products& pr, bool dx, int sms) {
  const int64_t pairs = sms / 2 > 0 ? sms / 2 : 1;
  Plan best{256, 1, 1, 0};
  double best_us = 1e30;
  for (int bn = 256; bn >= 128; bn -= 64)
    for (int px = 1; px <= MAX_PARTS; px += px < 4 ? 1 : 4) {
      if (px > 1 && (!dx || pr.x.stages < 2 * px || pr.x.tiles(bn) > 2 * pairs)) break;
      for (int pw = 1; pw <= MAX_PARTS; pw += pw < 4 ? 1 : 4) {
        const int64_t tiles_w = pr.w[0].tiles(bn) * 2 + pr.w[2].tiles(bn);
        if (pw > 1 && (pr.w[0].stages < 2 * pw || tiles_w > 2 * pairs)) break;
        const int64_t nx = dx ? pr.x.tiles(bn) * px : 0, nw = tiles_w * pw, rest = nx % pairs;
        const double a = round_us(bn, double(pr.x.stages) / px), b = round_us(bn, double(pr.w[0].stages) / pw);
        double bytes = px > 1 ? 8.0 * px * double(pr.x.samples * pr.x.M * pr.x.N) : 0.0;
        if (pw > 1)
          for (const Shape& w : pr.w) bytes += 8.0 * pw * double(w.M * w.N);
        // early rounds until the pairs without a further dx unit have caught up
        int64_t early = rest > 0 ? int64_t(a / b + 0.5) : 0;
        if (early * (pairs - rest) > nw) early = nw / (pairs - rest);
        const int64_t common = div_up(nw - early * (pairs - rest), pairs);
        const double with = double(div_up(nx, pairs)) * a, without = double(nx / pairs) * a + double(early) * b;
        const double us = fixed_us(bn) + (with > without ? with : without) + double(common) * b +
                          (bytes > 0 ? 2.5 + bytes / 5e6 : 0.0);
        if (us < best_us) {
          best_us = us;
          best = Plan{bn, px, pw, int(early)};
        }
      }
    }
  return best;
}

// Clusters of c CTAs of a kernel that the GPU holds at once (of eight CTAs of
// glu_cols_kernel, two an SM: 36, though 304 CTAs fit). One cluster more than fits
// doubles a kernel's time.
ClusterTable::Counts resident_clusters(const void* fn, int smem) {
  static ClusterTable table;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) cudaGetLastError();
  return table.get(dev, fn, smem, [&](int c) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(c);
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(c));
    cfg.blockDim = dim3(SOME_THREADS);
    cfg.dynamicSmemBytes = size_t(smem);
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, fn, &cfg) == cudaSuccess) return n;
    cudaGetLastError();
    return -1;
  });
}

// Does glu_some_kernel take the call? Its shape: features a CTA and CTAs that share K,
// so that the busiest SM stages the fewest bytes (it stages about 64 a ns; a byte of the
// sums that a cluster exchanges takes as long as five); stages as the shared memory has room
// for, or half of it where there is more than one round: then a CTA has its first loads
// in flight while the one before it ends.
constexpr int SOME_SMEM = 225 * 1024, SOME_SMEM_HALF = 112 * 1024, SOME_MAX_CS = 4;
bool some_rows(const ra_glu_args& a, const Params& p, const RowTensor (&x)[3], const void* fn, SomeParams& sp) {
  std::memset(&sp, 0, sizeof(sp));
  int most = 0;
  for (int j = 0; j < p.n_jobs; ++j) {
    const Job& job = p.job[j];
    SomeSeg& d = sp.seg[j];
    const int64_t nb = (int64_t(job.rows) + 7) / 8 * 8, n = (nb * x[j].B + 15) / 16 * 16;
    if (n > SOME_MAX) return false;
    d.B = job.samples, d.rows = job.rows, d.nb = int(nb), d.N = int(n), d.gated = job.gated;
    for (int z = 0; z < 3; ++z) d.out[z] = job.out[z];
    most = d.N > most ? d.N : most;
  }
  const int sms = num_sms();
  sp.F = a.F;
  sp.stages = int(div_up(a.C, 64));
  int64_t best = INT64_MAX, rounds = 1;
  const ClusterTable::Counts held = resident_clusters(fn, SOME_SMEM);
  for (int cs = 1; cs <= SOME_MAX_CS && cs <= sp.stages; ++cs)
    for (int f = 8; f <= 64; f += 8) {
      const int64_t units = div_up(a.F, f) * p.n_jobs;
      if (cs > 1 && units > held.of[cs]) continue;
      const int64_t turns = cs > 1 ? 1 : div_up(units, sms);
      const int64_t bytes = turns * (2 * f + most) * 128 * div_up(sp.stages, cs) + (cs > 1 ? 5 * most * 2 * f * 4 : 0);
      if (bytes < best) best = bytes, rounds = turns, sp.f = f, sp.cs = cs;
    }
  sp.stage_bytes = 128 * (2 * sp.f + most);
  sp.ring = ((rounds > 1 ? SOME_SMEM_HALF : SOME_SMEM) - SOME_SLACK) / sp.stage_bytes;
  if (sp.ring > SOME_RING) sp.ring = SOME_RING;
  if (sp.ring > div_up(sp.stages, sp.cs)) sp.ring = int(div_up(sp.stages, sp.cs));
  // the fp32 tile takes the place of the stages
  while (sp.ring * sp.stage_bytes < most * 2 * sp.f * 4) ++sp.ring;
  sp.tmem_cols = 32;
  while (sp.tmem_cols < most) sp.tmem_cols *= 2;
  return true;
}

// Rows up to which glu_cols_kernel takes du, and dx too: beside the weights' gradients,
// which are many short tiles, dx by tiles costs little more than they do. All
// gradients: 4 rows of 1024 -> 2736 34.8 us by tiles alone, 27.7; 30 of 2000 -> 3504
// 44.9, 38.9 (with dx here 44.9); 64 of 1024 -> 4096 35.2, 34.5; 128 rows even. dx
// alone: 30 rows 33.6 and 20.0, 128 of 2048 -> 5504 51.6 and 39.9, 200 of 1536 -> 4096
// 36.9 and 33.9, 400 of 512 -> 8192 36.0 and 42.2.
constexpr int COLS_ROWS_DU = 64, COLS_ROWS_DX = 16, COLS_ROWS_ALONE = 256;
int cols_box(int rows) {  // rows of a block, as launch_cols has them
  const int64_t blocks = div_up(rows, COLS_N);
  return int(div_up(div_up(rows, blocks), 16) * 16);
}
template <int KIND>
ra_status launch_cols(const char* who, void (*fn)(ColsParams), ColsParams& p, int samples, cudaStream_t st) {
  const int sms = num_sms();
  p.blocks = int(div_up(p.rows, COLS_N));
  p.N = cols_box(p.rows);
  p.col_tiles = int(div_up(p.cols, COLS_M));
  const int stages = p.spans * p.span_stages;
  const int64_t units = int64_t(samples) * p.blocks * p.col_tiles;
  const int stage_bytes = COLS_W_BYTES + p.N * 128;
  p.ring = (COLS_SMEM - 1024) / stage_bytes < COLS_RING ? (COLS_SMEM - 1024) / stage_bytes : COLS_RING;
  p.tmem_cols = 32;
  while (p.tmem_cols < p.N) p.tmem_cols *= 2;
  const ra_status as = ensure_dynamic_smem(reinterpret_cast<const void*>(fn), COLS_SMEM, who);
  if (as != RA_OK) return as;
  int cs = 1;
  double best = 1e30;
  const ClusterTable::Counts held = resident_clusters(reinterpret_cast<const void*>(fn), COLS_SMEM);
  for (int c = 1; c <= ClusterTable::MAX_CLUSTER && c <= stages; ++c) {
    if (held.of[c] < 1) continue;
    const double us = 2.0 * double(div_up(units, held.of[c])) +
                      0.2 * double(div_up(units * c, sms) * div_up(stages, c)) + 0.15 * c;
    if (us < best) best = us, cs = c;
  }
  cudaLaunchAttribute attr[2];
  attr[0] = pdl_attribute();
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(cs);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(units * cs));
  cfg.blockDim = dim3(SOME_THREADS);
  cfg.dynamicSmemBytes = size_t(p.ring) * stage_bytes + 1024;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, p);
  if (e != cudaSuccess) {
    set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
    cudaGetLastError();
    return RA_ECUDA;
  }
  return launch_status(who);
}

size_t partial_bytes(const Shape& s, int parts) {
  return parts > 1 ? size_t(parts) * size_t(s.samples) * size_t(s.M) * size_t(s.N) * 4 : 0;
}

}  // namespace glu
}  // namespace ra

extern "C" ra_status refadapt_glu(const ra_glu_args* a, void* stream) {
  using namespace ra;
  using namespace ra::glu;
  const char* who = "refadapt_glu";
  clear_error();
  if (!a) {
    set_error("%s: args is NULL", who);
    return RA_EINVAL;
  }
  if (a->B < 1 || a->n_seg < 1 || a->n_seg > 3 || a->C < 64 || a->C % 8 != 0 || a->F < 64 || a->F % 8 != 0 ||
      (a->act != RA_ACT_SILU && a->act != RA_ACT_GELU)) {
    set_error("%s: need B >= 1, 1 <= n_seg <= 3, C and F multiples of 8 and at least 64, a known activation (B=%d n_seg=%d "
              "C=%d F=%d act=%d)", who, a->B, a->n_seg, a->C, a->F, a->act);
    return RA_EINVAL;
  }
  Params p;
  std::memset(&p, 0, sizeof(p));
  p.mode = a->mode;
  p.err_word = a->err_word;
  p.budget_ns = wait_budget_ns();
  RowTensor x[3];
  RowSpan ins[9], all_out[9];  // of all segments
  int n_in = 0, n_out = 0;
  for (int g = 0; g < a->n_seg; ++g) {
    const ra_glu_seg& s = a->seg[g];
    if (s.rows < 0) {
      set_error("%s: seg %d rows < 0", who, g);
      return RA_EINVAL;
    }
    if (s.gated && !a->mode) {
      set_error("%s: seg %d is gated but mode is NULL", who, g);
      return RA_EINVAL;
    }
    if (s.rows == 0) continue;
    if (!s.w_gate || !s.w_up || !aligned16(s.w_gate) || !aligned16(s.w_up)) {
      set_error("%s: seg %d: w_gate and w_up must be given and 16-byte aligned", who, g);
      return RA_EINVAL;
    }
    if (!s.pre_gate != !s.pre_up) {
      set_error("%s: seg %d: pre_gate and pre_up go together", who, g);
      return RA_EINVAL;
    }
    RowTensor r{s.x, s.x_stride_s, s.x_stride_r, a->B, s.rows, a->C};
    RowTensor o[3] = {{s.out, s.out_stride_s, s.out_stride_r, a->B, s.rows, a->F},
                      {s.pre_gate, s.pre_gate_stride_s, s.pre_gate_stride_r, a->B, s.rows, a->F},
                      {s.pre_up, s.pre_up_stride_s, s.pre_up_stride_r, a->B, s.rows, a->F}};
    const int outs = s.pre_gate ? 3 : 1;
    if (!check_rows(who, "x", r, false) || !check_rows(who, "out", o[0], true) ||
        (s.pre_gate && (!check_rows(who, "pre_gate", o[1], true) || !check_rows(who, "pre_up", o[2], true))))
      return RA_EINVAL;
    if (int64_t(a->B) * s.rows >= (int64_t(1) << 30)) {
      set_error("%s: seg %d: too many rows", who, g);
      return RA_EINVAL;
    }
    ins[n_in++] = span_of(r);
    ins[n_in++] = span_of(s.w_gate, int64_t(2) * a->F * a->C);
    ins[n_in++] = span_of(s.w_up, int64_t(2) * a->F * a->C);
    for (int i = 0; i < outs; ++i) all_out[n_out++] = span_of(o[i]);
    // samples whose rows follow one another share row tiles
    bool flat = !s.gated && joins(r);
    for (int i = 0; i < outs; ++i) flat &= joins(o[i]);
    if (flat) {
      r.n *= r.B;
      r.B = 1;
    }
    const int j = p.n_jobs++;
    x[j] = r;
    Job& job = p.job[j];
    job.samples = r.B;
    job.rows = r.n;
    job.gated = s.gated ? 1 : 0;
    job.m_tiles = int32_t(div_up(r.n, TM));
    job.N = a->F;
    one_span<GLU>(job, a->C);
    for (int i = 0; i < outs; ++i)
      job.out[i] = Rows{static_cast<__nv_bfloat16*>(const_cast<void*>(o[i].ptr)), o[i].ss, o[i].sr};
  }
  if (p.n_jobs == 0) return RA_OK;
  if (overlapping(all_out, n_out, ins, n_in) >= 0) {
    set_error("%s: an output must not overlap an input or another output of any segment", who);
    return RA_EINVAL;
  }
  int most = 0;
  for (int g = 0; g < a->n_seg; ++g)
    if (int64_t(a->B) * a->seg[g].rows > most) most = a->B * a->seg[g].rows;
  if (few_rows(most, int64_t(4) * a->F * a->C)) {
    RowsParams r;
    std::memset(&r, 0, sizeof(r));
    r.B = a->B, r.F = a->F, r.C = a->C, r.mode = a->mode;
    int n = 0;
    for (int g = 0; g < a->n_seg; ++g) {
      const ra_glu_seg& s = a->seg[g];
      if (s.rows == 0) continue;
      RowsSeg& d = r.seg[n++];
      auto rows = [](const void* ptr, int64_t ss, int64_t sr) {
        return Rows{static_cast<__nv_bfloat16*>(const_cast<void*>(ptr)), ss, sr};
      };
      d.x = rows(s.x, s.x_stride_s, s.x_stride_r);
      d.w_gate = static_cast<const __nv_bfloat16*>(s.w_gate), d.w_up = static_cast<const __nv_bfloat16*>(s.w_up);
      d.out[0] = rows(s.out, s.out_stride_s, s.out_stride_r);
      d.out[1] = rows(s.pre_gate, s.pre_gate_stride_s, s.pre_gate_stride_r);
      d.out[2] = rows(s.pre_up, s.pre_up_stride_s, s.pre_up_stride_r);
      d.rows = s.rows;
      d.gated = s.gated ? 1 : 0;
    }
    const bool gelu = a->act == RA_ACT_GELU;
    void (*fn)(RowsParams) = most <= 8 ? (gelu ? glu_rows_kernel<RA_ACT_GELU, 1, 2> : glu_rows_kernel<RA_ACT_SILU, 1, 2>)
                                       : (gelu ? glu_rows_kernel<RA_ACT_GELU, 2, 1> : glu_rows_kernel<RA_ACT_SILU, 2, 1>);
    note_launch("few rows");
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(a->F / 8), unsigned(n));
    cfg.blockDim = dim3(32 * ROWS_WARPS);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr = pdl_attribute();
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, r);
    if (e != cudaSuccess) {
      set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
      cudaGetLastError();
      return RA_ECUDA;
    }
    return launch_status(who);
  }
  void (*some)(SomeParams) = a->act == RA_ACT_GELU ? glu_some_kernel<RA_ACT_GELU> : glu_some_kernel<RA_ACT_SILU>;
  SomeParams sp;
  if (most <= SOME_MAX) {
    const ra_status as = ensure_dynamic_smem(reinterpret_cast<const void*>(some), SOME_SMEM, who);
    if (as != RA_OK) return as;
  }
  if (most <= SOME_MAX && some_rows(*a, p, x, reinterpret_cast<const void*>(some), sp)) {
    sp.mode = a->mode, sp.err_word = a->err_word, sp.budget_ns = p.budget_ns;
    for (int g = 0, j = 0; g < a->n_seg; ++g) {
      const ra_glu_seg& s = a->seg[g];
      if (s.rows == 0) continue;
      SomeSeg& d = sp.seg[j];
      const RowTensor wg{s.w_gate, 0, a->C, 1, a->F, a->C}, wu{s.w_up, 0, a->C, 1, a->F, a->C};
      if (!encode(&d.x, x[j], d.nb) || !encode(&d.w[0], wg, sp.f) || !encode(&d.w[1], wu, sp.f)) return RA_EINVAL;
      ++j;
    }
    note_launch("some rows, %d features, clusters of %d", sp.f, sp.cs);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(div_up(a->F, sp.f) * sp.cs), unsigned(p.n_jobs));
    cfg.blockDim = dim3(SOME_THREADS);
    cfg.dynamicSmemBytes = size_t(sp.ring) * sp.stage_bytes + SOME_SLACK;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0] = pdl_attribute();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(sp.cs);
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = sp.cs > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, some, sp);
    if (e != cudaSuccess) {
      set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
      cudaGetLastError();
      return RA_ECUDA;
    }
    return launch_status(who);
  }
  const int64_t pairs = num_sms() / 2 > 0 ? num_sms() / 2 : 1;
  double best_us = 1e30;
  int64_t units = 0;
  for (int bn = 256; bn >= 64; bn -= 32) {
    int64_t n = 0;
    for (int j = 0; j < p.n_jobs; ++j) n += int64_t(p.job[j].samples) * p.job[j].m_tiles * div_up(a->F, bn / 2);
    const double us = fixed_us(bn) + round_us(bn, double(p.job[0].span_stages)) * double(div_up(n, pairs));
    if (us < best_us) best_us = us, p.bn = bn, units = n;
  }
  for (int g = 0, j = 0; g < a->n_seg; ++g) {
    const ra_glu_seg& s = a->seg[g];
    if (s.rows == 0) continue;
    p.job[j].cols = int32_t(div_up(a->F, p.bn / 2));
    const RowTensor wg{s.w_gate, 0, a->C, 1, a->F, a->C}, wu{s.w_up, 0, a->C, 1, a->F, a->C};
    if (!encode(&p.tm_a[j][0], x[j], 128) || !encode(&p.tm_b[j][0], wg, p.bn / 2) ||
        !encode(&p.tm_b[j][1], wu, p.bn / 2))
      return RA_EINVAL;
    ++j;
  }
  if (units > 2147483647) {
    set_error("%s: too many rows", who);
    return RA_EINVAL;
  }
  note_launch("CTA pairs, %d columns", p.bn / 2);
  return launch<GLU>(who, a->act == RA_ACT_GELU ? glu_kernel<GLU, RA_ACT_GELU> : glu_kernel<GLU, RA_ACT_SILU>, p, units, static_cast<cudaStream_t>(stream));
}

extern "C" size_t refadapt_glu_backward_workspace_size(int32_t B, int32_t rows, int32_t C, int32_t F, int32_t O) {
  using namespace ra::glu;
  if (B < 1 || rows < 0 || C < 64 || F < 64 || O < 64) return 0;
  const int sms = ra::num_sms();
  size_t most = 0;
  if (rows > 0)
    for (int flat = 0; flat < (B > 1 ? 4 : 1); ++flat) {
      const Products pr(B, rows, C, F, O, flat & 1, flat & 2);
      for (int dx = 0; dx < 2; ++dx) {
        const Plan plan = make_plan(pr, dx, sms);
        size_t b = partial_bytes(pr.x, plan.parts_x);
        for (const Shape& w : pr.w) b += partial_bytes(w, plan.parts_w);
        most = b > most ? b : most;
      }
    }
  return size_t(2) * size_t(B) * size_t(rows) * size_t(F) * 2 + most + 16;
}

extern "C" ra_status refadapt_glu_backward(const ra_glu_grad_args* a, void* stream) {
  using namespace ra;
  using namespace ra::glu;
  const char* who = "refadapt_glu_backward";
  clear_error();
  if (!a) {
    set_error("%s: args is NULL", who);
    return RA_EINVAL;
  }
  if (a->B < 1 || a->rows < 0 || a->C < 64 || a->C % 8 != 0 || a->F < 64 || a->F % 8 != 0 || a->O < 64 ||
      a->O % 8 != 0 || (a->act != RA_ACT_SILU && a->act != RA_ACT_GELU)) {
    set_error("%s: need B >= 1, rows >= 0, C, F and O multiples of 8 and at least 64, a known activation (B=%d rows=%d "
              "C=%d F=%d O=%d act=%d)", who, a->B, a->rows, a->C, a->F, a->O, a->act);
    return RA_EINVAL;
  }
  if (int64_t(a->B) * a->rows >= (int64_t(1) << 30)) {
    set_error("%s: too many rows", who);
    return RA_EINVAL;
  }
  if (!a->dx && !a->dw_gate && !a->dw_up && !a->dw_down) {
    set_error("%s: no gradient wanted", who);
    return RA_EINVAL;
  }
  if (!aligned16(a->dw_gate) || !aligned16(a->dw_up) || !aligned16(a->dw_down)) {
    set_error("%s: the weights' gradients must be 16-byte aligned", who);
    return RA_EINVAL;
  }
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->rows == 0) {  // sums of no rows
    const size_t fc = size_t(a->F) * a->C * 2, of = size_t(a->O) * a->F * 2;
    cudaError_t e = cudaSuccess;
    if (a->dw_gate) e = cudaMemsetAsync(a->dw_gate, 0, fc, st);
    if (e == cudaSuccess && a->dw_up) e = cudaMemsetAsync(a->dw_up, 0, fc, st);
    if (e == cudaSuccess && a->dw_down) e = cudaMemsetAsync(a->dw_down, 0, of, st);
    if (e != cudaSuccess) {
      set_error("%s: %s", who, cudaGetErrorString(e));
      cudaGetLastError();
      return RA_ECUDA;
    }
    return RA_OK;
  }
  const bool dgw = a->dx || a->dw_gate || a->dw_up;
  RowTensor dy{a->dy, a->dy_stride_s, a->dy_stride_r, a->B, a->rows, a->O};
  RowTensor x{a->x, a->x_stride_s, a->x_stride_r, a->B, a->rows, a->C};
  RowTensor g{a->pre_gate, a->pre_gate_stride_s, a->pre_gate_stride_r, a->B, a->rows, a->F};
  RowTensor w{a->pre_up, a->pre_up_stride_s, a->pre_up_stride_r, a->B, a->rows, a->F};
  RowTensor hid{a->hidden, a->hidden_stride_s, a->hidden_stride_r, a->B, a->rows, a->F};
  RowTensor dx{a->dx, a->dx_stride_s, a->dx_stride_r, a->B, a->rows, a->C};
  if (!check_rows(who, "dy", dy, false) ||
      (dgw && (!check_rows(who, "pre_gate", g, false) || !check_rows(who, "pre_up", w, false))) ||
      ((a->dw_gate || a->dw_up) && !check_rows(who, "x", x, false)) ||
      (a->dw_down && !check_rows(who, "hidden", hid, false)) || (a->dx && !check_rows(who, "dx", dx, true)))
    return RA_EINVAL;
  if ((dgw && (!a->w_down || !aligned16(a->w_down))) ||
      (a->dx && (!a->w_gate || !a->w_up || !aligned16(a->w_gate) || !aligned16(a->w_up)))) {
    set_error("%s: the weights that the wanted gradients need must be given and 16-byte aligned", who);
    return RA_EINVAL;
  }
  const size_t need = refadapt_glu_backward_workspace_size(a->B, a->rows, a->C, a->F, a->O);
  if (!a->workspace || !aligned16(a->workspace) || a->workspace_bytes < need) {
    set_error("%s: workspace NULL, not 16-byte aligned or smaller than refadapt_glu_backward_workspace_size() (%zu bytes)",
              who, need);
    return RA_EINVAL;
  }
  const int64_t fc = int64_t(2) * a->F * a->C, of = int64_t(2) * a->O * a->F;
  const RowSpan ins[] = {span_of(dy), span_of(x), span_of(g), span_of(w), span_of(hid), span_of(a->w_gate, fc),
                         span_of(a->w_up, fc), span_of(a->w_down, of)};
  const RowSpan outs[] = {span_of(dx), span_of(a->dw_gate, fc), span_of(a->dw_up, fc), span_of(a->dw_down, of),
                          span_of(a->workspace, int64_t(need))};
  if (overlapping(outs, 5, ins, 8) >= 0) {
    set_error("%s: dx, the weights' gradients and the workspace must not overlap an input or one another", who);
    return RA_EINVAL;
  }
  const int sms = num_sms();
  const int64_t all = int64_t(a->B) * a->rows;
  __nv_bfloat16* dg_ptr = static_cast<__nv_bfloat16*>(a->workspace);
  __nv_bfloat16* dw_ptr = dg_ptr + all * a->F;
  float* partial = reinterpret_cast<float*>(dw_ptr + all * a->F);
  const int64_t ss = int64_t(a->rows) * a->F;
  RowTensor dgt{dg_ptr, ss, a->F, a->B, a->rows, a->F}, dwt{dw_ptr, ss, a->F, a->B, a->rows, a->F};
  const RowTensor w_gate{a->w_gate, 0, a->C, 1, a->F, a->C}, w_up{a->w_up, 0, a->C, 1, a->F, a->C};
  const RowTensor w_down{a->w_down, 0, a->F, 1, a->O, a->F};
  auto flatten = [](RowTensor t) {
    t.n *= t.B;
    t.B = 1;
    return t;
  };
  Params p;
  std::memset(&p, 0, sizeof(p));
  p.err_word = a->err_word;
  p.budget_ns = wait_budget_ns();
  auto rows_of = [](const RowTensor& t) {
    return Rows{static_cast<__nv_bfloat16*>(const_cast<void*>(t.ptr)), t.ss, t.sr};
  };
  const int64_t pairs = sms / 2 > 0 ? sms / 2 : 1;
  auto cols_params = [&](const RowTensor& t, int cols, int spans, int k) {
    ColsParams c;
    std::memset(&c, 0, sizeof(c));
    c.rows = t.n, c.cols = cols, c.spans = spans;
    c.span_stages = int(div_up(k, COLS_BK));
    c.err_word = a->err_word, c.budget_ns = p.budget_ns;
    return c;
  };
  const bool alone = !(a->dw_gate || a->dw_up || a->dw_down);
  const bool du_cols = all <= (alone ? COLS_ROWS_ALONE : COLS_ROWS_DU), dx_cols = a->dx && du_cols && (alone || all <= COLS_ROWS_DX);
  if (dgw && du_cols) {
    const bool flat = joins(dy) && joins(g) && joins(w);
    auto one = [&](const RowTensor& t) { return flat ? flatten(t) : t; };
    const RowTensor src = one(dy);
    ColsParams c = cols_params(src, a->F, 1, a->O);
    c.out[0] = rows_of(one(dgt)), c.out[1] = rows_of(one(dwt));
    c.pre[0] = rows_of(one(g)), c.pre[1] = rows_of(one(w));
    if (!encode(&c.a[0], src, cols_box(src.n)) || !encode(&c.w[0], w_down, COLS_BK)) return RA_EINVAL;
    const ra_status r = launch_cols<GRAD>(who, a->act == RA_ACT_GELU ? glu_cols_kernel<GRAD, RA_ACT_GELU> : glu_cols_kernel<GRAD, RA_ACT_SILU>,
                                          c, src.B, st);
    if (r != RA_OK) return r;
  } else if (dgw) {
    const bool flat = joins(dy) && joins(g) && joins(w);
    const RowTensor src = flat ? flatten(dy) : dy;
    Job& job = p.job[0];
    p.n_jobs = 1;
    job.samples = src.B, job.rows = src.n;
    job.m_tiles = int32_t(div_up(src.n, TM));
    job.N = a->F;
    one_span<GRAD>(job, a->O);
    double best_us = 1e30;
    int64_t units = 0;
    for (int bn = 256; bn >= 64; bn -= 64) {
      const int64_t n = int64_t(job.samples) * job.m_tiles * div_up(a->F, bn);
      const double us = fixed_us(bn) + round_us(bn, double(job.span_stages) / 2) * double(div_up(n, pairs));
      if (us < best_us) best_us = us, p.bn = bn, units = n;
    }
    job.cols = int32_t(div_up(a->F, p.bn));
    if (!encode(&p.tm_a[0][0], src, 128) || !encode(&p.tm_b[0][0], w_down, Cfg<GRAD>::BK) ||
        !encode_tiles(&p.tm_tile[0], flat ? flatten(g) : g) || !encode_tiles(&p.tm_tile[1], flat ? flatten(w) : w) ||
        !encode_tiles(&p.tm_tile[2], flat ? flatten(dgt) : dgt) || !encode_tiles(&p.tm_tile[3], flat ? flatten(dwt) : dwt))
      return RA_EINVAL;
    if (units > 2147483647) {
      set_error("%s: too many rows", who);
      return RA_EINVAL;
    }
    const ra_status r = launch<GRAD>(who, a->act == RA_ACT_GELU ? glu_kernel<GRAD, RA_ACT_GELU> : glu_kernel<GRAD, RA_ACT_SILU>, p,
                               units, st);
    if (r != RA_OK) return r;
  }
  // dx and the weights' gradients, in one launch
  if (dx_cols) {
    const bool flat = joins(dx);
    auto one = [&](const RowTensor& t) { return flat ? flatten(t) : t; };
    const RowTensor src = one(dgt);
    ColsParams c = cols_params(src, a->C, 2, a->F);
    c.out[0] = rows_of(one(dx));
    if (!encode(&c.a[0], src, cols_box(src.n)) || !encode(&c.a[1], one(dwt), cols_box(src.n)) ||
        !encode(&c.w[0], w_gate, COLS_BK) || !encode(&c.w[1], w_up, COLS_BK))
      return RA_EINVAL;
    const ra_status r = launch_cols<STORE>(who, glu_cols_kernel<STORE, 0>, c, src.B, st);
    if (r != RA_OK) return r;
  }
  const bool dx_tiles = a->dx && !dx_cols;
  if (!dx_tiles && !a->dw_gate && !a->dw_up && !a->dw_down) return RA_OK;
  const bool flat_x = a->B == 1 || !a->dx || joins(dx);
  const bool flat_w = a->B == 1 || ((!(a->dw_gate || a->dw_up) || joins(x)) && (!a->dw_down || (joins(dy) && joins(hid))));
  const Products pr(a->B, a->rows, a->C, a->F, a->O, flat_x, flat_w);
  const Plan plan = make_plan(pr, dx_tiles, sms);
  std::memset(p.job, 0, sizeof(p.job));
  p.n_jobs = 0;
  p.bn = plan.bn;
  int64_t units = 0, vecs = 0;
  JoinParams join;
  join.n = 0;
  auto add = [&](const Shape& s, int parts, const Rows& out) -> Job& {
    Job& job = p.job[p.n_jobs++];
    job.samples = int32_t(s.samples), job.rows = int32_t(s.M), job.N = int32_t(s.N);
    job.m_tiles = int32_t(div_up(s.M, TM));
    job.cols = int32_t(div_up(s.N, plan.bn));
    job.out[0] = out;
    units += s.tiles(plan.bn) * parts;
    if (parts > 1) {
      job.partial = partial;
      JoinJob& q = join.job[join.n++];
      q.partial = partial;
      q.plane = s.samples * s.M * s.N;
      q.vecs = q.plane / 8;
      q.parts = parts, q.rows = job.rows, q.N = job.N;
      q.out = out;
      partial += q.plane * parts;
      vecs += q.vecs;
    }
    return job;
  };
  if (dx_tiles) {
    Job& job = add(pr.x, plan.parts_x, rows_of(dx));
    one_span<STORE>(job, a->F);
    job.spans = 2;
    job.parts = plan.parts_x;
    if (!encode(&p.tm_a[0][0], flat_x ? flatten(dgt) : dgt, 128) || !encode(&p.tm_a[0][1], flat_x ? flatten(dwt) : dwt, 128) ||
        !encode(&p.tm_b[0][0], w_gate, BK) || !encode(&p.tm_b[0][1], w_up, BK))
      return RA_EINVAL;
    p.order.longs = int32_t(units);
    p.order.early = plan.early;
  }
  void* out[3] = {a->dw_gate, a->dw_up, a->dw_down};
  for (int i = 0; i < 3; ++i) {
    if (!out[i]) continue;
    const int n = p.n_jobs;
    Job& job = add(pr.w[i], plan.parts_w, Rows{static_cast<__nv_bfloat16*>(out[i]), 0, pr.w[i].N});
    one_span<STORE>(job, flat_w ? int(all) : a->rows);
    job.spans = flat_w ? 1 : a->B;
    job.parts = plan.parts_w;
    job.rows_k = 1;
    const RowTensor at = i == 0 ? dgt : i == 1 ? dwt : dy, bt = i == 2 ? hid : x;
    if (!encode(&p.tm_a[n][0], flat_w ? flatten(at) : at, BK) || !encode(&p.tm_b[n][0], flat_w ? flatten(bt) : bt, BK))
      return RA_EINVAL;
  }
  if (units > 2147483647) {
    set_error("%s: too many rows", who);
    return RA_EINVAL;
  }
  const int64_t ctas = units < pairs ? units : pairs;
  // Fewer units than pairs: the plan's early rounds do not fit. A pair with one of dx's
  // units takes another `longs` units further on, and as many pairs take none.
  if (ctas < pairs) p.order.early = 0;
  const ra_status r = launch<STORE>(who, glu_kernel<STORE, 0>, p, units, st);
  if (r != RA_OK || join.n == 0) return r;
  cudaLaunchConfig_t cfg = {};
  const int64_t blocks = div_up(vecs, 256), most = int64_t(8) * sms;
  cfg.gridDim = dim3(unsigned(blocks < most ? blocks : most));
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, join_kernel, join);
  if (e != cudaSuccess) {
    set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
    cudaGetLastError();
    return RA_ECUDA;
  }
  return launch_status(who);
}
