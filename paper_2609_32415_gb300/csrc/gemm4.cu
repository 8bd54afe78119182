// refadapt_gemm4: the linear layers of refadapt_gemm with operands of 4 bits and a scale
// for every few columns,
//   D[r, n] = sum over blocks b of  sa[r, b] sw[n, b]  sum over k in b of  a[r, k] w[n, k]
// on the tensor cores' block-scaled 4-bit MMAs (tcgen05.mma kind::mxf4nvf4, K = 64),
// which multiply the scales in. Tiles and roles are gemm.cu's (one CTA on a tile of 128 rows, or
// a pair on 256); what differs:
//   * A stage holds 256 of K: 128 bytes of codes a row, the swizzled box of 64 bf16, four
//     MMAs; and the rows' scales, whose tiles of 128 rows by 4 blocks (512 bytes) lie in
//     memory as tensor memory wants them, so that a stage's are one TMA box for each operand.
//   * Before a stage's MMAs the issuer has the scales copied to TMEM (tcgen05.cp 32x128b, 32
//     rows by 16 bytes, to every warp's lanes): four columns for 128 rows and four blocks.
//     Buffers of them take turns; one is written again once the MMAs that read it have ended
//     (their commit has arrived).
//   * TMEM holds two accumulators of 192 columns or three of up to 128, and two to six stages' scales.
//     Tiles of 256 columns would leave either the scales or the second accumulator no room, and
//     an epilogue takes as long as the MMAs of K = 1536.
// What bounds it: a stage of a pair's 256 x 192 tile takes 212 to 217 ns (e8m0; e4m3, whose scales have two
// buffers, 240), its MMAs alone 198 (9.7 PFLOP/s), its loads less; a stage of 128 columns 200 (single CTAs 185), of
// which 190 are the issuing warp's waits, copies and commit. Long calls reach the power cap: 8192 rows, K =
// 16384, N = 7296 take 254 to 263 us with e8m0 (7.5 to 7.7 PFLOP/s, four times the bf16 rate), 264 with e4m3. Unrolling
// the issuer by two stages, its tiles from the producer, and two producers each measured even or slower.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>

#include "gemm_body.cuh"
#include "gemm4.h"
#include "launch_plan.h"

namespace ra {
namespace gemm4 {

using namespace gemm;

// A quarter of the TMEM lanes (32 rows) has three epilogue warps, which take the units of 64 columns of all
// tiles in turn: with two units to a tile all three are at work, on one tile and a half.
constexpr int WAYS = 3, EPI4_WARPS = 4 * WAYS, THREADS4 = 64 + 32 * EPI4_WARPS;
constexpr int UNIT = 64;     // columns of a warp
constexpr int CHUNK = 256;   // K of a stage
constexpr int MAX_ACCS = 3;  // accumulators
// Stages of weights that a call of few rows asks for early (130 rows, 2048 -> 8192, weights from memory, with the
// rows' quantisation: 9.1 us, 7.7).
constexpr int AHEAD_STAGES = 32;
constexpr int A_BYTES = BM * CHUNK / 2;
constexpr int SA_BYTES = 4 * 512;  // scales of 128 rows, up to four tiles (e4m3)
constexpr int VEC_BYTES = 2 * UNIT * 4;    // two vectors of its columns
// QKV: the rows' sums of squares of each 32 columns, by tile (one in three) and TMEM lane quarter.
constexpr int SUMS = (128 / 32) * 32, SUMS_BYTES = WAYS * 4 * SUMS * 4;
constexpr int TURN_BYTES = EPI_STAGE_BYTES;  // QKV: a warp's RoPE rows of 16 columns

// Stages of the ring: five, whose shared memory leaves room for a CTA of the kernel before or after this
// one (a block's gradients, with quantisations around the products: 64 us, 69 with six) and L1 for the
// outputs (single CTAs, GELU: 40 and 44 us). Pairs whose call is long take a sixth (16384 rows, K =
// 4096, N = 16384: 349 us, 367 with five; 4096 rows, K = 16384, N = 4096 with e8m0: 83 and 87, but
// 16384 rows, K = 4096: 84.4 and 83.5).
constexpr int FEW_STAGES = 5, MAX_STAGES = 6;
constexpr double LONG_CALL = 100;  // microseconds of the plan

// Shared memory of one CTA a tile, and of CTA pairs (each stages half of the tile's weight rows).
template <bool PAIR_, bool QKV>
struct Layout {
  static constexpr bool PAIR = PAIR_;
  static constexpr int MAX_BN = PAIR && !QKV ? 192 : 128;  // columns of a tile
  static constexpr int B_BYTES = (PAIR ? MAX_BN / 2 : MAX_BN) * CHUNK / 2;
  static constexpr int OFF_B = A_BYTES, OFF_SF = A_BYTES + B_BYTES;
  static constexpr int STAGE_BYTES = OFF_SF + SA_BYTES * (1 + (MAX_BN + 127) / 128);
  // behind the stages
  static constexpr int OFF_SUMS = EPI4_WARPS * VEC_BYTES;
  static constexpr int OFF_TURN = OFF_SUMS + (QKV ? SUMS_BYTES : 0);
  static constexpr int OFF_BAR = OFF_TURN + (QKV ? EPI4_WARPS * TURN_BYTES : 0);
  static constexpr int OFF_MISC = OFF_BAR + (2 * MAX_STAGES + 2 * MAX_ACCS + 1) * 8;  // full, empty, tfull, tempty, drain
  static constexpr int smem(int stages) { return stages * STAGE_BYTES + OFF_MISC + 16 + 1024; }
  static_assert(STAGE_BYTES % 1024 == 0 && OFF_SF % 1024 == 0, "swizzled tiles start on 1024 bytes");
};

static_assert(Layout<true, false>::smem(MAX_STAGES) <= 232448 && Layout<true, true>::smem(MAX_STAGES) <= 232448 &&
                  Layout<false, false>::smem(FEW_STAGES) <= 232448 && Layout<false, true>::smem(FEW_STAGES) <= 232448,
              "shared memory budget");

// TMEM columns of a stage's scales: four for each tile of A's and of the weight's.
constexpr int scale_cols(int groups, int w_tiles) { return 4 * groups * (1 + w_tiles); }
static_assert(2 * 192 + 2 * scale_cols(4, 2) <= TMEM_COLS, "TMEM columns");
static_assert(MAX_ACCS * 64 + MAX_STAGES * scale_cols(4, 1) <= TMEM_COLS && MAX_ACCS == WAYS,
              "tiles of one unit have as many accumulators as warps that take them in turn");

struct Params4 : Params {
  int32_t e8m0;                      // format
  int32_t groups;                    // scale tiles of a stage: 4 (e4m3) or 2 (e8m0)
  int32_t w_tiles;                   // scale tiles of a tile's weight rows: 1 or 2
  int32_t sf_cols, sf_bufs;          // TMEM columns of a stage's scales, buffers of them
  int32_t units, accs;               // of 64 columns in a tile; accumulators
  int32_t stages;                    // of the ring
  int32_t ahead;                     // stages of weights asked for before the kernel before this one has ended
  int32_t n[3], k[3], kb[3], nt[3];  // by segment: N, K, stages of a tile, column tiles
  int32_t rounds, light;             // Tiles
  uint32_t stage_tx;                 // bytes of a stage that one CTA loads
  int32_t wide[3];                   // rows of the epilogue's tensors start on 32 bytes
  CUtensorMap tm_sa[3], tm_sw[3];
};

// Instruction descriptor, kind::mxf4nvf4: e2m1 operands, fp32 sums, K = 64; scales e4m3
// (one for 16 of K) or e8m0 (for 32).
__device__ __forceinline__ uint32_t idesc_mx4(int M, int N, int e8m0) {
  return (1u << 7) | (1u << 10) | (uint32_t(N >> 3) << 17) | (uint32_t(e8m0) << 23) | (uint32_t(M >> 4) << 24);
}

// A stage's scales to TMEM columns sf.., then its MMAs (ksteps of 64, 1 to 4) and the commit that
// frees the stage, by one thread of a converged warp. One asm block, whose operands are the same
// in every lane and whose addresses are the first ones plus immediates (in units of 16 bytes;
// below the descriptors' 14 bits of address): issued one by one from a single lane, with descriptors
// made for each, 12 copies and 4 MMAs took 1.3 us, five times what they need. lo: the stage's shared
// address / 16; sw: columns of the weight's scales (behind A's, and behind the rows of their
// first tile that lie before the tile's first weight row).
#define RA_CP(GROUP, COL, UNITS)                                                                             \
  "add.u32 c, %1, " COL ";\n\tadd.u32 l, %2, " UNITS ";\n\tmov.b64 s, {l, %10};\n\t"                         \
  "@e tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [c], s;\n\t"
#define RA_MMA(GROUP, VEC, K, A_UNITS, IDESC, SA_COL, SW_COL, ACC)                                           \
  "setp.gt.and.s32 q, %5, " K ", e;\n\t"                                                                     \
  "add.u32 l, %2, " A_UNITS ";\n\tmov.b64 s, {l, %9};\n\t"                                                   \
  "add.u32 l, %7, " A_UNITS ";\n\tmov.b64 t, {l, %9};\n\t"                                                   \
  "add.u32 c, %1, " SA_COL ";\n\tadd.u32 w, %8, " SW_COL ";\n\t"                                             \
  "@q tcgen05.mma.cta_group::" GROUP ".kind::mxf4nvf4.block_scale.scale_vec::" VEC " [%0], s, t, " IDESC     \
  ", [c], [w], " ACC ";\n\t"
#define RA_STAGE(COPIES, MMAS, COMMIT)                                                                       \
  asm volatile(                                                                                              \
      "{\n\t.reg .pred e, p, q, o;\n\t.reg .b64 s, t;\n\t.reg .b32 c, w, i, l;\n\t"                         \
      "elect.sync _|e, 0xffffffff;\n\t"                                                                      \
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 o, %4, %4;\n\tor.b32 i, %3, 0x40000020;\n\t" COPIES MMAS COMMIT "}" ::"r"(d), \
      "r"(sf), "r"(lo), "r"(idesc), "r"(acc), "r"(ksteps), "r"(bar), "r"(lo + L::OFF_B / 16), "r"(sw),           \
      "r"(HI_SW128), "r"(HI_SCALES)                                                                          \
      : "memory")
// Scale tiles of a stage: e4m3 four for 64 of K each, e8m0 two for 128 each, whose halves the
// descriptor selects (bits 4-5 and 30-31). Columns: A's tiles, four each, then for every one of
// them the weight's, four or eight. The scales' units are counted from the stage on.
#define RA_COPIES_E4M3(GROUP, A0, A1, A2, A3, W0, W1, W2, W3)                                                \
  RA_CP(GROUP, "0", A0) RA_CP(GROUP, "16", W0) RA_CP(GROUP, "4", A1) RA_CP(GROUP, "20", W1)                    \
  RA_CP(GROUP, "8", A2) RA_CP(GROUP, "24", W2) RA_CP(GROUP, "12", A3) RA_CP(GROUP, "28", W3)
#define RA_COPIES_E4M3_2(GROUP, A0, A1, A2, A3, W0, W1, W2, W3, X0, X1, X2, X3)                              \
  RA_CP(GROUP, "0", A0) RA_CP(GROUP, "16", W0) RA_CP(GROUP, "20", X0) RA_CP(GROUP, "4", A1)                    \
  RA_CP(GROUP, "24", W1) RA_CP(GROUP, "28", X1) RA_CP(GROUP, "8", A2) RA_CP(GROUP, "32", W2)                   \
  RA_CP(GROUP, "36", X2) RA_CP(GROUP, "12", A3) RA_CP(GROUP, "40", W3) RA_CP(GROUP, "44", X3)
#define RA_COPIES_E8M0(GROUP, A0, A1, W0, W1)                                                                \
  RA_CP(GROUP, "0", A0) RA_CP(GROUP, "8", W0) RA_CP(GROUP, "4", A1) RA_CP(GROUP, "12", W1)
#define RA_COPIES_E8M0_2(GROUP, A0, A1, W0, W1, X0, X1)                                                      \
  RA_CP(GROUP, "0", A0) RA_CP(GROUP, "8", W0) RA_CP(GROUP, "12", X0) RA_CP(GROUP, "4", A1)                     \
  RA_CP(GROUP, "16", W1) RA_CP(GROUP, "20", X1)
#define RA_MMAS_E4M3(GROUP)                                                                                  \
  RA_MMA(GROUP, "4X", "0", "0", "%3", "0", "0", "p") RA_MMA(GROUP, "4X", "1", "2", "%3", "4", "4", "o")          \
  RA_MMA(GROUP, "4X", "2", "4", "%3", "8", "8", "o") RA_MMA(GROUP, "4X", "3", "6", "%3", "12", "12", "o")
#define RA_MMAS_E4M3_2(GROUP)                                                                                \
  RA_MMA(GROUP, "4X", "0", "0", "%3", "0", "0", "p") RA_MMA(GROUP, "4X", "1", "2", "%3", "4", "8", "o")          \
  RA_MMA(GROUP, "4X", "2", "4", "%3", "8", "16", "o") RA_MMA(GROUP, "4X", "3", "6", "%3", "12", "24", "o")
#define RA_MMAS_E8M0(GROUP)                                                                                  \
  RA_MMA(GROUP, "2X", "0", "0", "%3", "0", "0", "p") RA_MMA(GROUP, "2X", "1", "2", "i", "0", "0", "o")           \
  RA_MMA(GROUP, "2X", "2", "4", "%3", "4", "4", "o") RA_MMA(GROUP, "2X", "3", "6", "i", "4", "4", "o")
#define RA_MMAS_E8M0_2(GROUP)                                                                                \
  RA_MMA(GROUP, "2X", "0", "0", "%3", "0", "0", "p") RA_MMA(GROUP, "2X", "1", "2", "i", "0", "0", "o")           \
  RA_MMA(GROUP, "2X", "2", "4", "%3", "4", "8", "o") RA_MMA(GROUP, "2X", "3", "6", "i", "4", "8", "o")
#define RA_COMMIT_2                                                                                          \
  "mov.b32 c, 3;\n\t.reg .b16 m;\n\tcvt.u16.u32 m, c;\n\t"                                                  \
  "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%6], m;\n\t"
#define RA_COMMIT_1 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%6];\n\t"
// Units of the scales within a stage, as immediates: wide pairs, pairs, single CTAs.
#define RA_U3(N) RA_STR(1792 + N)
#define RA_U2(N) RA_STR(1536 + N)
#define RA_U1(N) RA_STR(2048 + N)
#define RA_STR(N) RA_STR2(N)
#define RA_STR2(N) #N
static_assert(Layout<true, false>::OFF_SF / 16 == 1792 && Layout<true, true>::OFF_SF / 16 == 1536 &&
                  Layout<false, false>::OFF_SF / 16 == 2048, "immediates of the copies");
template <class L, bool E8M0>
__device__ __forceinline__ void issue_stage(const Params4& p, uint32_t lo, uint32_t sf, uint32_t sw, uint32_t d,
                                            uint32_t idesc, int ksteps, bool first, uint32_t bar) {
  constexpr uint32_t HI_SW128 = (1024u >> 4) | (1u << 14) | (2u << 29);  // 8 rows after 1024 bytes; version; swizzle
  constexpr uint32_t HI_SCALES = 8u | (1u << 14);                        // 8 rows after 128 bytes; version
  const uint32_t acc = first ? 0u : 1u;
#define RA_ONE(GROUP, U, COMMIT)                                                                                 \
  if constexpr (E8M0)                                                                                            \
    RA_STAGE(RA_COPIES_E8M0(GROUP, U(0), U(32), U(128), U(160)), RA_MMAS_E8M0(GROUP), COMMIT);                   \
  else                                                                                                           \
    RA_STAGE(RA_COPIES_E4M3(GROUP, U(0), U(32), U(64), U(96), U(128), U(160), U(192), U(224)), RA_MMAS_E4M3(GROUP), \
             COMMIT)
  if constexpr (!L::PAIR) {
    RA_ONE("1", RA_U1, RA_COMMIT_1);
  } else if constexpr (L::MAX_BN == 128) {
    RA_ONE("2", RA_U2, RA_COMMIT_2);
  } else if (p.w_tiles == 1) {
    RA_ONE("2", RA_U3, RA_COMMIT_2);
  } else if constexpr (E8M0) {
    RA_STAGE(RA_COPIES_E8M0_2("2", RA_U3(0), RA_U3(32), RA_U3(128), RA_U3(160), RA_U3(192), RA_U3(224)),
             RA_MMAS_E8M0_2("2"), RA_COMMIT_2);
  } else {
    RA_STAGE(RA_COPIES_E4M3_2("2", RA_U3(0), RA_U3(32), RA_U3(64), RA_U3(96), RA_U3(128), RA_U3(160), RA_U3(192),
                              RA_U3(224), RA_U3(256), RA_U3(288), RA_U3(320), RA_U3(352)),
             RA_MMAS_E4M3_2("2"), RA_COMMIT_2);
  }
#undef RA_ONE
}
#undef RA_CP
#undef RA_MMA
#undef RA_STAGE

// umma_commit and umma_commit_pair by one thread of a converged warp (the one that elect.sync
// names is the same every time, so the commits cover what it issued).
template <bool PAIR>
__device__ __forceinline__ void commit_one(uint64_t* bar) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(
            smem_u32(bar)),
        "h"(uint16_t(3))
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
        : "memory");
}

__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(one));
  return one != 0;
}
// A converged warp's wait. False if it was given up.
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const WaitCtl& ctl) {
  return __all_sync(0xffffffffu, CLUSTER ? mbar_wait_cluster(bar, parity, ctl) : mbar_wait(bar, parity, ctl));
}
// Arrival on an mbarrier of another CTA of the cluster by a thread that publishes no memory with
// it (its TMEM loads have ended): with release it waits for the thread's stores, about 0.5 us.
__device__ __forceinline__ void mbar_arrive_remote_relaxed(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Has the phase completed? Asked before the work in front of it is issued, so that the answer's
// latency (50 ns) passes meanwhile. CLUSTER: what arrives may come from the other CTA of the pair.
template <bool CLUSTER = false>
__device__ __forceinline__ uint32_t peek(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  if constexpr (CLUSTER)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
  return ok;
}
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint32_t peeked, uint64_t* bar, uint32_t parity, const WaitCtl& ctl) {
  return __all_sync(0xffffffffu, peeked != 0) || warp_wait<CLUSTER>(bar, parity, ctl);
}
// A value that is the same in every lane, known to be so.
__device__ __forceinline__ int same(int v) { return __shfl_sync(0xffffffffu, v, 0); }
// Walk's order of the tiles (gemm_body.cuh) by counting on from the tile before, without
// divisions but in the last band: the issuer, whose stages take about as long to issue as their
// MMAs run, spent 0.6 us a tile on those.
// Two products in one launch are two segments, the one of the longer K first: where its tiles leave some CTAs
// one more than others, these (the first `light`) take no tile after `rounds` rounds of all, which
// is about when the others have taken their share of the rest.
template <int TM, int EPI>
struct Tiles {
  int g = 0, s = 0, cols = -1;  // the piece: a segment's sample, and its column tiles
  int band = 0;                 // first row tile of the band of GROUP_M
  uint32_t idx = 0;             // the tile's number within the band
  int taken = 0;
  __device__ __forceinline__ int piece_cols(const Params4& p) const {
    if (p.m_tiles[g] == 0) return 0;
    if (!p.gated[g]) return p.nt[g];
    Walk<TM, EPI> w;
    w.g = g;
    w.s = s;
    return w.piece_cols(p);
  }
  // The next tile of the CTA (or pair) t0 of `step`; false past the last one.
  __device__ __forceinline__ bool on(const Params4& p, uint32_t t0, uint32_t step, Tile& r) {
    if (cols < 0) cols = piece_cols(p);
    if (taken >= p.rounds && t0 < uint32_t(p.light)) return false;
    idx += taken == 0 ? t0 : taken < p.rounds ? step : step - uint32_t(p.light);
    ++taken;
    uint32_t rows = uint32_t(min(GROUP_M, p.m_tiles[g] - band));
    while (idx >= rows * uint32_t(cols)) {
      idx -= rows * uint32_t(cols);
      band += GROUP_M;
      if (cols == 0 || band >= p.m_tiles[g]) {
        band = 0;
        if (++s == p.B) {
          s = 0;
          if (++g == p.n_seg) return false;
        }
        cols = piece_cols(p);
      }
      rows = uint32_t(min(GROUP_M, p.m_tiles[g] - band));
    }
    const uint32_t n = rows == GROUP_M ? idx / GROUP_M : idx / rows;
    r.seg = g;
    r.s = s;
    r.m0 = (band + int(idx - n * rows)) * TM;
    r.n0 = int(n) * p.bn;
    return true;
  }
};
// The same for a converged warp, whose values are then known to be the same in every lane.
template <int TM, int EPI>
__device__ __forceinline__ bool warp_tile(const Params4& p, Tiles<TM, EPI>& tiles, uint32_t t0, uint32_t step,
                                          Tile& tl) {
  Tile r{0, 0, 0, 0};
  const int more = same(tiles.on(p, t0, step, r));
  tl = Tile{same(r.seg), same(r.s), same(r.m0), same(r.n0)};
  return more != 0;
}
// tma_load_4d and tma_load_4d_pair by one thread of a converged warp.
template <bool PAIR>
__device__ __forceinline__ void tma_load_one(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1,
                                             int32_t c2, int32_t c3) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
        : "memory");
}

// A tile to L2, by one thread of a converged warp.
__device__ __forceinline__ void tma_prefetch_one(const void* tmap, int32_t c0, int32_t c1, int32_t c2, int32_t c3) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];\n\t}" ::"l"(
          reinterpret_cast<uint64_t>(tmap)),
      "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}

// A stage of the ring and the parity of its barriers' next phase.
struct Ring {
  int st = 0;
  uint32_t ph = 0;
  __device__ __forceinline__ void next(const Params4& p) {
    if (++st == p.stages) {
      st = 0;
      ph ^= 1;
    }
  }
};

// The buffers of scales in TMEM, one for a stage's MMAs after another. A buffer is written
// again once the MMAs that read it, sf_bufs stages ago, have ended. As many buffers as
// stages: the stage itself was filled again after that.
struct Scales {
  Ring old;  // the stage whose MMAs read the buffer last
  int col = 0, end, wait;
  __device__ __forceinline__ explicit Scales(const Params4& p)
      : end(p.sf_cols * p.sf_bufs), wait(p.sf_bufs < p.stages ? p.sf_bufs : -1) {}
  __device__ __forceinline__ bool free(uint64_t* empty, const WaitCtl& ctl) const {
    if (wait != 0) return true;
    // it is about to be: a warp that polls goes on sooner than one that is woken (e4m3 pairs, two buffers:
    // 249 ns a stage, 264)
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (__all_sync(0xffffffffu, peek(empty + old.st, old.ph) != 0)) return true;
    return warp_wait(empty + old.st, old.ph, ctl);
  }
  __device__ __forceinline__ void next(const Params4& p) {
    col += p.sf_cols;
    if (col == end) col = 0;
    if (wait > 0) --wait;
    else if (wait == 0) old.next(p);
  }
};

// gelu_tanh2 (gemm_body.cuh) with one reciprocal for the two: 1 / d0 = d1 / (d0 d1). The
// exponents stop at 60, which x below -7.5 passes; the factor there is 2^-60, and x counts as
// GELU_END, so that the result is -6.5e-18 down to minus infinity (the formula's is closer to zero; with x itself
// it grew to minus infinity, and took 1 % less: 29.4 us, 29.6, 3858 rows, 1536 -> 6144). The special functions of a
// tile of 192 columns (two a value) take as long as the MMAs of K = 1536.
__device__ __forceinline__ void gelu_tanh2_1(float& x0, float& x1) {
  constexpr float c = -2.f * 0.7978845608028654f * 1.4426950408889634f;
  const uint64_t x = f2_pack(x0, x1);
  float z0, z1;
  f2_unpack(f2_mul(x, f2_fma(f2_mul(x, x), f2_pack(0.044715f * c, 0.044715f * c), f2_pack(c, c))), z0, z1);
  float d0, d1;
  f2_unpack(f2_add(f2_pack(ex2_approx(fminf(z0, 60.f)), ex2_approx(fminf(z1, 60.f))), f2_pack(1.f, 1.f)), d0, d1);
  const float r = rcp_approx(d0 * d1);
  const uint64_t y = f2_pack(max_nan(x0, GELU_END), max_nan(x1, GELU_END));
  f2_unpack(f2_mul(y, f2_mul(f2_pack(d1, d0), f2_pack(r, r))), x0, x1);
}

// 32 bytes of a row between global memory and a thread's registers, each row a thread's; WIDE: 32-byte
// aligned (16 otherwise). No staging buffer, whose traffic would come on top of the stages' (a
// buffer and TMA stores of whole lines: 47 us where this takes 42, 8192 rows, K = 2048, N = 7296). What an
// epilogue touches leaves L2 first: an output that streams through it otherwise takes the
// operands with it, which all CTAs read again and again (49 us; 36 without the stores).
template <bool WIDE>
__device__ __forceinline__ void store32(char* dst, const uint32_t (&v)[8]) {
  if (WIDE) {
    asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst),
                 "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
  } else {
    __stcs(reinterpret_cast<uint4*>(dst), make_uint4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<uint4*>(dst) + 1, make_uint4(v[4], v[5], v[6], v[7]));
  }
}
template <bool WIDE>
__device__ __forceinline__ void load32(const char* src, uint32_t (&v)[8]) {
  if (WIDE) {
    asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "l"(src)
                 : "memory");
  } else {
    const uint4 a = __ldcs(reinterpret_cast<const uint4*>(src)), b = __ldcs(reinterpret_cast<const uint4*>(src) + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
}
// A thread's row of 32 columns, rounded to bf16.
__device__ __forceinline__ void store_row(char* dst, bool wide, const float (&x)[32]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = pack_bf16x2(x[16 * i + 2 * e], x[16 * i + 2 * e + 1]);
    if (wide) store32<true>(dst + 32 * i, v);
    else store32<false>(dst + 32 * i, v);
  }
}

// What an epilogue warp works on: its 32 rows (row0 + lane, nrow of them in the segment), its unit of
// 64 columns, its shared memory and the TMEM address of its lanes in the tile's accumulator.
struct Epi4 {
  int row0, nrow, unit;
  uint8_t* turn;
  float *vec0, *vec1;
  uint32_t acc;
};

// STORE, GELU, RESID. release(): the accumulator has been read.
template <int EPI, class Ready, class Release>
__device__ __forceinline__ bool epilogue_linear4(const Params4& p, const Tile& tl, const Epi4& w, Ready ready,
                                                 Release release) {
  const Seg& sg = p.seg[tl.seg];
  const int lane = threadIdx.x & 31, n0 = tl.n0 + UNIT * w.unit;
  const bool on = w.nrow > 0 && n0 < p.n[tl.seg];  // N is a multiple of 64
  const bool mine = lane < w.nrow, wide = p.wide[tl.seg];
  uint32_t r[2][2][8];
  const char* res = nullptr;
  auto residual = [&](int j) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (wide) load32<true>(res + 64 * j + 32 * i, r[j][i]);
      else load32<false>(res + 64 * j + 32 * i, r[j][i]);
    }
  };
  __syncwarp();  // all lanes, those without a row too, have read the vectors of the warp's tile before
  if (on) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      w.vec0[32 * j + lane] = sg.bias ? sg.bias[n0 + 32 * j + lane] : 0.f;
      if (EPI == RA_EPI_RESID) w.vec1[32 * j + lane] = sg.gate[int64_t(tl.s) * sg.gate_ss + n0 + 32 * j + lane];
    }
    if (EPI == RA_EPI_RESID && mine) {
      res = reinterpret_cast<const char*>(sg.resid + int64_t(tl.s) * sg.res_ss + int64_t(w.row0 + lane) * sg.res_sr + n0);
      residual(0);
      residual(1);
    }
  }
  char* out = reinterpret_cast<char*>(sg.out + int64_t(tl.s) * sg.out_ss + int64_t(w.row0 + lane) * sg.out_sr + n0);
  __syncwarp();
  if (!ready()) return false;
  // RESID: 32 columns at a time, all would not fit the registers (spilled ones go through an L1 that
  // shared memory has left nothing of)
  constexpr int AHEAD = EPI == RA_EPI_RESID ? 1 : 2;
  uint32_t v[AHEAD][32];
  if (on) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) tmem_ld32(w.acc + UNIT * w.unit + 32 * j, v[j]);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) tmem_ld_wait_for(v[j]);
  }
  if (AHEAD == 2 || !on) release();
  if (!on) return true;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float x[32];
    if (AHEAD == 1 && j == 1) {
      tmem_ld_wait_for(v[0]);
      release();
    }
    add_cols<true>(v[j % AHEAD], sg.alpha, w.vec0 + 32 * j, x);
    if (AHEAD == 1 && j == 0) tmem_ld32(w.acc + UNIT * w.unit + 32, v[0]);
    if (EPI == RA_EPI_GELU) {
#pragma unroll
      for (int i = 0; i < 32; i += 2) gelu_tanh2_1(x[i], x[i + 1]);
    } else if (EPI == RA_EPI_RESID) {
      const float4* g4 = reinterpret_cast<const float4*>(w.vec1 + 32 * j);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float4 g = g4[q];
        const uint32_t lo = r[j][q / 4][2 * (q & 3)], hi = r[j][q / 4][2 * (q & 3) + 1];
        x[4 * q] = fmaf(g.x, x[4 * q], __uint_as_float(lo << 16));
        x[4 * q + 1] = fmaf(g.y, x[4 * q + 1], __uint_as_float(lo & 0xFFFF0000u));
        x[4 * q + 2] = fmaf(g.z, x[4 * q + 2], __uint_as_float(hi << 16));
        x[4 * q + 3] = fmaf(g.w, x[4 * q + 3], __uint_as_float(hi & 0xFFFF0000u));
      }
    }
    if (mine) store_row(out + 64 * j, wide, x);
  }
  return true;
}

// True where `ok` is in every thread of the two warps that share a tile's quarter, which both get here.
// Tiles in flight have barriers of their own (turn 0 to 2).
__device__ __forceinline__ bool both(int quarter, int turn, bool ok) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(uint32_t(ok)), "r"(1 + quarter * WAYS + turn), "n"(64)
      : "memory");
  return all != 0;
}

// QKV: sums the squares of its columns, which for heads of 128 meet the other warp's in shared memory;
// then the columns are normalised, turned and stored. `turn`: the tile's number modulo three. Its
// sums are written again three tiles on, by the same warps: that tile's accumulators are
// ready only after both have given this one's back, past their reads of the sums.
template <int D, class Ready, class Release>
__device__ __forceinline__ bool epilogue_qkv4(const Params4& p, const Tile& tl, const Epi4& w, float* sums, int turn,
                                              Ready ready, Release release) {
  const Seg& sg = p.seg[tl.seg];
  const int lane = threadIdx.x & 31, quarter = (threadIdx.x >> 5) & 3;
  const int part = tl.n0 / p.C;                       // 0 q, 1 k, 2 v
  const int c0 = tl.n0 - part * p.C + UNIT * w.unit;  // the unit's first column within the part
  const bool on = w.nrow > 0;
  // RoPE rows of the warp's positions: (cos, sin) of D / 2 pairs, 64 bytes for 16 columns, eight
  // rows an access (a row to a thread, 32 bytes each, took twice the whole tile's time)
  const char* rope = reinterpret_cast<const char*>(p.rope + int64_t(sg.pos_offset + w.row0) * (D / 4)) + 4 * (c0 % D);
  uint4 cs[2][4];
  auto turns = [&](int j) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) rows_fetch(rope + 64 * (2 * j + hf), 4 * D, w.nrow, cs[hf]);
  };
  __syncwarp();  // as in epilogue_linear4
  if (on) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = c0 + 32 * j + lane;
      w.vec0[32 * j + lane] = sg.bias ? sg.bias[part * p.C + c] : 0.f;
      if (part < 2) w.vec1[32 * j + lane] = sg.norm_w[part][c % D];
    }
    if (part < 2) turns(0);
  }
  __syncwarp();
  const bool ok = ready();
  uint32_t v[32];
  if (part < 2 && ok && on) {
    // a first pass over the accumulators for the squares
#pragma unroll 1
    for (int j = 0; j < 2; ++j) {
      float x[32], s0 = 0.f, s1 = 0.f;
      tmem_ld32(w.acc + UNIT * w.unit + 32 * j, v);
      tmem_ld_wait_for(v);
      add_cols<true>(v, sg.alpha, w.vec0 + 32 * j, x);
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        s0 = fmaf(x[i], x[i], s0);
        s1 = fmaf(x[i + 1], x[i + 1], s1);
      }
      sums[(2 * w.unit + j) * 32 + lane] = s0 + s1;
    }
  }
  // Both go on or neither does.
  if (!(D == 128 && part < 2 ? both(quarter, turn, ok) : ok)) return false;
  if (on) {
    float rstd = 1.f;
    if (part < 2) {
      float s = 0.f;
      const int first = D == 128 ? 0 : 2 * w.unit;  // 32 columns of the tile that the head starts with
#pragma unroll
      for (int c = 0; c < D / 32; ++c) s += sums[(first + c) * 32 + lane];
      rstd = rsqrtf(s / float(D) + p.norm_eps);
    }
    char* dst = reinterpret_cast<char*>(sg.dst[part] + tl.s * sg.dst_sb[part] + (c0 / D) * sg.dst_sh[part] +
                                        int64_t(w.row0 + lane) * sg.dst_sn[part] + c0 % D);
#pragma unroll 1
    for (int j = 0; j < 2; ++j) {
      float x[32];
      tmem_ld32(w.acc + UNIT * w.unit + 32 * j, v);
      tmem_ld_wait_for(v);
      if (j == 1) release();
      add_cols<true>(v, sg.alpha, w.vec0 + 32 * j, x);
      if (part < 2) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint4 own[4];
          rows_turn(w.turn, cs[hf], own);
          const float4* w4 = reinterpret_cast<const float4*>(w.vec1 + 32 * j + 16 * hf);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 wv = w4[q];
            const float c0 = __uint_as_float(own[q].x), s0 = __uint_as_float(own[q].y);
            const float c1 = __uint_as_float(own[q].z), s1 = __uint_as_float(own[q].w);
            float* xe = &x[16 * hf + 4 * q];
            const float a0 = xe[0] * rstd * wv.x, a1 = xe[1] * rstd * wv.y;
            const float b0 = xe[2] * rstd * wv.z, b1 = xe[3] * rstd * wv.w;
            xe[0] = a0 * c0 - a1 * s0;
            xe[1] = a0 * s0 + a1 * c0;
            xe[2] = b0 * c1 - b1 * s1;
            xe[3] = b0 * s1 + b1 * c1;
          }
        }
        if (j == 0) turns(1);
      }
      if (lane < w.nrow) store_row(dst + 64 * j, p.wide[tl.seg], x);
    }
  } else {
    release();
  }
  return true;
}

template <int EPI, int D, class Ready, class Release>
__device__ __forceinline__ bool epilogue4(const Params4& p, const Tile& tl, const Epi4& w, float* sums, int turn,
                                          Ready ready, Release release) {
  if constexpr (EPI == RA_EPI_QKV)
    return epilogue_qkv4<D>(p, tl, w, sums + turn * (4 * SUMS), turn, ready, release);
  else
    return epilogue_linear4<EPI>(p, tl, w, ready, release);
}

// One CTA on tiles of 128 rows, or CTA pairs on 256 (as gemm_pair_kernel): each CTA of a pair stages
// its own 128 rows of A with their scales, half of the tile's weight rows, and the scales of all
// of them, which each tensor core wants in its own TMEM; rank 0 issues the copies and MMAs of
// both, commits reach both, and what frees an accumulator arrives at rank 0.
//   warp 0      TMA producer     warp 1      TMEM allocator, MMA issuer (of a pair: rank 0's)
//   warps 2..13 epilogue (quarter = warp % 4, thread = output row = TMEM lane)
template <int EPI, int D, bool E8M0, bool PAIR>
__global__ void __launch_bounds__(THREADS4, 1) gemm4_kernel(const __grid_constant__ Params4 p) {
  using L = Layout<PAIR, EPI == RA_EPI_QKV>;
  constexpr int TM = PAIR ? P_TM : BM, CTAS = PAIR ? 2 : 1;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* rest = smem + p.stages * L::STAGE_BYTES;
  uint64_t* full = reinterpret_cast<uint64_t*>(rest + L::OFF_BAR);
  uint64_t* empty = full + MAX_STAGES;
  uint64_t* tfull = empty + MAX_STAGES;
  uint64_t* tempty = tfull + MAX_ACCS;
  uint64_t* drain = tempty + MAX_ACCS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(rest + L::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(rest + L::OFF_MISC + 4);
  const int warp = same(int(threadIdx.x >> 5)), lane = threadIdx.x & 31;
  const int rank = PAIR ? same(int(cluster_rank())) : 0;
  const uint32_t t0 = blockIdx.x / CTAS, step = gridDim.x / CTAS;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int b = 0; b < MAX_ACCS; ++b) {
      mbar_init(tfull + b, 1);
      mbar_init(tempty + b, uint32_t(CTAS * 4 * p.units));
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    if (PAIR) tmem_alloc_pair(tmem_slot, TMEM_COLS);
    else tmem_alloc(tmem_slot, TMEM_COLS);
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();  // both CTAs' barriers and TMEM exist before any cross-CTA use
  tc_fence_after();
  const uint32_t tmem = uint32_t(same(int(*tmem_slot)));
  const WaitCtl ctl{abort_flag, p.err_word, p.budget_ns};
  pdl_launch();
  if (warp != 0) pdl_wait();

  int64_t loads = 0;    // the producer's: stages whose loads may be on their way
  bool issued = false;  // the issuer's: MMAs may be on their way
  if (warp == 0) {
    // ---------------------------------------------------------------- producer (a converged warp)
    for (int g = 0; g < p.n_seg; ++g)
      if (p.rows[g] > 0) {
        tma_prefetch_desc(&p.tm_a[g]);
        tma_prefetch_desc(&p.tm_w[g]);
        tma_prefetch_desc(&p.tm_sa[g]);
        tma_prefetch_desc(&p.tm_sw[g]);
      }
    if (!p.ahead) pdl_wait();
    const uint32_t full0 = PAIR ? mapa_shared(smem_u32(full), 0) : smem_u32(full);  // a pair's are rank 0's
    Ring in;
    Tiles<TM, EPI> tiles;
    Tile tl;
    bool ok = true;
    while (ok && warp_tile(p, tiles, t0, step, tl)) {
      const int kblocks = same(p.kb[tl.seg]);
      if (p.ahead && loads == 0) {
        // the first tile's weights go to L2 while the kernel before this one runs (if that one writes them, it
        // writes to L2 as well)
        for (int kb = 0; kb < min(kblocks, p.ahead); ++kb) {
          tma_prefetch_one(&p.tm_w[tl.seg], kb * (CHUNK / 4), tl.n0 + rank * (p.bn / 2), 0, 0);
          tma_prefetch_one(&p.tm_sw[tl.seg], 0, kb * p.groups, tl.n0 / 128, 0);
        }
        pdl_wait();
      }
      for (int kb = 0; kb < kblocks; ++kb) {
        if (loads >= p.stages && !(ok = warp_wait(empty + in.st, in.ph ^ 1, ctl))) break;
        const uint32_t stage = smem_u32(smem) + in.st * L::STAGE_BYTES, bar = full0 + 8u * in.st;
        if (rank == 0 && elect_one()) mbar_arrive_expect_tx(full + in.st, CTAS * p.stage_tx);
        __syncwarp();
        tma_load_one<PAIR>(stage, &p.tm_a[tl.seg], bar, kb * (CHUNK / 4), tl.m0 + rank * 128, 0, tl.s);
        tma_load_one<PAIR>(stage + L::OFF_B, &p.tm_w[tl.seg], bar, kb * (CHUNK / 4), tl.n0 + rank * (p.bn / 2), 0, 0);
        tma_load_one<PAIR>(stage + L::OFF_SF, &p.tm_sa[tl.seg], bar, 0, kb * p.groups, tl.m0 / 128 + rank, tl.s);
        tma_load_one<PAIR>(stage + L::OFF_SF + SA_BYTES, &p.tm_sw[tl.seg], bar, 0, kb * p.groups, tl.n0 / 128, 0);
        ++loads;
        in.next(p);
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      // -------------------------------------------------------------- MMA issuer (a converged warp)
      const uint32_t idesc = idesc_mx4(TM, p.bn, E8M0);
      const uint32_t s0 = smem_u32(smem) >> 4, sf0 = tmem + uint32_t(p.accs * p.bn);
      int i = 0, buf = 0;   // tiles so far, the next one's accumulator
      uint32_t ph = 1;      // of its release
      uint32_t freed = 0;   // which was asked for early
      Ring in;              // stages as they are filled
      uint32_t filled = 0;  // asked for early
      Scales sf(p);
      Tiles<TM, EPI> tiles;
      Tile tl;
      bool ok = true;
      while (ok && warp_tile(p, tiles, t0, step, tl)) {
        if (i >= p.accs && !(ok = warp_wait<PAIR>(freed, tempty + buf, ph, ctl))) break;
        const uint32_t sw0 = sf0 + (E8M0 ? 8u : 16u) + (uint32_t(tl.n0 & 64) >> 5);
        const int kblocks = same(p.kb[tl.seg]), steps = same(p.k[tl.seg]) / 64;  // of 64 columns
        for (int kb = 0; kb < kblocks; ++kb) {
          if (!(ok = warp_wait(filled, full + in.st, in.ph, ctl) && sf.free(empty, ctl))) break;
          tc_fence_after();
          Ring next = in;
          next.next(p);
          // the next stage's answer: single CTAs ask before this one is issued (8.0 us, 8.5 after it; 256 rows, K =
          // 8192, N = 2048), pairs, whose stage takes longer, after it (5120 rows: 29.0 us, 30.3 before it)
          if (!PAIR) filled = peek(full + next.st, next.ph);
          issue_stage<L, E8M0>(p, s0 + uint32_t(in.st * (L::STAGE_BYTES / 16)), sf0 + sf.col, sw0 + sf.col,
                               tmem + uint32_t(buf * p.bn), idesc, min(CHUNK / 64, steps - kb * (CHUNK / 64)), kb == 0,
                               smem_u32(empty + in.st));
          if (PAIR) filled = peek(full + next.st, next.ph);
          issued = true;
          in = next;
          sf.next(p);
        }
        if (!ok) break;
        commit_one<PAIR>(tfull + buf);
        ++i;
        if (++buf == p.accs) {
          buf = 0;
          ph ^= 1;
        }
        freed = peek<PAIR>(tempty + buf, ph);
      }
    }
  } else {
    // ---------------------------------------------------------------- epilogue
    const int quarter = warp & 3;
    Epi4 w;
    const int way = (warp - 2) >> 2;
    w.turn = rest + L::OFF_TURN + (warp - 2) * TURN_BYTES;
    w.vec0 = reinterpret_cast<float*>(rest + (warp - 2) * VEC_BYTES);
    w.vec1 = w.vec0 + UNIT;
    float* sums = reinterpret_cast<float*>(rest + L::OFF_SUMS) + quarter * SUMS;
    const uint32_t tempty0 = PAIR ? mapa_shared(smem_u32(tempty), 0) : 0u;
    int turn = 0;    // the tile's number modulo three
    int unit = way;  // the tile's unit whose turn is this warp's; behind the last one: none
    int buf = 0;     // the tile's accumulator
    uint32_t ph = 0;
    bool ok = true;
    Tiles<TM, EPI> tiles;
    Tile tl;
    // The phase before the one that a warp waits for has ended: with two units to a tile it has taken one
    // of the two tiles before; with one it takes every third tile, whose accumulator is always the same.
    while (tiles.on(p, t0, step, tl)) {
      if (unit < p.units) {
        w.unit = unit;
        w.row0 = tl.m0 + rank * 128 + quarter * 32;
        w.nrow = min(32, p.rows[tl.seg] - w.row0);
        w.acc = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(buf * p.bn);
        ok = epilogue4<EPI, D>(
            p, tl, w, sums, turn,
            [&] {
              const bool there = ok && __all_sync(0xffffffffu, mbar_wait(tfull + buf, ph, ctl));
              tc_fence_after();
              return there;
            },
            [&] {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) {
                if (rank == 0) mbar_arrive(tempty + buf);
                else mbar_arrive_remote_relaxed(tempty0 + 8u * buf);
              }
            });
        // Where two warps meet at a barrier, one that gave up comes there for all its tiles: the other one
        // would wait for ever.
        if (!ok && !(EPI == RA_EPI_QKV && D == 128)) break;
      }
      unit -= p.units;
      if (unit < 0) unit += WAYS;
      if (++turn == WAYS) turn = 0;
      if (++buf == p.accs) {
        buf = 0;
        ph ^= 1;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  // No role waits any more, so the flag is final. What a CTA that gave up has on its way lands before
  // its shared memory and TMEM go. (A rank 0 that did not give up has seen every MMA end, and with
  // them the loads of both CTAs.)
  if (*abort_flag) {
    if (warp == 0 && lane == 0 && rank == 0) {
      // a pair's full barriers count both CTAs' bytes of every phase that rank 0 armed
      for (int st = 0; st < p.stages; ++st) {
        const int64_t n_s = (loads > st) ? (loads - st + p.stages - 1) / p.stages : 0;
        if (n_s > 0) mbar_wait_drain(full + st, uint32_t((n_s - 1) & 1), p.budget_ns);
      }
    }
    if (warp == 1 && issued) {
      commit_one<PAIR>(drain);
      mbar_wait_drain(drain, 0, p.budget_ns);
    }
    if (PAIR) pause_ns(kLandNs);  // rank 1's loads, and the commits' arrivals at rank 1
  }
  __syncwarp();
  if (PAIR) cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem, TMEM_COLS);
    else tmem_dealloc(tmem, TMEM_COLS);
  }
}

using Kernel = void (*)(Params4);
struct Kernels {
  Kernel single, pair;
};
template <int EPI, int D, bool E8M0>
Kernels kernels() {
  return {gemm4_kernel<EPI, D, E8M0, false>, gemm4_kernel<EPI, D, E8M0, true>};
}
template <bool E8M0>
Kernels pick(int epi, int d) {
  switch (epi) {
    case RA_EPI_STORE: return kernels<RA_EPI_STORE, 0, E8M0>();
    case RA_EPI_GELU: return kernels<RA_EPI_GELU, 0, E8M0>();
    case RA_EPI_RESID: return kernels<RA_EPI_RESID, 0, E8M0>();
    default: return d == 128 ? kernels<RA_EPI_QKV, 128, E8M0>() : kernels<RA_EPI_QKV, 64, E8M0>();
  }
}

struct Plan {
  bool pair;
  int bn, stages;
  double us;
  int32_t rounds, light;
};

// A cut's times (microseconds) by a model fitted to one, four and nine whole rounds of tiles at K = 256 to
// 4096 of every cut, format and epilogue (rms error 5.5 %): a round takes what its stages or its
// epilogue take, whichever is longer, and some of the other.
double round_us(const ra_gemm4_args& a, bool pair, int bn) {
  const double k = a.K / 1024.0;
  const bool e4m3 = a.format == RA_Q4_E4M3;
  const double epilogue = a.epilogue == RA_EPI_STORE ? 0.0047 : a.epilogue == RA_EPI_RESID ? 0.0116
                          : a.epilogue == RA_EPI_GELU ? 0.0076 : 0.019;  // of a tile, per column
  const double stages = k * (bn == 192 ? (e4m3 ? 1.18 : 1.0)
                                       : (pair ? 0.89 : bn == 128 ? 0.84 : 0.65) * (e4m3 ? 1.086 : 1.0)) + 0.16;
  const double ends = epilogue * bn * (!pair ? 1.0 : a.epilogue == RA_EPI_QKV ? 0.87 : 1.06);
  const double more = stages > ends ? stages : ends, less = stages > ends ? ends : stages;
  return more + 0.49 * less * less / more;
}
int64_t tiles_of(const ra_gemm4_args& a, int g, int tm, int bn) {
  const int64_t rows = a.seg[g].lin.rows;
  return rows > 0 ? int64_t(a.B) * ((rows + tm - 1) / tm) * ((a.N + bn - 1) / bn) : 0;
}

// The cheapest cut. Few tiles: 152 single CTAs of narrow tiles beat 76 pairs, whose set-up takes longer too.
// `then`: a second product in the launch, of a K no longer than the first one's.
Plan make_plan(const ra_gemm4_args& a, const ra_gemm4_args* then, int sms) {
  Plan best{false, 64, FEW_STAGES, 1e30, INT32_MAX, 0};
  for (int pair = 0; pair < 2; ++pair) {
    if ((a.tile_mode == 1 && pair) || (a.tile_mode == 2 && !pair) || (pair && sms < 2)) continue;
    const int tm = pair ? P_TM : BM, slots = pair ? sms / 2 : sms;
    for (int bn = pair && a.epilogue != RA_EPI_QKV ? 192 : 128; bn >= 64; bn -= 64) {
      if (a.epilogue == RA_EPI_QKV && bn % a.d != 0) continue;
      int64_t all = 0, open = 0;  // tiles, and those of segments that are not gated
      for (int g = 0; g < a.n_seg; ++g) {
        const int64_t t = tiles_of(a, g, tm, bn);
        all += t;
        if (!a.seg[g].lin.gated) open += t;
      }
      const double fixed = pair ? 4.0 + 0.0032 * bn : 3.7, round = round_us(a, pair, bn);
      Plan one{pair != 0, bn, FEW_STAGES, fixed, INT32_MAX, 0};
      if (!then) {
        one.us += round * double((all + slots - 1) / slots);
        if (open > 0 && open < all) one.us += fixed + round * double((open + slots - 1) / slots);
      } else {
        const int64_t total = all + tiles_of(*then, 0, tm, bn), ctas = total < slots ? total : slots;
        const double second = round_us(*then, pair, bn);
        // the first `light` CTAs have `most` tiles of the first product, the others one less
        const int64_t most = (all + ctas - 1) / ctas, light = all % ctas, whole = (total + ctas - 1) / ctas;
        const double even = double(most) * round + double(whole - most) * second;
        const int64_t r = int64_t((double(total) - (round / second - 1) * double(ctas - light)) / double(ctas));
        const int64_t rounds = r > most ? r : most, rest = total - rounds * ctas;
        if (light > 0 && rest > 0) {
          const double few = double(most) * round + double(rounds - most) * second;
          const double many = double(most - 1) * round +
                              double(rounds - most + 1 + (rest + ctas - light - 1) / (ctas - light)) * second;
          if ((few > many ? few : many) < even) {
            one.rounds = int32_t(rounds);
            one.light = int32_t(light);
          }
          one.us += one.light ? (few > many ? few : many) : even;
        } else {
          one.us += even;
        }
        // The fewer CTAs, the more of this launch and of the ones around it runs at once (quantisation and
        // both products of 130 rows, 1024 -> 1024: 160 tiles of 64 columns 8.8 us, 80 of 128 7.9).
        one.us += 0.008 * double(ctas * (pair ? 2 : 1));
      }
      if (pair && one.us > LONG_CALL) one.stages = MAX_STAGES;
      if (one.us < best.us) best = one;
    }
  }
  return best;
}

// Scales of one operand as a 4-D tensor map (512 bytes of a tile as 128 words, tiles along
// K, tiles along the rows, samples); boxes of `groups` by `tiles` tiles.
bool encode_scales(CUtensorMap* tm, const void* scales, int K, int rows, int B, int format, int groups, int tiles) {
  const int64_t along = (K + 4 * block_of(format) - 1) / (4 * block_of(format)), down = (rows + 127) / 128;
  return encode_words(tm, scales, 128, along, down, B, 512, 512 * along, 512 * along * down, groups, tiles);
}

ra_status run(const char* who, const ra_gemm4_args& a, cudaStream_t st, bool made, const ra_gemm4_args* then) {
  if (a.B < 1 || a.n_seg < 1 || a.n_seg > 3 || a.K < 64 || a.K % 64 != 0 || a.N < 64 || a.N % 64 != 0) {
    set_error("%s: need B >= 1, 1 <= n_seg <= 3, N and K positive multiples of 64 (B=%d n_seg=%d N=%d K=%d)", who, a.B,
              a.n_seg, a.N, a.K);
    return RA_EINVAL;
  }
  if (a.epilogue < RA_EPI_STORE || a.epilogue > RA_EPI_QKV) {
    set_error("%s: unknown epilogue %d", who, a.epilogue);
    return RA_EINVAL;
  }
  if (a.format != RA_Q4_E4M3 && a.format != RA_Q4_E8M0) {
    set_error("%s: unknown format %d", who, a.format);
    return RA_EINVAL;
  }
  if (a.tile_mode < 0 || a.tile_mode > 2) {
    set_error("%s: tile_mode %d (0 auto, 1 one CTA per tile, 2 CTA pairs)", who, a.tile_mode);
    return RA_EINVAL;
  }
  Params4 p;
  std::memset(static_cast<void*>(&p), 0, sizeof(p));
  p.n_seg = a.n_seg + (then ? 1 : 0);
  p.B = a.B;
  p.mode = a.mode;
  p.err_word = a.err_word;
  p.budget_ns = wait_budget_ns();
  p.norm_eps = a.norm_eps;
  p.e8m0 = a.format == RA_Q4_E8M0;
  p.groups = p.e8m0 ? 2 : 4;
  if (a.epilogue == RA_EPI_QKV) {
    if ((a.d != 64 && a.d != 128) || a.H < 1 || int64_t(3) * a.H * a.d != a.N || (a.H * a.d) % 256 != 0) {
      set_error("%s: QKV needs d in {64, 128}, N = 3 H d and H d a multiple of 256", who);
      return RA_EINVAL;
    }
    if (!a.rope || !aligned16(a.rope) || a.rope_len < 1 || !(a.norm_eps >= 0.f)) {
      set_error("%s: QKV needs a 16-byte aligned rope table, rope_len >= 1 and norm_eps >= 0", who);
      return RA_EINVAL;
    }
    p.C = a.H * a.d;
    p.rope = reinterpret_cast<const float4*>(a.rope);
    p.rope_len = a.rope_len;
  }
  const int sms = num_sms();
  const Plan plan = make_plan(a, then, sms);
  const bool pair = plan.pair;
  const int tm = pair ? P_TM : BM;
  p.bn = plan.bn;
  p.w_tiles = plan.bn > 128 ? 2 : 1;
  p.sf_cols = scale_cols(p.groups, p.w_tiles);
  const bool qkv = a.epilogue == RA_EPI_QKV;
  p.stages = plan.stages;
  p.units = plan.bn / UNIT;
  p.accs = MAX_ACCS * plan.bn + p.stages * p.sf_cols <= TMEM_COLS ? MAX_ACCS : 2;
  p.sf_bufs = (TMEM_COLS - p.accs * plan.bn) / p.sf_cols;
  if (p.sf_bufs > p.stages) p.sf_bufs = p.stages;
  p.stage_tx = A_BYTES + (pair ? plan.bn / 2 : plan.bn) * (CHUNK / 2) + p.groups * 512 * (1 + p.w_tiles);
  p.rounds = plan.rounds;
  p.light = plan.light;
  p.cols = (a.N + plan.bn - 1) / plan.bn;
  p.cols_q = p.C / plan.bn;
  int64_t tiles = 0;
  CallPlaces<9, 24> places;  // read: three of the call, seven of a segment
  if (a.mode) places.reads(place_of(a.mode, int64_t(a.B) * 4));
  if (a.epilogue == RA_EPI_QKV) places.reads(place_of(a.rope, int64_t(a.rope_len) * a.d * 4));
  if (a.err_word) places.reads(place_of(a.err_word, 4));
  // Segment g: a's, behind them the second product's.
  const auto call_of = [&](int g) -> const ra_gemm4_args& { return g < a.n_seg ? a : *then; };
  const auto seg_of = [&](int g) -> const ra_gemm4_seg& { return g < a.n_seg ? a.seg[g] : then->seg[0]; };
  for (int g = 0; g < p.n_seg; ++g) {
    const ra_gemm_seg& s = seg_of(g).lin;
    const int32_t N = call_of(g).N, K = call_of(g).K;
    p.n[g] = N;
    p.k[g] = K;
    p.kb[g] = (K + CHUNK - 1) / CHUNK;
    p.nt[g] = (N + plan.bn - 1) / plan.bn;
    if (s.rows < 0) {
      set_error("%s: seg %d rows < 0", who, g);
      return RA_EINVAL;
    }
    if (s.gated && !a.mode) {
      set_error("%s: seg %d is gated but mode is NULL", who, g);
      return RA_EINVAL;
    }
    p.rows[g] = s.rows;
    p.m_tiles[g] = int32_t((int64_t(s.rows) + tm - 1) / tm);
    p.gated[g] = s.gated ? 1 : 0;
    if (s.rows == 0) continue;
    const ra_gemm4_seg& q = seg_of(g);
    if (!s.a || !s.w || !q.a_scales || !q.w_scales || !aligned16(s.a) || !aligned16(s.w) || !aligned16(q.a_scales) ||
        !aligned16(q.w_scales) || s.a_stride_r % 16 != 0 || s.a_stride_s % 16 != 0 || s.a_stride_r < K / 2 ||
        s.a_stride_s < 0) {
      set_error("%s: seg %d: codes and scales of A and W must be 16-byte aligned, strides multiples of 16 bytes, "
                "a_stride_r >= K / 2", who, g);
      return RA_EINVAL;
    }
    // 2^128 is no fp32 number: the sums would count infinitely, zeros as NaN
    if (q.a_exponent < -64 || q.a_exponent > 64 || q.w_exponent < -64 || q.w_exponent > 64 ||
        q.a_exponent + q.w_exponent > 127 || (p.e8m0 && (q.a_exponent || q.w_exponent))) {
      set_error("%s: seg %d: exponents need -64 to 64, together at most 127, and 0 for RA_Q4_E8M0 (%d, %d)", who, g,
                q.a_exponent, q.w_exponent);
      return RA_EINVAL;
    }
    if (!fill_epilogue(who, call_of(g), g, s, p.seg[g])) return RA_EINVAL;
    auto on32 = [](const void* ptr, int64_t ss, int64_t sr, int64_t sh = 0) {  // strides in elements of 2 bytes
      return (reinterpret_cast<uintptr_t>(ptr) & 31u) == 0 && ss % 16 == 0 && sr % 16 == 0 && sh % 16 == 0;
    };
    const int e = q.a_exponent + q.w_exponent;
    p.seg[g].alpha = ldexpf(1.f, e);
    const int64_t rows = s.rows, group = 4 * block_of(a.format), spans = (rows + 127) / 128 * ((K + group - 1) / group);
    places.reads(place_of(s.a, K / 2, {a.B, s.a_stride_s}, {rows, s.a_stride_r}));
    places.reads(place_of(q.a_scales, spans * 512 * a.B));
    places.reads(place_of(s.w, int64_t(N) * (K / 2)));
    places.reads(place_of(q.w_scales, int64_t(refadapt_quant4_scales_size(N, K, a.format))));
    if (s.bias) places.reads(place_of(s.bias, int64_t(N) * 4));
    if (a.epilogue == RA_EPI_QKV) {
      places.reads(place_of(s.q_norm, int64_t(a.d) * 4));
      places.reads(place_of(s.k_norm, int64_t(a.d) * 4));
      p.wide[g] = 1;
      for (const ra_seg* o : {&s.q_out, &s.k_out, &s.v_out}) {
        places.writes(place_of(o->ptr, int64_t(a.d) * 2, {a.B, o->stride_b * 2}, {a.H, o->stride_h * 2},
                               {rows, o->stride_n * 2}));
        if ((a.B > 1 && o->stride_b < 1) || (a.H > 1 && o->stride_h < 1) || (rows > 1 && o->stride_n < a.d)) {
          set_error("%s: seg %d: strides of q_out, k_out and v_out must be positive, their rows' at least d", who, g);
          return RA_EINVAL;
        }
        p.wide[g] &= on32(o->ptr, o->stride_b, o->stride_n, o->stride_h);
      }
    } else {
      if (a.B > 1 && s.out_stride_s < 1) {
        set_error("%s: seg %d: out_stride_s must be positive", who, g);
        return RA_EINVAL;
      }
      places.writes(place_of(s.out, int64_t(N) * 2, {a.B, s.out_stride_s * 2}, {rows, s.out_stride_r * 2}));
      p.wide[g] = on32(s.out, s.out_stride_s, s.out_stride_r) &&
                  (a.epilogue != RA_EPI_RESID || on32(s.resid, s.resid_stride_s, s.resid_stride_r));
      if (a.epilogue == RA_EPI_RESID) {
        places.reads(place_of(s.gate, int64_t(N) * 4, {a.B, s.gate_stride_s * 4}));
        if (s.resid != s.out || s.resid_stride_s != s.out_stride_s || s.resid_stride_r != s.out_stride_r)
          places.reads(place_of(s.resid, int64_t(N) * 2, {a.B, s.resid_stride_s * 2}, {rows, s.resid_stride_r * 2}));
      }
    }
    if (int64_t(p.m_tiles[g]) * p.nt[g] > 2147483647) {
      set_error("%s: seg %d: too many rows", who, g);
      return RA_EINVAL;
    }
    tiles += int64_t(a.B) * p.m_tiles[g] * p.nt[g];
  }
  if (places.clash()) {
    set_error("%s: an output overlaps an input, another output or itself", who);
    return RA_EINVAL;
  }
  if (tiles == 0) return RA_OK;
  // Weights of few rows' tiles, which no other CTA asks for; of many rows', a ring full. Not behind gates, which
  // are read after the kernel before.
  p.ahead = made ? 0 : tiles <= 2 * p.cols ? AHEAD_STAGES : p.stages;
  for (int g = 0; g < a.n_seg; ++g)
    if (a.seg[g].lin.gated) p.ahead = 0;
  int64_t single = 0, more = 0;  // segments of one row, of more
  for (int g = 0; g < a.n_seg; ++g) {
    single += a.seg[g].lin.rows == 1;
    more += a.seg[g].lin.rows > 1;
  }
  if (!then && a.B == 1 && more == 0 && !qkv && a.tile_mode == 0 && a.K <= MAX_ROW_K && single * a.N <= int64_t(sms) * 64)
    return run_row(who, a, st);
  for (int g = 0; g < p.n_seg; ++g) {
    const ra_gemm4_seg& q = seg_of(g);
    const ra_gemm_seg& s = q.lin;
    if (s.rows == 0) continue;
    // Two bytes of codes as one element: a box of 64 is 128 bytes, 256 columns.
    ra_seg as{const_cast<void*>(s.a), s.a_stride_s / 2, 0, s.a_stride_r / 2, s.rows, 0};
    ra_seg ws{const_cast<void*>(s.w), 0, 0, p.k[g] / 4, p.n[g], 0};
    if (!encode_seg(&p.tm_a[g], as, a.B, 1, p.k[g] / 4, CHUNK / 4, BM, true) ||
        !encode_seg(&p.tm_w[g], ws, 1, 1, p.k[g] / 4, CHUNK / 4, pair ? plan.bn / 2 : plan.bn, true) ||
        !encode_scales(&p.tm_sa[g], q.a_scales, p.k[g], s.rows, a.B, a.format, p.groups, 1) ||
        !encode_scales(&p.tm_sw[g], q.w_scales, p.k[g], p.n[g], 1, a.format, p.groups, p.w_tiles))
      return RA_EINVAL;
  }
  const Kernels kn = p.e8m0 ? pick<true>(a.epilogue, a.d) : pick<false>(a.epilogue, a.d);
  const int64_t slots = pair ? (sms / 2 > 0 ? sms / 2 : 1) : sms;
  note_launch(pair ? (then ? "two products, CTA pairs, %d columns" : "CTA pairs, %d columns")
                   : (then ? "two products, single CTAs, %d columns" : "single CTAs, %d columns"), plan.bn);
  const auto smem = [&](int stages) {
    return pair ? (qkv ? Layout<true, true>::smem(stages) : Layout<true, false>::smem(stages))
                : (qkv ? Layout<false, true>::smem(stages) : Layout<false, false>::smem(stages));
  };
  const int64_t groups = tiles < slots ? tiles : slots;
  return launch(who, p, pair ? kn.pair : kn.single, smem(p.stages), pair ? 2 * groups : groups, pair ? 2 : 1, st, THREADS4,
                smem(pair ? MAX_STAGES : FEW_STAGES));
}

// Two products of one segment each in one launch, if that takes less than one after the other (the second
// one's first loads come while the first one ends).
ra_status run_two(const char* who, const ra_gemm4_args& a, const ra_gemm4_args& b, cudaStream_t st, bool made) {
  const int sms = num_sms();
  const ra_gemm4_args &first = a.K >= b.K ? a : b, &then = a.K >= b.K ? b : a;
  if (make_plan(first, &then, sms).us < make_plan(a, nullptr, sms).us + make_plan(b, nullptr, sms).us - 1)
    return run(who, first, st, made, &then);
  const ra_status r = run(who, a, st, made);
  return r != RA_OK ? r : run(who, b, st, made);
}

}  // namespace gemm4
}  // namespace ra

extern "C" ra_status refadapt_gemm4(const ra_gemm4_args* a, void* stream) {
  using namespace ra;
  clear_error();
  if (!a) {
    set_error("refadapt_gemm4: args is NULL");
    return RA_EINVAL;
  }
  return gemm4::run("refadapt_gemm4", *a, static_cast<cudaStream_t>(stream), false);
}
