// refadapt_gemm4: the linear layers of refadapt_gemm with operands of 4 bits and a scale
// for every few columns,
//   D[r, n] = sum over blocks b of  sa[r, b] sw[n, b]  sum over k in b of  a[r, k] w[n, k]
// on the tensor cores' block-scaled 4-bit MMAs (tcgen05.mma kind::mxf4nvf4, K = 64),
// which multiply the scales in. Tiles, roles and epilogues are gemm.cu's (gemm_body.cuh);
// what differs is how a K step reaches the tensor core:
//   * A stage holds 256 of K: 128 bytes of codes a row, the swizzled box of 64 bf16, four
//     MMAs; and the rows' scales, whose tiles of 128 rows by 4 blocks (512 bytes) lie in
//     memory as tensor memory wants them, so that a stage's are one TMA box for each operand.
//   * Before a stage's MMAs the issuer has the scales copied to TMEM (tcgen05.cp 32x128b, 32
//     rows by 16 bytes, to every warp's lanes): four columns for 128 rows and four blocks.
//     Two buffers of 48 columns take turns; a buffer is written again once the MMAs that
//     read it have ended (their commit, two stages ago, has arrived).
//   * TMEM holds two accumulators of up to 192 columns and the scales (480 of 512 columns).
//     Tiles of 256 columns would leave either the scales or the second accumulator no room,
//     and an epilogue takes as long as the MMAs of K = 2048.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstring>

#include "gemm_body.cuh"
#include "gemm4.h"
#include "launch_plan.h"

namespace ra {
namespace gemm4 {

using namespace gemm;

constexpr int CHUNK = 256;   // K of a stage
constexpr int MAX_BN = 192;  // columns of a tile
constexpr int A_BYTES = BM * CHUNK / 2;
constexpr int SA_BYTES = 4 * 512;  // scales of 128 rows, up to four tiles (e4m3)
constexpr int SF_BYTES = 3 * SA_BYTES;  // and of up to 256 weight rows

// One CTA a tile, and CTA pairs (each stages half of the tile's weight rows).
template <bool PAIR>
struct Layout {
  static constexpr int B_BYTES = (PAIR ? MAX_BN / 2 : MAX_BN) * CHUNK / 2;
  static constexpr int OFF_B = A_BYTES, OFF_SF = A_BYTES + B_BYTES;
  static constexpr int STAGE_BYTES = OFF_SF + SF_BYTES;
  static constexpr int STAGES = PAIR ? 5 : 4;
  static constexpr int OFF_BAR = STAGES * STAGE_BYTES;
  static constexpr int OFF_MISC = OFF_BAR + (2 * STAGES + 6) * 8;  // full, empty, tfull[2], tempty[2], drain, parts_full
  static constexpr int OFF_EPI = (OFF_MISC + 16 + 127) / 128 * 128;
  static constexpr int SMEM_ALLOC = OFF_EPI + EPI_WARPS * EPI_WARP_BYTES + 1024;
  static_assert(STAGE_BYTES % 1024 == 0 && OFF_SF % 1024 == 0, "swizzled tiles start on 1024 bytes");
  static_assert(SMEM_ALLOC <= 232448, "shared memory budget");
};
// split tiles: the parts to send and those received take the place of the stages
static_assert(2 * (MAX_SPLIT - 1) * (BM * 128 * 4 / MAX_SPLIT) <= Layout<false>::OFF_BAR &&
                  2 * (BM * MAX_BN * 4 / 2) <= Layout<false>::OFF_BAR, "parts fit the stages");

// TMEM columns of a stage's scales: four for each tile of A's and of the weight's.
constexpr int scale_cols(int groups, int w_tiles) { return 4 * groups * (1 + w_tiles); }
static_assert(2 * MAX_BN + 2 * scale_cols(4, 2) <= TMEM_COLS, "TMEM columns");

struct Params4 : Params {
  int32_t e8m0;                      // format
  int32_t groups;                    // scale tiles of a stage: 4 (e4m3) or 2 (e8m0)
  int32_t w_tiles;                   // scale tiles of a tile's weight rows: 1 or 2
  int32_t sf_cols, sf_bufs;          // TMEM columns of a stage's scales, buffers of them
  uint32_t stage_tx;                 // bytes of a stage that one CTA loads
  CUtensorMap tm_sa[3], tm_sw[3];
};

// Instruction descriptor, kind::mxf4nvf4: e2m1 operands, fp32 sums, K = 64; scales e4m3
// (one for 16 of K) or e8m0 (for 32).
__device__ __forceinline__ uint32_t idesc_mx4(int M, int N, int e8m0) {
  return (1u << 7) | (1u << 10) | (uint32_t(N >> 3) << 17) | (uint32_t(e8m0) << 23) | (uint32_t(M >> 4) << 24);
}
// Matrix descriptor of 32 rows of 16 bytes, 8 rows (128 bytes) after 8 rows, no swizzle.
__device__ __forceinline__ uint64_t sdesc_scales(uint32_t saddr) {
  return uint64_t((saddr >> 4) & 0x3FFFu) | (uint64_t(8) << 16) | (uint64_t(8) << 32) | (uint64_t(1) << 46);
}

// A stage's scales to TMEM columns sf.., then its MMAs (ksteps of 64, 1 to 4), by one thread of a
// converged warp. One asm block, whose operands are the same in every lane and whose
// addresses are the first ones plus immediates (tiles start on 1024 bytes, so that the sums never
// carry out of a descriptor's address field): issued one by one from a single lane, with
// descriptors made for each, 12 copies and 4 MMAs took 1.3 us, six times what the tensor core
// needs for them. half_cols: columns by which the tile's first weight row lies inside a scale tile.
#define RA_CP(GROUP, COL, DESC, UNITS)                                                                       \
  "add.u32 c, %1, " COL ";\n\tadd.s64 s, " DESC ", " UNITS ";\n\t"                                           \
  "@e tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [c], s;\n\t"
#define RA_MMA(GROUP, VEC, K, UNITS, IDESC, SA_COL, SW_COL, ACC)                                             \
  "setp.gt.and.s32 q, %8, " K ", e;\n\t"                                                                     \
  "add.s64 s, %4, " UNITS ";\n\tadd.s64 t, %5, " UNITS ";\n\tadd.u32 c, %1, " SA_COL ";\n\tadd.u32 w, %9, "  \
  SW_COL ";\n\t"                                                                                             \
  "@q tcgen05.mma.cta_group::" GROUP ".kind::mxf4nvf4.block_scale.scale_vec::" VEC " [%0], s, t, " IDESC     \
  ", [c], [w], " ACC ";\n\t"
#define RA_STAGE(COPIES, MMAS)                                                                   \
  asm volatile(                                                                                              \
      "{\n\t.reg .pred e, p, q, o;\n\t.reg .b64 s, t;\n\t.reg .b32 c, w, i;\n\t"                            \
      "elect.sync _|e, 0xffffffff;\n\t"                                                                      \
      "setp.ne.b32 p, %7, 0;\n\tsetp.eq.b32 o, %7, %7;\n\tor.b32 i, %6, 0x40000020;\n\t" COPIES MMAS "}" ::"r"(d), \
      "r"(sf), "l"(s_a), "l"(s_w), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(ksteps), "r"(sf + half_cols)      \
      : "memory")
// Scale tiles of a stage: e4m3 four for 64 of K each, e8m0 two for 128 each, whose halves the
// descriptor selects (bits 4-5 and 30-31). Columns: A's tiles, four each, then for every one of
// them the weight's, four or eight.
#define RA_COPIES_E4M3(GROUP)                                                                                \
  RA_CP(GROUP, "0", "%2", "0") RA_CP(GROUP, "16", "%3", "0") RA_CP(GROUP, "4", "%2", "32")                     \
  RA_CP(GROUP, "20", "%3", "32") RA_CP(GROUP, "8", "%2", "64") RA_CP(GROUP, "24", "%3", "64")                  \
  RA_CP(GROUP, "12", "%2", "96") RA_CP(GROUP, "28", "%3", "96")
#define RA_COPIES_E4M3_2(GROUP)                                                                              \
  RA_CP(GROUP, "0", "%2", "0") RA_CP(GROUP, "16", "%3", "0") RA_CP(GROUP, "20", "%3", "128")                   \
  RA_CP(GROUP, "4", "%2", "32") RA_CP(GROUP, "24", "%3", "32") RA_CP(GROUP, "28", "%3", "160")                 \
  RA_CP(GROUP, "8", "%2", "64") RA_CP(GROUP, "32", "%3", "64") RA_CP(GROUP, "36", "%3", "192")                 \
  RA_CP(GROUP, "12", "%2", "96") RA_CP(GROUP, "40", "%3", "96") RA_CP(GROUP, "44", "%3", "224")
#define RA_COPIES_E8M0(GROUP)                                                                                \
  RA_CP(GROUP, "0", "%2", "0") RA_CP(GROUP, "8", "%3", "0") RA_CP(GROUP, "4", "%2", "32") RA_CP(GROUP, "12", "%3", "32")
#define RA_COPIES_E8M0_2(GROUP)                                                                              \
  RA_CP(GROUP, "0", "%2", "0") RA_CP(GROUP, "8", "%3", "0") RA_CP(GROUP, "12", "%3", "64")                     \
  RA_CP(GROUP, "4", "%2", "32") RA_CP(GROUP, "16", "%3", "32") RA_CP(GROUP, "20", "%3", "96")
#define RA_MMAS_E4M3(GROUP)                                                                                  \
  RA_MMA(GROUP, "4X", "0", "0", "%6", "0", "16", "p") RA_MMA(GROUP, "4X", "1", "2", "%6", "4", "20", "o")        \
  RA_MMA(GROUP, "4X", "2", "4", "%6", "8", "24", "o") RA_MMA(GROUP, "4X", "3", "6", "%6", "12", "28", "o")
#define RA_MMAS_E4M3_2(GROUP)                                                                                \
  RA_MMA(GROUP, "4X", "0", "0", "%6", "0", "16", "p") RA_MMA(GROUP, "4X", "1", "2", "%6", "4", "24", "o")        \
  RA_MMA(GROUP, "4X", "2", "4", "%6", "8", "32", "o") RA_MMA(GROUP, "4X", "3", "6", "%6", "12", "40", "o")
#define RA_MMAS_E8M0(GROUP)                                                                                  \
  RA_MMA(GROUP, "2X", "0", "0", "%6", "0", "8", "p") RA_MMA(GROUP, "2X", "1", "2", "i", "0", "8", "o")           \
  RA_MMA(GROUP, "2X", "2", "4", "%6", "4", "12", "o") RA_MMA(GROUP, "2X", "3", "6", "i", "4", "12", "o")
#define RA_MMAS_E8M0_2(GROUP)                                                                                \
  RA_MMA(GROUP, "2X", "0", "0", "%6", "0", "8", "p") RA_MMA(GROUP, "2X", "1", "2", "i", "0", "8", "o")           \
  RA_MMA(GROUP, "2X", "2", "4", "%6", "4", "16", "o") RA_MMA(GROUP, "2X", "3", "6", "i", "4", "16", "o")
template <bool PAIR>
__device__ __forceinline__ void issue_stage(const Params4& p, uint32_t stage, uint32_t sf, uint32_t d, uint32_t idesc,
                                            uint32_t half_cols, int ksteps, bool first) {
  using L = Layout<PAIR>;
  const uint64_t a = sdesc_sw128(stage, 16, 1024), b = sdesc_sw128(stage + L::OFF_B, 16, 1024);
  const uint64_t s_a = sdesc_scales(stage + L::OFF_SF), s_w = sdesc_scales(stage + L::OFF_SF + SA_BYTES);
  const uint32_t acc = first ? 0u : 1u;
  if constexpr (PAIR) {
    if (p.e8m0) {
      if (p.w_tiles == 2) RA_STAGE(RA_COPIES_E8M0_2("2"), RA_MMAS_E8M0_2("2"));
      else RA_STAGE(RA_COPIES_E8M0("2"), RA_MMAS_E8M0("2"));
    } else {
      if (p.w_tiles == 2) RA_STAGE(RA_COPIES_E4M3_2("2"), RA_MMAS_E4M3_2("2"));
      else RA_STAGE(RA_COPIES_E4M3("2"), RA_MMAS_E4M3("2"));
    }
  } else {
    if (p.e8m0) {
      if (p.w_tiles == 2) RA_STAGE(RA_COPIES_E8M0_2("1"), RA_MMAS_E8M0_2("1"));
      else RA_STAGE(RA_COPIES_E8M0("1"), RA_MMAS_E8M0("1"));
    } else {
      if (p.w_tiles == 2) RA_STAGE(RA_COPIES_E4M3_2("1"), RA_MMAS_E4M3_2("1"));
      else RA_STAGE(RA_COPIES_E4M3("1"), RA_MMAS_E4M3("1"));
    }
  }
}
#undef RA_CP
#undef RA_MMA
#undef RA_STAGE

// umma_commit and umma_commit_pair by one thread of a converged warp (the one that elect.sync
// names is the same every time, so the commits cover what it issued).
template <bool PAIR>
__device__ __forceinline__ void commit_stage(uint64_t* bar) {
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

__device__ __forceinline__ int ksteps_of(const Params4& p, int kb) { return min(CHUNK, p.K - kb * CHUNK) / 64; }

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
// Has the phase completed? Asked before the work in front of it is issued, so that the answer's
// latency (50 ns) passes meanwhile.
__device__ __forceinline__ uint32_t peek(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok;
}
__device__ __forceinline__ bool warp_wait(uint32_t peeked, uint64_t* bar, uint32_t parity, const WaitCtl& ctl) {
  return __all_sync(0xffffffffu, peeked != 0) || warp_wait(bar, parity, ctl);
}
// A value that is the same in every lane, known to be so.
__device__ __forceinline__ int same(int v) { return __shfl_sync(0xffffffffu, v, 0); }
// Walk's order of the tiles (gemm_body.cuh) by counting on from the tile before, without
// divisions but in the last band: the issuer, whose stages take about as long to issue as their
// MMAs run, spent 0.6 us a tile on those.
template <int TM, int EPI>
struct Tiles {
  int g = 0, s = 0, cols = -1;  // the piece: a segment's sample, and its column tiles
  int band = 0;                 // first row tile of the band of GROUP_M
  uint32_t idx = 0;             // the tile's number within the band
  __device__ __forceinline__ int piece_cols(const Params& p) const {
    if (p.m_tiles[g] == 0) return 0;
    Walk<TM, EPI> w;
    w.g = g;
    w.s = s;
    return w.piece_cols(p);
  }
  // `by` tiles on (the first call: from the first one); false past the last one.
  __device__ __forceinline__ bool on(const Params& p, uint32_t by, Tile& r) {
    if (cols < 0) cols = piece_cols(p);
    idx += by;
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
__device__ __forceinline__ bool warp_tile(const Params& p, Tiles<TM, EPI>& tiles, uint32_t by, Tile& tl) {
  Tile r{0, 0, 0, 0};
  const int more = same(tiles.on(p, by, r));
  tl = Tile{same(r.seg), same(r.s), same(r.m0), same(r.n0)};
  return more != 0;
}
// tma_load_4d and tma_load_4d_pair by one thread of a converged warp.
__device__ __forceinline__ void tma_load_one(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1,
                                             int32_t c2, int32_t c3) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_one_pair(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1,
                                                  int32_t c2, int32_t c3) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
      : "memory");
}

// A stage of the ring and the parity of its barriers' next phase.
template <int STAGES>
struct Ring {
  int st = 0;
  uint32_t ph = 0;
  __device__ __forceinline__ void next() {
    if (++st == STAGES) {
      st = 0;
      ph ^= 1;
    }
  }
};

// The buffers of scales in TMEM, one for a stage's MMAs after another. A buffer is written
// again once the MMAs that read it, sf_bufs stages ago, have ended. As many buffers as
// stages: the stage itself was filled again after that.
template <int STAGES>
struct Scales {
  Ring<STAGES> old;  // the stage whose MMAs read the buffer last
  int col = 0, end, wait;
  __device__ __forceinline__ explicit Scales(const Params4& p)
      : end(p.sf_cols * p.sf_bufs), wait(p.sf_bufs < STAGES ? p.sf_bufs : -1) {}
  __device__ __forceinline__ bool free(uint64_t* empty, const WaitCtl& ctl) const {
    return wait != 0 || warp_wait(empty + old.st, old.ph, ctl);
  }
  __device__ __forceinline__ void next(const Params4& p) {
    col += p.sf_cols;
    if (col == end) col = 0;
    if (wait > 0) --wait;
    else if (wait == 0) old.next();
  }
};

// One CTA a tile of 128 rows. SPLIT: a cluster takes a tile, each rank a contiguous part
// of its K (merge_parts adds them up), then its share of the columns in the epilogue.
template <int EPI, int D, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1) gemm4_kernel(const __grid_constant__ Params4 p) {
  using L = Layout<false>;
  constexpr int STAGES = L::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  uint64_t* full = bars;
  uint64_t* empty = bars + STAGES;
  uint64_t* tfull = bars + 2 * STAGES;
  uint64_t* tempty = bars + 2 * STAGES + 2;
  uint64_t* drain = bars + 2 * STAGES + 4;
  uint64_t* parts_full = bars + 2 * STAGES + 5;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::OFF_MISC + 4);
  volatile int* live = reinterpret_cast<volatile int*>(smem + L::OFF_MISC + 8);
  const int warp = same(int(threadIdx.x >> 5)), lane = threadIdx.x & 31;
  const int rank = SPLIT ? int(cluster_rank()) : 0, cs = SPLIT ? int(cluster_size()) : 1;
  const uint32_t t0 = SPLIT ? blockIdx.x / cs : blockIdx.x, step = SPLIT ? gridDim.x / cs : gridDim.x;
  const int kb0 = SPLIT ? p.kblocks * rank / cs : 0;  // this CTA's stages of K
  const int kb1 = SPLIT ? p.kblocks * (rank + 1) / cs : p.kblocks;
  const int bn = p.bn;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull + b, 1);
      mbar_init(tempty + b, EPI_WARPS);
    }
    mbar_init(drain, 1);
    mbar_init(parts_full, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc(tmem_slot, TMEM_COLS);
  if (SPLIT && warp == 2) {
    pdl_wait();
    Tiles<BM, EPI> tiles;
    Tile tl;
    *live = tiles.on(p, t0, tl);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uint32_t(same(int(*tmem_slot)));
  if (SPLIT && !*live) {  // uniform over the cluster: the modes leave it no tile
    if (warp == 1) tmem_dealloc(tmem, TMEM_COLS);
    return;
  }
  const WaitCtl ctl{abort_flag, p.err_word, p.budget_ns};
  pdl_launch();
  if (warp != 0) pdl_wait();

  int64_t loads = 0;    // the producer's: stages whose loads may be on their way
  bool issued = false;  // the issuer's: MMAs may be on their way
  if (warp == 0) {
    {
      // -------------------------------------------------------------- producer (a converged warp)
      for (int g = 0; g < p.n_seg; ++g)
        if (p.rows[g] > 0) {
          tma_prefetch_desc(&p.tm_a[g]);
          tma_prefetch_desc(&p.tm_w[g]);
          tma_prefetch_desc(&p.tm_sa[g]);
          tma_prefetch_desc(&p.tm_sw[g]);
        }
      pdl_wait();
      Ring<STAGES> in;
      bool ok = true;
      Tiles<BM, EPI> tiles;
      Tile tl;
      for (uint32_t by = t0; ok && warp_tile(p, tiles, by, tl); by = step) {
        for (int kb = kb0; kb < kb1; ++kb) {
          if (loads >= STAGES && !(ok = warp_wait(empty + in.st, in.ph ^ 1, ctl))) break;
          const uint32_t stage = smem_u32(smem) + in.st * L::STAGE_BYTES, bar = smem_u32(full + in.st);
          const bool one = elect_one();
          if (one) mbar_arrive_expect_tx(full + in.st, p.stage_tx);
          __syncwarp();
          tma_load_one(stage, &p.tm_a[tl.seg], bar, kb * (CHUNK / 4), tl.m0, 0, tl.s);
          tma_load_one(stage + L::OFF_B, &p.tm_w[tl.seg], bar, kb * (CHUNK / 4), tl.n0, 0, 0);
          tma_load_one(stage + L::OFF_SF, &p.tm_sa[tl.seg], bar, 0, kb * p.groups, tl.m0 / 128, tl.s);
          tma_load_one(stage + L::OFF_SF + SA_BYTES, &p.tm_sw[tl.seg], bar, 0, kb * p.groups, tl.n0 / 128, 0);
          ++loads;
          in.next();
        }
      }
    }
  } else if (warp == 1) {
    {
      // -------------------------------------------------------------- MMA issuer (a converged warp)
      const uint32_t idesc = idesc_mx4(BM, bn, p.e8m0);
      const uint32_t s0 = smem_u32(smem), sf0 = tmem + uint32_t(2 * bn);
      int i = 0;
      Ring<STAGES> in;  // stages as they are filled
      uint32_t filled = 0;
      Scales<STAGES> sf(p);
      bool ok = true;
      Tiles<BM, EPI> tiles;
      Tile tl;
      for (uint32_t by = t0; ok && warp_tile(p, tiles, by, tl); by = step) {
        const int buf = i & 1, use = i >> 1;
        if (use > 0 && !(ok = warp_wait(tempty + buf, uint32_t((use - 1) & 1), ctl))) break;
        tc_fence_after();
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!(ok = warp_wait(filled, full + in.st, in.ph, ctl) && sf.free(empty, ctl))) break;
          tc_fence_after();
          Ring<STAGES> next = in;
          next.next();
          filled = peek(full + next.st, next.ph);
          issue_stage<false>(p, s0 + in.st * L::STAGE_BYTES, sf0 + sf.col, tmem + uint32_t(buf * bn), idesc,
                             uint32_t(tl.n0 & 64) >> 5, ksteps_of(p, kb), kb == kb0);
          commit_stage<false>(empty + in.st);
          issued = true;
          in = next;
          sf.next(p);
        }
        if (!ok) break;
        commit_stage<false>(tfull + buf);
        ++i;
      }
    }
  } else {
    // ---------------------------------------------------------------- epilogue
    const int quarter = warp & 3;
    EpiWarp w;
    w.half = (warp - 2) >> 2;
    w.stage = smem + L::OFF_EPI + (warp - 2) * EPI_WARP_BYTES;
    w.vec0 = reinterpret_cast<float*>(w.stage + EPI_STAGE_BYTES);
    w.vec1 = w.vec0 + 128;
    int i = 0;
    Tiles<BM, EPI> tiles;
    Tile tl;
    for (uint32_t by = t0; tiles.on(p, by, tl); by = step) {
      const int buf = i & 1, use = i >> 1;
      w.row0 = tl.m0 + quarter * 32;
      w.nrow = min(32, p.rows[tl.seg] - w.row0);
      w.acc = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(buf * bn);
      w.cols = bn;
      const uint32_t acc = w.acc;
      if (SPLIT) {
        w.cols /= cs;
        w.acc += uint32_t(rank * w.cols);
        tl.n0 += rank * w.cols;
      }
      if (!epilogue_tile<EPI, D, true>(p, tl, w, [&] {
            bool ok = __all_sync(0xffffffffu, mbar_wait(tfull + buf, uint32_t(use & 1), ctl));
            tc_fence_after();
            if (SPLIT) ok = merge_parts(ctl, smem, parts_full, acc, ok, bn, w.half, quarter, rank, cs);
            return ok;
          }))
        break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(tempty + buf);
      ++i;
    }
  }
  if (SPLIT) {
    // Warps 0 and 1 meet the epilogue's cluster barrier here. No CTA exits before
    // every part has been read from it and received.
    __syncwarp();
    if (warp < 2) cluster_sync_all();
    cluster_sync_all();
  }
  tc_fence_before();
  __syncthreads();
  // No role waits any more, so the flag is final. What this CTA has on its way lands first.
  if (*abort_flag) {
    if (warp == 0 && lane == 0)
      for (int st = 0; st < STAGES; ++st) {
        const int64_t n_s = (loads > st) ? (loads - st + STAGES - 1) / STAGES : 0;
        if (n_s > 0) mbar_wait_drain(full + st, uint32_t((n_s - 1) & 1), p.budget_ns);
      }
    if (warp == 1 && issued) {
      commit_stage<false>(drain);
      mbar_wait_drain(drain, 0, p.budget_ns);
    }
  }
  __syncwarp();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
  }
}

// CTA pairs on tiles of 256 rows (as gemm_pair_kernel): each CTA stages its own 128 rows of
// A with their scales, half of the tile's weight rows, and the scales of all of them, which
// each tensor core wants in its own TMEM; rank 0 issues the copies and MMAs of both.
template <int EPI, int D>
__global__ void __launch_bounds__(THREADS, 1) gemm4_pair_kernel(const __grid_constant__ Params4 p) {
  using L = Layout<true>;
  constexpr int STAGES = L::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  uint64_t* full = bars;
  uint64_t* empty = bars + STAGES;
  uint64_t* tfull = bars + 2 * STAGES;
  uint64_t* tempty = bars + 2 * STAGES + 2;
  uint64_t* drain = bars + 2 * STAGES + 4;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::OFF_MISC + 4);
  const int warp = same(int(threadIdx.x >> 5)), lane = threadIdx.x & 31;
  const uint32_t rank = uint32_t(same(int(cluster_rank())));
  const uint32_t cid = blockIdx.x >> 1, ncl = gridDim.x >> 1;
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
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc_pair(tmem_slot, TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // both CTAs' barriers and TMEM exist before any cross-CTA use
  tc_fence_after();
  const uint32_t tmem = uint32_t(same(int(*tmem_slot)));
  const WaitCtl ctl{abort_flag, p.err_word, p.budget_ns};
  pdl_launch();
  if (warp != 0) pdl_wait();

  int64_t loads = 0;    // the producer's: stages that it loaded
  bool issued = false;  // the issuer's: it has issued MMAs
  if (warp == 0) {
    {
      // -------------------------------------------------------------- producer (both CTAs, a converged warp)
      for (int g = 0; g < p.n_seg; ++g)
        if (p.rows[g] > 0) {
          tma_prefetch_desc(&p.tm_a[g]);
          tma_prefetch_desc(&p.tm_w[g]);
          tma_prefetch_desc(&p.tm_sa[g]);
          tma_prefetch_desc(&p.tm_sw[g]);
        }
      pdl_wait();
      const uint32_t full0 = mapa_shared(smem_u32(full), 0);  // rank 0's full barriers
      Ring<STAGES> in;
      bool ok = true;
      Tiles<P_TM, EPI> tiles;
      Tile tl;
      for (uint32_t by = cid; ok && warp_tile(p, tiles, by, tl); by = ncl) {
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (loads >= STAGES && !(ok = warp_wait(empty + in.st, in.ph ^ 1, ctl))) break;
          const uint32_t stage = smem_u32(smem) + in.st * L::STAGE_BYTES, bar = full0 + 8u * in.st;
          const bool one = elect_one();
          if (one && rank == 0) mbar_arrive_expect_tx(full + in.st, 2 * p.stage_tx);
          __syncwarp();
          tma_load_one_pair(stage, &p.tm_a[tl.seg], bar, kb * (CHUNK / 4), tl.m0 + int(rank) * 128, 0, tl.s);
          tma_load_one_pair(stage + L::OFF_B, &p.tm_w[tl.seg], bar, kb * (CHUNK / 4), tl.n0 + int(rank) * (p.bn / 2), 0,
                           0);
          tma_load_one_pair(stage + L::OFF_SF, &p.tm_sa[tl.seg], bar, 0, kb * p.groups, tl.m0 / 128 + int(rank), tl.s);
          tma_load_one_pair(stage + L::OFF_SF + SA_BYTES, &p.tm_sw[tl.seg], bar, 0, kb * p.groups, tl.n0 / 128, 0);
          ++loads;
          in.next();
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      // -------------------------------------------------------------- MMA issuer (rank 0, a converged warp)
      const uint32_t idesc = idesc_mx4(P_TM, p.bn, p.e8m0);
      const uint32_t s0 = smem_u32(smem), sf0 = tmem + uint32_t(2 * p.bn);
      int i = 0;
      Ring<STAGES> in;  // stages as they are filled
      uint32_t filled = 0;
      Scales<STAGES> sf(p);
      bool ok = true;
      Tiles<P_TM, EPI> tiles;
      Tile tl;
      for (uint32_t by = cid; ok && warp_tile(p, tiles, by, tl); by = ncl) {
        const int buf = i & 1, use = i >> 1;
        if (use > 0 && !(ok = warp_wait<true>(tempty + buf, uint32_t((use - 1) & 1), ctl))) break;
        tc_fence_after();
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (!(ok = warp_wait(filled, full + in.st, in.ph, ctl) && sf.free(empty, ctl))) break;
          tc_fence_after();
          Ring<STAGES> next = in;
          next.next();
          filled = peek(full + next.st, next.ph);
          issue_stage<true>(p, s0 + in.st * L::STAGE_BYTES, sf0 + sf.col, tmem + uint32_t(buf * p.bn), idesc,
                            uint32_t(tl.n0 & 64) >> 5, ksteps_of(p, kb), kb == 0);
          commit_stage<true>(empty + in.st);
          issued = true;
          in = next;
          sf.next(p);
        }
        if (!ok) break;
        commit_stage<true>(tfull + buf);
        ++i;
      }
    }
  } else {
    // ---------------------------------------------------------------- epilogue (both CTAs)
    const int quarter = warp & 3;
    EpiWarp w;
    w.half = (warp - 2) >> 2;
    w.stage = smem + L::OFF_EPI + (warp - 2) * EPI_WARP_BYTES;
    w.vec0 = reinterpret_cast<float*>(w.stage + EPI_STAGE_BYTES);
    w.vec1 = w.vec0 + 128;
    const uint32_t tempty0 = mapa_shared(smem_u32(tempty), 0);
    int i = 0;
    Tiles<P_TM, EPI> tiles;
    Tile tl;
    for (uint32_t by = cid; tiles.on(p, by, tl); by = ncl) {
      const int buf = i & 1, use = i >> 1;
      w.row0 = tl.m0 + int(rank) * 128 + quarter * 32;
      w.cols = p.bn;
      w.nrow = min(32, p.rows[tl.seg] - w.row0);
      w.acc = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(buf * p.bn);
      if (!epilogue_tile<EPI, D, true>(p, tl, w, [&] {
            const bool ok = __all_sync(0xffffffffu, mbar_wait(tfull + buf, uint32_t(use & 1), ctl));
            tc_fence_after();
            return ok;
          }))
        break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (rank == 0)
          mbar_arrive(tempty + buf);
        else
          mbar_arrive_remote(tempty0 + 8u * buf);
      }
      ++i;
    }
  }
  tc_fence_before();
  __syncthreads();
  // No role waits any more, so the flag is final. What a CTA that gave up has on its way
  // lands before the pair's shared memory and TMEM go. (A rank 0 that did not give up has
  // seen every MMA end, and with them the loads of both CTAs.)
  if (*abort_flag) {
    if (warp == 0 && lane == 0 && rank == 0) {
      // rank 0's full barriers count both CTAs' bytes of every phase it armed
      for (int st = 0; st < STAGES; ++st) {
        const int64_t n_s = (loads > st) ? (loads - st + STAGES - 1) / STAGES : 0;
        if (n_s > 0) mbar_wait_drain(full + st, uint32_t((n_s - 1) & 1), p.budget_ns);
      }
    }
    if (warp == 1 && issued) {
      // the peer's barrier of this name is not waited for and has its own CTA's life
      commit_stage<true>(drain);
      mbar_wait_drain(drain, 0, p.budget_ns);
    }
    pause_ns(kLandNs);  // rank 1's loads, and the commits' arrivals at rank 1
  }
  __syncwarp();
  cluster_sync_all();
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem, TMEM_COLS);
}

using Kernel = void (*)(Params4);
struct Kernels {
  Kernel single, pair, split;  // split: STORE, GELU and RESID
};
template <int EPI, int D>
Kernels kernels() {
  if constexpr (EPI == RA_EPI_QKV)
    return {gemm4_kernel<EPI, D, false>, gemm4_pair_kernel<EPI, D>, nullptr};
  else
    return {gemm4_kernel<EPI, D, false>, gemm4_pair_kernel<EPI, D>, gemm4_kernel<EPI, D, true>};
}
Kernels pick(int epi, int d) {
  switch (epi) {
    case RA_EPI_STORE: return kernels<RA_EPI_STORE, 0>();
    case RA_EPI_GELU: return kernels<RA_EPI_GELU, 0>();
    case RA_EPI_RESID: return kernels<RA_EPI_RESID, 0>();
    default: return d == 128 ? kernels<RA_EPI_QKV, 128>() : kernels<RA_EPI_QKV, 64>();
  }
}

// Clusters of cs CTAs of a split kernel that run at once (ClusterTable asks 1 to 8; only
// sizes up to MAX_SPLIT are used).
int max_clusters(Kernel fn, int cs) {
  static ClusterTable table;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  const int smem = Layout<false>::SMEM_ALLOC;
  return table
      .get(dev, reinterpret_cast<const void*>(fn), smem,
           [&](int c) {
             cudaLaunchAttribute attr[1];
             attr[0].id = cudaLaunchAttributeClusterDimension;
             attr[0].val.clusterDim.x = c;
             attr[0].val.clusterDim.y = 1;
             attr[0].val.clusterDim.z = 1;
             cudaLaunchConfig_t cfg;
             std::memset(&cfg, 0, sizeof(cfg));
             cfg.gridDim = dim3(c, 1, 1);
             cfg.blockDim = dim3(THREADS, 1, 1);
             cfg.dynamicSmemBytes = smem;
             cfg.attrs = attr;
             cfg.numAttrs = 1;
             int found = 0;
             if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
                 cudaOccupancyMaxActiveClusters(&found, fn, &cfg) != cudaSuccess) {
               cudaGetLastError();
               return -1;
             }
             return found;
           })
      .of[cs];
}

struct Plan {
  bool pair;
  int bn, cs;
};

// The cheapest cut: rounds of tiles on the SMs, each as long as its MMAs or its epilogue.
Plan make_plan(const ra_gemm4_args& a, int sms) {
  Plan best{false, 64, 1};
  double best_us = 1e30;
  auto tiles_of = [&](int tm, int bn, int64_t* all, int64_t* open) {
    const int64_t cols = (a.N + bn - 1) / bn;
    *all = *open = 0;  // tiles, and those of segments that are not gated
    for (int g = 0; g < a.n_seg; ++g) {
      const int64_t t = a.seg[g].lin.rows > 0 ? int64_t(a.B) * ((a.seg[g].lin.rows + tm - 1) / tm) * cols : 0;
      *all += t;
      if (!a.seg[g].lin.gated) *open += t;
    }
  };
  const double k = a.K / 1024.0;
  for (int pair = 0; pair < 2; ++pair) {
    if ((a.tile_mode == 1 && pair) || (a.tile_mode == 2 && !pair) || (pair && sms < 2)) continue;
    const int tm = pair ? P_TM : BM, slots = pair ? sms / 2 : sms;
    for (int bn = MAX_BN; bn >= 64; bn -= 64) {
      if (a.epilogue == RA_EPI_QKV && (bn % a.d != 0 || (a.H * a.d) % bn != 0)) continue;
      int64_t all, open;
      tiles_of(tm, bn, &all, &open);
      const double epilogue = 0.0085 * bn;  // of a tile, hidden behind the next one's MMAs
      double round = k * (pair ? 0.8 + 0.0020 * bn : 0.9 + 0.0034 * bn);
      round = round > epilogue ? round : epilogue;
      const double fixed = (pair ? 4.4 : 3.6) + 0.0088 * bn;
      double us = fixed + round * double((all + slots - 1) / slots);
      if (open > 0 && open < all) us += fixed + round * double((open + slots - 1) / slots);
      if (us < best_us) {
        best_us = us;
        best = Plan{pair != 0, bn, 1};
      }
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

// The checks that need no epilogue, and the launch. `who` names the entry point in errors.
ra_status run(const char* who, const ra_gemm4_args& a, cudaStream_t st) {
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
  p.n_seg = a.n_seg;
  p.B = a.B;
  p.N = a.N;
  p.K = a.K;
  p.kblocks = (a.K + CHUNK - 1) / CHUNK;
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
  const Plan plan = make_plan(a, sms);
  const bool pair = plan.pair;
  const int tm = pair ? P_TM : BM;
  p.bn = plan.bn;
  p.w_tiles = plan.bn > 128 ? 2 : 1;
  p.sf_cols = scale_cols(p.groups, p.w_tiles);
  p.sf_bufs = (TMEM_COLS - 2 * plan.bn) / p.sf_cols;
  const int stages = pair ? Layout<true>::STAGES : Layout<false>::STAGES;
  if (p.sf_bufs > stages) p.sf_bufs = stages;
  p.stage_tx = A_BYTES + (pair ? plan.bn / 2 : plan.bn) * (CHUNK / 2) + p.groups * 512 * (1 + p.w_tiles);
  const int64_t cols = (a.N + plan.bn - 1) / plan.bn;
  p.cols = int32_t(cols);
  p.cols_q = p.C / plan.bn;
  int64_t tiles = 0;
  RowSpan out[9], in[21];
  int n_out = 0, n_in = 0;
  for (int g = 0; g < a.n_seg; ++g) {
    const ra_gemm_seg& s = a.seg[g].lin;
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
    const ra_gemm4_seg& q = a.seg[g];
    if (!s.a || !s.w || !q.a_scales || !q.w_scales || !aligned16(s.a) || !aligned16(s.w) || !aligned16(q.a_scales) ||
        !aligned16(q.w_scales) || s.a_stride_r % 16 != 0 || s.a_stride_s % 16 != 0 || s.a_stride_r < a.K / 2 ||
        s.a_stride_s < 0) {
      set_error("%s: seg %d: codes and scales of A and W must be 16-byte aligned, strides multiples of 16 bytes, "
                "a_stride_r >= K / 2", who, g);
      return RA_EINVAL;
    }
    if (q.a_exponent < -64 || q.a_exponent > 64 || q.w_exponent < -64 || q.w_exponent > 64 ||
        (p.e8m0 && (q.a_exponent || q.w_exponent))) {
      set_error("%s: seg %d: exponents need -64 to 64, and 0 for RA_Q4_E8M0 (%d, %d)", who, g, q.a_exponent,
                q.w_exponent);
      return RA_EINVAL;
    }
    if (!fill_epilogue(who, a, g, s, p.seg[g])) return RA_EINVAL;
    const int e = q.a_exponent + q.w_exponent;
    p.seg[g].alpha = ldexpf(1.f, e);
    const int64_t rows = s.rows, spans = (rows + 127) / 128 * ((a.K + 4 * block_of(a.format) - 1) / (4 * block_of(a.format)));
    in[n_in++] = RowSpan{s.a, s.a_stride_s, s.a_stride_r, a.B, rows, a.K / 2};
    in[n_in++] = RowSpan{q.a_scales, spans * 512, 0, a.B, 1, spans * 512};
    in[n_in++] = RowSpan{s.w, 0, a.K / 2, 1, a.N, a.K / 2};
    in[n_in++] = RowSpan{q.w_scales, 0, 0, 1, 1, int64_t(refadapt_quant4_scales_size(a.N, a.K, a.format))};
    if (s.bias) in[n_in++] = RowSpan{s.bias, 0, 0, 1, 1, int64_t(a.N) * 4};
    if (a.epilogue == RA_EPI_QKV) {
      // the rows of the first head: outputs may interleave their heads
      for (const ra_seg* o : {&s.q_out, &s.k_out, &s.v_out})
        out[n_out++] = RowSpan{o->ptr, o->stride_b * 2, o->stride_n * 2, a.B, rows, int64_t(a.d) * 2};
    } else {
      if (a.B > 1 && s.out_stride_s < 1) {
        set_error("%s: seg %d: out_stride_s must be positive", who, g);
        return RA_EINVAL;
      }
      out[n_out++] = RowSpan{s.out, s.out_stride_s * 2, s.out_stride_r * 2, a.B, rows, int64_t(a.N) * 2};
      if (a.epilogue == RA_EPI_RESID) {
        in[n_in++] = RowSpan{s.gate, s.gate_stride_s * 4, 0, a.B, 1, int64_t(a.N) * 4};
        if (s.resid != s.out || s.resid_stride_s != s.out_stride_s || s.resid_stride_r != s.out_stride_r)
          in[n_in++] = RowSpan{s.resid, s.resid_stride_s * 2, s.resid_stride_r * 2, a.B, rows, int64_t(a.N) * 2};
      }
    }
    // Two bytes of codes as one element: a box of 64 is 128 bytes, 256 columns.
    ra_seg as{const_cast<void*>(s.a), s.a_stride_s / 2, 0, s.a_stride_r / 2, s.rows, 0};
    ra_seg ws{const_cast<void*>(s.w), 0, 0, a.K / 4, a.N, 0};
    if (!encode_seg(&p.tm_a[g], as, a.B, 1, a.K / 4, CHUNK / 4, BM, true) ||
        !encode_seg(&p.tm_w[g], ws, 1, 1, a.K / 4, CHUNK / 4, pair ? plan.bn / 2 : plan.bn, true) ||
        !encode_scales(&p.tm_sa[g], q.a_scales, a.K, s.rows, a.B, a.format, p.groups, 1) ||
        !encode_scales(&p.tm_sw[g], q.w_scales, a.K, a.N, 1, a.format, p.groups, p.w_tiles))
      return RA_EINVAL;
    if (int64_t(p.m_tiles[g]) * cols > 2147483647) {
      set_error("%s: seg %d: too many rows", who, g);
      return RA_EINVAL;
    }
    tiles += int64_t(a.B) * p.m_tiles[g] * cols;
  }
  if (overlapping(out, n_out, in, n_in) >= 0) {
    set_error("%s: an output overlaps an input or another output", who);
    return RA_EINVAL;
  }
  if (tiles == 0) return RA_OK;
  const Kernels kn = pick(a.epilogue, a.d);
  const int64_t slots = pair ? (sms / 2 > 0 ? sms / 2 : 1) : sms;
  if (pair) note_launch("CTA pairs, %d columns", plan.bn);
  else if (plan.cs > 1) note_launch("clusters of %d, %d columns", plan.cs, plan.bn);
  else note_launch("single CTAs, %d columns", plan.bn);
  if (pair) return launch(who, p, kn.pair, Layout<true>::SMEM_ALLOC, 2 * (tiles < slots ? tiles : slots), 2, st);
  if (plan.cs > 1) return launch(who, p, kn.split, Layout<false>::SMEM_ALLOC, tiles * plan.cs, plan.cs, st);
  return launch(who, p, kn.single, Layout<false>::SMEM_ALLOC, tiles < slots ? tiles : slots, 1, st);
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
  return gemm4::run("refadapt_gemm4", *a, static_cast<cudaStream_t>(stream));
}
