// refadapt_gemm: the linear layers of the DiT block around the attention
// (QKV projection, output projection, MLP), bf16 in, fp32 accumulate in TMEM,
// with the elementwise work that follows each layer fused into the epilogue.
//
//   D[r, n] = sum_k A[r, k] W[n, k]        (A rows of one segment and sample,
//                                           W in nn.Linear layout [N][K])
//
// Two kernels: CTA pairs on 256-row output tiles (gemm_pair_kernel, below) and
// one CTA per SM on 128-row tiles (gemm_kernel), both persistent, tiles up to
// 256 columns wide. Calls of few tiles and a long K go to a third form, where
// the CTAs of a cluster share a 128-row tile's K (gemm_kernel, SPLIT). make_plan()
// picks the form and the width. Live tiles
// (those the modes do not skip) are numbered segment-major, then sample, then
// in bands of GROUP_M row tiles, rows fastest inside a band (so the CTAs that
// run at once share a few A row blocks and a few W column blocks, both held in
// L2); CTA c takes tiles c, c + G, c + 2G, ...
//   warp 0      TMA producer: per K step one 128 x 64 A box and one W box of the
//               tile's width x 64 (128-byte swizzle, rows past a segment's end read as
//               zeros) into a 4-stage ring.
//   warp 1      TMEM allocator (512 columns: two 256-column accumulators) and
//               MMA issuer: tcgen05.mma kind::f16, M = 128, N = the tile's
//               width, K = 16, four per stage; commits free the stage and, after a tile's
//               last step, hand the accumulator to the epilogue.
//   warps 2..9  epilogue: two warps per TMEM lane quarter (quarter = warp % 4,
//               thread = output row = TMEM lane), which take the tile's 32-column
//               chunks (QKV: heads) in turn; the next tile's MMAs run into the
//               other accumulator meanwhile.
// Epilogues (fp32 until the final bf16 rounding):
//   STORE  out = acc + bias
//   GELU   out = gelu_tanh(acc + bias)
//   RESID  out = resid + gate[sample] * (acc + bias)        (gated residual)
//   QKV    columns [q | k | v] of H heads of width d: q and k RMS-normalised
//          per head with a [d] weight, then rotated by RoPE on interleaved
//          pairs at the row's joint position; written head-major.
// A tile whose MMAs take 4 us (K = 1024) left the epilogue of four warps, with
// 16-byte accesses 32 rows apart and a global-load latency per 32 columns, as
// the longer part (11 us a tile with GELU). So the per-column vectors of a tile
// go to shared memory and the first residuals to registers before its
// accumulator is ready, and global rows are read and written through a 2 KB
// staging buffer per warp, 64 contiguous bytes of eight rows per instruction.
// Reference segments may be gated on the per-sample mode: their tiles are
// skipped when the mode is REUSE (Algorithm 1 skips reference rows) and, for
// QKV, the K and V column tiles also when it is BOUNDARY (the block keeps its
// cached reference K/V). Every mbarrier wait is bounded; on a timeout the CTA
// drains its own TMA and MMA work, frees TMEM, flags the error word and returns.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>
#include <mutex>

#include "gemm_body.cuh"

namespace ra {
namespace gemm {

constexpr int BN = 256, BK = 64;
constexpr int STAGES = 4;
constexpr int A_BYTES = BM * BK * 2;
constexpr int B_BYTES = BN * BK * 2;
constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int OFF_BAR = STAGES * STAGE_BYTES;
constexpr int NUM_BARS = 2 * STAGES + 2 + 2 + 1 + 1;  // full, empty, tfull[2], tempty[2], drain, parts_full
constexpr int OFF_MISC = OFF_BAR + NUM_BARS * 8;
constexpr int OFF_EPI = (OFF_MISC + 16 + 127) / 128 * 128;
constexpr int SMEM_BYTES = OFF_EPI + EPI_WARPS * EPI_WARP_BYTES;
constexpr int SMEM_ALLOC = SMEM_BYTES + 1024;
static_assert(SMEM_ALLOC <= 232448, "shared memory budget");
// split tiles: the parts to send and those received take the place of the stages
static_assert(2 * (MAX_SPLIT - 1) * (BM * BN * 4 / MAX_SPLIT) <= OFF_BAR, "parts fit the stages");

// CTA-pair kernel: 256-row output tiles; each CTA stages its 128 rows of A
// and its half of the W tile (up to 128 columns), 128 of K per stage (two 128-byte
// swizzle chunks per operand, 64 KB per stage, 3 stages): half the stage
// hand-offs of 64-wide stages, which the fused epilogues gained from (GELU
// +3 %); a K % 128 == 64 tail is a half stage.
constexpr int P_STAGES = 3;
constexpr int P_BK = 128;              // K per stage: two 64-column chunks per operand
constexpr int P_CHUNK = 128 * 64 * 2;  // 128 rows x 64 K of one operand (one 128-byte swizzle span)
constexpr int P_A_BYTES = 128 * P_BK * 2;
constexpr int P_B_BYTES = 128 * P_BK * 2;
constexpr int P_STAGE_BYTES = P_A_BYTES + P_B_BYTES;
constexpr int P_OFF_BAR = P_STAGES * P_STAGE_BYTES;
constexpr int P_NUM_BARS = 2 * P_STAGES + 2 + 2 + 1;
constexpr int P_OFF_MISC = P_OFF_BAR + P_NUM_BARS * 8;
constexpr int P_OFF_EPI = (P_OFF_MISC + 16 + 127) / 128 * 128;
constexpr int P_SMEM_BYTES = P_OFF_EPI + EPI_WARPS * EPI_WARP_BYTES;
constexpr int P_SMEM_ALLOC = P_SMEM_BYTES + 1024;
static_assert(P_SMEM_ALLOC <= 232448, "shared memory budget");

// SPLIT: a cluster takes one tile, each rank a contiguous part of its K
// (merge_parts adds them up), then its share of the columns in the epilogue.
template <int EPI, int D, bool SPLIT = false>
__global__ void __launch_bounds__(THREADS, 1) gemm_kernel(const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint64_t* full = bars;
  uint64_t* empty = bars + STAGES;
  uint64_t* tfull = bars + 2 * STAGES;
  uint64_t* tempty = bars + 2 * STAGES + 2;
  uint64_t* drain = bars + 2 * STAGES + 4;
  uint64_t* parts_full = bars + 2 * STAGES + 5;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + OFF_MISC + 4);
  volatile int* live = reinterpret_cast<volatile int*>(smem + OFF_MISC + 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = SPLIT ? int(cluster_rank()) : 0, cs = SPLIT ? int(cluster_size()) : 1;
  const int64_t t0 = SPLIT ? blockIdx.x / cs : blockIdx.x, step = SPLIT ? gridDim.x / cs : gridDim.x;
  const int kb0 = SPLIT ? p.kblocks * rank / cs : 0;  // this CTA's K steps
  const int kb1 = SPLIT ? p.kblocks * (rank + 1) / cs : p.kblocks;
  const int bn = SPLIT && p.rest_max > 0 ? REST_BN : p.bn;
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
    // The modes may leave this cluster no tile: it goes now, before the barriers
    // of the merge (reuse rows of a call planned with a rest 75.8 -> 72.2 us).
    pdl_wait();
    Walk<BM, EPI> walk;
    Tile tl;
    *live = tile_at<EPI, SPLIT>(p, walk, t0, tl);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem0 = SPLIT ? 0 : *tmem_slot;  // SPLIT reads it per role: 0.3 us less there, 0.1 more without
  if (SPLIT && !*live) {  // uniform over the cluster
    if (warp == 1) tmem_dealloc(*tmem_slot, TMEM_COLS);
    return;
  }
  const WaitCtl ctl{abort_flag, p.err_word, p.budget_ns};
  pdl_launch();
  if (warp != 0) pdl_wait();

  int64_t loads = 0;    // the producer's: K steps whose loads may be on their way
  bool issued = false;  // the issuer's: MMAs may be on their way
  if (warp == 0) {
    if (lane == 0) {
      // -------------------------------------------------------------- producer
      for (int g = 0; g < p.n_seg; ++g)
        if (p.rows[g] > 0) {
          tma_prefetch_desc(&p.tm_a[g]);
          tma_prefetch_desc(&p.tm_w[g]);
        }
      pdl_wait();
      int64_t it = 0;  // K steps issued
      bool ok = true;
      Walk<BM, EPI> walk;
      Tile tl;
      for (int64_t t = t0; ok && tile_at<EPI, SPLIT>(p, walk, t, tl); t += step) {
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          const int st = int(it % STAGES);
          if (it >= STAGES && !(ok = mbar_wait(empty + st, uint32_t((it / STAGES - 1) & 1), ctl))) break;
          uint8_t* sa = smem + st * STAGE_BYTES;
          mbar_arrive_expect_tx(full + st, A_BYTES + bn * BK * 2);
          tma_load_4d(sa, &p.tm_a[tl.seg], full + st, kb * BK, tl.m0, 0, tl.s);
          tma_load_4d(sa + A_BYTES, &p.tm_w[tl.seg], full + st, kb * BK, tl.n0, 0, 0);
        }
      }
      if (*abort_flag) {
        for (int st = 0; st < STAGES; ++st) {
          const int64_t n_s = (it > st) ? (it - st + STAGES - 1) / STAGES : 0;
          if (n_s > 0) mbar_wait_drain(full + st, uint32_t((n_s - 1) & 1), p.budget_ns);
        }
      } else {
        loads = it;
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      // -------------------------------------------------------------- MMA issuer
      const uint32_t idesc = idesc_bf16_f32(BM, bn, 0, 0);
      const uint32_t s0 = smem_u32(smem), tmem = SPLIT ? *tmem_slot : tmem0;
      int64_t it = 0;
      int i = 0;
      bool ok = true;
      Walk<BM, EPI> walk;
      Tile tl;
      for (int64_t t = t0; ok && tile_at<EPI, SPLIT>(p, walk, t, tl); t += step) {
        const int buf = i & 1, use = i >> 1;
        if (use > 0 && !(ok = mbar_wait(tempty + buf, uint32_t((use - 1) & 1), ctl))) break;
        tc_fence_after();
        const uint32_t d_t = tmem + uint32_t(buf * BN);
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          const int st = int(it % STAGES);
          if (!(ok = mbar_wait(full + st, uint32_t((it / STAGES) & 1), ctl))) break;
          tc_fence_after();
          const uint32_t sa = s0 + st * STAGE_BYTES, sb = sa + A_BYTES;
#pragma unroll
          for (int kk = 0; kk < BK / 16; ++kk)
            umma_ss(d_t, sdesc_sw128(sa + kk * 32, 16, 1024), sdesc_sw128(sb + kk * 32, 16, 1024), idesc,
                    (kb > kb0 || kk > 0) ? 1u : 0u);
          umma_commit(empty + st);
          issued = true;
        }
        if (!ok) break;
        umma_commit(tfull + buf);
        ++i;
      }
      if (!ok && issued) {
        umma_commit(drain);
        mbar_wait_drain(drain, 0, p.budget_ns);
        issued = false;
      }
    }
  } else {
    // ---------------------------------------------------------------- epilogue
    const int quarter = warp & 3;
    const uint32_t tmem = SPLIT ? *tmem_slot : tmem0;
    EpiWarp w;
    w.half = (warp - 2) >> 2;
    w.stage = smem + OFF_EPI + (warp - 2) * EPI_WARP_BYTES;
    w.vec0 = reinterpret_cast<float*>(w.stage + EPI_STAGE_BYTES);
    w.vec1 = w.vec0 + 128;
    int i = 0;
    Walk<BM, EPI> walk;
    Tile tl;
    for (int64_t t = t0; tile_at<EPI, SPLIT>(p, walk, t, tl); t += step) {
      const int buf = i & 1, use = i >> 1;
      w.row0 = tl.m0 + quarter * 32;
      w.nrow = min(32, p.rows[tl.seg] - w.row0);
      w.acc = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(buf * BN);
      w.cols = bn;
      const uint32_t acc = w.acc;
      if (SPLIT) {
        w.cols /= cs;
        w.acc += uint32_t(rank * w.cols);
        tl.n0 += rank * w.cols;
      }
      if (!epilogue_tile<EPI, D>(p, tl, w, [&] {
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
  // No role waits any more, so the flag is final: it may have been raised after the
  // producer and the issuer were through. What this CTA has on its way lands first.
  if (*abort_flag && lane == 0) {
    if (warp == 0)
      for (int st = 0; st < STAGES; ++st) {
        const int64_t n_s = (loads > st) ? (loads - st + STAGES - 1) / STAGES : 0;
        if (n_s > 0) mbar_wait_drain(full + st, uint32_t((n_s - 1) & 1), p.budget_ns);
      }
    if (warp == 1 && issued) {
      umma_commit(drain);
      mbar_wait_drain(drain, 0, p.budget_ns);
    }
  }
  __syncwarp();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(SPLIT ? *tmem_slot : tmem0, TMEM_COLS);
  }
}


// CTA-pair variant (cluster of two, cta_group::2). Both CTAs walk the same
// tile sequence (cluster c takes tiles c, c + G/2, ...); per K step each CTA's
// producer loads its own 128 A rows and its half of the W tile, and both
// loads complete on rank 0's full barrier (rank 0 arms it for both CTAs'
// bytes). Rank 0's MMA thread issues M = 256 MMAs of the tile's width; commits are
// multicast to both CTAs (stage free, accumulator ready). Each CTA's epilogue
// reads its own TMEM rows and arrives on rank 0's accumulator-free barrier
// (count 16). The two CTAs meet at a cluster barrier before TMEM is freed and
// before either exits, so no remote arrive or MMA outlives its target.
template <int EPI, int D>
__global__ void __launch_bounds__(THREADS, 1) gemm_pair_kernel(const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + P_OFF_BAR);
  uint64_t* full = bars;
  uint64_t* empty = bars + P_STAGES;
  uint64_t* tfull = bars + 2 * P_STAGES;
  uint64_t* tempty = bars + 2 * P_STAGES + 2;
  uint64_t* drain = bars + 2 * P_STAGES + 4;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + P_OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + P_OFF_MISC + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int64_t cid = blockIdx.x >> 1, ncl = gridDim.x >> 1;
  if (threadIdx.x == 0) {
    for (int s = 0; s < P_STAGES; ++s) {
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
  const uint32_t tmem = *tmem_slot;
  const WaitCtl ctl{abort_flag, p.err_word, p.budget_ns};
  pdl_launch();
  if (warp != 0) pdl_wait();

  int64_t loads = 0;    // the producer's: stages that it loaded
  bool issued = false;  // the issuer's: it has issued MMAs
  if (warp == 0) {
    if (lane == 0) {
      // -------------------------------------------------------------- producer (both CTAs)
      for (int g = 0; g < p.n_seg; ++g)
        if (p.rows[g] > 0) {
          tma_prefetch_desc(&p.tm_a[g]);
          tma_prefetch_desc(&p.tm_w[g]);
        }
      pdl_wait();
      const uint32_t full0 = mapa_shared(smem_u32(full), 0);  // rank 0's full barriers
      int64_t it = 0;
      bool ok = true;
      Walk<P_TM, EPI> walk;
      Tile tl;
      const int64_t end = round_tiles<P_TM, EPI>(p);
      for (int64_t t = cid; ok && t < end && walk.at(p, t, tl); t += ncl) {
        for (int kb = 0; kb < (p.kblocks + 1) / 2; ++kb, ++it) {
          const int st = int(it % P_STAGES);
          if (it >= P_STAGES && !(ok = mbar_wait(empty + st, uint32_t((it / P_STAGES - 1) & 1), ctl))) break;
          uint8_t* sa = smem + st * P_STAGE_BYTES;
          const int chunks = (2 * kb + 1 < p.kblocks) ? 2 : 1;  // K % 128 == 64: the last stage is half
          if (rank == 0) mbar_arrive_expect_tx(full + st, chunks * (2 * P_CHUNK + p.bn * 128));
          for (int c = 0; c < chunks; ++c) {
            tma_load_4d_pair(sa + c * P_CHUNK, &p.tm_a[tl.seg], full0 + 8u * st, kb * P_BK + c * 64,
                             tl.m0 + int(rank) * 128, 0, tl.s);
            tma_load_4d_pair(sa + P_A_BYTES + c * P_CHUNK, &p.tm_w[tl.seg], full0 + 8u * st, kb * P_BK + c * 64,
                             tl.n0 + int(rank) * (p.bn / 2), 0, 0);
          }
        }
      }
      loads = it;
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      // -------------------------------------------------------------- MMA issuer (rank 0)
      const uint32_t idesc = idesc_bf16_f32(P_TM, p.bn, 0, 0);
      const uint32_t s0 = smem_u32(smem);
      int64_t it = 0;
      int i = 0;
      bool ok = true;
      Walk<P_TM, EPI> walk;
      Tile tl;
      const int64_t end = round_tiles<P_TM, EPI>(p);
      for (int64_t t = cid; ok && t < end && walk.at(p, t, tl); t += ncl) {
        const int buf = i & 1, use = i >> 1;
        if (use > 0 && !(ok = mbar_wait_cluster(tempty + buf, uint32_t((use - 1) & 1), ctl))) break;
        tc_fence_after();
        const uint32_t d_t = tmem + uint32_t(buf * BN);
        for (int kb = 0; kb < (p.kblocks + 1) / 2; ++kb, ++it) {
          const int st = int(it % P_STAGES);
          if (!(ok = mbar_wait(full + st, uint32_t((it / P_STAGES) & 1), ctl))) break;
          tc_fence_after();
          const uint32_t sa = s0 + st * P_STAGE_BYTES, sb = sa + P_A_BYTES;
          const int ksteps = (2 * kb + 1 < p.kblocks) ? P_BK / 16 : 64 / 16;
#pragma unroll
          for (int kk = 0; kk < P_BK / 16; ++kk) {
            if (kk >= ksteps) break;
            const uint32_t o = uint32_t((kk >> 2) * P_CHUNK + (kk & 3) * 32);
            umma_ss_pair(d_t, sdesc_sw128(sa + o, 16, 1024), sdesc_sw128(sb + o, 16, 1024), idesc,
                         (kb > 0 || kk > 0) ? 1u : 0u);
          }
          umma_commit_pair(empty + st, 0x3);
          issued = true;
        }
        if (!ok) break;
        umma_commit_pair(tfull + buf, 0x3);
        ++i;
      }
    }
  } else {
    // ---------------------------------------------------------------- epilogue (both CTAs)
    const int quarter = warp & 3;
    EpiWarp w;
    w.half = (warp - 2) >> 2;
    w.stage = smem + P_OFF_EPI + (warp - 2) * EPI_WARP_BYTES;
    w.vec0 = reinterpret_cast<float*>(w.stage + EPI_STAGE_BYTES);
    w.vec1 = w.vec0 + 128;
    const uint32_t tempty0 = mapa_shared(smem_u32(tempty), 0);
    int i = 0;
    Walk<P_TM, EPI> walk;
    Tile tl;
    const int64_t end = round_tiles<P_TM, EPI>(p);
    for (int64_t t = cid; t < end && walk.at(p, t, tl); t += ncl) {
      const int buf = i & 1, use = i >> 1;
      w.row0 = tl.m0 + int(rank) * 128 + quarter * 32;
      w.cols = p.bn;
      w.nrow = min(32, p.rows[tl.seg] - w.row0);
      w.acc = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(buf * BN);
      if (!epilogue_tile<EPI, D>(p, tl, w, [&] {
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
  if (*abort_flag && lane == 0) {
    if (warp == 0 && rank == 0) {
      // rank 0's full barriers count both CTAs' bytes of every phase it armed
      for (int st = 0; st < P_STAGES; ++st) {
        const int64_t n_s = (loads > st) ? (loads - st + P_STAGES - 1) / P_STAGES : 0;
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

__global__ void rope_table_kernel(float* table, int32_t n_pos, int32_t d, double base) {
  const int64_t n = int64_t(n_pos) * (d / 2);
  for (int64_t i = blockIdx.x * int64_t(blockDim.x) + threadIdx.x; i < n; i += int64_t(gridDim.x) * blockDim.x) {
    const int64_t pos = i / (d / 2);
    const int pair = int(i % (d / 2));
    const double ang = double(pos) * pow(base, -2.0 * pair / double(d));
    double s, c;
    sincos(ang, &s, &c);
    table[2 * i] = float(c);
    table[2 * i + 1] = float(s);
  }
}

// The kernels by epilogue (QKV: by head dim too), one CTA per tile and CTA pairs.
using Kernel = void (*)(Params);
struct Kernels {
  Kernel single, pair, split;  // split: STORE, GELU and RESID
};
Kernels pick(int epi, int d) {
  switch (epi) {
    case RA_EPI_STORE: return {gemm_kernel<RA_EPI_STORE, 0>, gemm_pair_kernel<RA_EPI_STORE, 0>, gemm_kernel<RA_EPI_STORE, 0, true>};
    case RA_EPI_GELU: return {gemm_kernel<RA_EPI_GELU, 0>, gemm_pair_kernel<RA_EPI_GELU, 0>, gemm_kernel<RA_EPI_GELU, 0, true>};
    case RA_EPI_RESID: return {gemm_kernel<RA_EPI_RESID, 0>, gemm_pair_kernel<RA_EPI_RESID, 0>, gemm_kernel<RA_EPI_RESID, 0, true>};
    default:
      return d == 128 ? Kernels{gemm_kernel<RA_EPI_QKV, 128>, gemm_pair_kernel<RA_EPI_QKV, 128>, nullptr}
                      : Kernels{gemm_kernel<RA_EPI_QKV, 64>, gemm_pair_kernel<RA_EPI_QKV, 64>, nullptr};
  }
}

// How a call is cut into tiles: CTA pairs or single CTAs, tile columns, and the
// CTAs of a cluster that share a tile's K (1: a CTA has a tile of its own).
// rest_max > 0: pair tiles of 256 columns in whole rounds, and a rest of at most
// this many split, each into four tiles of clusters of cs CTAs, by a second launch.
struct Plan {
  bool pair;
  int bn, cs, rest_max;
};

// Clusters of cs CTAs of a split kernel that can run at once on the current
// device (they live inside one GPC, so the floorplan decides; every split kernel
// has the same launch shape); cached per device. 0: none, or the query failed,
// and nothing is split.
int max_clusters(Kernel fn, int cs) {
  static std::mutex mu;
  static int cache[64][MAX_SPLIT + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return 0;
  }
  std::lock_guard<std::mutex> lk(mu);
  int& n = cache[dev][cs];
  if (n > 0) return n;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(cs, 1, 1);
  cfg.blockDim = dim3(THREADS, 1, 1);
  cfg.dynamicSmemBytes = SMEM_ALLOC;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int found = 0;
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_ALLOC) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&found, fn, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  return n = found;
}

// The cheapest cut by a model of the two kernels' time (microseconds), fitted to
// single waves of 256 to 64 columns at K = 1024 and 4096 on a GB300 (each within
// 6 %): what one round of tiles takes grows with the operand bytes a CTA stages
// per K step (each is written to shared memory once and read once, which fills
// its port before the tensor core is full), so a narrower tile costs nearly as
// much as a wide one (256 columns 5.1 us per 1024 of K, 128 columns 4.0) and
// pays only where it saves a round: 13 row tiles of 256 by N = 3072 make 156
// tiles of 256 columns (three rounds of 76 pairs, the last one nearly empty;
// 188 us at K = 12288) or 208 of 192 columns (three shorter rounds, 164 us).
// Few tiles of a long K leave SMs idle (a small model's MLP output, 377 rows by
// N = 1024, K = 4096, is 64 narrow tiles, 19.2 us): there two or four CTAs of a
// cluster share a tile's K, which costs a merge and pays from about K = 3072 up
// while the clusters fit the GPU at once (12.1 us in clusters of four on tiles of
// 128 columns; 516 rows, K = 12288, N = 3072 58.9 -> 50.3 in clusters of two;
// at K = 1024 it loses, 7.3 -> 8.2). Not for QKV, whose epilogue needs whole heads,
// nor where the caller chose the tiles.
// Whole rounds of pair tiles and a small rest: the rest's tiles are cut into
// quarters and split in the same way by a second launch, which costs 13 us and
// its share of K, so only a long K gains (K = 12288, N = 3072: 13 row tiles, two
// rounds and 4 tiles, 162 -> 157 us; 1572 rows, one round and 8, 105 -> 95). Its
// 256-column tiles also suit what the modes leave better than narrow ones.
// Calls with gated segments are weighed with and without them.
Plan make_plan(const ra_gemm_args& a, int sms) {
  Plan best{false, 256, 1, 0};
  double best_us = 1e30;
  auto tiles_of = [&](int tm, int bn, int64_t* all, int64_t* open) {
    const int64_t cols = (a.N + bn - 1) / bn;
    *all = *open = 0;  // tiles, and those of segments that are not gated
    for (int g = 0; g < a.n_seg; ++g) {
      const int64_t t = a.seg[g].rows > 0 ? int64_t(a.B) * ((a.seg[g].rows + tm - 1) / tm) * cols : 0;
      *all += t;
      if (!a.seg[g].gated) *open += t;
    }
  };
  // Many column tiles that all read the same few rows of A contend for the L2
  // lines these lie in (4 rows, K = 2048, N = 8192: 21.7 us in 128 tiles of 64
  // columns, 11.8 in 32 of 256; from 32 rows on 10.3 and 11.9).
  bool few_rows = false;
  for (int g = 0; g < a.n_seg; ++g) few_rows |= a.seg[g].rows > 0 && a.seg[g].rows < 32;
  for (int pair = 0; pair < 2; ++pair) {
    if ((a.tile_mode == 1 && pair) || (a.tile_mode == 2 && !pair) || (pair && sms < 2)) continue;
    const int tm = pair ? P_TM : BM, slots = pair ? sms / 2 : sms;
    for (int bn = 256; bn >= 64; bn -= 32) {
      if (a.epilogue == RA_EPI_QKV && (bn % a.d != 0 || (a.H * a.d) % bn != 0)) continue;
      if (few_rows && bn < 256 && a.N / bn > 40) continue;
      int64_t all, open;
      tiles_of(tm, bn, &all, &open);
      const double epilogue = 0.0085 * bn;  // of a tile, hidden behind the next one's MMAs
      double round = a.K / 1024.0 * (pair ? 3.11 + 0.00766 * bn : 3.4 + 0.0127 * bn);
      round = round > epilogue ? round : epilogue;
      const double fixed = pair ? 4.4 + 0.0088 * bn : 3.6;
      double us = fixed + round * double((all + slots - 1) / slots);
      if (open > 0 && open < all) us += fixed + round * double((open + slots - 1) / slots);
      if (us < best_us) {
        best_us = us;
        best = Plan{pair != 0, bn, 1, 0};
      }
    }
  }
  if (a.epilogue == RA_EPI_QKV || a.tile_mode != 0) return best;
  const double merge = 4.0;
  for (int cs = 2; cs <= MAX_SPLIT; cs *= 2) {
    if (a.K / BK < 4 * cs) break;
    const int clusters = max_clusters(pick(a.epilogue, a.d).split, cs);
    if (clusters == 0) continue;
    for (int bn = 256; bn >= 32 * cs; bn /= 2) {
      int64_t all, open;
      tiles_of(BM, bn, &all, &open);
      const double wave = 3.6 + merge + a.K / 1024.0 / cs * (3.4 + 0.0127 * bn);
      double us = wave * double((all + clusters - 1) / clusters);
      if (open > 0 && open < all) us += wave * double((open + clusters - 1) / clusters);
      if (us < 0.97 * best_us) {
        best_us = us;
        best = Plan{false, bn, cs, 0};
      }
    }
    const int slots = sms / 2;
    const double round = a.K / 1024.0 * (3.11 + 0.00766 * BN), fixed = 4.4 + 0.0088 * BN;
    const double wave = 13.3 + a.K / 1024.0 / cs * (3.4 + 0.0127 * REST_BN);
    int64_t all, open;
    tiles_of(P_TM, BN, &all, &open);
    int64_t rest_max = int64_t(round / wave) * clusters / 4;
    if (rest_max > slots - 1) rest_max = slots - 1;
    if (slots < 1 || rest_max < 1 || all < slots) continue;
    auto time = [&](int64_t tiles) {
      const int64_t rest = tiles % slots;
      const bool split = rest <= rest_max;
      return fixed + round * double(split ? tiles / slots : tiles / slots + 1) +
             wave * double(split ? (4 * rest + clusters - 1) / clusters : 0);
    };
    const double us = time(all) + (open > 0 && open < all ? time(open) : 0.0);
    if (us < 0.97 * best_us) {
      best_us = us;
      best = Plan{true, BN, cs, int(rest_max)};
    }
  }
  return best;
}

}  // namespace gemm
}  // namespace ra

extern "C" ra_status refadapt_rope_table(float* table, int32_t n_pos, int32_t d, double base, void* stream) {
  using namespace ra;
  clear_error();
  if (!table || n_pos < 1 || d < 2 || d % 4 != 0 || !(base > 1.0)) {
    set_error("refadapt_rope_table: table NULL, n_pos < 1, d not a multiple of 4 or base <= 1");
    return RA_EINVAL;
  }
  const int64_t n = int64_t(n_pos) * (d / 2);
  const int blocks = int((n + 255) / 256 < 4096 ? (n + 255) / 256 : 4096);
  gemm::rope_table_kernel<<<blocks, 256, 0, static_cast<cudaStream_t>(stream)>>>(table, n_pos, d, base);
  return launch_status("refadapt_rope_table");
}

extern "C" ra_status refadapt_gemm(const ra_gemm_args* a, void* stream) {
  using namespace ra;
  using namespace ra::gemm;
  clear_error();
  if (!a) {
    set_error("refadapt_gemm: args is NULL");
    return RA_EINVAL;
  }
  if (a->B < 1 || a->n_seg < 1 || a->n_seg > 3 || a->K < BK || a->K % BK != 0 || a->N < BN || a->N % BN != 0) {
    set_error("refadapt_gemm: need B >= 1, 1 <= n_seg <= 3, K a positive multiple of 64, N of 256 "
              "(B=%d n_seg=%d N=%d K=%d)", a->B, a->n_seg, a->N, a->K);
    return RA_EINVAL;
  }
  if (a->epilogue < RA_EPI_STORE || a->epilogue > RA_EPI_QKV) {
    set_error("refadapt_gemm: unknown epilogue %d", a->epilogue);
    return RA_EINVAL;
  }
  Params p;
  std::memset(&p, 0, sizeof(p));
  p.n_seg = a->n_seg;
  p.B = a->B;
  p.N = a->N;
  p.K = a->K;
  p.kblocks = a->K / BK;
  p.mode = a->mode;
  p.err_word = a->err_word;
  p.budget_ns = wait_budget_ns();
  p.norm_eps = a->norm_eps;
  if (a->epilogue == RA_EPI_QKV) {
    if ((a->d != 64 && a->d != 128) || a->H < 1 || int64_t(3) * a->H * a->d != a->N || (a->H * a->d) % BN != 0) {
      set_error("refadapt_gemm: QKV needs d in {64, 128}, N = 3 H d and H d a multiple of 256");
      return RA_EINVAL;
    }
    if (!a->rope || !aligned16(a->rope) || a->rope_len < 1 || !(a->norm_eps >= 0.f)) {
      set_error("refadapt_gemm: QKV needs a 16-byte aligned rope table, rope_len >= 1 and norm_eps >= 0");
      return RA_EINVAL;
    }
    p.C = a->H * a->d;
    p.rope = reinterpret_cast<const float4*>(a->rope);
    p.rope_len = a->rope_len;
  }
  if (a->tile_mode < 0 || a->tile_mode > 2) {
    set_error("refadapt_gemm: tile_mode %d (0 auto, 1 one CTA per tile, 2 CTA pairs)", a->tile_mode);
    return RA_EINVAL;
  }
  const int sms = num_sms();
  const Plan plan = make_plan(*a, sms);
  const bool pair = plan.pair;
  const int tm = pair ? P_TM : BM;
  p.bn = plan.bn;
  const int64_t cols = (a->N + plan.bn - 1) / plan.bn;
  p.cols = int32_t(cols);
  p.cols_q = p.C / plan.bn;
  int64_t tiles = 0;
  for (int g = 0; g < a->n_seg; ++g) {
    const ra_gemm_seg& s = a->seg[g];
    Seg& d = p.seg[g];
    if (s.rows < 0) {
      set_error("refadapt_gemm: seg %d rows < 0", g);
      return RA_EINVAL;
    }
    p.rows[g] = s.rows;
    p.m_tiles[g] = (s.rows + tm - 1) / tm;
    p.gated[g] = s.gated ? 1 : 0;
    if (s.gated && !a->mode) {
      set_error("refadapt_gemm: seg %d is gated but mode is NULL", g);
      return RA_EINVAL;
    }
    if (s.rows == 0) continue;
    if (!s.a || !s.w || !aligned16(s.a) || !aligned16(s.w) || s.a_stride_r % 8 != 0 || s.a_stride_s % 8 != 0 ||
        s.a_stride_r < a->K || s.a_stride_s < 0) {
      set_error("refadapt_gemm: seg %d: A and W must be 16-byte aligned, strides multiples of 8 elements, "
                "a_stride_r >= K", g);
      return RA_EINVAL;
    }
    if (!fill_epilogue("refadapt_gemm", *a, g, s, d)) return RA_EINVAL;
    ra_seg as{const_cast<void*>(s.a), s.a_stride_s, 0, s.a_stride_r, s.rows, 0};
    ra_seg ws{const_cast<void*>(s.w), 0, 0, a->K, a->N, 0};
    // The pair kernel loads half a tile's rows of W per CTA.
    if (!encode_seg(&p.tm_a[g], as, a->B, 1, a->K, BK, BM, true) ||
        !encode_seg(&p.tm_w[g], ws, 1, 1, a->K, BK, pair ? plan.bn / 2 : plan.bn, true))
      return RA_EINVAL;
    if (int64_t(p.m_tiles[g]) * cols > 2147483647) {
      set_error("refadapt_gemm: seg %d: too many rows", g);
      return RA_EINVAL;
    }
    tiles += int64_t(a->B) * p.m_tiles[g] * cols;
  }
  if (tiles == 0) return RA_OK;
  const Kernels kn = pick(a->epilogue, a->d);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int64_t slots = pair ? (sms / 2 > 0 ? sms / 2 : 1) : sms;
  p.slots = int32_t(slots);
  p.rest_max = plan.rest_max;
  if (plan.rest_max > 0) {
    note_launch("rounds of CTA pairs, up to %d tiles in clusters of %d", plan.rest_max, plan.cs);
    // No modes leave more whole rounds than all tiles do, or a larger split rest.
    const int64_t rest = tiles % slots, whole = rest <= plan.rest_max ? tiles - rest : tiles;
    const ra_status r = launch("refadapt_gemm", p, kn.pair, P_SMEM_ALLOC, 2 * (whole < slots ? whole : slots), 2, st);
    if (r != RA_OK) return r;
    return launch("refadapt_gemm", p, kn.split, SMEM_ALLOC, int64_t(4) * plan.rest_max * plan.cs, plan.cs, st);
  }
  if (pair) note_launch("CTA pairs, %d columns", plan.bn);
  else if (plan.cs > 1) note_launch("clusters of %d, %d columns", plan.cs, plan.bn);
  else note_launch("single CTAs, %d columns", plan.bn);
  if (pair) return launch("refadapt_gemm", p, kn.pair, P_SMEM_ALLOC, 2 * (tiles < slots ? tiles : slots), 2, st);
  if (plan.cs > 1) return launch("refadapt_gemm", p, kn.split, SMEM_ALLOC, tiles * plan.cs, plan.cs, st);
  return launch("refadapt_gemm", p, kn.single, SMEM_ALLOC, tiles < slots ? tiles : slots, 1, st);
}
