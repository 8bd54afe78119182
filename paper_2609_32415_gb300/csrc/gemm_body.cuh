// Parts of the GEMM kernels. Of 16-bit and of 4-bit operands: the tiles' order (Walk), a segment's epilogue tensors
// and their checks, bias and scale (add_cols), the launch; the one-row kernel of 4-bit operands: gelu_tanh2. Of 16-bit
// operands alone: round_tiles and tile_at, the epilogues (epilogue_*), the merge of tiles whose K is shared (4-bit
// tiles have epilogues of their own, gemm4.cu, and share no K).
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstring>

#include "api_common.h"
#include "epi_rows.cuh"
#include "tc_ptx.cuh"

namespace ra {
namespace gemm {

constexpr int BM = 128;    // rows of a tile of one CTA
constexpr int P_TM = 256;  // of a CTA pair's
constexpr int EPI_WARPS = 8;
constexpr int EPI_STAGE_BYTES = 32 * 64;                  // 32 rows x 32 bf16 (or 16 fp32) of one warp
constexpr int EPI_WARP_BYTES = EPI_STAGE_BYTES + 2 * 512;  // and two per-column vectors of its 128 columns
constexpr int THREADS = 64 + 32 * EPI_WARPS;
constexpr int TMEM_COLS = 512;
constexpr int MAX_SPLIT = 4;  // CTAs of a cluster that share one tile's K

struct Seg {
  int32_t pos_offset, reserved;
  const float* bias;
  __nv_bfloat16* out;
  int64_t out_ss, out_sr;
  const __nv_bfloat16* resid;
  int64_t res_ss, res_sr;
  const float* gate;
  int64_t gate_ss;
  __nv_bfloat16* dst[3];  // QKV: q, k, v, head-major
  int64_t dst_sb[3], dst_sh[3], dst_sn[3];
  const float* norm_w[2];  // QKV: q, k
  float alpha;             // SCALED: the sums count this much (a power of two)
};

// What every role reads before its first tile comes first: a kernel starts with
// a cold constant cache, and each line it touches costs hundreds of cycles.
struct Params {
  int32_t n_seg, B, N, C, kblocks;
  int32_t bn;                // columns of a tile
  int32_t slots, rest_max;   // rest_max > 0: whole rounds of `slots` pair tiles, a rest of up to rest_max split
  int32_t cols, cols_q;      // column tiles of N; of the query part (QKV)
  int32_t rows[3], m_tiles[3], gated[3];
  int32_t K;
  const int32_t* mode;
  int32_t* err_word;
  uint64_t budget_ns;
  const float4* rope;  // [pos][d/4]: (cos, sin) of two consecutive pairs
  int32_t rope_len;
  float norm_eps;
  Seg seg[3];
  CUtensorMap tm_a[3], tm_w[3];
};

struct Tile {
  int seg, s, m0, n0;
};

constexpr int GROUP_M = 16;  // tile rows per band of the tile order

// Walks the live tiles in order; tile indices only grow. A piece is the tiles
// of one (segment, sample): all column tiles, or none when the segment is gated
// and the sample reuses, or only the query's (QKV at the boundary, which keeps
// its cached K and V).
template <int TM, int EPI>  // TM: output rows per tile, 128 (one CTA) or 256 (a CTA pair)
struct Walk {
  int g = 0, s = 0, cols = -1;  // cols: column tiles of the piece
  int64_t begin = 0;            // first tile of the piece

  __device__ __forceinline__ int piece_cols(const Params& p) const {
    if (p.gated[g]) {
      const int m = p.mode[s];
      if (m == RA_MODE_REUSE) return 0;
      if (EPI == RA_EPI_QKV && m == RA_MODE_BOUNDARY) return p.cols_q;
    }
    return p.cols;
  }
  // Tile t, or false past the last one.
  __device__ __forceinline__ bool at(const Params& p, int64_t t, Tile& r) {
    if (cols < 0) cols = piece_cols(p);
    while (t - begin >= int64_t(p.m_tiles[g]) * cols) {
      begin += int64_t(p.m_tiles[g]) * cols;
      ++s;
      if (p.m_tiles[g] == 0) {
        s = p.B;
      } else if (p.B > 4 && !p.gated[g] && t - begin <= 0xffffffff) {
        // the samples' pieces are alike: count them off at once
        const uint32_t n = uint32_t(p.m_tiles[g]) * uint32_t(cols), k = uint32_t(t - begin) / n;
        const int pass = int(min(k, uint32_t(p.B - s)));
        begin += int64_t(n) * pass;
        s += pass;
      }
      if (s == p.B) {
        s = 0;
        if (++g == p.n_seg) return false;
      }
      cols = piece_cols(p);
    }
    r.seg = g;
    r.s = s;
    const uint32_t rem = uint32_t(t - begin);
    // Grouped order: bands of GROUP_M tile rows, rows fastest inside a band, so
    // the tiles in flight at once (one per CTA pair) share a few A row blocks
    // and a few W column blocks that stay in L2, and W streams from HBM once per
    // band instead of once per wave.
    const uint32_t band_tiles = uint32_t(GROUP_M) * uint32_t(cols);
    const uint32_t band = rem / band_tiles, idx = rem - band * band_tiles;
    const int m_first = int(band) * GROUP_M;
    const uint32_t rows = uint32_t(min(GROUP_M, p.m_tiles[g] - m_first));
    r.m0 = (m_first + int(idx % rows)) * TM;
    r.n0 = int(idx / rows) * p.bn;
    return true;
  }
};

// The tiles of a call's whole rounds; those past them, if at most p.rest_max, are
// its rest. Every tile where the call has no rest.
template <int TM, int EPI>
__device__ __forceinline__ int64_t round_tiles(const Params& p) {
  if (p.rest_max == 0) return INT64_MAX;
  Walk<TM, EPI> w;
  int64_t live = 0;
  for (w.g = 0; w.g < p.n_seg; ++w.g)
    for (w.s = 0; w.s < p.B; ++w.s) live += int64_t(p.m_tiles[w.g]) * w.piece_cols(p);
  const int64_t rest = live % p.slots;
  return rest <= p.rest_max ? live - rest : live;
}

// The tile of item t of a launch. SPLIT: where the call has a rest, a quarter
// (128 rows by REST_BN columns) of a pair tile of it; p.m_tiles and p.bn are the
// pair kernel's then.
constexpr int REST_BN = 128;
template <int EPI, bool SPLIT>
__device__ __forceinline__ bool tile_at(const Params& p, Walk<BM, EPI>& walk, int64_t t, Tile& tl) {
  if (!SPLIT || p.rest_max == 0) return walk.at(p, t, tl);
  if (!walk.at(p, round_tiles<P_TM, EPI>(p) + (t >> 2), tl)) return false;
  tl.m0 = 2 * tl.m0 + (t & 1 ? BM : 0);
  tl.n0 += t & 2 ? REST_BN : 0;
  return tl.m0 < p.rows[tl.seg];
}

// GELU, tanh form, of two values through the identity
// 0.5 x (1 + tanh(u)) = x / (1 + e^(-2u)), u = sqrt(2/pi) (x + 0.044715 x^3),
// with e^(-2u) = 2^(x (c + 0.044715 c x^2)), c = -2 sqrt(2/pi) log2(e): one
// exponential and one reciprocal (an exponential that overflows to +inf for
// very negative x gives -0).
__device__ __forceinline__ void gelu_tanh2(float& x0, float& x1) {
  constexpr float c = -2.f * 0.7978845608028654f * 1.4426950408889634f;
  const uint64_t x = f2_pack(x0, x1);
  float z0, z1;
  f2_unpack(f2_mul(x, f2_fma(f2_mul(x, x), f2_pack(0.044715f * c, 0.044715f * c), f2_pack(c, c))), z0, z1);
  float d0, d1;
  f2_unpack(f2_add(f2_pack(ex2_approx(z0), ex2_approx(z1)), f2_pack(1.f, 1.f)), d0, d1);
  f2_unpack(f2_mul(x, f2_pack(rcp_approx(d0), rcp_approx(d1))), x0, x1);
}

// What an epilogue warp works on: its 32 rows (row0 + lane, nrow of them in
// the segment), its share of the tile's columns (half 0 or 1), its shared
// memory (staging buffer, two vectors of 128 per-column values) and the TMEM
// address of its lanes in the tile's accumulator; cols: columns of the tile.
struct EpiWarp {
  int row0, nrow, half, cols;
  uint8_t* stage;
  float* vec0;
  float* vec1;
  uint32_t acc;
};

// 32 accumulators, SCALED: times alpha, plus 32 per-column values from shared memory.
template <bool SCALED>
__device__ __forceinline__ void add_cols(const uint32_t (&v)[32], float alpha, const float* cols, float (&x)[32]) {
  const float4* c4 = reinterpret_cast<const float4*>(cols);
  auto sum = [&](uint32_t a, float c) { return SCALED ? fmaf(__uint_as_float(a), alpha, c) : __uint_as_float(a) + c; };
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float4 c = c4[i];
    x[4 * i] = sum(v[4 * i], c.x);
    x[4 * i + 1] = sum(v[4 * i + 1], c.y);
    x[4 * i + 2] = sum(v[4 * i + 2], c.z);
    x[4 * i + 3] = sum(v[4 * i + 3], c.w);
  }
}

// STORE, GELU, RESID: chunk j of the warp is tile columns 32 (half + 2 j) ...
template <int EPI, class Ready>
__device__ __forceinline__ bool epilogue_linear(const Params& p, const Tile& tl, const EpiWarp& w, Ready ready) {
  const Seg& sg = p.seg[tl.seg];
  const int lane = threadIdx.x & 31, n0 = tl.n0 + 32 * w.half;
  // this warp's; the last tile of a row may reach past N (a multiple of 32)
  const int chunks = (min(w.cols, p.N - tl.n0) / 32 + 1 - w.half) >> 1;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (j >= chunks) break;
    w.vec0[32 * j + lane] = sg.bias ? sg.bias[n0 + 64 * j + lane] : 0.f;
    if (EPI == RA_EPI_RESID) w.vec1[32 * j + lane] = sg.gate[int64_t(tl.s) * sg.gate_ss + n0 + 64 * j + lane];
  }
  const char* res = nullptr;
  uint4 ra[4], rb[4];  // residuals of the next even and odd chunk
  if (EPI == RA_EPI_RESID && chunks > 0) {
    res = reinterpret_cast<const char*>(sg.resid + int64_t(tl.s) * sg.res_ss + int64_t(w.row0) * sg.res_sr + n0);
    rows_fetch(res, 2 * sg.res_sr, w.nrow, ra);
    if (chunks > 1) rows_fetch(res + 128, 2 * sg.res_sr, w.nrow, rb);
  }
  char* out = reinterpret_cast<char*>(sg.out + int64_t(tl.s) * sg.out_ss + int64_t(w.row0) * sg.out_sr + n0);
  __syncwarp();
  if (!ready()) return false;
  if (w.nrow <= 0 || chunks <= 0) return true;
  uint32_t v[32];
  if (EPI != RA_EPI_RESID) tmem_ld32(w.acc + 32 * w.half, v);
  auto chunk = [&](int j, uint4 (&rc)[4]) {
    float x[32];
    uint4 r[4];
    if (EPI == RA_EPI_RESID) {
      // Residuals two chunks ahead (one ahead left about 1000 cycles of global
      // latency in every chunk); the accumulators are not loaded ahead in
      // exchange, the registers allow one of the two without spills.
      tmem_ld32(w.acc + 32 * w.half + 64 * j, v);
      rows_turn(w.stage, rc, r);
      if (j + 2 < chunks) rows_fetch(res + 128 * (j + 2), 2 * sg.res_sr, w.nrow, rc);
    }
    tmem_ld_wait_for(v);
    add_cols<false>(v, 1.f, w.vec0 + 32 * j, x);
    if (EPI != RA_EPI_RESID && j + 1 < chunks) tmem_ld32(w.acc + 32 * w.half + 64 * (j + 1), v);
    if (EPI == RA_EPI_GELU) {
#pragma unroll
      for (int i = 0; i < 32; i += 2) gelu_tanh2(x[i], x[i + 1]);
    } else if (EPI == RA_EPI_RESID) {
      const float4* g4 = reinterpret_cast<const float4*>(w.vec1 + 32 * j);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t rw[4] = {r[q].x, r[q].y, r[q].z, r[q].w};
        const float4 g0 = g4[2 * q], g1 = g4[2 * q + 1];
        const float gv[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[8 * q + 2 * e] = fmaf(gv[2 * e], x[8 * q + 2 * e], __uint_as_float(rw[e] << 16));
          x[8 * q + 2 * e + 1] = fmaf(gv[2 * e + 1], x[8 * q + 2 * e + 1], __uint_as_float(rw[e] & 0xFFFF0000u));
        }
      }
    }
    rows_store(w.stage, x, out + 128 * j, 2 * sg.out_sr, w.nrow);
  };
#pragma unroll 1
  for (int j = 0; j < chunks; j += 2) {
    chunk(j, ra);
    if (j + 1 < chunks) chunk(j + 1, rb);
  }
  return true;
}

// QKV: heads half, half + 2, ... of the tile.
template <int D, class Ready>
__device__ __forceinline__ bool epilogue_qkv(const Params& p, const Tile& tl, const EpiWarp& w, Ready ready) {
  constexpr int CH = D / 32;
  const int heads = (p.bn / D + 1 - w.half) >> 1;  // this warp's
  const Seg& sg = p.seg[tl.seg];
  const int lane = threadIdx.x & 31;
  const int part = tl.n0 / p.C;  // 0 q, 1 k, 2 v
  const int h0 = (tl.n0 - part * p.C) / D + w.half;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (j / CH >= heads) break;
    const int c = 32 * (j % CH) + lane;  // column within head h0 + 2 (j / CH)
    w.vec0[32 * j + lane] = sg.bias ? sg.bias[part * p.C + (h0 + 2 * (j / CH)) * D + c] : 0.f;
    if (part < 2) w.vec1[32 * j + lane] = sg.norm_w[part][c];
  }
  __syncwarp();
  // RoPE rows of the warp's positions: (cos, sin) of D / 2 pairs, 64 bytes = 16 columns at a time
  const char* rope = reinterpret_cast<const char*>(p.rope + int64_t(sg.pos_offset + w.row0) * (D / 4));
  uint4 cnext[4];
  if (part < 2) rows_fetch(rope, 4 * D, w.nrow, cnext);
  if (!ready()) return false;
  if (w.nrow <= 0 || heads <= 0) return true;
  char* dst0 = reinterpret_cast<char*>(sg.dst[part] + tl.s * sg.dst_sb[part] + int64_t(w.row0) * sg.dst_sn[part]);
#pragma unroll 1
  for (int hh = 0; hh < heads; ++hh) {
    const uint32_t acc = w.acc + (w.half + 2 * hh) * D;
    const float* bias = w.vec0 + 32 * CH * hh;
    const float* nw = w.vec1 + 32 * CH * hh;
    uint32_t v[32];
    float rstd = 0.f;
    tmem_ld32(acc, v);
    if (part < 2) {
      // a first pass over the head's accumulators for the mean square
      float s0 = 0.f, s1 = 0.f;
#pragma unroll 1
      for (int c = 0; c < CH; ++c) {
        float x[32];
        tmem_ld_wait_for(v);
        add_cols<false>(v, 1.f, bias + 32 * c, x);
        tmem_ld32(acc + 32 * ((c + 1) % CH), v);
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
          s0 = fmaf(x[i], x[i], s0);
          s1 = fmaf(x[i + 1], x[i + 1], s1);
        }
      }
      rstd = rsqrtf((s0 + s1) / float(D) + p.norm_eps);
    }
    char* dst = dst0 + 2 * int64_t(h0 + 2 * hh) * sg.dst_sh[part];
#pragma unroll 1
    for (int c = 0; c < CH; ++c) {
      float x[32];
      tmem_ld_wait_for(v);
      add_cols<false>(v, 1.f, bias + 32 * c, x);
      if (c + 1 < CH) tmem_ld32(acc + 32 * (c + 1), v);
      if (part < 2) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint4 own[4];
          rows_turn(w.stage, cnext, own);
          // the next 16 columns' table entries (the next head starts over)
          const int nx = (2 * c + hf + 1) % (2 * CH);
          if (nx != 0 || hh + 1 < heads) rows_fetch(rope + 64 * nx, 4 * D, w.nrow, cnext);
          const float4* w4 = reinterpret_cast<const float4*>(nw + 32 * c + 16 * hf);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 wv = w4[q];
            const float cs[4] = {__uint_as_float(own[q].x), __uint_as_float(own[q].y), __uint_as_float(own[q].z),
                                 __uint_as_float(own[q].w)};
            float* xe = &x[16 * hf + 4 * q];
            const float a0 = xe[0] * rstd * wv.x, a1 = xe[1] * rstd * wv.y;
            const float b0 = xe[2] * rstd * wv.z, b1 = xe[3] * rstd * wv.w;
            xe[0] = a0 * cs[0] - a1 * cs[1];
            xe[1] = a0 * cs[1] + a1 * cs[0];
            xe[2] = b0 * cs[2] - b1 * cs[3];
            xe[3] = b0 * cs[3] + b1 * cs[2];
          }
        }
      }
      rows_store(w.stage, x, dst + 64 * c, 2 * sg.dst_sn[part], w.nrow);
    }
  }
  return true;
}

// Epilogue of one warp's share of an output tile; ready() waits for the
// accumulator (false: the wait was given up). D: head dim (QKV).
template <int EPI, int D, class Ready>
__device__ __forceinline__ bool epilogue_tile(const Params& p, const Tile& tl, const EpiWarp& w, Ready ready) {
  if constexpr (EPI == RA_EPI_QKV)
    return epilogue_qkv<D>(p, tl, w, ready);
  else
    return epilogue_linear<EPI>(p, tl, w, ready);
}

// A split tile: each CTA of the cluster has the sums over its part of K in its
// own TMEM; afterwards rank r has columns [r, r + 1) * bn / cs of the whole sums
// there. Each rank hands every other rank that one's columns, in fp32, by a bulk
// copy between the CTAs' shared memory (the stages are idle by then), and adds
// its own columns up in rank order. Every thread of the cluster takes part in
// the cluster barrier: before it every rank's barriers exist, its stages are idle
// and its parts are written, after it they are copied (a cluster barrier of its
// own in the set-up cost 0.2 us). ok: this warp's accumulator is complete. Every
// rank sends and waits for what it receives, also after a wait of this CTA was
// given up: no CTA exits with a copy into it, or out of it, in flight.
// The merge of a 128 x 256 tile between two CTAs (64 KB each way) takes 2.6 us.
__device__ __forceinline__ bool merge_parts(const WaitCtl& ctl, uint8_t* smem, uint64_t* parts_full, uint32_t acc,
                                            bool ok, int bn, int half, int quarter, int rank, int cs) {
  const int lane = threadIdx.x & 31, row = quarter * 32 + lane;
  const int cw = bn / cs;                            // columns per rank
  const uint32_t part_bytes = uint32_t(BM) * cw * 4;  // [column / 4][row] of 16 bytes
  uint8_t* send = smem;                              // parts for the other ranks, in rank order
  uint8_t* recv = smem + (cs - 1) * part_bytes;      // parts from the other ranks, in rank order
  const bool leader = quarter == 0 && half == 0 && lane == 0;
  if (leader) mbar_arrive_expect_tx(parts_full, (cs - 1) * part_bytes);
#pragma unroll 1
  for (int c0 = 32 * half; c0 < bn; c0 += 64) {
    const int q = c0 / cw;
    if (q == rank) continue;
    uint32_t v[32];
    tmem_ld32(acc + c0, v);
    tmem_ld_wait_for(v);
    if (!ok) {  // what was given up is NaN on every rank
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = 0x7fffffffu;
    }
    uint4* dst = reinterpret_cast<uint4*>(send + (q - (q > rank ? 1 : 0)) * part_bytes) +
                 ((c0 - q * cw) >> 2) * BM + row;
#pragma unroll
    for (int i = 0; i < 32; i += 4) dst[(i >> 2) * BM] = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  }
  fence_proxy_async_smem();  // the parts are next read by bulk copies
  cluster_sync_all();
  if (leader)
    for (int q = 0; q < cs; ++q)
      if (q != rank)
        bulk_copy_to_cta(mapa_shared(smem_u32(recv + (rank - (rank > q ? 1 : 0)) * part_bytes), q),
                         send + (q - (q > rank ? 1 : 0)) * part_bytes, part_bytes,
                         mapa_shared(smem_u32(parts_full), q));
  const bool got = __all_sync(0xffffffffu, mbar_wait(parts_full, 0, ctl) ||
                                               mbar_wait_drain(parts_full, 0, ctl.budget_ns));
  if (!got || !ok) return false;
#pragma unroll 1
  for (int c0 = 32 * half; c0 < cw; c0 += 64) {
    uint32_t v[32];
    float x[32];
    tmem_ld32(acc + rank * cw + c0, v);
    tmem_ld_wait_for(v);
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = 0.f;
#pragma unroll 1
    for (int r = 0; r < cs; ++r) {
      const float4* src = reinterpret_cast<const float4*>(recv + (r - (r > rank ? 1 : 0)) * part_bytes) +
                          (c0 >> 2) * BM + row;
#pragma unroll
      for (int i = 0; i < 32; i += 4) {
        const float4 y = r == rank ? make_float4(__uint_as_float(v[i]), __uint_as_float(v[i + 1]),
                                                 __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]))
                                   : src[(i >> 2) * BM];
        x[i] += y.x;
        x[i + 1] += y.y;
        x[i + 2] += y.z;
        x[i + 3] += y.w;
      }
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(x[i]);
    tmem_st32(acc + rank * cw + c0, v);
  }
  tmem_st_wait();
  return true;
}

inline bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

// Launches `ctas` CTAs in clusters of cs.
template <class P>
ra_status launch(const char* who, const P& p, void (*fn)(P), int smem, int64_t ctas, int cs, cudaStream_t st,
                 int threads = THREADS, int most_smem = 0) {
  const ra_status as =
      ensure_dynamic_smem(reinterpret_cast<const void*>(fn), most_smem > smem ? most_smem : smem, who);
  if (as != RA_OK) return as;
  cudaLaunchAttribute attr[2];
  attr[0] = pdl_attribute();
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cs;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(unsigned(ctas), 1, 1);
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = cs > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, p);
  if (e != cudaSuccess) {
    set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
    cudaGetLastError();
    return RA_ECUDA;
  }
  return launch_status(who);
}


// A segment's epilogue tensors, checked (Args: ra_gemm_args or ra_gemm4_args); false: the reason is recorded.
template <class Args>
bool fill_epilogue(const char* who, const Args& a, int g, const ra_gemm_seg& s, Seg& d) {
  d.pos_offset = s.pos_offset;
  d.bias = s.bias;
  d.alpha = 1.f;
  if (s.bias && !aligned16(s.bias)) {
    set_error("%s: seg %d: bias must be 16-byte aligned", who, g);
    return false;
  }
  if (a.epilogue == RA_EPI_QKV) {
    const ra_seg* dst[3] = {&s.q_out, &s.k_out, &s.v_out};
    const char* nm[3] = {"q_out", "k_out", "v_out"};
    for (int z = 0; z < 3; ++z) {
      if (dst[z]->n != s.rows || !check_seg(*dst[z], nm[z], false)) {
        if (dst[z]->n != s.rows) set_error("%s: seg %d: %s.n must equal rows", who, g, nm[z]);
        return false;
      }
      d.dst[z] = static_cast<__nv_bfloat16*>(dst[z]->ptr);
      d.dst_sb[z] = dst[z]->stride_b;
      d.dst_sh[z] = dst[z]->stride_h;
      d.dst_sn[z] = dst[z]->stride_n;
    }
    if (!s.q_norm || !s.k_norm || !aligned16(s.q_norm) || !aligned16(s.k_norm)) {
      set_error("%s: seg %d: QKV needs 16-byte aligned q_norm and k_norm", who, g);
      return false;
    }
    if (s.pos_offset < 0 || int64_t(s.pos_offset) + s.rows > a.rope_len) {
      set_error("%s: seg %d: positions [%d, %d) outside the rope table (%d)", who, g, s.pos_offset,
                s.pos_offset + s.rows, a.rope_len);
      return false;
    }
    d.norm_w[0] = s.q_norm;
    d.norm_w[1] = s.k_norm;
  } else {
    if (!s.out || !aligned16(s.out) || s.out_stride_r % 8 != 0 || s.out_stride_s % 8 != 0 ||
        s.out_stride_r < a.N) {
      set_error("%s: seg %d: out must be 16-byte aligned with strides multiples of 8 elements, "
                "out_stride_r >= N", who, g);
      return false;
    }
    d.out = static_cast<__nv_bfloat16*>(s.out);
    d.out_ss = s.out_stride_s;
    d.out_sr = s.out_stride_r;
    if (a.epilogue == RA_EPI_RESID) {
      if (!s.resid || !s.gate || !aligned16(s.resid) || !aligned16(s.gate) || s.resid_stride_r % 8 != 0 ||
          s.resid_stride_s % 8 != 0 || s.gate_stride_s % 4 != 0) {
        set_error("%s: seg %d: RESID needs 16-byte aligned resid and gate, resid strides "
                  "multiples of 8 elements, gate_stride_s of 4", who, g);
        return false;
      }
      d.resid = static_cast<const __nv_bfloat16*>(s.resid);
      d.res_ss = s.resid_stride_s;
      d.res_sr = s.resid_stride_r;
      d.gate = s.gate;
      d.gate_ss = s.gate_stride_s;
    }
  }
  return true;
}

}  // namespace gemm
}  // namespace ra
