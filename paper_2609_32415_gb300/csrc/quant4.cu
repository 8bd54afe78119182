// refadapt_quant4: bf16 rows to microscaled 4 bits, along the features, along the rows
// (the transposed matrix), or both; and refadapt_linear4_backward, which is that and two
// products of gemm4.cu.
//
// Per block of 16 (e4m3 scales) or 32 (e8m0) values: amax, the scale s, and x / s rounded to
// e2m1. Quotients: x has 8 significant bits, s four, and the borders between two e2m1 values
// (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5) three, so x / s is a border or at least 2^-15 of
// it away. Hence x times 1/s rounded up, the product cut towards zero, falls on the border
// exactly where x / s does (an excess below one unit in the last place is cut off) and on
// the right side elsewhere: one multiplication a value, and the conversion instruction.
//
// 2 bytes read and 0.53 to 0.56 written a value. Along the features memory bounds it (16384 x 4096 in 28.5 us, 6 TB/s),
// along the rows the instructions' issue (tokens_kernel).
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstring>

#include "api_common.h"
#include "gemm4.h"
#include "launch_plan.h"
#include "tc_ptx.cuh"

namespace ra {
namespace quant4 {

constexpr int THREADS = 256;
constexpr int ROWS = 32, COLS = 256;  // of a CTA, along the features
constexpr int T_TOKENS = 128, T_COLS = 64;  // of a CTA, along the rows

struct Block {
  uint32_t byte;  // as stored
  float factor;   // x times this, cut towards zero, is rounded to e2m1
};

// The scale of a block whose largest magnitude has the bf16 bits `amax`; down = 2^-exponent.
template <bool E8M0>
__device__ __forceinline__ Block block_scale(uint32_t amax, float down) {
  if (amax >= 0x7f80u) return Block{E8M0 ? 0xffu : 0x7fu, 0.f};
  if (E8M0) {
    // amax = m 2^a, m in [1, 2): 6 2^e covers it from e = a - 2 (m <= 1.5) or a - 1
    const int byte = max(1, int((amax << 16) + 0x3fffffu >> 23) - 2);
    return Block{uint32_t(byte), __uint_as_float(uint32_t(254 - byte) << 23)};
  }
  const float top = __uint_as_float(amax << 16) * down;
  const uint32_t byte = __nv_cvt_float_to_fp8(__fdiv_rn(top, 6.f), __NV_SATFINITE, __NV_E4M3);
  const float s = __half2float(__half(__nv_cvt_fp8_to_halfraw(__nv_fp8_storage_t(byte), __NV_E4M3)));
  return Block{byte, byte ? __frcp_ru(s) * down : 0.f};
}

// Eight values to e2m1, the first in the lowest bits.
__device__ __forceinline__ uint32_t to_e2m1(const float (&x)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return r;
}
// Two values times a factor, cut towards zero.
__device__ __forceinline__ uint64_t mul2_rz(uint64_t x, uint64_t f) {
  uint64_t r;
  asm("mul.rz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(f));
  return r;
}
// Eight bf16 in four words.
__device__ __forceinline__ uint32_t codes_of(const uint32_t (&w)[4], float factor) {
  const uint64_t f = f2_pack(factor, factor);
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) f2_unpack(mul2_rz(bf2_unpack(w[i]), f), x[2 * i], x[2 * i + 1]);
  return to_e2m1(x);
}
// The larger magnitudes of two pairs of bf16 (NaN above infinity above the rest); the signs of the
// result say nothing.
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {
  uint32_t m;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  return m;
}
__device__ __forceinline__ uint32_t top2(uint32_t a) { return max(a & 0x7fffu, (a >> 16) & 0x7fffu); }

struct Seg {
  const char* x;
  int64_t x_ss, x_sr;  // bytes
  uint8_t* codes;
  int64_t c_ss, c_sr;
  uint8_t* scales;
  uint8_t* codes_t;
  int64_t t_stride;
  uint8_t* scales_t;
  int32_t rows, gated;
  float down;          // 2^-exponent
  int32_t samples;     // along the rows: of the matrix
  int32_t C;
  int64_t first;       // CTA of the launch that the segment starts with
};
struct Params {
  int32_t n_seg, B, C;
  Seg seg[3];
  const int32_t* mode;
};

// Blocks along the features. A CTA: 32 rows of one sample (those behind its last, up to a
// multiple of 128, have zero scales) by 256 columns; a thread: 16 columns of two rows.
template <bool E8M0>
__global__ void __launch_bounds__(THREADS) rows_kernel(const __grid_constant__ Params p) {
  pdl_wait();
  pdl_launch();
  int g = 0;
  while (g + 1 < p.n_seg && int64_t(blockIdx.x) >= p.seg[g + 1].first) ++g;
  const Seg& sg = p.seg[g];
  const uint32_t at = blockIdx.x - uint32_t(sg.first);
  const uint32_t col_tiles = (p.C + COLS - 1) / COLS, row_tiles = 4 * uint32_t((sg.rows + 127) / 128);
  const uint32_t ct = at % col_tiles, rest = at / col_tiles, rt = rest % row_tiles, s = rest / row_tiles;
  if (sg.gated && p.mode[s] == RA_MODE_REUSE) return;
  const int unit = threadIdx.x & 15, col = int(ct) * COLS + 16 * unit;
  constexpr int GROUP = E8M0 ? 128 : 64;  // columns of a scale tile
  const int64_t groups = (p.C + GROUP - 1) / GROUP;
  uint8_t* tiles = sg.scales + (int64_t(s) * (row_tiles / 4) + rt / 4) * groups * 512;
  uint4 v[2][2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int row = int(rt) * ROWS + (threadIdx.x >> 4) + 16 * k;
    const bool on = row < sg.rows && col < p.C;
    const uint4* src = reinterpret_cast<const uint4*>(sg.x + s * sg.x_ss + row * sg.x_sr + 2 * int64_t(col));
    v[k][0] = on ? src[0] : make_uint4(0, 0, 0, 0);
    v[k][1] = on ? src[1] : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int row = int(rt) * ROWS + (threadIdx.x >> 4) + 16 * k;
    const bool on = row < sg.rows && col < p.C;
    const uint32_t a[4] = {v[k][0].x, v[k][0].y, v[k][0].z, v[k][0].w}, b[4] = {v[k][1].x, v[k][1].y, v[k][1].z, v[k][1].w};
    uint32_t m = top2(max_abs2(max_abs2(max_abs2(a[0], a[1]), max_abs2(a[2], a[3])),
                               max_abs2(max_abs2(b[0], b[1]), max_abs2(b[2], b[3]))));
    if (E8M0) m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    const Block blk = block_scale<E8M0>(m, sg.down);
    if (on)
      *reinterpret_cast<uint2*>(sg.codes + s * sg.c_ss + row * sg.c_sr + col / 2) =
          make_uint2(codes_of(a, blk.factor), codes_of(b, blk.factor));
    // four blocks' bytes, in the first of their threads
    uint32_t w = on ? blk.byte : 0u;
    if (E8M0) {
      w |= __shfl_down_sync(0xffffffffu, w, 2) << 8;
      w |= __shfl_down_sync(0xffffffffu, w, 4) << 16;
    } else {
      w |= __shfl_down_sync(0xffffffffu, w, 1) << 8;
      w |= __shfl_down_sync(0xffffffffu, w, 2) << 16;
    }
    const int64_t group = col / GROUP;
    if ((unit & (E8M0 ? 7 : 3)) == 0 && group < groups)
      *reinterpret_cast<uint32_t*>(tiles + group * 512 + 16 * (row & 31) + 4 * ((row >> 5) & 3)) = w;
  }
}

// Blocks along the rows (tokens: all samples' rows, one after another), and along the
// features where codes are wanted too. A CTA: 128 tokens by 64 columns, kept in shared
// memory, 16 KB. A thread loads 16 columns of two tokens (and rounds them along the features),
// then takes two columns of 16 tokens from there, a word of both a token; the eight threads of
// a column pair write 64 contiguous bytes of each column. 16-byte pieces of a token are permuted by
// its group of 16 and its parity, which keeps both accesses free of conflicts.
// Bound by instruction issue (77 % of the slots, memory 51 %): 13 to 15 instructions a value, 16384 x 4096 in both
// forms 41 us; 24 and 48 us where a thread took 8 columns and then 32 tokens of one column with 16-bit loads.
template <bool E8M0>
__global__ void __launch_bounds__(THREADS) tokens_kernel(const __grid_constant__ Params p) {
  __shared__ __align__(16) uint8_t tile[T_TOKENS * T_COLS * 2];
  auto piece_at = [&](int token, int piece) {
    return reinterpret_cast<uint4*>(tile + token * (T_COLS * 2) + ((piece ^ (token >> 4) ^ (token & 1)) << 4));
  };
  pdl_wait();
  pdl_launch();
  int g = 0;
  while (g + 1 < p.n_seg && int64_t(blockIdx.x) >= p.seg[g + 1].first) ++g;
  const Seg& sg = p.seg[g];
  const uint32_t at = blockIdx.x - uint32_t(sg.first);
  const uint32_t col_tiles = (sg.C + T_COLS - 1) / T_COLS;
  const int ct = int(at % col_tiles), tt = int(at / col_tiles);
  const int tokens = sg.rows * sg.samples, c0 = ct * T_COLS, t0 = tt * T_TOKENS;
  {
    const int unit = threadIdx.x & 3, col = c0 + 16 * unit;
    uint4 v[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int t = t0 + (threadIdx.x >> 2) + 64 * k;
      const uint32_t s = sg.samples > 1 ? uint32_t(t) / uint32_t(sg.rows) : 0u, r = uint32_t(t) - s * uint32_t(sg.rows);
      const uint4* src = reinterpret_cast<const uint4*>(sg.x + s * sg.x_ss + r * sg.x_sr + 2 * int64_t(col));
      v[k][0] = t < tokens && col < sg.C ? src[0] : make_uint4(0, 0, 0, 0);  // C is a multiple of 8
      v[k][1] = t < tokens && col + 8 < sg.C ? src[1] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int tl = (threadIdx.x >> 2) + 64 * k, t = t0 + tl;
      *piece_at(tl, 2 * unit) = v[k][0];
      *piece_at(tl, 2 * unit + 1) = v[k][1];
      if (sg.codes) {
        const uint32_t a[4] = {v[k][0].x, v[k][0].y, v[k][0].z, v[k][0].w};
        const uint32_t b[4] = {v[k][1].x, v[k][1].y, v[k][1].z, v[k][1].w};
        uint32_t m = top2(max_abs2(max_abs2(max_abs2(a[0], a[1]), max_abs2(a[2], a[3])),
                                   max_abs2(max_abs2(b[0], b[1]), max_abs2(b[2], b[3]))));
        if (E8M0) m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        const Block blk = block_scale<E8M0>(m, sg.down);
        const bool on = t < tokens && col < sg.C;  // C is a multiple of 64 here
        if (on)
          *reinterpret_cast<uint2*>(sg.codes + t * sg.c_sr + col / 2) =
              make_uint2(codes_of(a, blk.factor), codes_of(b, blk.factor));
        // the scale tile of these 128 tokens: e4m3 four blocks are its 64 columns, e8m0 two are half of 128
        uint32_t w = on ? blk.byte : 0u;
        constexpr int GROUP = E8M0 ? 128 : 64;
        const int64_t groups = (sg.C + GROUP - 1) / GROUP;
        uint8_t* dst = sg.scales + (tt * groups + c0 / GROUP) * 512 + 16 * (tl & 31) + 4 * ((tl >> 5) & 3);
        if (E8M0) {
          w |= __shfl_down_sync(0xffffffffu, w, 2) << 8;
          if (unit == 0) {
            if (ct & 1)
              *reinterpret_cast<uint16_t*>(dst + 2) = uint16_t(w);
            else if (ct + 1 == int(col_tiles))
              *reinterpret_cast<uint32_t*>(dst) = w & 0xffffu;
            else
              *reinterpret_cast<uint16_t*>(dst) = uint16_t(w);
          }
        } else {
          w |= __shfl_down_sync(0xffffffffu, w, 1) << 8;
          w |= __shfl_down_sync(0xffffffffu, w, 2) << 16;
          if (unit == 0) *reinterpret_cast<uint32_t*>(dst) = w;
        }
      }
    }
  }
  if (!sg.codes_t) return;
  __syncthreads();
  const int tg = threadIdx.x & 7, pair = threadIdx.x >> 3, col = c0 + 2 * pair;  // 16 tokens from 16 tg on; C is even
  const int padded = (tokens + 63) / 64 * 64, first = t0 + 16 * tg;
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = reinterpret_cast<const uint32_t*>(piece_at(16 * tg + i, pair >> 2))[pair & 3];
  uint32_t m = w[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) m = max_abs2(m, w[i]);
  uint32_t top[2] = {m & 0x7fffu, (m >> 16) & 0x7fffu};
  Block b[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    if (E8M0) top[c] = max(top[c], __shfl_xor_sync(0xffffffffu, top[c], 1));
    b[c] = block_scale<E8M0>(top[c], sg.down);
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const uint64_t f = f2_pack(b[c].factor, b[c].factor);
    uint32_t q[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const uint32_t lo = w[8 * h + i], hi = w[8 * h + i + 1];
        const uint64_t y = c == 0 ? f2_pack(__uint_as_float(lo << 16), __uint_as_float(hi << 16))
                                  : f2_pack(__uint_as_float(lo & 0xffff0000u), __uint_as_float(hi & 0xffff0000u));
        f2_unpack(mul2_rz(y, f), x[i], x[i + 1]);
      }
      q[h] = to_e2m1(x);
    }
    if (col < sg.C && first < padded)
      *reinterpret_cast<uint2*>(sg.codes_t + int64_t(col + c) * sg.t_stride + first / 2) = make_uint2(q[0], q[1]);
  }
  // Scales of the transposed matrix: 64 of a tile's 128 rows; those behind the last column are zero.
  // Four blocks' bytes of both columns meet in the first of their threads.
  constexpr int STEP = E8M0 ? 2 : 1;  // threads from block to block
  uint32_t e = b[0].byte | b[1].byte << 16;
  if (col >= sg.C || first >= padded) e = 0;
  e |= __shfl_down_sync(0xffffffffu, e, STEP) << 8;
  const uint32_t o = __shfl_down_sync(0xffffffffu, e, 2 * STEP);
  const int64_t groups = E8M0 ? (padded + 127) / 128 : padded / 64;
  const int64_t group = E8M0 ? tt : 2 * tt + tg / 4;
  const int rows_up = (sg.C + 127) / 128 * 128;
  if (tg % (4 * STEP) == 0 && group < groups) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = col + c;
      uint8_t* dst = sg.scales_t + (int64_t(r >> 7) * groups + group) * 512 + 16 * (r & 31) + 4 * ((r >> 5) & 3);
      *reinterpret_cast<uint32_t*>(dst) = c == 0 ? (e & 0xffffu) | o << 16 : e >> 16 | (o & 0xffff0000u);
      // the half tile behind the last columns has no CTA of its own
      if (ct + 1 == int(col_tiles) && c0 + T_COLS < rows_up) *reinterpret_cast<uint32_t*>(dst + 8) = 0;
    }
  }
}

inline bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

ra_status launch(const char* who, const Params& p, void (*fn)(Params), int64_t ctas, cudaStream_t st) {
  cudaLaunchAttribute attr[1] = {pdl_attribute()};
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(unsigned(ctas), 1, 1);
  cfg.blockDim = dim3(THREADS, 1, 1);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, p);
  if (e != cudaSuccess) {
    set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
    cudaGetLastError();
    return RA_ECUDA;
  }
  return launch_status(who);
}

int64_t rows_ctas(int64_t B, int64_t rows, int64_t C) {
  return B * ((rows + 127) / 128 * 4) * ((C + COLS - 1) / COLS);
}
int64_t tokens_ctas(int64_t tokens, int64_t C) {
  return (tokens + T_TOKENS - 1) / T_TOKENS * ((C + T_COLS - 1) / T_COLS);
}

// Along the rows; p.seg[].first is set here.
ra_status launch_tokens(const char* who, Params& p, int format, cudaStream_t st) {
  int64_t ctas = 0;
  for (int g = 0; g < p.n_seg; ++g) {
    p.seg[g].first = ctas;
    ctas += tokens_ctas(int64_t(p.seg[g].rows) * p.seg[g].samples, p.seg[g].C);
  }
  if (ctas == 0) return RA_OK;
  if (ctas > 2147483647) {
    set_error("%s: too many rows", who);
    return RA_EINVAL;
  }
  return launch(who, p, format == RA_Q4_E8M0 ? tokens_kernel<true> : tokens_kernel<false>, ctas, st);
}

}  // namespace quant4
}  // namespace ra

extern "C" size_t refadapt_quant4_scales_size(int32_t rows, int32_t K, int32_t format) {
  if (rows < 0 || K < 0 || (format != RA_Q4_E4M3 && format != RA_Q4_E8M0)) return 0;
  const size_t group = 4 * size_t(ra::block_of(format));
  return (size_t(rows) + 127) / 128 * ((size_t(K) + group - 1) / group) * 512;
}

extern "C" ra_status refadapt_quant4(const ra_quant4_args* a, void* stream) {
  using namespace ra;
  using namespace ra::quant4;
  clear_error();
  if (!a) {
    set_error("refadapt_quant4: args is NULL");
    return RA_EINVAL;
  }
  if (a->B < 1 || a->n_seg < 1 || a->n_seg > 3 || a->C < 8 || a->C % 8 != 0) {
    set_error("refadapt_quant4: need B >= 1, 1 <= n_seg <= 3, C a positive multiple of 8 (B=%d n_seg=%d C=%d)", a->B,
              a->n_seg, a->C);
    return RA_EINVAL;
  }
  if (a->format != RA_Q4_E4M3 && a->format != RA_Q4_E8M0) {
    set_error("refadapt_quant4: unknown format %d", a->format);
    return RA_EINVAL;
  }
  Params rows, tokens;  // segments along the features only, and the others
  std::memset(&rows, 0, sizeof(rows));
  rows.B = a->B;
  rows.C = a->C;
  rows.mode = a->mode;
  tokens = rows;
  int64_t ctas = 0;
  CallPlaces<12, 4> places;
  if (a->mode) places.reads(place_of(a->mode, int64_t(a->B) * 4));
  for (int g = 0; g < a->n_seg; ++g) {
    const ra_quant4_seg& s = a->seg[g];
    if (s.rows < 0 || int64_t(a->B) * s.rows >= (int64_t(1) << 30)) {
      set_error("refadapt_quant4: seg %d: rows need 0 <= rows and B * rows < 2^30", g);
      return RA_EINVAL;
    }
    if ((s.codes != nullptr) != (s.scales != nullptr) || (s.codes_t != nullptr) != (s.scales_t != nullptr)) {
      set_error("refadapt_quant4: seg %d: codes go with scales, codes_t with scales_t", g);
      return RA_EINVAL;
    }
    if (s.gated && (!a->mode || s.codes_t)) {
      set_error("refadapt_quant4: seg %d is gated but %s", g, a->mode ? "has codes_t" : "mode is NULL");
      return RA_EINVAL;
    }
    if (s.exponent < -64 || s.exponent > 64 || (a->format == RA_Q4_E8M0 && s.exponent != 0)) {
      set_error("refadapt_quant4: seg %d: exponent needs -64 to 64, and 0 for RA_Q4_E8M0 (%d)", g, s.exponent);
      return RA_EINVAL;
    }
    if (s.rows == 0) continue;
    if (!s.codes && !s.codes_t) {
      set_error("refadapt_quant4: seg %d has no outputs", g);
      return RA_EINVAL;
    }
    if (!s.x || !aligned16(s.x) || s.x_stride_r % 8 != 0 || s.x_stride_s % 8 != 0 || s.x_stride_r < a->C ||
        s.x_stride_s < 0) {
      set_error("refadapt_quant4: seg %d: x must be 16-byte aligned, strides multiples of 8 elements, x_stride_r >= C",
                g);
      return RA_EINVAL;
    }
    const int64_t n = int64_t(a->B) * s.rows, padded = (n + 63) / 64 * 64;
    if (s.codes) {
      if (a->C % 64 != 0 || !aligned16(s.codes) || !aligned16(s.scales) || s.codes_stride_r % 16 != 0 ||
          s.codes_stride_s % 16 != 0 || s.codes_stride_r < a->C / 2 || (a->B > 1 && s.codes_stride_s < 1)) {
        set_error("refadapt_quant4: seg %d: codes need C a multiple of 64, 16-byte aligned pointers, strides "
                  "multiples of 16 bytes, codes_stride_r >= C / 2", g);
        return RA_EINVAL;
      }
      places.writes(place_of(s.codes, a->C / 2, {a->B, s.codes_stride_s}, {s.rows, s.codes_stride_r}));
      places.writes(place_of(s.scales, a->B * int64_t(refadapt_quant4_scales_size(s.rows, a->C, a->format))));
    }
    if (s.codes_t) {
      if (!aligned16(s.codes_t) || !aligned16(s.scales_t) || s.codes_t_stride % 16 != 0 ||
          s.codes_t_stride < padded / 2) {
        set_error("refadapt_quant4: seg %d: codes_t need 16-byte aligned pointers and a stride that is a multiple of "
                  "16 bytes and holds all rows", g);
        return RA_EINVAL;
      }
      places.writes(place_of(s.codes_t, padded / 2, {a->C, s.codes_t_stride}));
      places.writes(place_of(s.scales_t, int64_t(refadapt_quant4_scales_size(a->C, int32_t(padded), a->format))));
    }
    places.reads(place_of(s.x, int64_t(a->C) * 2, {a->B, s.x_stride_s * 2}, {s.rows, s.x_stride_r * 2}));
    Seg d;
    std::memset(&d, 0, sizeof(d));
    d.x = static_cast<const char*>(s.x);
    d.x_ss = 2 * s.x_stride_s;
    d.x_sr = 2 * s.x_stride_r;
    d.codes = static_cast<uint8_t*>(s.codes);
    d.c_ss = s.codes_stride_s;
    d.c_sr = s.codes_stride_r;
    d.scales = static_cast<uint8_t*>(s.scales);
    d.codes_t = static_cast<uint8_t*>(s.codes_t);
    d.t_stride = s.codes_t_stride;
    d.scales_t = static_cast<uint8_t*>(s.scales_t);
    d.rows = s.rows;
    d.gated = s.gated ? 1 : 0;
    d.down = ldexpf(1.f, -s.exponent);
    d.samples = a->B;
    d.C = a->C;
    // One sample's rows are read once for both; the scale tiles of several do not lie
    // with 128 tokens, so these take a pass each.
    const bool both = s.codes && s.codes_t && a->B == 1;
    if (s.codes && !both) {
      d.first = ctas;
      ctas += rows_ctas(a->B, s.rows, a->C);
      rows.seg[rows.n_seg++] = d;
    }
    if (s.codes_t) {
      if (!both) d.codes = nullptr;
      tokens.seg[tokens.n_seg++] = d;
    }
  }
  if (places.clash()) {
    set_error("refadapt_quant4: an output overlaps an input, another output or itself");
    return RA_EINVAL;
  }
  if (ctas > 2147483647) {
    set_error("refadapt_quant4: too many rows");
    return RA_EINVAL;
  }
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (ctas > 0) {
    const ra_status r =
        launch("refadapt_quant4", rows, a->format == RA_Q4_E8M0 ? rows_kernel<true> : rows_kernel<false>, ctas, st);
    if (r != RA_OK) return r;
  }
  return tokens.n_seg > 0 ? launch_tokens("refadapt_quant4", tokens, a->format, st) : RA_OK;
}

// ------------------------------------------------------------------ gradients of a layer
namespace ra {
namespace linear4 {

// A 4-bit matrix in the workspace.
struct Matrix {
  size_t codes, scales;  // offsets
};
struct Plan {
  Matrix dy, wt, dyt, xt;
  size_t bytes;
  int64_t tokens;  // padded to 64
};
Plan plan(int64_t n, int32_t K, int32_t N) {
  Plan p;
  p.tokens = (n + 63) / 64 * 64;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t r = at;
    at += (bytes + 255) / 256 * 256;
    return r;
  };
  auto matrix = [&](int64_t rows, int64_t cols) {
    const size_t c = take(size_t(rows) * size_t(cols / 2));
    return Matrix{c, take(refadapt_quant4_scales_size(int32_t(rows), int32_t(cols), RA_Q4_E8M0))};
  };
  p.dy = matrix(n, N);
  p.wt = matrix(K, N);
  p.dyt = matrix(N, p.tokens);
  p.xt = matrix(K, p.tokens);
  p.bytes = at;
  return p;
}

}  // namespace linear4
}  // namespace ra

extern "C" size_t refadapt_linear4_backward_workspace_size(int32_t B, int32_t rows, int32_t K, int32_t N) {
  if (B < 1 || rows < 0 || K < 1 || N < 1 || int64_t(B) * rows >= (int64_t(1) << 30)) return 0;
  const size_t n = ra::linear4::plan(int64_t(B) * rows, K, N).bytes;
  return n > 16 ? n : 16;
}

extern "C" ra_status refadapt_linear4_backward(const ra_linear4_grad_args* a, void* stream) {
  using namespace ra;
  using namespace ra::quant4;
  const char* who = "refadapt_linear4_backward";
  clear_error();
  if (!a) {
    set_error("%s: args is NULL", who);
    return RA_EINVAL;
  }
  const int64_t n = int64_t(a->B) * a->rows;
  if (a->B < 1 || a->rows < 0 || n >= (int64_t(1) << 30) || a->K < 64 || a->K % 64 != 0 || a->N < 64 || a->N % 64 != 0) {
    set_error("%s: need B >= 1, rows >= 0, B * rows < 2^30, K and N positive multiples of 64 (B=%d rows=%d K=%d N=%d)",
              who, a->B, a->rows, a->K, a->N);
    return RA_EINVAL;
  }
  if (!a->dx && !a->dw) {
    set_error("%s: neither dx nor dw", who);
    return RA_EINVAL;
  }
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dw && !aligned16(a->dw)) {
    set_error("%s: dw must be 16-byte aligned", who);
    return RA_EINVAL;
  }
  if (n == 0) {
    if (!a->dw) return RA_OK;
    if (cudaMemsetAsync(a->dw, 0, size_t(a->N) * size_t(a->K) * 2, st) != cudaSuccess) {
      set_error("%s: cudaMemsetAsync: %s", who, cudaGetErrorString(cudaGetLastError()));
      return RA_ECUDA;
    }
    return RA_OK;
  }
  auto bad_rows = [&](const void* ptr, int64_t ss, int64_t sr, int F) {
    return !ptr || !aligned16(ptr) || ss % 8 != 0 || sr % 8 != 0 || sr < F || ss < 0;
  };
  if (bad_rows(a->dy, a->dy_stride_s, a->dy_stride_r, a->N) ||
      (a->dw && bad_rows(a->x, a->x_stride_s, a->x_stride_r, a->K)) ||
      (a->dx && (bad_rows(a->dx, a->dx_stride_s, a->dx_stride_r, a->K) || !a->w || !aligned16(a->w)))) {
    set_error("%s: dy, x (with dw), w and dx (with dx) must be given, 16-byte aligned, strides multiples of 8 "
              "elements and at least a row", who);
    return RA_EINVAL;
  }
  // the samples' rows are one matrix to the product
  const int64_t dx_sr = a->rows == 1 ? a->dx_stride_s : a->dx_stride_r;
  if (a->dx && a->B > 1 && (dx_sr < a->K || a->dx_stride_s != a->rows * dx_sr)) {
    set_error("%s: dx: the rows of a sample must follow those of the one before", who);
    return RA_EINVAL;
  }
  const linear4::Plan pl = linear4::plan(n, a->K, a->N);
  if (!a->workspace || !aligned16(a->workspace) || a->workspace_bytes < pl.bytes) {
    set_error("%s: the workspace must be 16-byte aligned and hold %zu bytes (%zu given)", who, pl.bytes,
              a->workspace_bytes);
    return RA_EINVAL;
  }
  CallPlaces<3, 4> places;
  places.writes(place_of(a->workspace, int64_t(pl.bytes)));
  if (a->dx) places.writes(place_of(a->dx, int64_t(a->K) * 2, {a->B, a->dx_stride_s * 2}, {a->rows, a->dx_stride_r * 2}));
  if (a->dw) places.writes(place_of(a->dw, int64_t(a->N) * a->K * 2));
  places.reads(place_of(a->dy, int64_t(a->N) * 2, {a->B, a->dy_stride_s * 2}, {a->rows, a->dy_stride_r * 2}));
  if (a->dw) places.reads(place_of(a->x, int64_t(a->K) * 2, {a->B, a->x_stride_s * 2}, {a->rows, a->x_stride_r * 2}));
  if (a->dx) places.reads(place_of(a->w, int64_t(a->N) * a->K * 2));
  if (a->err_word) places.reads(place_of(a->err_word, 4));
  if (places.clash()) {
    set_error("%s: an output or the workspace overlaps an input or another output", who);
    return RA_EINVAL;
  }
  uint8_t* ws = static_cast<uint8_t*>(a->workspace);
  // dy both ways, x along the tokens and w along its outputs, in one launch.
  Params p;
  std::memset(&p, 0, sizeof(p));
  auto add = [&](const void* x, int64_t ss, int64_t sr, int samples, int rows, int C, const linear4::Matrix& t) {
    Seg& d = p.seg[p.n_seg++];
    d.x = static_cast<const char*>(x);
    d.x_ss = 2 * ss;
    d.x_sr = 2 * sr;
    d.rows = rows;
    d.samples = samples;
    d.C = C;
    d.down = 1.f;
    d.codes_t = ws + t.codes;
    d.scales_t = ws + t.scales;
    d.t_stride = (int64_t(samples) * rows + 63) / 64 * 32;
    return &d;
  };
  if (a->dw) add(a->x, a->x_stride_s, a->x_stride_r, a->B, a->rows, a->K, pl.xt);
  if (a->dx) add(a->w, 0, a->K, 1, a->N, a->K, pl.wt);
  Seg* d = add(a->dy, a->dy_stride_s, a->dy_stride_r, a->B, a->rows, a->N, pl.dyt);
  if (!a->dw) d->codes_t = d->scales_t = nullptr;
  if (a->dx) {
    d->codes = ws + pl.dy.codes;
    d->scales = ws + pl.dy.scales;
    d->c_sr = a->N / 2;
  }
  const ra_status r = launch_tokens(who, p, RA_Q4_E8M0, st);
  if (r != RA_OK) return r;
  auto product = [&](const linear4::Matrix& am, const linear4::Matrix& wm, int64_t rows, int32_t N, int32_t K) {
    ra_gemm4_args g;
    std::memset(&g, 0, sizeof(g));
    g.B = 1;
    g.N = N;
    g.K = K;
    g.epilogue = RA_EPI_STORE;
    g.n_seg = 1;
    g.format = RA_Q4_E8M0;
    g.err_word = a->err_word;
    ra_gemm4_seg& s = g.seg[0];
    s.lin.a = ws + am.codes;
    s.lin.a_stride_r = K / 2;
    s.lin.rows = int32_t(rows);
    s.lin.w = ws + wm.codes;
    s.a_scales = ws + am.scales;
    s.w_scales = ws + wm.scales;
    return g;
  };
  ra_gemm4_args dw, dx;
  if (a->dw) {
    dw = product(pl.dyt, pl.xt, a->N, a->K, int32_t(pl.tokens));
    dw.seg[0].lin.out = a->dw;
    dw.seg[0].lin.out_stride_r = a->K;
  }
  if (a->dx) {
    dx = product(pl.dy, pl.wt, n, a->K, a->N);
    dx.seg[0].lin.out = a->dx;
    dx.seg[0].lin.out_stride_r = n == 1 ? a->K : (a->B == 1 ? a->dx_stride_r : dx_sr);
  }
  return a->dw && a->dx ? gemm4::run_two(who, dw, dx, st, true) : gemm4::run(who, a->dw ? dw : dx, st, true);
}
