// refadapt_gemm4 for one row (a pooled or conditioning token; STORE, GELU, RESID): the weights' bytes are
// all there is to move, and the tensor cores' way there (TMEM, rings, tiles of 128 rows) costs more than
// the work.
//
// A warp takes eight weight rows (those whose scales lie in the same 32 bytes: rows 2 i, 2 i + 1
// of each 32 of a scale tile), 32 codes of each to a lane; K is shared by the warps of a CTA and
// their sums meet in shared memory, in a fixed order. A's row is in shared memory as fp16. The
// products of 16 codes are summed in fp16 exactly: values are multiples of 1/2 up to 6, products
// of 1/4 up to 36, and half of the 16 in each half of a register, at most 8 x 36 = 288 =
// 1152 quarters, below fp16's 2048. The block's sum times both scales is exact in fp32 (12 + 8
// bits), the blocks are summed in fp32.
//
// Bound by latency in small calls and by the conversions in large ones (16 codes take eight, at a quarter
// of the products' rate): the time goes with N K. Tensor core tiles cover 64 columns each at about the
// speed of one SM's loads, so that theirs goes with K alone until every SM has one: K = 2048, N = 8192
// (e4m3, 9.5 MB) takes 5.1 us here, 7.0 there; K = 4096, N = 8192 8.3 and 10.5; K = 8192, N = 2048 5.2
// and 9.6; K = 16384, N = 4096 12.7 and 29.1; K = N = 1024 3.8 and 4.1. Beyond that they are the faster
// ones: K = 2048, N = 16384 7.8 and 7.4, K = 4096 13.5 and 11.5 (N = 12288: 11.1 and 11.7, e8m0 11.9 and
// 11.3). A second row here costs another 4 us at K = 2048, N = 8192, there nothing.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>

#include "api_common.h"
#include "gemm4.h"
#include "gemm_body.cuh"
#include "tc_ptx.cuh"

namespace ra {
namespace gemm4 {
namespace {

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int STEP = 1024;  // of K: 32 codes a lane
constexpr int N_ROWS = 8;   // weight rows of a warp
constexpr int row_smem(int K) { return K * 2 + K / 16 * 4; }

struct RowSeg {
  const uint8_t* a;
  const uint8_t* a_scales;
  const uint8_t* w;
  const uint8_t* w_scales;
  const float* bias;
  __nv_bfloat16* out;
  const __nv_bfloat16* resid;
  const float* gate;
  float alpha;
  int32_t gated, first;  // first: CTA that the segment starts with
};
struct RowParams {
  int32_t n_seg, N, K, e8m0, epilogue;
  int32_t share;  // warps that share a unit's K: 1, 2, 4 or 8
  const int32_t* mode;
  RowSeg seg[3];
};

// Eight codes (a word) as four pairs of fp16.
__device__ __forceinline__ void values4(uint32_t w, __half2 (&h)[4]) {
  uint32_t r[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
      : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = *reinterpret_cast<__half2*>(&r[i]);
}
__device__ __forceinline__ float scale_of(uint32_t byte, int e8m0) {
  if (e8m0) return byte == 255u ? __int_as_float(0x7fffffff) : byte == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(__nv_fp8_storage_t(byte), __NV_E4M3)));
}
// Place of the 16-byte piece q (8 values) of a lane's 32 in shared memory: the four pieces of
// lanes two apart are permuted, so that a warp's reads have no conflicts.
__device__ __forceinline__ int piece_at(int chunk, int q) { return chunk * 4 + (q ^ ((chunk >> 1) & 3)); }

__device__ __forceinline__ void prefetch_l2(const void* ptr) { asm volatile("prefetch.global.L2 [%0];" ::"l"(ptr)); }

__global__ void __launch_bounds__(THREADS) row_kernel(const __grid_constant__ RowParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float sums[WARPS * N_ROWS];
  uint4* av = reinterpret_cast<uint4*>(smem);              // K / 8 pieces of 8 fp16
  float* as = reinterpret_cast<float*>(smem + p.K * 2);    // the scales of 16 of K
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int g = 0;
  while (g + 1 < p.n_seg && int(blockIdx.x) >= p.seg[g + 1].first) ++g;
  const RowSeg& sg = p.seg[g];
  const int units = WARPS / p.share;
  const int unit = (int(blockIdx.x) - sg.first) * units + warp / p.share, part = warp % p.share;
  const int tile = unit >> 4, i2 = 2 * (unit & 15);  // weight rows 128 tile + 32 q + i2 + i
  const int block = p.e8m0 ? 32 : 16;
  const int64_t groups = (p.K + 4 * block - 1) / (4 * block);
  const bool mine = tile * 128 < p.N;
  // What the warp reads of the weights goes to L2 while the kernel before this one runs: with the row's
  // quantisation 7.3 us, 6.5 (2048 -> 8192). (If that one writes them, it writes to L2 as well.)
  for (int step = part; mine && step * STEP < p.K; step += p.share) {
    const int n = tile * 128 + 32 * (lane >> 3) + i2 + ((lane >> 2) & 1), k = step * STEP + 256 * (lane & 3);
    if (n < p.N && k < p.K) prefetch_l2(sg.w + int64_t(n) * (p.K / 2) + k / 2);
    const int ks = step * STEP + 4 * block * lane;
    if (ks < min(p.K, (step + 1) * STEP)) prefetch_l2(sg.w_scales + (tile * groups + ks / (4 * block)) * 512 + 16 * i2);
  }
  pdl_wait();
  pdl_launch();
  if (sg.gated && *p.mode == RA_MODE_REUSE) return;
  // the first step's weights are on their way while A is unpacked
  uint4 c[N_ROWS], s[2];
  auto fetch = [&](int step) {
    const int k0 = step * STEP + 32 * lane;
    const bool on = mine && k0 < p.K;
#pragma unroll
    for (int e = 0; e < N_ROWS; ++e) {
      const int n = tile * 128 + 32 * (e >> 1) + i2 + (e & 1);
      c[e] = on && n < p.N ? *reinterpret_cast<const uint4*>(sg.w + int64_t(n) * (p.K / 2) + k0 / 2)
                           : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      s[i] = on ? *reinterpret_cast<const uint4*>(sg.w_scales + (tile * groups + k0 / (4 * block)) * 512 + 16 * (i2 + i))
                : make_uint4(0, 0, 0, 0);
  };
  fetch(part);
  // A's row: eight codes a thread
  for (int k8 = threadIdx.x; k8 < p.K / 8; k8 += THREADS) {
    __half2 h[4];
    values4(reinterpret_cast<const uint32_t*>(sg.a)[k8], h);
    av[piece_at(k8 >> 2, k8 & 3)] = *reinterpret_cast<uint4*>(h);
  }
  for (int i = threadIdx.x; i < p.K / 16; i += THREADS) {
    const int j = i * 16 / block;
    as[i] = scale_of(sg.a_scales[j / 4 * 512 + j % 4], p.e8m0);
  }
  __syncthreads();
  float acc[N_ROWS] = {};
  for (int step = part; step * STEP < p.K; step += p.share) {
    const int k0 = step * STEP + 32 * lane;
    uint4 cc[N_ROWS], ss[2];
#pragma unroll
    for (int e = 0; e < N_ROWS; ++e) cc[e] = c[e];
    ss[0] = s[0], ss[1] = s[1];
    if ((step + p.share) * STEP < p.K) fetch(step + p.share);
    if (k0 >= p.K) continue;
    const int chunk = k0 / 32, j0 = (k0 / block) & 3;  // the first of the lane's blocks within its scale tile
#pragma unroll
    for (int b = 0; b < 2; ++b) {  // 16 codes
      const uint4 x[2] = {av[piece_at(chunk, 2 * b)], av[piece_at(chunk, 2 * b + 1)]};
      const __half2* y = reinterpret_cast<const __half2*>(x);
      const float sa = as[k0 / 16 + b];
#pragma unroll
      for (int e = 0; e < N_ROWS; ++e) {
        __half2 w[8];
        {
          const uint32_t lo = b == 0 ? cc[e].x : cc[e].z, hi = b == 0 ? cc[e].y : cc[e].w;
          __half2 h[4];
          values4(lo, h);
          w[0] = h[0], w[1] = h[1], w[2] = h[2], w[3] = h[3];
          values4(hi, h);
          w[4] = h[0], w[5] = h[1], w[6] = h[2], w[7] = h[3];
        }
        const uint4& sq = ss[e & 1];
        const uint32_t word = (e >> 1) == 0 ? sq.x : (e >> 1) == 1 ? sq.y : (e >> 1) == 2 ? sq.z : sq.w;
        const float sw = scale_of((word >> (8 * (j0 + (p.e8m0 ? 0 : b)))) & 0xffu, p.e8m0);
        __half2 t = __hmul2(y[0], w[0]);
#pragma unroll
        for (int q = 1; q < 8; ++q) t = __hfma2(y[q], w[q], t);
        const float2 f = __half22float2(t);
        acc[e] = fmaf(f.x + f.y, sa * sw, acc[e]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < N_ROWS; ++e) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], d);
    if (lane == 0) sums[warp * N_ROWS + e] = acc[e];
  }
  __syncthreads();
  // One thread an output.
  const int u = threadIdx.x / N_ROWS, e = threadIdx.x % N_ROWS;
  if (u >= units) return;
  const int unit_o = (int(blockIdx.x) - sg.first) * units + u;
  const int n = (unit_o >> 4) * 128 + 32 * (e >> 1) + 2 * (unit_o & 15) + (e & 1);
  if (n >= p.N) return;
  float v = 0.f;
  for (int q = 0; q < p.share; ++q) v += sums[(u * p.share + q) * N_ROWS + e];
  v = fmaf(v, sg.alpha, sg.bias ? sg.bias[n] : 0.f);
  if (p.epilogue == RA_EPI_GELU) {
    float other = 0.f;
    v = max_nan(v, GELU_END);
    gemm::gelu_tanh2(v, other);
  } else if (p.epilogue == RA_EPI_RESID) {
    v = fmaf(sg.gate[n], v, __bfloat162float(sg.resid[n]));
  }
  sg.out[n] = __float2bfloat16_rn(v);
}

}  // namespace

ra_status run_row(const char* who, const ra_gemm4_args& a, cudaStream_t st) {
  RowParams p;
  std::memset(&p, 0, sizeof(p));
  p.N = a.N;
  p.K = a.K;
  p.e8m0 = a.format == RA_Q4_E8M0;
  p.epilogue = a.epilogue;
  p.mode = a.mode;
  p.share = 1;
  while (p.share < WARPS && p.share * STEP < a.K) p.share *= 2;
  const int units = (a.N + 127) / 128 * 16, per = WARPS / p.share, ctas = (units + per - 1) / per;
  for (int g = 0; g < a.n_seg; ++g) {
    const ra_gemm4_seg& q = a.seg[g];
    const ra_gemm_seg& s = q.lin;
    if (s.rows == 0) continue;
    RowSeg& d = p.seg[p.n_seg];
    d.a = static_cast<const uint8_t*>(s.a);
    d.a_scales = static_cast<const uint8_t*>(q.a_scales);
    d.w = static_cast<const uint8_t*>(s.w);
    d.w_scales = static_cast<const uint8_t*>(q.w_scales);
    d.bias = s.bias;
    d.out = static_cast<__nv_bfloat16*>(s.out);
    d.resid = static_cast<const __nv_bfloat16*>(s.resid);
    d.gate = s.gate;
    d.alpha = ldexpf(1.f, q.a_exponent + q.w_exponent);
    d.gated = s.gated ? 1 : 0;
    d.first = ctas * p.n_seg++;
  }
  note_launch("one row, %d warps to a row of weights", p.share);
  const ra_status as = ensure_dynamic_smem(reinterpret_cast<const void*>(row_kernel), row_smem(MAX_ROW_K), who);
  if (as != RA_OK) return as;
  cudaLaunchAttribute attr[1] = {pdl_attribute()};
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(unsigned(ctas * p.n_seg), 1, 1);
  cfg.blockDim = dim3(THREADS, 1, 1);
  cfg.dynamicSmemBytes = row_smem(a.K);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, row_kernel, p);
  if (e != cudaSuccess) {
    set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
    cudaGetLastError();
    return RA_ECUDA;
  }
  return launch_status(who);
}

}  // namespace gemm4
}  // namespace ra
