// refadapt_grad_norm and refadapt_adamw: the global norm of the gradients with the factor
// that clips them, and a step of AdamW over many tensors in one launch, with moments in
// fp32 or in 8 bits.
//
// The tensors' descriptions travel as kernel arguments (up to 256 a launch; calls of more
// launch again), so a call copies nothing to the device and can be captured. Each tensor is
// cut into chunks of a few thousand elements; a CTA finds its chunk's tensor by bisection of the
// first chunks' numbers.
//
// Bandwidth-bound: bytes a weight of the step are 8 (p) + 2 or 4 (g) + 2 (w) + 16 with
// fp32 moments, + 4.13 with 8-bit ones; the norm reads g.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "api_common.h"
#include "tc_ptx.cuh"

namespace ra {
namespace opt {

constexpr int THREADS = 256;
// Elements of a CTA's share of a tensor: long ones have more loads on their way in a thread (the
// norm) or in front of its computations (8-bit moments); the plain streams of the step with
// fp32 moments took 1262 us at 4096, 1296 at 8192 (317 M weights).
constexpr int CHUNK = 8192;
template <int BITS>
constexpr int STEP_CHUNK = BITS == 8 ? CHUNK : CHUNK / 2;
// Tensors of a launch; calls of few tensors take kernels whose arguments (2.6 KB, not 20) are copied in
// less time than these run.
constexpr int MAX_TENSORS = 256, FEW_TENSORS = 32;

// ------------------------------------------------------------------ norm
constexpr int NORM_CTAS = 2048;  // at most, over all launches of a call
// Workspace: a ticket, the number of finite norms, then a partial sum of squares (fp64) per CTA.
constexpr size_t NORM_WORKSPACE = 16 + NORM_CTAS * sizeof(double);

struct NormTensor {
  const void* g;
  int64_t n;
  uint32_t first;  // chunk of the launch that the tensor starts with
  int32_t bf16;
};
template <int MAX>
struct NormParams {
  int32_t n_tensors;
  uint32_t chunks;
  int32_t base, total;  // CTAs of the launches before, of all
  float max_norm;
  float* out;
  uint32_t* ticket;
  double* partial;
  NormTensor t[MAX];
};

// The tensor whose chunks include `chunk` (the last one that starts at or before it).
template <class T>
__device__ __forceinline__ int tensor_of(const T* t, int n, uint32_t chunk) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t[mid].first <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The CTA's sum of what the first lanes of its warps have, in thread 0.
__device__ __forceinline__ double block_sum(double v, double* warps) {
  static_assert(THREADS / 32 == 8, "eight warps");
  if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0;
  if (threadIdx.x < 8) {
    s = warps[threadIdx.x];
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) s += __shfl_xor_sync(0xffu, s, d);
  }
  __syncthreads();
  return s;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// Sums in an order that the sizes and alignments alone decide: a warp's squares of a chunk in fp32 (16 in a row, two
// of these a thread, 32 threads; 32 in a row where a chunk is not whole or not aligned), its chunks, the CTA's warps
// and the CTAs in fp64; the CTA that takes the last ticket of the call adds the CTAs' sums up. This GPU adds two fp64
// numbers a clock and SM: trees of all threads' in fp64 took 8 us beside the loads (21 M bf16 gradients: 16.7 us, now
// 8.8; 317 M: 94 us, 6.7 TB/s).
template <int MAX>
__global__ void __launch_bounds__(THREADS, 8) norm_kernel(const __grid_constant__ NormParams<MAX> p) {
  __shared__ double warps[THREADS / 32];
  __shared__ bool last;
  pdl_wait();
  pdl_launch();
  double sum = 0;
  for (uint32_t c = blockIdx.x; c < p.chunks; c += gridDim.x) {
    const NormTensor& t = p.t[tensor_of(p.t, p.n_tensors, c)];
    const int64_t i0 = int64_t(c - t.first) * CHUNK;
    const int n = int(min(int64_t(CHUNK), t.n - i0));
    uint64_t s = f2_pack(0.f, 0.f);  // two sums
    if (t.bf16) {
      const __nv_bfloat16* g = static_cast<const __nv_bfloat16*>(t.g) + i0;
      if (n == CHUNK && (reinterpret_cast<uintptr_t>(g) & 15) == 0) {
        constexpr int PIECES = CHUNK / (8 * THREADS);
        uint4 v[PIECES];
#pragma unroll
        for (int k = 0; k < PIECES; ++k) v[k] = reinterpret_cast<const uint4*>(g)[threadIdx.x + k * THREADS];
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
          const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint64_t a = bf2_unpack(w[i]);
            s = f2_fma(a, a, s);
          }
        }
      } else {
        for (int i = threadIdx.x; i < n; i += THREADS) {
          const uint64_t a = f2_pack(__bfloat162float(g[i]), 0.f);
          s = f2_fma(a, a, s);
        }
      }
    } else {
      const float* g = static_cast<const float*>(t.g) + i0;
      if (n == CHUNK && (reinterpret_cast<uintptr_t>(g) & 15) == 0) {
        constexpr int PIECES = CHUNK / (8 * THREADS);
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          float4 v[PIECES];
#pragma unroll
          for (int k = 0; k < PIECES; ++k)
            v[k] = reinterpret_cast<const float4*>(g)[threadIdx.x + (h * PIECES + k) * THREADS];
#pragma unroll
          for (int k = 0; k < PIECES; ++k) {
            const uint64_t a = f2_pack(v[k].x, v[k].y), b = f2_pack(v[k].z, v[k].w);
            s = f2_fma(a, a, s);
            s = f2_fma(b, b, s);
          }
        }
      } else {
        for (int i = threadIdx.x; i < n; i += THREADS) {
          const uint64_t a = f2_pack(g[i], 0.f);
          s = f2_fma(a, a, s);
        }
      }
    }
    float s0, s1;
    f2_unpack(s, s0, s1);
    sum += double(warp_sum(s0 + s1));
  }
  sum = block_sum(sum, warps);
  if (threadIdx.x == 0) {
    p.partial[p.base + blockIdx.x] = sum;
    __threadfence();
    last = atomicAdd(p.ticket, 1u) + 1 == uint32_t(p.total);
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  sum = 0;
  for (int i = threadIdx.x; i < p.total; i += THREADS) sum += __ldcg(p.partial + i);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  sum = block_sum(sum, warps);
  if (threadIdx.x == 0) {
    // root and quotient in fp32 (half a unit of the result each) wherever the sum is far from its ends
    const float norm = sum > 1e-30 && sum < 1e30 ? sqrtf(float(sum)) : float(sqrt(sum));
    p.out[0] = norm;
    p.out[1] = !isfinite(norm) ? __int_as_float(0x7fffffff) : norm > p.max_norm ? p.max_norm / norm : 1.f;
    p.ticket[0] = 0;
    if (isfinite(norm)) ++p.ticket[1];
  }
}

// ------------------------------------------------------------------ step
struct StepTensor {
  float* p;
  const void* g;
  void* m;
  void* v;
  uint8_t* m_scale;
  uint8_t* v_scale;
  __nv_bfloat16* w;
  int64_t n;
  uint64_t counter;  // number of the first element in the call
  uint32_t first;    // chunk of the launch that the tensor starts with
  uint8_t bf16, wide, pad[2];  // wide: pointers allow 16-byte access
};
struct StepRates {
  int32_t n_tensors;
  float lr, beta1, beta2, rest1, rest2, eps, decay;  // rest: 1 - beta
  float log1, log2;                                  // natural logarithms of the betas
  uint32_t step, seed_lo, seed_hi;
  const float* lr_dev;
  const int32_t* step_dev;
  const float* grad_scale;
};
template <int MAX>
struct StepParams : StepRates {
  StepTensor t[MAX];
};

// A mix of 32 bits in which every input bit reaches every output bit, of the published form of integer finalisers (shift
// and exclusive or around two products); the factors are the first 32 binary digits of the fractions of pi and e, odd.
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x243f6a89u;
  x = (x ^ (x >> 15)) * 0xb7e15163u;
  return x ^ (x >> 16);
}

struct Rates {
  float lr1, root2, decay, c;  // lr / (1 - beta1^t), 2^-12 / sqrt(1 - beta2^t), lr times the decay
};

// Eight elements' update; b1, b2: the betas, times the scales of what m and v hold (powers of two:
// the product with the scale is exact wherever it stands). m and v by the fp32 operations
// that the formula names, each rounded: their 8-bit forms depend on the last bit. The root and the
// quotient are the hardware's (2 ulp), of which the weight takes lr times.
__device__ __forceinline__ void update(const StepRates& h, const Rates& r, float b1, float b2, const float (&g)[8],
                                       float (&p)[8], float (&m)[8], float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float gc = __fmul_rn(g[i], r.c);
    m[i] = __fadd_rn(__fmul_rn(b1, m[i]), __fmul_rn(h.rest1, gc));
    v[i] = __fadd_rn(__fmul_rn(b2, v[i]), __fmul_rn(h.rest2, __fmul_rn(gc, gc)));
  }
  // lr m / (1 - beta1^t) / (sqrt(v) / sqrt(1 - beta2^t) + eps)
  auto move = [&](int i, float up, float root2) {
    float root, q;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root) : "f"(v[i] * up));
    asm("div.approx.ftz.f32 %0, %1, %2;" : "=f"(q) : "f"(r.lr1 * m[i]), "f"(fmaf(root, root2, h.eps)));
    p[i] = fmaf(-r.decay, p[i], p[i]) - q;
  };
  // The root of 2^24 v, which is no denormal number, so that the short form of the root will do; of v itself
  // where that could pass fp32's end (gradients beyond 10^16). Looking for those costs 5 of 924 us with 8-bit moments
  // (the step and its norm, 317 M weights).
  float top = fmaxf(v[0], v[1]);
#pragma unroll
  for (int i = 2; i < 8; i += 2) top = fmaxf(top, fmaxf(v[i], v[i + 1]));
  if (top < 0x1p100f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) move(i, 16777216.f, r.root2);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool big = v[i] >= 0x1p100f;
      move(i, big ? 1.f : 16777216.f, big ? r.root2 * 4096.f : r.root2);
    }
  }
}

// The smallest power of two with amax <= 448 s (448 = 1.75 2^8), as its biased exponent.
__device__ __forceinline__ uint32_t block_scale8(float amax) {
  const uint32_t bits = __float_as_uint(amax) & 0x7fffffffu;
  if (bits >= 0x7f800000u) return 0xffu;
  const int b = int((bits + 0x1fffffu) >> 23) - 8;
  return uint32_t(min(max(b, 1), 254));
}
template <bool WIDE>
__device__ __forceinline__ void load8(const float* src, int n, float (&x)[8]) {
  if (WIDE) {
    const float4 a = reinterpret_cast<const float4*>(src)[0], b = reinterpret_cast<const float4*>(src)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? src[i] : 0.f;
  }
}
template <bool WIDE>
__device__ __forceinline__ void store8(float* dst, int n, const float (&x)[8]) {
  if (WIDE) {
    reinterpret_cast<float4*>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) dst[i] = x[i];
  }
}
template <bool WIDE>
__device__ __forceinline__ void load8(const __nv_bfloat16* src, int n, float (&x)[8]) {
  if (WIDE) {
    const uint4 v = *reinterpret_cast<const uint4*>(src);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? __bfloat162float(src[i]) : 0.f;
  }
}
// Eight e4m3 bytes and back.
template <bool WIDE>
__device__ __forceinline__ uint2 load_bytes(const uint8_t* src, int n) {
  if (WIDE) return *reinterpret_cast<const uint2*>(src);
  uint2 r = make_uint2(0, 0);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) (i < 4 ? r.x : r.y) |= uint32_t(src[i]) << (8 * (i & 3));
  return r;
}
template <bool WIDE>
__device__ __forceinline__ void store_bytes(uint8_t* dst, int n, uint2 v) {
  if (WIDE) {
    *reinterpret_cast<uint2*>(dst) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) dst[i] = uint8_t((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
  }
}
__device__ __forceinline__ void values8(uint2 codes, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? codes.x : codes.y;
    const __half2 h(__nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(w >> (16 * (i & 1))), __NV_E4M3));
    const float2 f = __half22float2(h);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ float scale_value(uint32_t scale) {
  return scale == 0xffu ? __int_as_float(0x7fffffff)
                        : scale == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(scale << 23);
}
// Four threads (8 elements each) have a block of 32.
__device__ __forceinline__ uint32_t scale_of_block(const float (&x)[8]) {
  float top = max_nan(fabsf(x[0]), fabsf(x[1]));
#pragma unroll
  for (int i = 2; i < 8; i += 2) top = max_nan(top, fabsf(x[i]), fabsf(x[i + 1]));
  top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2));
  return block_scale8(top);
}
// The e4m3 bytes of eight moments under their scale, each rounded by 16 random bits. SECOND: the
// second moment, whose random bits are the upper halves and which stays above zero.
// y 2^-120, |y| <= 448, has e4m3's exponent in the fp32 pattern's exponent field, and where e4m3
// is denormal so is fp32: bits 20 and up of the pattern are the code, those below what lies
// between two codes. Sixteen patterns plus 256 random numbers plus 128 leave the code in the
// upper byte.
template <bool SECOND>
__device__ __forceinline__ uint2 codes8(const float (&x)[8], uint32_t scale, const uint32_t (&r)[8]) {
  if (scale == 0xffu) return make_uint2(0, 0);
  const float f = __uint_as_float((254u - scale) << 23);
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t y = __float_as_uint(__fmul_rn(__fmul_rn(x[i], f), 7.52316384526264e-37f));  // 2^-120
    const uint32_t random = __byte_perm(r[i], 0x80u, SECOND ? 0x5324 : 0x5104);  // r16 << 8 | 0x80
    c[i] = y * 16u + random;
    if (SECOND)  // 2^24 x has an exponent where x is not zero
      c[i] = max(c[i], min(__float_as_uint(x[i] * 16777216.f), 1u << 24));
    else
      c[i] = (c[i] & 0x7fffffffu) | (y & 0x80000000u);
  }
  return make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410),
                    __byte_perm(__byte_perm(c[4], c[5], 0x0073), __byte_perm(c[6], c[7], 0x0073), 0x5410));
}

// The new weights and their rounding to bf16.
template <bool WIDE>
__device__ __forceinline__ void store_weights(const StepTensor& t, int64_t at, int n, const float (&p)[8]) {
  store8<WIDE>(t.p + at, n, p);
  if (!t.w) return;
  if (WIDE) {
    *reinterpret_cast<uint4*>(t.w + at) =
        make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) t.w[at + i] = __float2bfloat16_rn(p[i]);
  }
}
// Rounds eight elements' moments to 8 bits and stores them and the weights.
template <bool WIDE>
__device__ __forceinline__ void finish8(const StepTensor& t, uint32_t key, int64_t at, int n, const float (&p)[8],
                                        const float (&m)[8], const float (&v)[8]) {
  const uint32_t ms = scale_of_block(m), vs = scale_of_block(v);
  uint32_t bits[8];
  const uint64_t c = t.counter + uint64_t(at);
  const uint32_t k = (c >> 32) ? mix(key ^ uint32_t(c >> 32)) : key;  // a run of 8 from a multiple of 8 on
#pragma unroll
  for (int i = 0; i < 8; ++i) bits[i] = mix(((uint32_t(c) + i) * 0x9e3779b1u) ^ k);
  if (n <= 0) return;
  store_bytes<WIDE>(static_cast<uint8_t*>(t.m) + at, n, codes8<false>(m, ms, bits));
  store_bytes<WIDE>(static_cast<uint8_t*>(t.v) + at, n, codes8<true>(v, vs, bits));
  if ((at & 31) == 0) {
    t.m_scale[at >> 5] = uint8_t(ms);
    t.v_scale[at >> 5] = uint8_t(vs);
  }
  store_weights<WIDE>(t, at, n, p);
}

// Eight elements of a tensor from `at` on, n of them in the tensor (at most 0: none, but
// the thread takes part in its block's scale).
template <int BITS, bool WIDE>
__device__ __forceinline__ void step8(const StepRates& h, const StepTensor& t, const Rates& r, uint32_t key,
                                      int64_t at, int n) {
  float p[8], g[8], m[8], v[8], b1 = h.beta1, b2 = h.beta2;
  if (n > 0) {
    load8<WIDE>(t.p + at, n, p);
    if (t.bf16)
      load8<WIDE>(static_cast<const __nv_bfloat16*>(t.g) + at, n, g);
    else
      load8<WIDE>(static_cast<const float*>(t.g) + at, n, g);
    if (BITS == 32) {
      load8<WIDE>(static_cast<const float*>(t.m) + at, n, m);
      load8<WIDE>(static_cast<const float*>(t.v) + at, n, v);
    } else {
      const uint2 mc = load_bytes<WIDE>(static_cast<const uint8_t*>(t.m) + at, n);
      const uint2 vc = load_bytes<WIDE>(static_cast<const uint8_t*>(t.v) + at, n);
      b1 *= scale_value(t.m_scale[at >> 5]);
      b2 *= scale_value(t.v_scale[at >> 5]);
      values8(mc, m);
      values8(vc, v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = g[i] = m[i] = v[i] = 0.f;
  }
  update(h, r, b1, b2, g, p, m, v);
  if (BITS == 8) {
    if (n < 8) {  // what is not in the tensor has no part in the block
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= n) m[i] = v[i] = 0.f;
    }
    finish8<WIDE>(t, key, at, n, p, m, v);
  } else if (n > 0) {
    store8<WIDE>(static_cast<float*>(t.m) + at, n, m);
    store8<WIDE>(static_cast<float*>(t.v) + at, n, v);
    store_weights<WIDE>(t, at, n, p);
  }
}

// What eight elements with 8-bit moments need, as it lies in memory.
template <bool BF16>
struct Raw8 {
  float4 p[2];
  uint4 g[BF16 ? 1 : 2];
  uint2 m, v;
  uint32_t m_scale, v_scale;
  __device__ __forceinline__ void load(const StepTensor& t, int64_t at) {
    p[0] = reinterpret_cast<const float4*>(t.p + at)[0];
    p[1] = reinterpret_cast<const float4*>(t.p + at)[1];
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const char*>(t.g) + at * (BF16 ? 2 : 4));
    g[0] = src[0];
    if (!BF16) g[BF16 ? 0 : 1] = src[1];
    m = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.m) + at);
    v = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + at);
    m_scale = t.m_scale[at >> 5];
    v_scale = t.v_scale[at >> 5];
  }
};

// A whole chunk with 8-bit moments: the loads of the next eight elements are on their way while
// these are computed (70 instructions an element); without, the warps waited for memory half
// their time: 1144 -> 833 us for 317 M weights, 6.1 TB/s.
template <bool BF16>
__device__ __forceinline__ void whole_chunk(const StepRates& h, const StepTensor& t, const Rates& r, uint32_t key,
                                            int64_t i0) {
  constexpr int PASSES = CHUNK / (8 * THREADS);
  int64_t at = i0 + int(threadIdx.x) * 8;
  Raw8<BF16> next;
  next.load(t, at);
#pragma unroll 1
  for (int k = 0; k < PASSES; ++k, at += 8 * THREADS) {
    const Raw8<BF16> in = next;
    if (k + 1 < PASSES) next.load(t, at + 8 * THREADS);
    float p[8] = {in.p[0].x, in.p[0].y, in.p[0].z, in.p[0].w, in.p[1].x, in.p[1].y, in.p[1].z, in.p[1].w};
    float g[8], m[8], v[8];
    const uint32_t* w = reinterpret_cast<const uint32_t*>(in.g);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      g[i] = BF16 ? __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16) : __uint_as_float(w[i]);
    values8(in.m, m);
    values8(in.v, v);
    update(h, r, h.beta1 * scale_value(in.m_scale), h.beta2 * scale_value(in.v_scale), g, p, m, v);
    finish8<true>(t, key, at, 8, p, m, v);
  }
}

template <int BITS, int MAX>
__global__ void __launch_bounds__(THREADS, BITS == 8 ? 3 : 4) step_kernel(const __grid_constant__ StepParams<MAX> h) {
  pdl_wait();
  pdl_launch();
  const uint32_t chunk = blockIdx.x;
  const StepTensor& t = h.t[tensor_of(h.t, h.n_tensors, chunk)];
  Rates r;
  r.c = h.grad_scale ? *h.grad_scale : 1.f;
  if (!isfinite(r.c)) return;
  const float lr = h.lr_dev ? *h.lr_dev : h.lr;
  r.decay = lr * h.decay;
  const uint32_t step = h.step_dev ? uint32_t(max(*h.step_dev, 1)) : h.step;
  // 1 - beta^t = -expm1(t ln beta): no cancellation at small t
  r.lr1 = h.beta1 > 0.f ? -lr / expm1f(float(step) * h.log1) : lr;
  r.root2 = h.beta2 > 0.f ? rsqrtf(-expm1f(float(step) * h.log2)) : 1.f;
  r.root2 *= 0.000244140625f;  // of the root of 2^24 v
  const uint32_t key = mix(mix(mix(h.seed_lo) ^ h.seed_hi) ^ step);
  const int64_t i0 = int64_t(chunk - t.first) * STEP_CHUNK<BITS>;
  if (BITS == 8 && t.wide && t.n - i0 >= STEP_CHUNK<BITS>) {
    if (t.bf16)
      whole_chunk<true>(h, t, r, key, i0);
    else
      whole_chunk<false>(h, t, r, key, i0);
    return;
  }
#pragma unroll
  for (int k = 0; k < STEP_CHUNK<BITS> / (8 * THREADS); ++k) {
    const int64_t at = i0 + (k * THREADS + int(threadIdx.x)) * 8;
    const int n = int(min(int64_t(8), t.n - at));
    if (t.wide && n == 8)
      step8<BITS, true>(h, t, r, key, at, n);
    else
      step8<BITS, false>(h, t, r, key, at, n);
  }
}

template <class P>
ra_status launch(const char* who, const P& p, void (*fn)(P), int64_t ctas, cudaStream_t st) {
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

bool aligned(const void* ptr, uintptr_t to) { return reinterpret_cast<uintptr_t>(ptr) % to == 0; }

// Ranges of memory; `out` ones may meet no other.
struct Range {
  uintptr_t begin, end;
  bool out;
};
// Do an output and any other range meet?
bool meet(std::vector<Range>& r) {
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t in_end = 0, out_end = 0;  // of what starts at or before
  for (const Range& x : r) {
    if (x.begin < out_end || (x.out && x.begin < in_end)) return true;
    uintptr_t& end = x.out ? out_end : in_end;
    if (x.end > end) end = x.end;
  }
  return false;
}

struct NormCall {
  const ra_grad* tensors;
  int32_t n_tensors;
  float max_norm;
  float* out;
  void* workspace;
  int64_t most;  // CTAs of a launch
  cudaStream_t st;
};
template <int MAX>
ra_status launch_norm(const NormCall& c) {
  NormParams<MAX> p;
  std::memset(&p, 0, sizeof(p));
  p.max_norm = c.max_norm;
  p.out = c.out;
  p.ticket = static_cast<uint32_t*>(c.workspace);
  p.partial = reinterpret_cast<double*>(static_cast<char*>(c.workspace) + 16);
  auto ctas_of = [&](int64_t n) { return n < 1 ? 1 : n < c.most ? n : c.most; };
  for (int pass = 0; pass < 2; ++pass) {  // counts the CTAs, then launches
    int32_t base = 0, i = 0;
    do {
      p.n_tensors = 0;
      int64_t first = 0;
      for (; i < c.n_tensors && p.n_tensors < MAX; ++i) {
        if (c.tensors[i].n == 0) continue;
        p.t[p.n_tensors++] = NormTensor{c.tensors[i].g, c.tensors[i].n, uint32_t(first), c.tensors[i].type == RA_BF16};
        first += (c.tensors[i].n + CHUNK - 1) / CHUNK;
      }
      while (i < c.n_tensors && c.tensors[i].n == 0) ++i;
      p.chunks = uint32_t(first);
      p.base = base;
      const int64_t ctas = ctas_of(first);
      base += int32_t(ctas);
      if (pass == 1) {
        const ra_status r = opt::launch("refadapt_grad_norm", p, norm_kernel<MAX>, ctas, c.st);
        if (r != RA_OK) return r;
      }
    } while (i < c.n_tensors);
    p.total = base;
  }
  return RA_OK;
}

template <int BITS, int MAX>
ra_status launch_step(const ra_adamw_args& a, cudaStream_t st) {
  StepParams<MAX> p;
  std::memset(static_cast<void*>(&p), 0, sizeof(p));
  p.lr = float(a.lr);
  p.beta1 = float(a.beta1);
  p.beta2 = float(a.beta2);
  p.rest1 = float(1.0 - a.beta1);
  p.rest2 = float(1.0 - a.beta2);
  p.eps = float(a.eps);
  p.decay = float(a.decay);
  p.log1 = a.beta1 > 0 ? float(std::log(a.beta1)) : 0.f;
  p.log2 = a.beta2 > 0 ? float(std::log(a.beta2)) : 0.f;
  p.step = uint32_t(a.step);
  p.seed_lo = uint32_t(a.seed);
  p.seed_hi = uint32_t(a.seed >> 32);
  p.lr_dev = a.lr_dev;
  p.step_dev = a.step_dev;
  p.grad_scale = a.grad_scale;
  uint64_t counter = 0;
  int64_t chunks = 0;
  constexpr int chunk = STEP_CHUNK<BITS>, states = BITS == 8 ? 8 : 16;  // states: what vectors of moments align to
  auto flush = [&]() {
    if (p.n_tensors == 0) return RA_OK;
    const ra_status r = opt::launch("refadapt_adamw", p, step_kernel<BITS, MAX>, chunks, st);
    p.n_tensors = 0;
    chunks = 0;
    return r;
  };
  for (int32_t i = 0; i < a.n_tensors; ++i) {
    const ra_adamw_tensor& t = a.tensors[i];
    if (t.n == 0) continue;
    const int64_t mine = (t.n + chunk - 1) / chunk;
    if (p.n_tensors == MAX || chunks + mine > 2147483647) {
      const ra_status r = flush();
      if (r != RA_OK) return r;
    }
    StepTensor& d = p.t[p.n_tensors++];
    d.p = static_cast<float*>(t.p);
    d.g = t.g;
    d.m = t.m;
    d.v = t.v;
    d.m_scale = static_cast<uint8_t*>(t.m_scale);
    d.v_scale = static_cast<uint8_t*>(t.v_scale);
    d.w = static_cast<__nv_bfloat16*>(t.w);
    d.n = t.n;
    d.counter = counter;
    d.first = uint32_t(chunks);
    d.bf16 = t.g_type == RA_BF16;
    d.wide = aligned(t.p, 16) && aligned(t.g, 16) && aligned(t.m, states) && aligned(t.v, states) &&
             aligned(t.w, 16);
    chunks += mine;
    counter += uint64_t(t.n + 31) / 32 * 32;
  }
  return flush();
}

}  // namespace opt
}  // namespace ra

extern "C" size_t refadapt_grad_norm_workspace_size(void) { return ra::opt::NORM_WORKSPACE; }

extern "C" ra_status refadapt_grad_norm(const ra_grad* tensors, int32_t n_tensors, float max_norm, float* out,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  using namespace ra;
  using namespace ra::opt;
  clear_error();
  if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !(max_norm > 0.f)) {
    set_error("refadapt_grad_norm: need n_tensors >= 0 with their array, and max_norm > 0");
    return RA_EINVAL;
  }
  if (!out || !aligned(out, 4) || !workspace || !aligned(workspace, 16) || workspace_bytes < NORM_WORKSPACE) {
    set_error("refadapt_grad_norm: need out and a 16-byte aligned workspace of %zu bytes", NORM_WORKSPACE);
    return RA_EINVAL;
  }
  const uintptr_t o = reinterpret_cast<uintptr_t>(out), w = reinterpret_cast<uintptr_t>(workspace);
  if (o < w + NORM_WORKSPACE && w < o + 8) {
    set_error("refadapt_grad_norm: out and the workspace overlap");
    return RA_EINVAL;
  }
  int32_t used = 0;
  int64_t chunks = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const ra_grad& t = tensors[i];
    if (t.n < 0 || t.n > (int64_t(1) << 42) || (t.type != RA_F32 && t.type != RA_BF16) ||
        (t.n > 0 && (!t.g || !aligned(t.g, t.type == RA_BF16 ? 2 : 4)))) {
      set_error("refadapt_grad_norm: tensor %d: need 0 <= n <= 2^42, a known type and a pointer aligned to it", i);
      return RA_EINVAL;
    }
    const uintptr_t g = reinterpret_cast<uintptr_t>(t.g), ge = g + uintptr_t(t.n) * (t.type == RA_BF16 ? 2 : 4);
    if (t.n > 0 && ((g < o + 8 && o < ge) || (g < w + NORM_WORKSPACE && w < ge))) {
      set_error("refadapt_grad_norm: tensor %d overlaps out or the workspace", i);
      return RA_EINVAL;
    }
    used += t.n > 0;
    chunks += (t.n + CHUNK - 1) / CHUNK;
  }
  const int64_t launches = used > 0 ? (used + MAX_TENSORS - 1) / MAX_TENSORS : 1;
  if (launches > NORM_CTAS || chunks > (int64_t(1) << 31)) {
    set_error("refadapt_grad_norm: too many tensors or elements");
    return RA_EINVAL;
  }
  // CTAs of a launch: eight for an SM, as many as the workspace has room for
  const int64_t most = std::min<int64_t>(int64_t(num_sms()) * 8, NORM_CTAS / launches);
  const NormCall call{tensors, n_tensors, max_norm, out, workspace, most, static_cast<cudaStream_t>(stream)};
  return used <= FEW_TENSORS ? launch_norm<FEW_TENSORS>(call) : launch_norm<MAX_TENSORS>(call);
}

extern "C" ra_status refadapt_adamw(const ra_adamw_args* a, void* stream) {
  using namespace ra;
  using namespace ra::opt;
  clear_error();
  if (!a) {
    set_error("refadapt_adamw: args is NULL");
    return RA_EINVAL;
  }
  if (a->n_tensors < 0 || (a->n_tensors > 0 && !a->tensors) || (a->bits != 32 && a->bits != 8)) {
    set_error("refadapt_adamw: need n_tensors >= 0 with their array, and bits 32 or 8");
    return RA_EINVAL;
  }
  // The rates count in fp32: eps as 2^-126 or more there (the quotient takes denormal numbers for zero, and an
  // element without moments would be 0 / 0), the others as finite.
  if (!(a->beta1 >= 0 && a->beta1 < 1 && a->beta2 >= 0 && a->beta2 < 1 && float(a->eps) >= FLT_MIN &&
        std::isfinite(float(a->eps)) && a->decay >= 0 && std::isfinite(float(a->decay)) && a->lr >= 0 &&
        std::isfinite(float(a->lr))) ||
      (!a->step_dev && (a->step < 1 || a->step > 2147483647))) {
    set_error("refadapt_adamw: need betas in [0, 1), eps >= 2^-126, lr and decay >= 0, all finite in fp32, 1 <= step < 2^31");
    return RA_EINVAL;
  }
  const bool small = a->bits == 8;
  try {
    std::vector<Range> ranges;
    ranges.reserve(size_t(a->n_tensors) * (small ? 7 : 5) + 3);
    auto add = [&](const void* ptr, int64_t bytes, bool out) {
      const uintptr_t b = reinterpret_cast<uintptr_t>(ptr);
      if (ptr && bytes > 0) ranges.push_back(Range{b, b + uintptr_t(bytes), out});
    };
    for (int32_t i = 0; i < a->n_tensors; ++i) {
      const ra_adamw_tensor& t = a->tensors[i];
      if (t.n < 0 || t.n > (int64_t(1) << 42) || (t.g_type != RA_F32 && t.g_type != RA_BF16)) {
        set_error("refadapt_adamw: tensor %d: need 0 <= n <= 2^42 and a known type", i);
        return RA_EINVAL;
      }
      if (t.n == 0) continue;
      if (!t.p || !t.g || !t.m || !t.v || (small && (!t.m_scale || !t.v_scale)) || !aligned(t.p, 4) ||
          !aligned(t.g, t.g_type == RA_BF16 ? 2 : 4) || (!small && (!aligned(t.m, 4) || !aligned(t.v, 4))) ||
          !aligned(t.w, 2)) {
        set_error("refadapt_adamw: tensor %d: p, g, m, v%s must be given and aligned to their types", i,
                  small ? ", m_scale, v_scale" : "");
        return RA_EINVAL;
      }
      const int64_t blocks = (t.n + 31) / 32;
      add(t.p, t.n * 4, true);
      add(t.g, t.n * (t.g_type == RA_BF16 ? 2 : 4), false);
      add(t.m, t.n * (small ? 1 : 4), true);
      add(t.v, t.n * (small ? 1 : 4), true);
      add(t.w, t.n * 2, true);
      if (small) {
        add(t.m_scale, blocks, true);
        add(t.v_scale, blocks, true);
      }
    }
    add(a->lr_dev, 4, false);
    add(a->step_dev, 4, false);
    add(a->grad_scale, 4, false);
    if (meet(ranges)) {
      set_error("refadapt_adamw: an output overlaps an input or another output");
      return RA_EINVAL;
    }
  } catch (const std::bad_alloc&) {
    set_error("refadapt_adamw: out of host memory");
    return RA_EINVAL;
  }
  int32_t used = 0;
  for (int32_t i = 0; i < a->n_tensors; ++i) used += a->tensors[i].n > 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (small) return used <= FEW_TENSORS ? launch_step<8, FEW_TENSORS>(*a, st) : launch_step<8, MAX_TENSORS>(*a, st);
  return used <= FEW_TENSORS ? launch_step<32, FEW_TENSORS>(*a, st) : launch_step<32, MAX_TENSORS>(*a, st);
}
