// refadapt_rope_axes, refadapt_rope_axes_table: rotary positions with several
// axes, forward and inverse.
//
//   (x[2i], x[2i+1]) -> (x[2i] c - x[2i+1] s, x[2i] s + x[2i+1] c),
//   (c, s) = (cos, sin)(pos[row][axis(i)] * base^(-2 i' / axis_dim)), i' within the axis
//
// HBM-bound: every element read and written once (4 bytes), the angles computed
// from the row's coordinates (4 bytes an axis) instead of read from a table.
// A thread has eight columns (four pairs) of one row: it forms their sines and
// cosines once, in registers, and turns the same columns of a run of heads of q
// and k with them, AHEAD loads in flight.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>

#include "api_common.h"
#include "tc_ptx.cuh"

namespace ra {
namespace rope {

constexpr int MAX_PAIRS = 128;
constexpr int THREADS = 256;
constexpr int AHEAD = 4;
constexpr uint8_t NO_AXIS = 255;

// Turns per unit of position, base^(-2i/D) / (2 pi), as a sum of two floats.
struct Freqs {
  float2 f[MAX_PAIRS];
  uint8_t axis[MAX_PAIRS];
};

struct Tensor {
  const __nv_bfloat16* x;
  __nv_bfloat16* out;
  int64_t x_sb, x_sh, x_sn, o_sb, o_sh, o_sn;
};

struct Params {
  Tensor t[2];
  const float* pos;
  int64_t pos_ss;
  int32_t n_axes, vecs;  // vecs: eight-column pieces of a sample's rows, n * d / 8
  int32_t row_vecs;      // of a row
  int32_t heads0, heads; // of the first tensor, of both
  int32_t run;           // heads of a thread
  int32_t blocks, runs;  // blocks over vecs, runs over the heads
  float sign;
  Freqs freqs;
};

// cos and sin of the angle pos * f turns. The product's whole turns are taken
// off while it is exact (p and its rounding error e), so the angle is good to
// fp32 however many turns it has.
__device__ __forceinline__ void turn(float pos, float2 f, float& c, float& s) {
  const float p = pos * f.x, e = fmaf(pos, f.x, -p);
  const float r = (p - rintf(p)) + fmaf(pos, f.y, e);
  sincospif(2.f * r, &s, &c);
}

__device__ __forceinline__ uint32_t turn_pair(uint32_t v, float c, float s) {
  const float a = __uint_as_float(v << 16), b = __uint_as_float(v & 0xFFFF0000u);
  return pack_bf16x2(a * c - b * s, a * s + b * c);
}

__global__ void __launch_bounds__(THREADS) rope_kernel(const __grid_constant__ Params p) {
  pdl_launch();
  const uint32_t blk = blockIdx.x % uint32_t(p.blocks), rest = blockIdx.x / uint32_t(p.blocks);
  const int run = int(rest % uint32_t(p.runs)), s = int(rest / uint32_t(p.runs));
  const uint32_t v = blk * THREADS + threadIdx.x;
  if (v >= uint32_t(p.vecs)) return;
  const uint32_t row = v / uint32_t(p.row_vecs), vec = v - row * uint32_t(p.row_vecs);
  pdl_wait();
  const float* pos = p.pos + s * p.pos_ss + int64_t(row) * p.n_axes;
  float c[4], sn[4];
  uint32_t keep = 0;  // pairs that no axis turns
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int a = p.freqs.axis[4 * vec + i];
    c[i] = 1.f, sn[i] = 0.f;
    if (a == NO_AXIS) {
      keep |= 1u << i;
    } else {
      turn(pos[a], p.freqs.f[4 * vec + i], c[i], sn[i]);
      sn[i] *= p.sign;
    }
  }
  const int h_end = min((run + 1) * p.run, p.heads);
  for (int h = run * p.run; h < h_end; h += AHEAD) {
    uint4 u[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (h + k >= h_end) break;
      const bool second = h + k >= p.heads0;
      const Tensor& t = p.t[second];
      u[k] = *reinterpret_cast<const uint4*>(t.x + s * t.x_sb + int64_t(h + k - (second ? p.heads0 : 0)) * t.x_sh +
                                             int64_t(row) * t.x_sn + 8 * vec);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (h + k >= h_end) break;
      const bool second = h + k >= p.heads0;
      const Tensor& t = p.t[second];
      uint4 y = make_uint4(turn_pair(u[k].x, c[0], sn[0]), turn_pair(u[k].y, c[1], sn[1]),
                           turn_pair(u[k].z, c[2], sn[2]), turn_pair(u[k].w, c[3], sn[3]));
      if (keep) {  // copied, not turned by a zero angle: an infinity beside a zero sine would be NaN
        if (keep & 1) y.x = u[k].x;
        if (keep & 2) y.y = u[k].y;
        if (keep & 4) y.z = u[k].z;
        if (keep & 8) y.w = u[k].w;
      }
      *reinterpret_cast<uint4*>(t.out + s * t.o_sb + int64_t(h + k - (second ? p.heads0 : 0)) * t.o_sh +
                                int64_t(row) * t.o_sn + 8 * vec) = y;
    }
  }
}

__global__ void table_kernel(float2* table, const float* pos, int64_t n, int n_axes, int pairs,
                             const __grid_constant__ Freqs fr) {
  for (int64_t i = blockIdx.x * int64_t(blockDim.x) + threadIdx.x; i < n * pairs; i += int64_t(gridDim.x) * blockDim.x) {
    const int64_t row = i / pairs;
    const int pair = int(i - row * pairs), a = fr.axis[pair];
    float c = 1.f, s = 0.f;
    if (a != NO_AXIS) turn(pos[row * n_axes + a], fr.f[pair], c, s);
    table[i] = make_float2(c, s);
  }
}

// The frequencies of `pairs` pairs; false with the reason recorded if the axes
// do not fit the head.
bool make_freqs(Freqs& fr, const char* who, int n_axes, const int32_t* axis_dim, int d, double base) {
  if (n_axes < 1 || n_axes > 4 || !(base > 1.0) || !std::isfinite(base)) {
    set_error("%s: need 1 to 4 axes and a finite base > 1 (n_axes=%d base=%g)", who, n_axes, base);
    return false;
  }
  int64_t sum = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (axis_dim[a] < 2 || axis_dim[a] % 2 != 0) {
      set_error("%s: axis %d has %d columns: an even number >= 2 is needed", who, a, axis_dim[a]);
      return false;
    }
    sum += axis_dim[a];
  }
  if (sum > d) {
    set_error("%s: the axes have %lld columns, a head %d", who, static_cast<long long>(sum), d);
    return false;
  }
  const double two_pi = 6.283185307179586476925;
  int pair = 0;
  for (int a = 0; a < n_axes; ++a)
    for (int i = 0; i < axis_dim[a] / 2; ++i, ++pair) {
      const double f = std::pow(base, -2.0 * i / axis_dim[a]) / two_pi;
      fr.f[pair].x = float(f);
      fr.f[pair].y = float(f - double(fr.f[pair].x));
      fr.axis[pair] = uint8_t(a);
    }
  for (; pair < MAX_PAIRS; ++pair) {
    fr.f[pair] = make_float2(0.f, 0.f);
    fr.axis[pair] = NO_AXIS;
  }
  return true;
}

}  // namespace rope
}  // namespace ra

extern "C" ra_status refadapt_rope_axes(const ra_rope_args* a, void* stream) {
  using namespace ra;
  using namespace ra::rope;
  clear_error();
  if (!a) {
    set_error("refadapt_rope_axes: args is NULL");
    return RA_EINVAL;
  }
  if (a->B < 1 || a->n < 0 || a->d < 8 || a->d % 8 != 0 || a->d > 2 * MAX_PAIRS || a->n_tensors < 1 ||
      a->n_tensors > 2 || a->inverse < 0 || a->inverse > 1) {
    set_error("refadapt_rope_axes: need B >= 1, n >= 0, d a multiple of 8 in [8, 256], one or two tensors, inverse 0 "
              "or 1 (B=%d n=%d d=%d n_tensors=%d inverse=%d)", a->B, a->n, a->d, a->n_tensors, a->inverse);
    return RA_EINVAL;
  }
  Params p;
  std::memset(&p, 0, sizeof(p));
  if (!make_freqs(p.freqs, "refadapt_rope_axes", a->n_axes, a->axis_dim, a->d, a->base)) return RA_EINVAL;
  const int64_t vecs = int64_t(a->n) * (a->d / 8);
  if (vecs > 2147483647 - THREADS) {
    set_error("refadapt_rope_axes: too many rows (n=%d d=%d)", a->n, a->d);
    return RA_EINVAL;
  }
  int64_t heads = 0;
  for (int i = 0; i < a->n_tensors; ++i) {
    const ra_rope_tensor& t = a->t[i];
    if (t.heads < 0 || t.x.n != a->n || t.out.n != a->n) {
      set_error("refadapt_rope_axes: tensor %d: heads < 0, or its rows differ from n", i);
      return RA_EINVAL;
    }
    if (t.heads == 0) continue;
    if (!check_seg(t.x, "refadapt_rope_axes: x") || !check_seg(t.out, "refadapt_rope_axes: out")) return RA_EINVAL;
    heads += t.heads;
    p.t[i] = Tensor{static_cast<const __nv_bfloat16*>(t.x.ptr), static_cast<__nv_bfloat16*>(t.out.ptr),
                    t.x.stride_b, t.x.stride_h, t.x.stride_n, t.out.stride_b, t.out.stride_h, t.out.stride_n};
  }
  if (a->n == 0 || heads == 0) return RA_OK;
  if (!a->pos || reinterpret_cast<uintptr_t>(a->pos) % 4 != 0 || a->pos_stride_s < 0) {
    set_error("refadapt_rope_axes: pos NULL or not 4-byte aligned, or pos_stride_s < 0");
    return RA_EINVAL;
  }
  if (heads > 65535) {
    set_error("refadapt_rope_axes: too many heads");
    return RA_EINVAL;
  }
  p.pos = a->pos;
  p.pos_ss = a->pos_stride_s;
  p.n_axes = a->n_axes;
  p.vecs = int32_t(vecs);
  p.row_vecs = a->d / 8;
  p.heads0 = a->t[0].heads;
  p.heads = int32_t(heads);
  p.sign = a->inverse ? -1.f : 1.f;
  p.blocks = int32_t((vecs + THREADS - 1) / THREADS);
  // Heads of a thread: as many as leave two full loads of the GPU's threads.
  const int64_t want = int64_t(2) * 2048 * num_sms() / THREADS, have = int64_t(p.blocks) * a->B;
  int64_t runs = (want + have - 1) / have;
  if (runs > heads) runs = heads;
  p.run = int32_t((heads + runs - 1) / runs);
  p.runs = int32_t((heads + p.run - 1) / p.run);
  const int64_t grid = int64_t(p.blocks) * p.runs * a->B;
  if (grid > 2147483647) {
    set_error("refadapt_rope_axes: too many rows and samples");
    return RA_EINVAL;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(grid));
  cfg.blockDim = dim3(THREADS);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, rope_kernel, p);
  if (e != cudaSuccess) {
    set_error("refadapt_rope_axes: launch failed: %s", cudaGetErrorString(e));
    cudaGetLastError();
    return RA_ECUDA;
  }
  return launch_status("refadapt_rope_axes");
}

extern "C" ra_status refadapt_rope_axes_table(float* table, const float* pos, int32_t n, int32_t d, int32_t n_axes,
                                              const int32_t* axis_dim, double base, void* stream) {
  using namespace ra;
  using namespace ra::rope;
  clear_error();
  if (!table || !pos || !axis_dim || reinterpret_cast<uintptr_t>(table) % 16 != 0 ||
      reinterpret_cast<uintptr_t>(pos) % 4 != 0 || n < 1 || d < 4 || d % 4 != 0 || d > 2 * MAX_PAIRS) {
    set_error("refadapt_rope_axes_table: table, pos or axis_dim NULL or misaligned, n < 1, or d not a multiple of 4 in "
              "[4, 256] (n=%d d=%d)", n, d);
    return RA_EINVAL;
  }
  Freqs fr;
  if (!make_freqs(fr, "refadapt_rope_axes_table", n_axes, axis_dim, d, base)) return RA_EINVAL;
  const int64_t total = int64_t(n) * (d / 2), blocks = (total + 255) / 256;
  table_kernel<<<unsigned(blocks < 4096 ? blocks : 4096), 256, 0, static_cast<cudaStream_t>(stream)>>>(
      reinterpret_cast<float2*>(table), pos, n, n_axes, d / 2, fr);
  return launch_status("refadapt_rope_axes_table");
}
