// refadapt_rope_axes, refadapt_rope_axes_table: rotary positions with several
// axes, forward and inverse.
//
//   (x[2i], x[2i+1]) -> (x[2i] c - x[2i+1] s, x[2i] s + x[2i+1] c),
//   (c, s) = (cos, sin)(pos[row][axis(i)] * base^(-2 i' / axis_dim)), i' within the axis
//
// HBM-bound: every element read and written once (4 bytes), the angles computed
// from the row's coordinates (4 bytes an axis) instead of read from a table.
// A thread has eight columns (four pairs) of one row, a slot, and turns them in
// every HEAD_GROUPS-th head of q and k, AHEAD loads in flight, the first of them
// while the angles are formed. A CTA's threads form the sines and cosines of its
// slots once, one pair each, and share them (each thread its own four pairs: 2745
// rows, 20 heads of 64, two samples 11.7 us, here 9.0). 16,128 rows, 48 heads of 128:
// 59.7 us, 6.6 TB/s = 98 % of a plain copy (64.3 before; AHEAD = 4: 63.2, 8: 60.9).
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
constexpr int AHEAD = 6;
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
  int32_t heads, reserved;
};

struct Params {
  Tensor t[2];
  const float* pos;
  int64_t pos_ss;
  int32_t n_tensors;
  int32_t n_axes, vecs;  // vecs: eight-column pieces of a sample's rows, n * d / 8
  int32_t row_vecs;      // of a row
  int32_t blocks;        // of a sample
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

// SLOTS slots a CTA, THREADS / SLOTS groups of heads.
template <int SLOTS>
__global__ void __launch_bounds__(THREADS, 4) rope_kernel(const __grid_constant__ Params p) {
  constexpr int HEAD_GROUPS = THREADS / SLOTS;
  static_assert(4 * SLOTS <= THREADS, "one pair a thread");
  __shared__ float4 turns[SLOTS][2];  // (cos, sin) of a slot's pairs
  __shared__ uint8_t axis[SLOTS][4];
  pdl_launch();
  const uint32_t s = blockIdx.x / uint32_t(p.blocks), v0 = (blockIdx.x - s * uint32_t(p.blocks)) * SLOTS;
  const int slot = threadIdx.x % SLOTS, h0 = threadIdx.x / SLOTS;
  const uint32_t v = v0 + slot, row = v / uint32_t(p.row_vecs), vec = v - row * uint32_t(p.row_vecs);
  const bool in = v < uint32_t(p.vecs);
  const __nv_bfloat16* x;
  int64_t step;
  uint4 u[AHEAD];
  auto start = [&](const Tensor& t) {
    x = t.x + s * t.x_sb + int64_t(row) * t.x_sn + 8 * vec + h0 * t.x_sh;
    step = HEAD_GROUPS * t.x_sh;
  };
  auto load = [&](int h, int heads) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (in && h + k * HEAD_GROUPS < heads) u[k] = *reinterpret_cast<const uint4*>(x);
      x += step;
    }
  };
  pdl_wait();
  start(p.t[0]);
  load(h0, p.t[0].heads);  // on their way while the angles are formed
  if (threadIdx.x < 4 * SLOTS) {
    const uint32_t w = v0 + threadIdx.x / 4, i = threadIdx.x % 4;
    if (w < uint32_t(p.vecs)) {
      const uint32_t r = w / uint32_t(p.row_vecs), pair = 4 * (w - r * uint32_t(p.row_vecs)) + i;
      const int a = p.freqs.axis[pair];
      float c = 1.f, sn = 0.f;
      if (a != NO_AXIS) turn(p.pos[s * p.pos_ss + int64_t(r) * p.n_axes + a], p.freqs.f[pair], c, sn);
      reinterpret_cast<float2*>(turns[threadIdx.x / 4])[i] = make_float2(c, p.sign * sn);
      axis[threadIdx.x / 4][i] = uint8_t(a);
    }
  }
  __syncthreads();
  if (!in) return;
  const float4 t0 = turns[slot][0], t1 = turns[slot][1];
  uint32_t keep = 0;  // pairs that no axis turns
#pragma unroll
  for (int i = 0; i < 4; ++i) keep |= axis[slot][i] == NO_AXIS ? 1u << i : 0u;
#pragma unroll 1
  for (int z = 0; z < p.n_tensors; ++z) {
    const Tensor& t = p.t[z];
    if (z > 0) {
      start(t);
      load(h0, t.heads);
    }
    __nv_bfloat16* out = t.out + s * t.o_sb + int64_t(row) * t.o_sn + 8 * vec + h0 * t.o_sh;
    const int64_t out_step = HEAD_GROUPS * t.o_sh;
#pragma unroll 1
    for (int h = h0; h < t.heads; h += AHEAD * HEAD_GROUPS) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        if (h + k * HEAD_GROUPS >= t.heads) break;
        uint4 y = make_uint4(turn_pair(u[k].x, t0.x, t0.y), turn_pair(u[k].y, t0.z, t0.w),
                             turn_pair(u[k].z, t1.x, t1.y), turn_pair(u[k].w, t1.z, t1.w));
        if (keep) {  // copied, not turned by a zero angle: an infinity beside a zero sine would be NaN
          if (keep & 1) y.x = u[k].x;
          if (keep & 2) y.y = u[k].y;
          if (keep & 4) y.z = u[k].z;
          if (keep & 8) y.w = u[k].w;
        }
        *reinterpret_cast<uint4*>(out) = y;
        out += out_step;
      }
      load(h + AHEAD * HEAD_GROUPS, t.heads);
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
  const double two_pi = 6.283185307179586476925, log2_base = std::log2(base);
  int pair = 0;
  for (int a = 0; a < n_axes; ++a)
    for (int i = 0; i < axis_dim[a] / 2; ++i, ++pair) {
      const double f = std::exp2(log2_base * (-2.0 * i / axis_dim[a])) / two_pi;
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

// An output has a place for each row, and that of an input in place is the input's own.
// Strides of axes with one entry say nothing.
bool check_out(const ra_rope_args& a, const ra_rope_tensor& t, int i) {
  const int64_t longer[3] = {a.B, t.heads, a.n};
  const int64_t in[3] = {t.x.stride_b, t.x.stride_h, t.x.stride_n}, out[3] = {t.out.stride_b, t.out.stride_h, t.out.stride_n};
  bool same = true, apart = true;
  for (int k = 0; k < 3; ++k) {
    if (longer[k] < 2) continue;
    same &= in[k] == out[k];
    apart &= out[k] >= a.d;
  }
  if (!apart) {
    set_error("refadapt_rope_axes: tensor %d: the output's rows lie on one another", i);
    return false;
  }
  if (t.x.ptr == t.out.ptr && !same) {
    set_error("refadapt_rope_axes: tensor %d: an output in place needs its input's strides", i);
    return false;
  }
  const ra_rope_tensor& other = a.t[1 - i];
  if (a.n_tensors == 2 && other.heads > 0 && (t.out.ptr == other.out.ptr || t.out.ptr == other.x.ptr)) {
    set_error("refadapt_rope_axes: tensor %d: the output is the other's input or output", i);
    return false;
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
    if (a->n > 0 && !check_out(*a, t, i)) return RA_EINVAL;
    heads += t.heads;
    p.t[i] = Tensor{static_cast<const __nv_bfloat16*>(t.x.ptr), static_cast<__nv_bfloat16*>(t.out.ptr),
                    t.x.stride_b, t.x.stride_h, t.x.stride_n, t.out.stride_b, t.out.stride_h, t.out.stride_n, t.heads, 0};
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
  p.n_tensors = a->n_tensors;
  p.sign = a->inverse ? -1.f : 1.f;
  // 64 slots a CTA; 16, and the heads in more groups, where that leaves SMs idle.
  const bool few = (vecs + 63) / 64 * a->B < 2 * num_sms();
  const int slots = few ? 16 : 64;
  p.blocks = int32_t((vecs + slots - 1) / slots);
  const int64_t grid = int64_t(p.blocks) * a->B;
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, few ? rope_kernel<16> : rope_kernel<64>, p);
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
