// refadapt_residual_norm and its backward pass: the norm after a branch, the
// branch's gate, the residual sum and the modulated norm before the next branch.
//
//   h' = alpha h + gate o N_post(y) post_w,   x = N_pre(h') pre_w (1 + scale) + shift
//
// and, from h', y, dx and dh' (N^ the normalised row, r its 1 / deviation, m the
// row mean; the terms in brackets for LAYER only):
//   e = dx pre_w (1 + scale);  dH = dh' + r (e - [m(e)] - x^ m(e x^));  dh = alpha dH
//   f = dH gate post_w;        dy = r_y (f - [m(f)] - y^ m(f y^))
//   per sample S0 = sum dx, S1 = sum dx x^, S2 = sum dH y^ over its rows:
//   dshift = S0, dscale = pre_w S1, dgate = post_w S2,
//   dpre_w = sum_s (1 + scale_s) S1_s,  dpost_w = sum_s gate_s S2_s
//
// HBM-bound: 8 C bytes a row forward (h, y read, h', x written), 12 C backward.
// A row belongs to a group of warps, eight columns per thread and piece, so that
// what a sample's rows share (gate, scale, shift; the column sums) stays in
// registers while a CTA walks its rows: read per row instead, the fp32 vectors
// would be 12 C bytes through L1, more than the row. Each thread copies its own
// pieces of the rows to come into a ring of its own in shared memory (cp.async),
// which needs no barrier and keeps S - 1 rows a group in flight. A warp reduces
// the mean and then the squares around it with shuffles; the warps of a group
// join theirs (count, sum, squares) through shared memory with one barrier.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstring>

#include "api_common.h"
#include "row_walk.cuh"
#include "tc_ptx.cuh"

namespace ra {
namespace resnorm {

constexpr int MAX_C = 5120;
constexpr int FWD_STAGES = 4, BWD_STAGES = 3;
constexpr int FWD_THREADS = 512, BWD_THREADS = 384;  // at most, per CTA: 128 and 168 registers a thread

struct Seg {
  const __nv_bfloat16* h;
  int64_t h_ss, h_sr;
  const __nv_bfloat16* y;
  int64_t y_ss, y_sr;
  __nv_bfloat16* h_out;
  int64_t o_ss, o_sr;
  __nv_bfloat16* x;
  int64_t x_ss, x_sr;
  const float* gate;
  int64_t gate_ss;
  const float* scale;
  const float* shift;
  int64_t mod_ss;
  const float* post_w;
  const float* pre_w;
  int32_t rows, gated;
};

struct Params {
  int32_t n_seg, B, C, post, pre;
  int32_t warps, groups;  // warps of a group, groups of a CTA
  float eps, alpha;
  const int32_t* mode;
  Seg seg[3];
};

struct GradParams {
  int32_t B, C, rows, post, pre;
  int32_t warps, groups;
  int32_t parts;  // CTAs that share a sample's rows
  float eps, alpha;
  const __nv_bfloat16 *h, *y, *dx, *dh_out;
  int64_t h_ss, h_sr, y_ss, y_sr, dx_ss, dx_sr, dho_ss, dho_sr;
  __nv_bfloat16 *dh, *dy;
  int64_t dh_ss, dh_sr, dy_ss, dy_sr;
  const float *gate, *scale, *post_w, *pre_w;
  int64_t gate_ss, mod_ss;
  float* partial;  // [B][parts][3][C]
};

// ------------------------------------------------------------------ pieces of a row
__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void widen(uint4 u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 narrow(const float (&v)[8]) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                    pack_bf16x2(v[6], v[7]));
}
// Eight values of an fp32 vector, or `none` where the caller gave no vector.
__device__ __forceinline__ void vec8(const float* src, int col, float none, float (&v)[8]) {
  if (!src) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = none;
    return;
  }
  const float4 a = reinterpret_cast<const float4*>(src + col)[0], b = reinterpret_cast<const float4*>(src + col)[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

// This thread's place: piece j of a row is columns 8 (lane_g + j threads).
struct Place {
  int group, warp, lane_g, threads;  // group of the CTA, warp of the group, thread of the group, threads of a group
  int C, pieces;
  __device__ __forceinline__ Place(int warps, int C_) {
    threads = 32 * warps;
    group = threadIdx.x / threads;
    lane_g = threadIdx.x - group * threads;
    warp = lane_g >> 5;
    C = C_;
    pieces = C >> 3;
  }
  __device__ __forceinline__ bool has(int j) const { return lane_g + j * threads < pieces; }
  __device__ __forceinline__ int col(int j) const { return 8 * (lane_g + j * threads); }
  // Elements of a row in warp w of the group.
  template <int V>
  __device__ __forceinline__ float count(int w) const {
    int n = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) n += min(max(pieces - (32 * w + j * threads), 0), 32);
    return float(8 * n);
  }
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Values that the warps of a group hand one another: two float2 per warp, two
// sets in turn, so that one barrier an exchange is enough.
constexpr int MAX_WARPS = 16;
struct Exchange {
  float2* mem;  // of the group: [2][warps][2]
  int warps, bar, set;
  __device__ __forceinline__ Exchange(float2* base, const Place& at, int warps_)
      : mem(base + at.group * 4 * warps_), warps(warps_), bar(1 + at.group), set(0) {}
  // Puts the warp's a and b and returns the group's (entry w: a at [2 w], b at [2 w + 1]).
  __device__ __forceinline__ const float2* swap(int warp, float2 a, float2 b) {
    float2* m = mem + set * 2 * warps;
    set ^= 1;
    if ((threadIdx.x & 31) == 0) m[2 * warp] = a, m[2 * warp + 1] = b;
    if (warps == 1)
      __syncwarp();
    else
      named_bar_sync(bar, 32 * warps);
    return m;
  }
  // Sums of two values over the group.
  __device__ __forceinline__ float2 sums(int warp, float a, float b) {
    a = warp_sum(a), b = warp_sum(b);
    if (warps == 1) return make_float2(a, b);
    const float2* m = swap(warp, make_float2(a, b), make_float2(0.f, 0.f));
    float2 r = make_float2(0.f, 0.f);
    for (int w = 0; w < warps; ++w) r.x += m[2 * w].x, r.y += m[2 * w].y;
    return r;
  }
};

// A warp's share of a norm's statistics: its mean and the squares around it
// (LAYER), or zero and the squares (RMS).
template <int V>
__device__ __forceinline__ float2 warp_stats(int kind, const Place& at, const float (&v)[V][8], float n_warp) {
  if (kind == RA_NORM_NONE) return make_float2(0.f, 0.f);
  float mean = 0.f;
  if (kind == RA_NORM_LAYER) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[j][i];  // absent pieces are zeros
    mean = warp_sum(sum) / fmaxf(n_warp, 1.f);
  }
  float sq = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (at.has(j)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sq = fmaf(v[j][i] - mean, v[j][i] - mean, sq);
    }
  return make_float2(mean, warp_sum(sq));
}
// Mean and 1 / deviation of the row from its warps' shares (share w at m[2 w + which]).
template <int V>
__device__ __forceinline__ float2 join_stats(int kind, const Place& at, int warps, const float2* m, int which,
                                             float eps) {
  if (kind == RA_NORM_NONE) return make_float2(0.f, 1.f);
  const float inv_c = 1.f / float(at.C);
  float mean = 0.f, sq = 0.f;
  if (kind == RA_NORM_LAYER) {
    for (int w = 0; w < warps; ++w) mean = fmaf(at.count<V>(w), m[2 * w + which].x, mean);
    mean *= inv_c;
  }
  for (int w = 0; w < warps; ++w) {
    const float2 s = m[2 * w + which];
    sq += s.y;
    if (kind == RA_NORM_LAYER) {
      const float d = s.x - mean;
      sq = fmaf(at.count<V>(w) * d, d, sq);
    }
  }
  return make_float2(mean, rsqrtf(sq * inv_c + eps));
}

// ------------------------------------------------------------------ forward
template <int V>
__global__ void __launch_bounds__(FWD_THREADS, 1) residual_norm_kernel(const __grid_constant__ Params p) {
  constexpr int S = FWD_STAGES;
  extern __shared__ __align__(16) uint8_t smem[];
  // ring[stage][y, h][piece][thread of the CTA], then the exchange
  uint4* ring = reinterpret_cast<uint4*>(smem) + threadIdx.x;
  const int stride = blockDim.x;
  auto slot = [&](int stage, int which, int j) { return ring + ((stage * 2 + which) * V + j) * stride; };
  const Place at(p.warps, p.C);
  Exchange ex(reinterpret_cast<float2*>(smem + size_t(S) * 2 * V * 16 * stride), at, p.warps);
  const float n_warp = at.count<V>(at.warp);
  pdl_launch();
  pdl_wait();
  const int total = live_rows(p);
  const int share = total / int(gridDim.x), more = total - share * int(gridDim.x), cta = int(blockIdx.x);
  const int lo = share * cta + min(cta, more), hi = lo + share + (cta < more ? 1 : 0);
  Piece ld;
  if (lo < hi && p.B > 4) ld.jump(p, lo);
  Piece w = ld;
  int ld_i = lo + at.group;
  auto load = [&](int stage) {
    if (ld_i < hi) {
      ld.seek(p, ld_i);
      const Seg& sg = p.seg[ld.g];
      const int64_t r = ld_i - ld.begin;
      const __nv_bfloat16* h = sg.h + ld.s * sg.h_ss + r * sg.h_sr;
      const __nv_bfloat16* y = sg.y ? sg.y + ld.s * sg.y_ss + r * sg.y_sr : nullptr;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (at.has(j)) {
          if (y) cp_async16(slot(stage, 0, j), y + at.col(j));
          cp_async16(slot(stage, 1, j), h + at.col(j));
        }
    }
    ld_i += p.groups;
    cp_async_commit();
  };
#pragma unroll
  for (int k = 0; k < S - 1; ++k) load(k);
  float gate[V][8], mul[V][8], add[V][8];
  int cur_g = -1, cur_s = -1, stage = 0;
  for (int i = lo + at.group; i < hi; i += p.groups) {
    w.seek(p, i);
    const Seg& sg = p.seg[w.g];
    if (w.g != cur_g || w.s != cur_s) {  // another sample's rows: its vectors
      cur_g = w.g, cur_s = w.s;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (!at.has(j)) continue;
        float t[8];
        vec8(sg.gate ? sg.gate + w.s * sg.gate_ss : nullptr, at.col(j), 1.f, gate[j]);
        vec8(sg.post_w, at.col(j), 1.f, t);
#pragma unroll
        for (int k = 0; k < 8; ++k) gate[j][k] *= t[k];
        vec8(sg.scale ? sg.scale + w.s * sg.mod_ss : nullptr, at.col(j), 0.f, mul[j]);
        vec8(sg.pre_w, at.col(j), 1.f, t);
#pragma unroll
        for (int k = 0; k < 8; ++k) mul[j][k] = (1.f + mul[j][k]) * t[k];
        vec8(sg.shift ? sg.shift + w.s * sg.mod_ss : nullptr, at.col(j), 0.f, add[j]);
      }
    }
    load(stage == 0 ? S - 1 : stage - 1);
    cp_async_wait<S - 1>();
    float v[V][8];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const bool in = at.has(j) && sg.y;
      widen(in ? *slot(stage, 0, j) : make_uint4(0, 0, 0, 0), v[j]);
    }
    float2 st = make_float2(0.f, 1.f);
    if (p.post != RA_NORM_NONE) {
      const float2 mine = warp_stats<V>(p.post, at, v, n_warp);
      st = join_stats<V>(p.post, at, p.warps, ex.swap(at.warp, mine, mine), 0, p.eps);
    }
    const int64_t r = i - w.begin;
    __nv_bfloat16* h_out = sg.h_out ? sg.h_out + w.s * sg.o_ss + r * sg.o_sr : nullptr;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!at.has(j)) continue;
      float h[8];
      widen(*slot(stage, 1, j), h);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        // without y the branch adds nothing, whatever the gate (0 times an infinite gate would be NaN)
        const float z = sg.y ? gate[j][k] * ((v[j][k] - st.x) * st.y) : 0.f;
        v[j][k] = fmaf(p.alpha, h[k], z);
      }
      if (h_out) *reinterpret_cast<uint4*>(h_out + at.col(j)) = narrow(v[j]);
    }
    if (sg.x) {
      if (p.pre != RA_NORM_NONE) {
        const float2 mine = warp_stats<V>(p.pre, at, v, n_warp);
        st = join_stats<V>(p.pre, at, p.warps, ex.swap(at.warp, mine, mine), 0, p.eps);
      } else {
        st = make_float2(0.f, 1.f);
      }
      __nv_bfloat16* x = sg.x + w.s * sg.x_ss + r * sg.x_sr;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (!at.has(j)) continue;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[j][k] = fmaf((v[j][k] - st.x) * st.y, mul[j][k], add[j][k]);
        *reinterpret_cast<uint4*>(x + at.col(j)) = narrow(v[j]);
      }
    }
    if (++stage == S) stage = 0;
  }
}

// ------------------------------------------------------------------ backward
template <int V>
__global__ void __launch_bounds__(BWD_THREADS, 1) residual_norm_grad_kernel(const __grid_constant__ GradParams p) {
  constexpr int S = BWD_STAGES;
  extern __shared__ __align__(16) uint8_t smem[];
  uint4* ring = reinterpret_cast<uint4*>(smem) + threadIdx.x;
  const int stride = blockDim.x;
  auto slot = [&](int stage, int which, int j) { return ring + ((stage * 4 + which) * V + j) * stride; };
  const Place at(p.warps, p.C);
  Exchange ex(reinterpret_cast<float2*>(smem + size_t(S) * 4 * V * 16 * stride), at, p.warps);
  const float n_warp = at.count<V>(at.warp), inv_c = 1.f / float(p.C);
  pdl_launch();
  pdl_wait();
  const int s = int(blockIdx.x) / p.parts, part = int(blockIdx.x) - s * p.parts;
  const int lo = int(int64_t(p.rows) * part / p.parts), hi = int(int64_t(p.rows) * (part + 1) / p.parts);
  const __nv_bfloat16* src[4] = {p.h + s * p.h_ss, p.y ? p.y + s * p.y_ss : nullptr,
                                 p.dx ? p.dx + s * p.dx_ss : nullptr, p.dh_out ? p.dh_out + s * p.dho_ss : nullptr};
  const int64_t sr[4] = {p.h_sr, p.y_sr, p.dx_sr, p.dho_sr};
  int ld_i = lo + at.group;
  auto load = [&](int stage) {
    if (ld_i < hi) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (!src[q]) continue;
        const __nv_bfloat16* row = src[q] + ld_i * sr[q];
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (at.has(j)) cp_async16(slot(stage, q, j), row + at.col(j));
      }
    }
    ld_i += p.groups;
    cp_async_commit();
  };
#pragma unroll
  for (int k = 0; k < S - 1; ++k) load(k);
  float mul[V][8], gate[V][8];             // pre_w (1 + scale), gate post_w
  float s0[V][8], s1[V][8], s2[V][8];      // column sums of the group's rows
#pragma unroll
  for (int j = 0; j < V; ++j) {
#pragma unroll
    for (int k = 0; k < 8; ++k) s0[j][k] = s1[j][k] = s2[j][k] = mul[j][k] = gate[j][k] = 0.f;
    if (!at.has(j)) continue;
    float t[8];
    vec8(p.scale ? p.scale + s * p.mod_ss : nullptr, at.col(j), 0.f, mul[j]);
    vec8(p.pre_w, at.col(j), 1.f, t);
#pragma unroll
    for (int k = 0; k < 8; ++k) mul[j][k] = (1.f + mul[j][k]) * t[k];
    vec8(p.gate ? p.gate + s * p.gate_ss : nullptr, at.col(j), 1.f, gate[j]);
    vec8(p.post_w, at.col(j), 1.f, t);
#pragma unroll
    for (int k = 0; k < 8; ++k) gate[j][k] *= t[k];
  }
  int stage = 0;
  for (int i = lo + at.group; i < hi; i += p.groups) {
    load(stage == 0 ? S - 1 : stage - 1);
    cp_async_wait<S - 1>();
    float a[V][8], b[V][8];  // x^ and then dH; y^
    auto fetch = [&](int q, int j, float (&v)[8]) {
      widen(src[q] && at.has(j) ? *slot(stage, q, j) : make_uint4(0, 0, 0, 0), v);
    };
#pragma unroll
    for (int j = 0; j < V; ++j) fetch(0, j, a[j]), fetch(1, j, b[j]);
    float2 sa = make_float2(0.f, 1.f), sb = sa;
    if (p.pre != RA_NORM_NONE || p.post != RA_NORM_NONE) {
      const float2 ma = warp_stats<V>(p.pre, at, a, n_warp), mb = warp_stats<V>(p.post, at, b, n_warp);
      const float2* m = ex.swap(at.warp, ma, mb);
      sa = join_stats<V>(p.pre, at, p.warps, m, 0, p.eps);
      sb = join_stats<V>(p.post, at, p.warps, m, 1, p.eps);
    }
    // the norm before the next branch
    float e0 = 0.f, e1 = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float dx[8];
      fetch(2, j, dx);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        a[j][k] = at.has(j) ? (a[j][k] - sa.x) * sa.y : 0.f;
        s0[j][k] += dx[k];
        s1[j][k] = fmaf(dx[k], a[j][k], s1[j][k]);
        const float e = dx[k] * mul[j][k];
        e0 += e;
        e1 = fmaf(e, a[j][k], e1);
      }
    }
    float2 m = make_float2(0.f, 0.f);
    if (p.pre != RA_NORM_NONE && p.dx) {
      m = ex.sums(at.warp, e0, e1);
      m.x = p.pre == RA_NORM_LAYER ? m.x * inv_c : 0.f;
      m.y *= inv_c;
    }
    __nv_bfloat16* dh = p.dh ? p.dh + s * p.dh_ss + i * p.dh_sr : nullptr;
    float f0 = 0.f, f1 = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!at.has(j)) continue;
      float dx[8], dho[8], out[8];
      fetch(2, j, dx);
      fetch(3, j, dho);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        a[j][k] = fmaf(sa.y, dx[k] * mul[j][k] - m.x - a[j][k] * m.y, dho[k]);
        b[j][k] = (b[j][k] - sb.x) * sb.y;
        out[k] = p.alpha * a[j][k];
        s2[j][k] = fmaf(a[j][k], b[j][k], s2[j][k]);
        a[j][k] *= gate[j][k];
        f0 += a[j][k];
        f1 = fmaf(a[j][k], b[j][k], f1);
      }
      if (dh) *reinterpret_cast<uint4*>(dh + at.col(j)) = narrow(out);
    }
    // the norm after the branch
    if (p.dy) {
      m = make_float2(0.f, 0.f);
      if (p.post != RA_NORM_NONE) {
        m = ex.sums(at.warp, f0, f1);
        m.x = p.post == RA_NORM_LAYER ? m.x * inv_c : 0.f;
        m.y *= inv_c;
      }
      __nv_bfloat16* dy = p.dy + s * p.dy_ss + i * p.dy_sr;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (!at.has(j)) continue;
        float out[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) out[k] = sb.y * (a[j][k] - m.x - b[j][k] * m.y);
        *reinterpret_cast<uint4*>(dy + at.col(j)) = narrow(out);
      }
    }
    if (++stage == S) stage = 0;
  }
  // The CTA's column sums: its groups' in order, through the ring's memory.
  cp_async_wait<0>();
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);  // [group][3][C]
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (!at.has(j)) continue;
    float* at0 = sums + size_t(at.group) * 3 * p.C + at.col(j);
#pragma unroll
    for (int k = 0; k < 8; ++k) at0[k] = s0[j][k], at0[p.C + k] = s1[j][k], at0[2 * p.C + k] = s2[j][k];
  }
  __syncthreads();
  float* out = p.partial + int64_t(blockIdx.x) * 3 * p.C;
  for (int c = threadIdx.x; c < 3 * p.C; c += blockDim.x) {
    float v = 0.f;
    for (int g = 0; g < p.groups; ++g) v += sums[size_t(g) * 3 * p.C + c];
    out[c] = v;
  }
}

// Sums of a sample's parts: 32 columns by 32 slices of the parts a CTA, the
// slices then added in order. Writes the sample's gradients, and S1 and S2
// (over its first part) where weights want them summed over the samples.
struct SumParams {
  int32_t B, C, parts;
  float* partial;
  const float *post_w, *pre_w;
  float *dgate, *dscale, *dshift;
  bool keep;
};
__global__ void __launch_bounds__(1024) column_sum_kernel(const SumParams p) {
  __shared__ float red[3][32][33];
  pdl_launch();
  pdl_wait();
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, s = blockIdx.y;
  const int c = blockIdx.x * 32 + lane;
  float v[3] = {0.f, 0.f, 0.f};
  if (c < p.C)
    for (int q = slice; q < p.parts; q += 32) {
      const float* src = p.partial + (int64_t(s) * p.parts + q) * 3 * p.C + c;
#pragma unroll
      for (int z = 0; z < 3; ++z) v[z] += src[int64_t(z) * p.C];
    }
#pragma unroll
  for (int z = 0; z < 3; ++z) red[z][slice][lane] = v[z];
  __syncthreads();
  if (slice >= 3 || c >= p.C) return;
  const int z = slice;
  float t = 0.f;
#pragma unroll
  for (int q = 0; q < 32; ++q) t += red[z][q][lane];
  const int64_t at = int64_t(s) * p.C + c;
  if (z == 0) {
    if (p.dshift) p.dshift[at] = t;
  } else if (z == 1) {
    if (p.dscale) p.dscale[at] = p.pre_w ? p.pre_w[c] * t : t;
  } else {
    if (p.dgate) p.dgate[at] = p.post_w ? p.post_w[c] * t : t;
  }
  // every part of these columns of the sample has been read (the barrier above)
  if (p.keep && p.parts > 0) p.partial[int64_t(s) * p.parts * 3 * p.C + int64_t(z) * p.C + c] = t;
}

// dpre_w and dpost_w: sums over the samples, in order.
__global__ void __launch_bounds__(128) weight_sum_kernel(const float* partial, int B, int C, int parts,
                                                         const float* gate, int64_t gate_ss, const float* scale,
                                                         int64_t mod_ss, float* dpost_w, float* dpre_w) {
  pdl_launch();
  pdl_wait();
  const int c = blockIdx.x * 128 + threadIdx.x;
  if (c >= C) return;
  float pre = 0.f, post = 0.f;
  if (parts > 0)
#pragma unroll 4
    for (int s = 0; s < B; ++s) {
      const float* src = partial + int64_t(s) * parts * 3 * C + c;
      pre = fmaf(scale ? 1.f + scale[s * mod_ss + c] : 1.f, src[C], pre);
      post = fmaf(gate ? gate[s * gate_ss + c] : 1.f, src[2 * C], post);
    }
  if (dpre_w) dpre_w[c] = pre;
  if (dpost_w) dpost_w[c] = post;
}

// ------------------------------------------------------------------ host
bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

// A row tensor (or none): 16-byte aligned, strides whole 16-byte pieces, rows not
// overlapping; an output of B > 1 samples (out_b) has a place for each.
bool check_rows(const char* who, const char* what, const void* ptr, int64_t ss, int64_t sr, int C, int out_b = 0) {
  if (!ptr || (aligned16(ptr) && ss % 8 == 0 && sr % 8 == 0 && ss >= (out_b > 1 ? C : 0) && sr >= C)) return true;
  set_error("%s: %s must be 16-byte aligned with strides multiples of 8 elements, row stride >= C (and sample stride of "
            "an output)", who, what);
  return false;
}
bool check_vec(const char* who, const char* what, const void* ptr, int64_t ss) {
  if (aligned16(ptr) && ss % 4 == 0 && ss >= 0) return true;
  set_error("%s: %s must be 16-byte aligned, its row stride a multiple of 4", who, what);
  return false;
}
// Where an output shares memory with an input only in place: `a` may be `b` or lie apart from it.
bool same_or_apart(const void* a, int64_t a_ss, int64_t a_sr, const void* b, int64_t b_ss, int64_t b_sr) {
  return a != b || (a_ss == b_ss && a_sr == b_sr);
}

template <class P>
ra_status launch(const char* who, void (*fn)(P), const P& p, dim3 grid, int threads, int smem, cudaStream_t st) {
  if (smem > 48 * 1024) {
    const ra_status as = ensure_dynamic_smem(reinterpret_cast<const void*>(fn), 200 * 1024, who);
    if (as != RA_OK) return as;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, p);
  if (e != cudaSuccess) {
    set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
    cudaGetLastError();
    return RA_ECUDA;
  }
  return launch_status(who);
}

// Pieces per thread, warps of a row's group, groups of a CTA.
struct Shape {
  int V, warps, groups;
};
Shape make_shape(int C, int max_threads) {
  Shape s;
  s.V = C <= 256 ? 1 : 2;
  s.warps = (C / 8 + 32 * s.V - 1) / (32 * s.V);
  s.groups = max_threads / (32 * s.warps);
  if (s.groups > 15) s.groups = 15;  // named barriers
  return s;
}

// CTAs that share a sample's rows: as many as make the fewest rounds of rows.
int grad_parts(int B, int rows, int sms) {
  int best = 1;
  int64_t best_cost = INT64_MAX;
  for (int parts = 1; parts <= rows && int64_t(parts) * B <= int64_t(2) * sms + B; ++parts) {
    const int64_t rounds = (int64_t(parts) * B + sms - 1) / sms, cost = rounds * ((rows + parts - 1) / parts);
    if (cost < best_cost) best_cost = cost, best = parts;
  }
  return best;
}

}  // namespace resnorm
}  // namespace ra

extern "C" ra_status refadapt_residual_norm(const ra_resnorm_args* a, void* stream) {
  using namespace ra;
  using namespace ra::resnorm;
  const char* who = "refadapt_residual_norm";
  clear_error();
  if (!a) {
    set_error("%s: args is NULL", who);
    return RA_EINVAL;
  }
  if (a->B < 1 || a->n_seg < 1 || a->n_seg > 3 || a->C < 8 || a->C % 8 != 0 || a->C > MAX_C || !(a->eps >= 0.f) ||
      a->post < RA_NORM_NONE || a->post > RA_NORM_RMS || a->pre < RA_NORM_NONE || a->pre > RA_NORM_RMS) {
    set_error("%s: need B >= 1, 1 <= n_seg <= 3, C a multiple of 8 in [8, 5120], eps >= 0 and known norms (B=%d n_seg=%d "
              "C=%d post=%d pre=%d)", who, a->B, a->n_seg, a->C, a->post, a->pre);
    return RA_EINVAL;
  }
  Params p;
  std::memset(&p, 0, sizeof(p));
  p.n_seg = a->n_seg;
  p.B = a->B;
  p.C = a->C;
  p.post = a->post;
  p.pre = a->pre;
  p.eps = a->eps;
  p.alpha = a->alpha;
  p.mode = a->mode;
  int64_t rows = 0;
  for (int g = 0; g < a->n_seg; ++g) {
    const ra_resnorm_seg& s = a->seg[g];
    Seg& d = p.seg[g];
    if (s.rows < 0) {
      set_error("%s: seg %d rows < 0", who, g);
      return RA_EINVAL;
    }
    d.rows = s.rows;
    d.gated = s.gated ? 1 : 0;
    if (s.gated && !a->mode) {
      set_error("%s: seg %d is gated but mode is NULL", who, g);
      return RA_EINVAL;
    }
    if (s.rows == 0) continue;
    if (!s.h || (!s.h_out && !s.x)) {
      set_error("%s: seg %d: h is NULL, or both outputs are", who, g);
      return RA_EINVAL;
    }
    if (!check_rows(who, "h", s.h, s.h_stride_s, s.h_stride_r, a->C) ||
        !check_rows(who, "y", s.y, s.y_stride_s, s.y_stride_r, a->C) ||
        !check_rows(who, "h_out", s.h_out, s.h_out_stride_s, s.h_out_stride_r, a->C, a->B) ||
        !check_rows(who, "x", s.x, s.x_stride_s, s.x_stride_r, a->C, a->B) ||
        !check_vec(who, "gate", s.gate, s.gate_stride_s) || !check_vec(who, "scale", s.scale, s.mod_stride_s) ||
        !check_vec(who, "shift", s.shift, s.mod_stride_s) || !check_vec(who, "post_w", s.post_w, 0) ||
        !check_vec(who, "pre_w", s.pre_w, 0))
      return RA_EINVAL;
    if (s.x && s.x == s.h_out) {
      set_error("%s: seg %d: h_out and x are the same tensor", who, g);
      return RA_EINVAL;
    }
    if (!same_or_apart(s.h_out, s.h_out_stride_s, s.h_out_stride_r, s.h, s.h_stride_s, s.h_stride_r) ||
        !same_or_apart(s.h_out, s.h_out_stride_s, s.h_out_stride_r, s.y, s.y_stride_s, s.y_stride_r) ||
        !same_or_apart(s.x, s.x_stride_s, s.x_stride_r, s.h, s.h_stride_s, s.h_stride_r) ||
        !same_or_apart(s.x, s.x_stride_s, s.x_stride_r, s.y, s.y_stride_s, s.y_stride_r)) {
      set_error("%s: seg %d: an output in place needs its input's strides", who, g);
      return RA_EINVAL;
    }
    d.h = static_cast<const __nv_bfloat16*>(s.h);
    d.h_ss = s.h_stride_s, d.h_sr = s.h_stride_r;
    d.y = static_cast<const __nv_bfloat16*>(s.y);
    d.y_ss = s.y_stride_s, d.y_sr = s.y_stride_r;
    d.h_out = static_cast<__nv_bfloat16*>(s.h_out);
    d.o_ss = s.h_out_stride_s, d.o_sr = s.h_out_stride_r;
    d.x = static_cast<__nv_bfloat16*>(s.x);
    d.x_ss = s.x_stride_s, d.x_sr = s.x_stride_r;
    d.gate = s.gate, d.gate_ss = s.gate_stride_s;
    d.scale = s.scale, d.shift = s.shift, d.mod_ss = s.mod_stride_s;
    d.post_w = s.post_w, d.pre_w = s.pre_w;
    rows += int64_t(a->B) * s.rows;
  }
  if (rows == 0) return RA_OK;
  if (rows >= (int64_t(1) << 30)) {
    set_error("%s: too many rows", who);
    return RA_EINVAL;
  }
  const Shape sh = make_shape(a->C, FWD_THREADS);
  p.warps = sh.warps;
  p.groups = sh.groups;
  const int threads = 32 * sh.warps * sh.groups;
  const int smem = FWD_STAGES * 2 * sh.V * 16 * threads + sh.groups * 4 * sh.warps * int(sizeof(float2));
  const int64_t sms = num_sms();
  return launch(who, sh.V == 1 ? residual_norm_kernel<1> : residual_norm_kernel<2>, p,
                dim3(unsigned(rows < sms ? rows : sms)), threads, smem, static_cast<cudaStream_t>(stream));
}

extern "C" size_t refadapt_residual_norm_backward_workspace_size(int32_t B, int32_t rows, int32_t C) {
  using namespace ra::resnorm;
  if (B < 1 || rows < 0 || C < 8 || C > MAX_C) return 0;
  const size_t parts = rows > 0 ? size_t(grad_parts(B, rows, ra::num_sms())) : 1;
  return size_t(B) * parts * 3 * size_t(C) * sizeof(float);
}

extern "C" ra_status refadapt_residual_norm_backward(const ra_resnorm_grad_args* a, void* stream) {
  using namespace ra;
  using namespace ra::resnorm;
  const char* who = "refadapt_residual_norm_backward";
  clear_error();
  if (!a) {
    set_error("%s: args is NULL", who);
    return RA_EINVAL;
  }
  if (a->B < 1 || a->rows < 0 || a->C < 8 || a->C % 8 != 0 || a->C > MAX_C || !(a->eps >= 0.f) ||
      a->post < RA_NORM_NONE || a->post > RA_NORM_RMS || a->pre < RA_NORM_NONE || a->pre > RA_NORM_RMS) {
    set_error("%s: need B >= 1, rows >= 0, C a multiple of 8 in [8, 5120], eps >= 0 and known norms (B=%d rows=%d C=%d "
              "post=%d pre=%d)", who, a->B, a->rows, a->C, a->post, a->pre);
    return RA_EINVAL;
  }
  if (int64_t(a->B) * a->rows >= (int64_t(1) << 30) || a->B > 65535) {
    set_error("%s: too many rows or samples", who);
    return RA_EINVAL;
  }
  if (a->rows > 0) {
    if (!a->h || (!a->dx && !a->dh_out)) {
      set_error("%s: h is NULL, or dx and dh_out both are", who);
      return RA_EINVAL;
    }
    if (!check_rows(who, "h", a->h, a->h_stride_s, a->h_stride_r, a->C) ||
        !check_rows(who, "y", a->y, a->y_stride_s, a->y_stride_r, a->C) ||
        !check_rows(who, "dx", a->dx, a->dx_stride_s, a->dx_stride_r, a->C) ||
        !check_rows(who, "dh_out", a->dh_out, a->dh_out_stride_s, a->dh_out_stride_r, a->C) ||
        !check_rows(who, "dh", a->dh, a->dh_stride_s, a->dh_stride_r, a->C, a->B) ||
        !check_rows(who, "dy", a->dy, a->dy_stride_s, a->dy_stride_r, a->C, a->B))
      return RA_EINVAL;
    if (!a->y && (a->dy || a->dgate || a->dpost_w)) {
      set_error("%s: without y there is no dy, dgate or dpost_w", who);
      return RA_EINVAL;
    }
    if ((a->dy && a->dy == a->dh) ||
        !same_or_apart(a->dh, a->dh_stride_s, a->dh_stride_r, a->dh_out, a->dh_out_stride_s, a->dh_out_stride_r) ||
        !same_or_apart(a->dh, a->dh_stride_s, a->dh_stride_r, a->dx, a->dx_stride_s, a->dx_stride_r) ||
        !same_or_apart(a->dy, a->dy_stride_s, a->dy_stride_r, a->y, a->y_stride_s, a->y_stride_r)) {
      set_error("%s: dh and dy are the same tensor, or an output in place has other strides than its input", who);
      return RA_EINVAL;
    }
  }
  if (!check_vec(who, "gate", a->gate, a->gate_stride_s) || !check_vec(who, "scale", a->scale, a->mod_stride_s) ||
      !check_vec(who, "post_w", a->post_w, 0) || !check_vec(who, "pre_w", a->pre_w, 0))
    return RA_EINVAL;
  if (!a->workspace || !aligned16(a->workspace) ||
      a->workspace_bytes < refadapt_residual_norm_backward_workspace_size(a->B, a->rows, a->C)) {
    set_error("%s: workspace NULL, not 16-byte aligned or smaller than "
              "refadapt_residual_norm_backward_workspace_size(%d, %d, %d)", who, a->B, a->rows, a->C);
    return RA_EINVAL;
  }
  GradParams p;
  std::memset(&p, 0, sizeof(p));
  p.B = a->B, p.C = a->C, p.rows = a->rows, p.post = a->post, p.pre = a->pre;
  p.eps = a->eps, p.alpha = a->alpha;
  p.h = static_cast<const __nv_bfloat16*>(a->h), p.h_ss = a->h_stride_s, p.h_sr = a->h_stride_r;
  p.y = static_cast<const __nv_bfloat16*>(a->y), p.y_ss = a->y_stride_s, p.y_sr = a->y_stride_r;
  p.dx = static_cast<const __nv_bfloat16*>(a->dx), p.dx_ss = a->dx_stride_s, p.dx_sr = a->dx_stride_r;
  p.dh_out = static_cast<const __nv_bfloat16*>(a->dh_out);
  p.dho_ss = a->dh_out_stride_s, p.dho_sr = a->dh_out_stride_r;
  p.dh = static_cast<__nv_bfloat16*>(a->dh), p.dh_ss = a->dh_stride_s, p.dh_sr = a->dh_stride_r;
  p.dy = static_cast<__nv_bfloat16*>(a->dy), p.dy_ss = a->dy_stride_s, p.dy_sr = a->dy_stride_r;
  p.gate = a->gate, p.gate_ss = a->gate_stride_s;
  p.scale = a->scale, p.mod_ss = a->mod_stride_s;
  p.post_w = a->post_w, p.pre_w = a->pre_w;
  p.partial = static_cast<float*>(a->workspace);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const Shape sh = make_shape(a->C, BWD_THREADS);
  p.warps = sh.warps;
  p.groups = sh.groups;
  p.parts = a->rows > 0 ? grad_parts(a->B, a->rows, num_sms()) : 0;
  if (a->rows > 0) {
    const int threads = 32 * sh.warps * sh.groups;
    const int ring = BWD_STAGES * 4 * sh.V * 16 * threads;
    const int smem = ring + sh.groups * 4 * sh.warps * int(sizeof(float2));
    const ra_status r = launch(who, sh.V == 1 ? residual_norm_grad_kernel<1> : residual_norm_grad_kernel<2>, p,
                               dim3(unsigned(a->B * p.parts)), threads, smem, st);
    if (r != RA_OK) return r;
  }
  const bool weights = a->dpre_w || a->dpost_w;
  if (!weights && !a->dgate && !a->dscale && !a->dshift) return RA_OK;
  SumParams q;
  q.B = a->B, q.C = a->C, q.parts = p.parts, q.partial = p.partial;
  q.post_w = a->post_w, q.pre_w = a->pre_w;
  q.dgate = a->dgate, q.dscale = a->dscale, q.dshift = a->dshift;
  q.keep = weights;
  const ra_status r = launch(who, column_sum_kernel, q, dim3((a->C + 31) / 32, a->B), 1024, 0, st);
  if (r != RA_OK || !weights) return r;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((a->C + 127) / 128);
  cfg.blockDim = dim3(128);
  cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, weight_sum_kernel, static_cast<const float*>(p.partial), int(a->B),
                                           int(a->C), int(p.parts), a->gate, a->gate_stride_s, a->scale,
                                           a->mod_stride_s, a->dpost_w, a->dpre_w);
  if (e != cudaSuccess) {
    set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
    cudaGetLastError();
    return RA_ECUDA;
  }
  return launch_status(who);
}
