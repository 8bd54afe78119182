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
  int32_t groups;  // of a CTA
  float eps, alpha;
  const int32_t* mode;
  Seg seg[3];
};

struct GradParams {
  int32_t B, C, rows, post, pre;
  int32_t groups;
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

// Eight values as four packed pairs (the FMA pipe's two-wide instructions).
struct Vec {
  uint64_t p[4];
};
__device__ __forceinline__ uint64_t both(float v) { return f2_pack(v, v); }
__device__ __forceinline__ Vec widen(uint4 u) { return {{bf2_unpack(u.x), bf2_unpack(u.y), bf2_unpack(u.z), bf2_unpack(u.w)}}; }
__device__ __forceinline__ uint32_t narrow2(uint64_t v) {
  float a, b;
  f2_unpack(v, a, b);
  return pack_bf16x2(a, b);
}
__device__ __forceinline__ uint4 narrow(const Vec& v) {
  return make_uint4(narrow2(v.p[0]), narrow2(v.p[1]), narrow2(v.p[2]), narrow2(v.p[3]));
}
__device__ __forceinline__ Vec all(float v) { return {{both(v), both(v), both(v), both(v)}}; }
// Eight values of an fp32 vector, or `none` where the caller gave no vector.
__device__ __forceinline__ Vec vec8(const float* src, int col, float none) {
  if (!src) return all(none);
  const ulonglong2 a = reinterpret_cast<const ulonglong2*>(src + col)[0], b = reinterpret_cast<const ulonglong2*>(src + col)[1];
  return {{a.x, a.y, b.x, b.y}};
}
__device__ __forceinline__ Vec operator+(const Vec& a, const Vec& b) {
  Vec r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.p[i] = f2_add(a.p[i], b.p[i]);
  return r;
}
__device__ __forceinline__ Vec operator*(const Vec& a, const Vec& b) {
  Vec r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.p[i] = f2_mul(a.p[i], b.p[i]);
  return r;
}
__device__ __forceinline__ Vec fma(const Vec& a, const Vec& b, const Vec& c) {
  Vec r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.p[i] = f2_fma(a.p[i], b.p[i], c.p[i]);
  return r;
}
__device__ __forceinline__ float sum2(uint64_t v) {
  float a, b;
  f2_unpack(v, a, b);
  return a + b;
}

// This thread's place in its group of T warps: piece j < V of a row is columns
// 8 (lane_g + 32 T j); only the last piece can be missing.
template <int V, int T>
struct Place {
  int group, warp, lane_g;
  int pieces;
  bool last;
  float n_warp, inv_n;  // elements of a row in this warp
  __device__ __forceinline__ explicit Place(int C) {
    group = threadIdx.x / (32 * T);
    lane_g = threadIdx.x - group * (32 * T);
    warp = lane_g >> 5;
    pieces = C >> 3;
    last = lane_g + 32 * T * (V - 1) < pieces;
    int n = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) n += min(max(pieces - 32 * (warp + T * j), 0), 32);
    n_warp = float(8 * n);
    inv_n = 1.f / fmaxf(n_warp, 1.f);
  }
  __device__ __forceinline__ bool has(int j) const { return j < V - 1 || last; }
  __device__ __forceinline__ int col(int j) const { return 8 * (lane_g + 32 * T * j); }
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// What the warps of a group hand one another: two entries of four floats per
// warp, two sets in turn, so that one barrier an exchange is enough.
template <int T>
struct Exchange {
  float4* mem;  // of the group: [2][T][2]
  int bar, set;
  __device__ __forceinline__ Exchange(void* base, int group)
      : mem(reinterpret_cast<float4*>(base) + group * 4 * T), bar(1 + group), set(0) {}
  static constexpr int BYTES = 4 * T * int(sizeof(float4));  // of a group
  // Returns the group's entries: warp w's at [2 w] and [2 w + 1].
  __device__ __forceinline__ const float4* swap(int warp, float4 a, float4 b) {
    float4* m = mem + set * 2 * T;
    set ^= 1;
    if ((threadIdx.x & 31) == 0) m[2 * warp] = a, m[2 * warp + 1] = b;
    if (T == 1)
      __syncwarp();
    else
      named_bar_sync(bar, 32 * T);
    return m;
  }
  // Sums of two values over the group.
  __device__ __forceinline__ float2 sums(int warp, float a, float b) {
    a = warp_sum(a), b = warp_sum(b);
    if (T == 1) return make_float2(a, b);
    const float4 e = make_float4(a, b, 0.f, 0.f);
    float4* m = mem + set * 2 * T;
    set ^= 1;
    if ((threadIdx.x & 31) == 0) m[warp] = e;
    named_bar_sync(bar, 32 * T);
    float2 r = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < T; ++w) {
      const float4 t = m[w];
      r.x += t.x, r.y += t.y;
    }
    return r;
  }
};

// A warp's share of a norm's statistics: its mean, the squares around it and
// their count (LAYER), or zero and the squares (RMS).
template <int V, int T>
__device__ __forceinline__ float4 warp_stats(int kind, const Place<V, T>& at, const Vec (&v)[V]) {
  float mean = 0.f;
  uint64_t acc0 = both(0.f), acc1 = acc0;
  if (kind == RA_NORM_LAYER) {
#pragma unroll
    for (int j = 0; j < V; ++j) {  // a missing piece is zeros
      acc0 = f2_add(acc0, f2_add(v[j].p[0], v[j].p[1]));
      acc1 = f2_add(acc1, f2_add(v[j].p[2], v[j].p[3]));
    }
    mean = warp_sum(sum2(f2_add(acc0, acc1))) * at.inv_n;
    acc0 = acc1 = both(0.f);
    const uint64_t neg = both(-mean);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (at.has(j)) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          const uint64_t d0 = f2_add(v[j].p[i], neg), d1 = f2_add(v[j].p[i + 1], neg);
          acc0 = f2_fma(d0, d0, acc0);
          acc1 = f2_fma(d1, d1, acc1);
        }
      }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        acc0 = f2_fma(v[j].p[i], v[j].p[i], acc0);
        acc1 = f2_fma(v[j].p[i + 1], v[j].p[i + 1], acc1);
      }
  }
  return make_float4(mean, warp_sum(sum2(f2_add(acc0, acc1))), at.n_warp, 0.f);
}
// -mean and 1 / deviation of the row from its warps' shares (warp w's at m[2 w]).
template <int T>
__device__ __forceinline__ float2 join_stats(int kind, const float4* m, float inv_c, float eps) {
  float mean = 0.f, sq = 0.f;
  if (kind == RA_NORM_LAYER) {
#pragma unroll
    for (int w = 0; w < T; ++w) {
      const float4 t = m[2 * w];
      mean = fmaf(t.z, t.x, mean);
    }
    mean *= inv_c;
    asm volatile("" ::: "memory");  // read again: 3 T registers would spill
#pragma unroll
    for (int w = 0; w < T; ++w) {
      const float4 t = m[2 * w];
      const float d = t.x - mean;
      sq = fmaf(t.z * d, d, sq + t.y);
    }
  } else {
#pragma unroll
    for (int w = 0; w < T; ++w) sq += m[2 * w].y;
  }
  return make_float2(-mean, rsqrtf(fmaf(sq, inv_c, eps)));
}

// ------------------------------------------------------------------ forward
template <int V, int T>
__global__ void __launch_bounds__(FWD_THREADS, 1) residual_norm_kernel(const __grid_constant__ Params p) {
  constexpr int S = FWD_STAGES;
  extern __shared__ __align__(16) uint8_t smem[];
  // ring[stage][piece of y, of h][thread of the CTA], then the exchange
  const uint32_t piece_bytes = 16 * blockDim.x, stage_bytes = 2 * V * piece_bytes;
  uint8_t* const ring = smem + 16 * threadIdx.x;
  const Place<V, T> at(p.C);
  Exchange<T> ex(smem + S * stage_bytes, at.group);
  const float inv_c = 1.f / float(p.C);
  pdl_launch();
  pdl_wait();
  const int total = live_rows(p);
  const int share = total / int(gridDim.x), more = total - share * int(gridDim.x), cta = int(blockIdx.x);
  const int lo = share * cta + min(cta, more), hi = lo + share + (cta < more ? 1 : 0);
  Piece ld;
  if (lo < hi && p.B > 4) ld.jump(p, lo);
  Piece w = ld;
  // This thread's first piece of the next row to copy and of the row at work, and
  // the steps to the group's next rows; found anew where a (segment, sample) ends.
  const __nv_bfloat16 *h_src = nullptr, *y_src = nullptr;
  __nv_bfloat16 *h_dst = nullptr, *x_dst = nullptr;
  int64_t h_step = 0, y_step = 0, h_out_step = 0, x_step = 0;
  int ld_i = lo + at.group, ld_end = lo, w_end = lo;
  auto load = [&](uint32_t off) {
    if (ld_i < hi) {
      if (ld_i >= ld_end) {
        ld.seek(p, ld_i);
        const Seg& sg = p.seg[ld.g];
        ld_end = ld.begin + sg.rows;
        const int64_t r = ld_i - ld.begin;
        h_src = sg.h + ld.s * sg.h_ss + r * sg.h_sr + at.col(0);
        y_src = sg.y ? sg.y + ld.s * sg.y_ss + r * sg.y_sr + at.col(0) : nullptr;
        h_step = p.groups * sg.h_sr, y_step = sg.y ? p.groups * sg.y_sr : 0;
      }
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (at.has(j)) {
          if (y_src) cp_async16(ring + off + j * piece_bytes, y_src + 256 * T * j);
          cp_async16(ring + off + (V + j) * piece_bytes, h_src + 256 * T * j);
        }
      h_src += h_step, y_src += y_step;
    }
    ld_i += p.groups;
    cp_async_commit();
  };
#pragma unroll
  for (int k = 0; k < S - 1; ++k) load(k * stage_bytes);
  Vec gate[V], mul[V], add[V];
  bool has_y = false;
  uint32_t off = 0, ld_off = (S - 1) * stage_bytes;
  for (int i = lo + at.group; i < hi; i += p.groups) {
    if (i >= w_end) {  // another sample's rows: its vectors
      w.seek(p, i);
      const Seg& sg = p.seg[w.g];
      w_end = w.begin + sg.rows;
      const int64_t r = i - w.begin;
      has_y = sg.y != nullptr;
      h_dst = sg.h_out ? sg.h_out + w.s * sg.o_ss + r * sg.o_sr + at.col(0) : nullptr;
      x_dst = sg.x ? sg.x + w.s * sg.x_ss + r * sg.x_sr + at.col(0) : nullptr;
      h_out_step = sg.h_out ? p.groups * sg.o_sr : 0, x_step = sg.x ? p.groups * sg.x_sr : 0;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (!at.has(j)) continue;
        const int c = at.col(j);
        gate[j] = vec8(sg.gate ? sg.gate + w.s * sg.gate_ss : nullptr, c, 1.f) * vec8(sg.post_w, c, 1.f);
        mul[j] = (vec8(sg.scale ? sg.scale + w.s * sg.mod_ss : nullptr, c, 0.f) + all(1.f)) * vec8(sg.pre_w, c, 1.f);
        add[j] = vec8(sg.shift ? sg.shift + w.s * sg.mod_ss : nullptr, c, 0.f);
      }
    }
    load(ld_off);
    ld_off = off;
    cp_async_wait<S - 1>();
    Vec v[V];
    auto fetch = [&](int q, int j) {
      return widen(at.has(j) ? *reinterpret_cast<const uint4*>(ring + off + (q * V + j) * piece_bytes)
                             : make_uint4(0, 0, 0, 0));
    };
    if (has_y) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = fetch(0, j);
      if (p.post != RA_NORM_NONE) {
        const float4 mine = warp_stats<V, T>(p.post, at, v);
        const float2 st = join_stats<T>(p.post, ex.swap(at.warp, mine, mine), inv_c, p.eps);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (v[j] + all(st.x)) * all(st.y);
      }
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (at.has(j)) v[j] = fma(v[j], gate[j], all(p.alpha) * fetch(1, j));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = all(p.alpha) * fetch(1, j);
    }
    if (!at.last) v[V - 1] = all(0.f);
    if (h_dst) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (at.has(j)) *reinterpret_cast<uint4*>(h_dst + 256 * T * j) = narrow(v[j]);
      h_dst += h_out_step;
    }
    if (x_dst) {
      float2 st = make_float2(0.f, 1.f);
      if (p.pre != RA_NORM_NONE) {
        const float4 mine = warp_stats<V, T>(p.pre, at, v);
        st = join_stats<T>(p.pre, ex.swap(at.warp, mine, mine), inv_c, p.eps);
      }
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (at.has(j))
          *reinterpret_cast<uint4*>(x_dst + 256 * T * j) = narrow(fma((v[j] + all(st.x)) * all(st.y), mul[j], add[j]));
      x_dst += x_step;
    }
    off += stage_bytes;
    if (off == S * stage_bytes) off = 0;
  }
}

// ------------------------------------------------------------------ backward
template <int V, int T>
__global__ void __launch_bounds__(BWD_THREADS, 1) residual_norm_grad_kernel(const __grid_constant__ GradParams p) {
  constexpr int S = BWD_STAGES;
  extern __shared__ __align__(16) uint8_t smem[];
  const uint32_t piece_bytes = 16 * blockDim.x, stage_bytes = 4 * V * piece_bytes;
  uint8_t* const ring = smem + 16 * threadIdx.x;
  const Place<V, T> at(p.C);
  Exchange<T> ex(smem + S * stage_bytes, at.group);
  const float inv_c = 1.f / float(p.C);
  pdl_launch();
  pdl_wait();
  const int s = int(blockIdx.x) / p.parts, part = int(blockIdx.x) - s * p.parts;
  const int lo = int(int64_t(p.rows) * part / p.parts), hi = int(int64_t(p.rows) * (part + 1) / p.parts);
  const int first = lo + at.group;
  // this thread's first piece of the group's next row of h, y, dx and dh_out
  auto start = [&](const __nv_bfloat16* t, int64_t ss, int64_t sr) {
    return t ? t + s * ss + first * sr + at.col(0) : nullptr;
  };
  const __nv_bfloat16 *h = start(p.h, p.h_ss, p.h_sr), *y = start(p.y, p.y_ss, p.y_sr),
                      *dx = start(p.dx, p.dx_ss, p.dx_sr), *dho = start(p.dh_out, p.dho_ss, p.dho_sr);
  const bool has_y = y != nullptr, has_dx = dx != nullptr, has_dho = dho != nullptr;
  int ld_i = first;
  const int64_t h_step = p.groups * p.h_sr, y_step = p.groups * p.y_sr, dx_step = p.groups * p.dx_sr,
                dho_step = p.groups * p.dho_sr;
  auto load = [&](uint32_t off) {
    if (ld_i < hi) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (at.has(j)) {
          uint8_t* to = ring + off + j * piece_bytes;
          cp_async16(to, h + 256 * T * j);
          if (has_y) cp_async16(to + V * piece_bytes, y + 256 * T * j);
          if (has_dx) cp_async16(to + 2 * V * piece_bytes, dx + 256 * T * j);
          if (has_dho) cp_async16(to + 3 * V * piece_bytes, dho + 256 * T * j);
        }
      h += h_step, y += y_step, dx += dx_step, dho += dho_step;
    }
    ld_i += p.groups;
    cp_async_commit();
  };
#pragma unroll
  for (int k = 0; k < S - 1; ++k) load(k * stage_bytes);
  Vec mul[V], gate[V];          // pre_w (1 + scale), gate post_w
  Vec s0[V], s1[V], s2[V];      // column sums of the group's rows
#pragma unroll
  for (int j = 0; j < V; ++j) {
    s0[j] = s1[j] = s2[j] = mul[j] = gate[j] = all(0.f);
    if (!at.has(j)) continue;
    const int c = at.col(j);
    mul[j] = (vec8(p.scale ? p.scale + s * p.mod_ss : nullptr, c, 0.f) + all(1.f)) * vec8(p.pre_w, c, 1.f);
    gate[j] = vec8(p.gate ? p.gate + s * p.gate_ss : nullptr, c, 1.f) * vec8(p.post_w, c, 1.f);
  }
  auto place = [&](__nv_bfloat16* t, int64_t ss, int64_t sr) {
    return t ? t + s * ss + first * sr + at.col(0) : nullptr;
  };
  __nv_bfloat16 *dh = place(p.dh, p.dh_ss, p.dh_sr), *dy = place(p.dy, p.dy_ss, p.dy_sr);
  const int64_t dh_step = p.groups * p.dh_sr, dy_step = p.groups * p.dy_sr;
  uint32_t off = 0, ld_off = (S - 1) * stage_bytes;
  for (int i = first; i < hi; i += p.groups) {
    load(ld_off);
    ld_off = off;
    cp_async_wait<S - 1>();
    auto fetch = [&](bool given, int q, int j) {
      return widen(given && at.has(j) ? *reinterpret_cast<const uint4*>(ring + off + (q * V + j) * piece_bytes)
                                      : make_uint4(0, 0, 0, 0));
    };
    Vec a[V], b[V];  // x^, then dH and what follows from it; y^
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] = fetch(true, 0, j), b[j] = fetch(has_y, 1, j);
    float2 sa = make_float2(0.f, 1.f), sb = sa;
    if (p.pre != RA_NORM_NONE || p.post != RA_NORM_NONE) {
      const float4 ma = warp_stats<V, T>(p.pre, at, a), mb = warp_stats<V, T>(p.post, at, b);
      const float4* m = ex.swap(at.warp, ma, mb);
      if (p.pre != RA_NORM_NONE) sa = join_stats<T>(p.pre, m, inv_c, p.eps);
      if (p.post != RA_NORM_NONE) sb = join_stats<T>(p.post, m + 1, inv_c, p.eps);
    }
    // the norm before the next branch
    uint64_t e0 = both(0.f), e1 = e0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      a[j] = (a[j] + all(sa.x)) * all(sa.y);
      if (!at.has(j)) a[j] = all(0.f);
      const Vec d = fetch(has_dx, 2, j), e = d * mul[j];
      s0[j] = s0[j] + d;
      s1[j] = fma(d, a[j], s1[j]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        e0 = f2_add(e0, e.p[k]);
        e1 = f2_fma(e.p[k], a[j].p[k], e1);
      }
    }
    float2 m = make_float2(0.f, 0.f);
    if (p.pre != RA_NORM_NONE && has_dx) {
      m = ex.sums(at.warp, sum2(e0), sum2(e1));
      m.x = p.pre == RA_NORM_LAYER ? -m.x * inv_c : 0.f;
      m.y *= -inv_c;
    }
    e0 = e1 = both(0.f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      // dH = dh' + r (e - m(e) - x^ m(e x^))
      const Vec e = fma(a[j], all(m.y), fma(fetch(has_dx, 2, j), mul[j], all(m.x)));
      a[j] = fma(e, all(sa.y), fetch(has_dho, 3, j));
      if (!at.has(j)) a[j] = all(0.f);
      b[j] = (b[j] + all(sb.x)) * all(sb.y);
      if (dh && at.has(j)) *reinterpret_cast<uint4*>(dh + 256 * T * j) = narrow(a[j] * all(p.alpha));
      s2[j] = fma(a[j], b[j], s2[j]);
      a[j] = a[j] * gate[j];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        e0 = f2_add(e0, a[j].p[k]);
        e1 = f2_fma(a[j].p[k], b[j].p[k], e1);
      }
    }
    if (dh) dh += dh_step;
    // the norm after the branch
    if (dy) {
      m = make_float2(0.f, 0.f);
      if (p.post != RA_NORM_NONE) {
        m = ex.sums(at.warp, sum2(e0), sum2(e1));
        m.x = p.post == RA_NORM_LAYER ? -m.x * inv_c : 0.f;
        m.y *= -inv_c;
      }
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (at.has(j))
          *reinterpret_cast<uint4*>(dy + 256 * T * j) = narrow(fma(b[j], all(m.y), a[j] + all(m.x)) * all(sb.y));
      dy += dy_step;
    }
    off += stage_bytes;
    if (off == S * stage_bytes) off = 0;
  }
  // The CTA's column sums: its groups' in order, through the ring's memory.
  cp_async_wait<0>();
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);  // [group][3][C]
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (!at.has(j)) continue;
    float* to = sums + at.group * 3 * p.C + at.col(j);
    auto put = [](float* dst, const Vec& v) {
      reinterpret_cast<ulonglong2*>(dst)[0] = make_ulonglong2(v.p[0], v.p[1]);
      reinterpret_cast<ulonglong2*>(dst)[1] = make_ulonglong2(v.p[2], v.p[3]);
    };
    put(to, s0[j]);
    put(to + p.C, s1[j]);
    put(to + 2 * p.C, s2[j]);
  }
  __syncthreads();
  float* out = p.partial + int64_t(blockIdx.x) * 3 * p.C;
  for (int c = threadIdx.x; c < 3 * p.C; c += blockDim.x) {
    float v = 0.f;
    for (int g = 0; g < p.groups; ++g) v += sums[g * 3 * p.C + c];
    out[c] = v;
  }
}

// The column sums of the samples and what follows from them: 32 columns a CTA, up
// to 32 samples at once, whose parts are divided among its 32 warps; the warps'
// sums are then added in order.
struct SumParams {
  int32_t B, C, parts;
  const float* partial;
  const float *gate, *scale, *post_w, *pre_w;
  int64_t gate_ss, mod_ss;
  float *dgate, *dscale, *dshift, *dpost_w, *dpre_w;
};
__global__ void __launch_bounds__(1024) column_sum_kernel(const __grid_constant__ SumParams p) {
  __shared__ float red[3][32][33];
  pdl_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  const bool in = c < p.C;
  pdl_wait();
  float weight = 0.f;  // of dpre_w (warp 1), dpost_w (warp 2)
  for (int s0 = 0; s0 < p.B; s0 += 32) {
    const int n = min(32, p.B - s0), per = 32 / n, mine = warp / per;  // samples, warps of each, this warp's
    float v[3] = {0.f, 0.f, 0.f};
    if (in && mine < n) {
      const float* src = p.partial + (int64_t(s0 + mine) * p.parts + warp % per) * 3 * p.C + c;
#pragma unroll 4
      for (int q = warp % per; q < p.parts; q += per, src += int64_t(per) * 3 * p.C) {
        v[0] += src[0];
        v[1] += src[p.C];
        v[2] += src[2 * p.C];
      }
    }
#pragma unroll
    for (int z = 0; z < 3; ++z) red[z][warp][lane] = v[z];
    __syncthreads();
    if (warp < 3 && in) {
      // warp 0: S0, dshift; 1: S1, dscale and dpre_w; 2: S2, dgate and dpost_w
      float* out = warp == 0 ? p.dshift : warp == 1 ? p.dscale : p.dgate;
      const float* vec = warp == 0 ? nullptr : warp == 1 ? p.scale : p.gate;
      const int64_t vec_ss = warp == 1 ? p.mod_ss : p.gate_ss;
      const float* w = warp == 0 ? nullptr : warp == 1 ? p.pre_w : p.post_w;
      const float own = w ? w[c] : 1.f;
#pragma unroll 4
      for (int s = 0; s < n; ++s) {
        const float f = vec ? vec[(s0 + s) * vec_ss + c] : warp == 1 ? 0.f : 1.f;
        float t = 0.f;
        for (int k = 0; k < per; ++k) t += red[warp][s * per + k][lane];
        if (out) out[int64_t(s0 + s) * p.C + c] = own * t;
        weight = fmaf(warp == 1 ? 1.f + f : f, t, weight);
      }
    }
    __syncthreads();
  }
  if (in && warp == 1 && p.dpre_w) p.dpre_w[c] = weight;
  if (in && warp == 2 && p.dpost_w) p.dpost_w[c] = weight;
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
  int threads() const { return 32 * warps * groups; }
  int exchange() const { return groups * 4 * warps * int(sizeof(float4)); }
};
Shape make_shape(int C, int max_threads) {
  Shape s;
  s.V = C <= 256 ? 1 : 2;
  s.warps = (C / 8 + 32 * s.V - 1) / (32 * s.V);
  s.groups = max_threads / (32 * s.warps);
  if (s.groups > 15) s.groups = 15;  // named barriers
  return s;
}
using Fwd = void (*)(Params);
using Bwd = void (*)(GradParams);
#define RA_RESNORM_PICK(kernel, s)                                                                          \
  (s.V == 1 ? kernel<1, 1>                                                                                  \
   : s.warps == 1 ? kernel<2, 1> : s.warps == 2 ? kernel<2, 2> : s.warps == 3 ? kernel<2, 3>                \
   : s.warps == 4 ? kernel<2, 4> : s.warps == 5 ? kernel<2, 5> : s.warps == 6 ? kernel<2, 6>                \
   : s.warps == 7 ? kernel<2, 7> : s.warps == 8 ? kernel<2, 8> : s.warps == 9 ? kernel<2, 9> : kernel<2, 10>)
static_assert(MAX_C <= 10 * 512, "a group has at most ten warps");

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
  p.groups = sh.groups;
  const int smem = FWD_STAGES * 2 * sh.V * 16 * sh.threads() + sh.exchange();
  const int64_t sms = num_sms();
  const Fwd fn = RA_RESNORM_PICK(residual_norm_kernel, sh);
  return launch(who, fn, p, dim3(unsigned(rows < sms ? rows : sms)), sh.threads(), smem,
                static_cast<cudaStream_t>(stream));
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
  p.groups = sh.groups;
  p.parts = a->rows > 0 ? grad_parts(a->B, a->rows, num_sms()) : 0;
  if (a->rows > 0) {
    const int smem = BWD_STAGES * 4 * sh.V * 16 * sh.threads() + sh.exchange();
    const Bwd fn = RA_RESNORM_PICK(residual_norm_grad_kernel, sh);
    const ra_status r = launch(who, fn, p, dim3(unsigned(a->B * p.parts)), sh.threads(), smem, st);
    if (r != RA_OK) return r;
  }
  if (!a->dpre_w && !a->dpost_w && !a->dgate && !a->dscale && !a->dshift) return RA_OK;
  SumParams q;
  q.B = a->B, q.C = a->C, q.parts = p.parts, q.partial = p.partial;
  q.gate = a->gate, q.gate_ss = a->gate_stride_s, q.scale = a->scale, q.mod_ss = a->mod_stride_s;
  q.post_w = a->post_w, q.pre_w = a->pre_w;
  q.dgate = a->dgate, q.dscale = a->dscale, q.dshift = a->dshift;
  q.dpost_w = a->dpost_w, q.dpre_w = a->dpre_w;
  return launch(who, column_sum_kernel, q, dim3((a->C + 31) / 32), 1024, 0, st);
}
