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
// What holds it up is the latency of the reductions between. A row belongs to a
// group of warps, one or two pieces of eight columns a thread. Forward, a group works
// on two rows of a sample at once: their reductions share shuffles and barriers, and
// their instructions fill each other's latencies (backward, the norms' two reductions
// go together likewise; two rows would spill). A thread copies its own pieces of the
// rows to come into a ring of its own in shared memory (cp.async: no barrier);
// what a sample's rows share (gate, scale, shift with the weights; 12 C bytes, more
// than the row) lies in shared memory, the column sums of the backward pass in
// registers. A warp reduces the mean and then the squares around it; the warps of a
// group join theirs (count, mean, squares) through shared memory with one barrier.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstring>

#include "api_common.h"
#include "row_walk.cuh"
#include "tc_ptx.cuh"

namespace ra {
namespace resnorm {

constexpr int MAX_C = 5120;
constexpr int MAX_PIECES = 2;                        // of a row, a thread's at most
constexpr int FWD_THREADS = 640, BWD_THREADS = 384;  // of a CTA at most: 96 and 168 registers a thread
constexpr int MAX_STAGES = 4;                        // rows of a group in its ring
constexpr int SMEM_MAX = 227 * 1024;

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
  int32_t groups, stages;  // of a CTA; of a ring
  float eps, alpha;
  const int32_t* mode;
  Seg seg[3];
};

struct GradParams {
  int32_t B, C, rows, post, pre;
  int32_t groups, stages;
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
// All but the newest n of this thread's copies have landed.
__device__ __forceinline__ void cp_async_wait_upto(int n) {
  static_assert(MAX_STAGES == 4, "one case per ring length");
  if (n == 1)
    cp_async_wait<1>();
  else if (n == 2)
    cp_async_wait<2>();
  else
    cp_async_wait<3>();
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
// 8 (lane_g + 32 T j); the last piece can be missing.
template <int V, int T>
struct Place {
  int group, warp, lane_g;
  bool last;
  float inv_n;  // 1 / elements of a row in this warp
  __device__ __forceinline__ explicit Place(int C) {
    group = threadIdx.x / (32 * T);
    lane_g = threadIdx.x - group * (32 * T);
    warp = lane_g >> 5;
    const int pieces = C >> 3;
    last = lane_g + 32 * T * (V - 1) < pieces;
    inv_n = 1.f / fmaxf(count(warp, pieces), 1.f);
  }
  __device__ __forceinline__ bool has(int j) const { return j < V - 1 || last; }
  __device__ __forceinline__ int col(int j) const { return 8 * (lane_g + 32 * T * j); }
  // Elements of a row in warp w of the group.
  static __device__ __forceinline__ float count(int w, int pieces) {
    return float(256 * (V - 1) + 8 * min(max(pieces - 32 * (w + T * (V - 1)), 0), 32));
  }
};

// Two sums in the shuffles of one: even lanes get a's, odd lanes b's.
__device__ __forceinline__ float warp_sum2(float a, float b) {
  const bool odd = threadIdx.x & 1;
  float v = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
#pragma unroll
  for (int o = 16; o > 1; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// What the warps of a group hand one another: four floats per warp, two sets in
// turn, so that one barrier an exchange is enough.
template <int T>
struct Exchange {
  float4* mem;  // of the group: [2][T]
  int bar, set;
  static constexpr int BYTES = 2 * T * 16;
  __device__ __forceinline__ Exchange(void* base, int group)
      : mem(reinterpret_cast<float4*>(base) + group * 2 * T), bar(1 + group), set(0) {}
  __device__ __forceinline__ float* entries() {
    float4* m = mem + set * T;
    set ^= 1;
    return reinterpret_cast<float*>(m);
  }
  __device__ __forceinline__ void meet() {
    if (T == 1)
      __syncwarp();
    else
      named_bar_sync(bar, 32 * T);
  }
  // Sums of two values over the group.
  __device__ __forceinline__ float2 sums(int warp, float a, float b) {
    const float v = warp_sum2(a, b);
    float* m = entries();
    if ((threadIdx.x & 30) == 0) m[2 * warp + (threadIdx.x & 1)] = v;
    meet();
    const float2* e = reinterpret_cast<const float2*>(m);
    float2 r = e[0];
#pragma unroll
    for (int w = 1; w < T; ++w) {
      const float2 t = e[w];
      r.x += t.x, r.y += t.y;
    }
    return r;
  }
};

template <int V>
__device__ __forceinline__ float sum_of(const Vec (&v)[V]) {  // missing pieces are zeros
  uint64_t a = f2_add(v[0].p[0], v[0].p[1]), b = f2_add(v[0].p[2], v[0].p[3]);
#pragma unroll
  for (int j = 1; j < V; ++j) {
    a = f2_add(a, f2_add(v[j].p[0], v[j].p[1]));
    b = f2_add(b, f2_add(v[j].p[2], v[j].p[3]));
  }
  return sum2(f2_add(a, b));
}
template <int V, int T>
__device__ __forceinline__ float squares_around(const Place<V, T>& at, const Vec (&v)[V], float mean) {
  uint64_t a = both(0.f), b = a;
  const uint64_t neg = both(-mean);
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (at.has(j)) {
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const uint64_t d0 = f2_add(v[j].p[i], neg), d1 = f2_add(v[j].p[i + 1], neg);
        a = f2_fma(d0, d0, a);
        b = f2_fma(d1, d1, b);
      }
    }
  return sum2(f2_add(a, b));
}
template <int V>
__device__ __forceinline__ float squares_of(const Vec (&v)[V]) {
  uint64_t a = both(0.f), b = a;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      a = f2_fma(v[j].p[i], v[j].p[i], a);
      b = f2_fma(v[j].p[i + 1], v[j].p[i + 1], b);
    }
  return sum2(f2_add(a, b));
}

// -mean and 1 / deviation of two rows from their warps' shares, four floats each:
// mean and squares around it of the one row and of the other. layer: the means
// count (those of RMS are zeros).
template <int V, int T>
__device__ __forceinline__ float4 join_stats(bool layer, const float4* m, int pieces, float inv_c, float eps) {
  float mean0 = 0.f, mean1 = 0.f, sq0 = 0.f, sq1 = 0.f;
  if (T == 1) {
    const float4 t = m[0];
    mean0 = t.x, sq0 = t.y, mean1 = t.z, sq1 = t.w;
  } else if (layer) {
#pragma unroll
    for (int w = 0; w < T; ++w) {
      const float n = Place<V, T>::count(w, pieces);
      const float4 t = m[w];
      mean0 = fmaf(n, t.x, mean0), mean1 = fmaf(n, t.z, mean1);
    }
    mean0 *= inv_c, mean1 *= inv_c;
    asm volatile("" ::: "memory");  // read again: the entries of all warps would spill
#pragma unroll
    for (int w = 0; w < T; ++w) {
      const float n = Place<V, T>::count(w, pieces);
      const float4 t = m[w];
      const float d0 = t.x - mean0, d1 = t.z - mean1;
      sq0 = fmaf(n * d0, d0, sq0 + t.y), sq1 = fmaf(n * d1, d1, sq1 + t.w);
    }
  } else {
#pragma unroll
    for (int w = 0; w < T; ++w) {
      const float4 t = m[w];
      sq0 += t.y, sq1 += t.w;
    }
  }
  return make_float4(-mean0, rsqrtf(fmaf(sq0, inv_c, eps)), -mean1, rsqrtf(fmaf(sq1, inv_c, eps)));
}

// The statistics of two rows, of kinds k0 and k1 (one at least is a norm).
template <int V, int T>
__device__ __forceinline__ float4 row_stats(int k0, int k1, const Place<V, T>& at, Exchange<T>& ex, const Vec (&v0)[V],
                                            const Vec (&v1)[V], int pieces, float inv_c, float eps) {
  float* m = ex.entries();
  const int lane = threadIdx.x & 31;
  const bool layer = k0 == RA_NORM_LAYER || k1 == RA_NORM_LAYER;
  float mean = 0.f, sq;  // of the row that the lane's parity says
  if (layer) {
    mean = warp_sum2(sum_of(v0), sum_of(v1)) * at.inv_n;
    if (k0 != k1 && (lane & 1 ? k1 : k0) != RA_NORM_LAYER) mean = 0.f;
    const float other = __shfl_xor_sync(0xffffffffu, mean, 1);
    sq = warp_sum2(squares_around(at, v0, lane & 1 ? other : mean), squares_around(at, v1, lane & 1 ? mean : other));
  } else {
    sq = warp_sum2(squares_of(v0), squares_of(v1));
  }
  if (lane < 2) *reinterpret_cast<float2*>(m + 4 * at.warp + 2 * lane) = make_float2(mean, sq);
  ex.meet();
  return join_stats<V, T>(layer, reinterpret_cast<const float4*>(m), pieces, inv_c, eps);
}

// A sample's vector in shared memory, piece by piece: a piece's halves apart, so
// that a warp's 16-byte reads meet no bank conflicts.
template <int V, int T>
struct SharedVec {
  ulonglong2* mem;  // [V][2][32 T]
  static constexpr int BYTES = V * 2 * 32 * T * 16;
  __device__ __forceinline__ void put(int j, int lane_g, const Vec& v) const {
    mem[(2 * j) * 32 * T + lane_g] = make_ulonglong2(v.p[0], v.p[1]);
    mem[(2 * j + 1) * 32 * T + lane_g] = make_ulonglong2(v.p[2], v.p[3]);
  }
  __device__ __forceinline__ Vec get(int j, int lane_g) const {
    const ulonglong2 a = mem[(2 * j) * 32 * T + lane_g], b = mem[(2 * j + 1) * 32 * T + lane_g];
    return {{a.x, a.y, b.x, b.y}};
  }
};

// ------------------------------------------------------------------ forward
// The pairs of rows that a group takes: a CTA's share [lo, hi) of the live rows
// goes sample by sample (piece); of a piece's pairs group g takes g, g + groups, ...
struct Cursor {
  Piece w;
  int lo, hi, at;  // the piece's rows in the share; the pair's first row
  template <class P>
  __device__ __forceinline__ void enter(const P& p, int row, int share_hi, int group) {
    w.seek(p, row);
    lo = row;
    hi = min(share_hi, w.begin + p.seg[w.g].rows);
    at = lo + 2 * group;
  }
};

template <int V, int T>
__global__ void __launch_bounds__(FWD_THREADS, 1) residual_norm_kernel(const __grid_constant__ Params p) {
  extern __shared__ __align__(16) uint8_t smem[];
  // gate, mul, add of the sample; the exchange; ring[stage][row of the pair][piece of y, of h][thread of the CTA]
  using Shared = SharedVec<V, T>;
  const Shared gate{reinterpret_cast<ulonglong2*>(smem)}, mul{reinterpret_cast<ulonglong2*>(smem + Shared::BYTES)},
      add{reinterpret_cast<ulonglong2*>(smem + 2 * Shared::BYTES)};
  const Place<V, T> at(p.C);
  Exchange<T> ex(smem + 3 * Shared::BYTES, at.group);
  const uint32_t piece_bytes = 16 * blockDim.x, row_bytes = 2 * V * piece_bytes, stage_bytes = 2 * row_bytes;
  uint8_t* const ring = smem + 3 * Shared::BYTES + p.groups * Exchange<T>::BYTES + 16 * threadIdx.x;
  const float inv_c = 1.f / float(p.C);
  const int pieces = p.C >> 3, S = p.stages;
  pdl_launch();
  pdl_wait();
  const int total = live_rows(p);
  const int share = total / int(gridDim.x), more = total - share * int(gridDim.x), cta = int(blockIdx.x);
  const int lo = share * cta + min(cta, more), hi = lo + share + (cta < more ? 1 : 0);
  if (lo == hi) return;
  Cursor cur, ld;
  if (p.B > 4) cur.w.jump(p, lo);
  ld = cur;
  ld.enter(p, lo, hi, at.group);
  // this thread's first piece of the next pair's first row, found anew for each piece
  const __nv_bfloat16 *h_src = nullptr, *y_src = nullptr;
  bool fresh = true;
  auto load = [&](uint32_t off) {
    while (ld.at >= ld.hi && ld.hi < hi) {
      ld.enter(p, ld.hi, hi, at.group);
      fresh = true;
    }
    if (ld.at < ld.hi) {
      const Seg& sg = p.seg[ld.w.g];
      if (fresh) {
        const int64_t r = ld.at - ld.w.begin;
        h_src = sg.h + ld.w.s * sg.h_ss + r * sg.h_sr + at.col(0);
        y_src = sg.y ? sg.y + ld.w.s * sg.y_ss + r * sg.y_sr + at.col(0) : nullptr;
        fresh = false;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (k == 1 && ld.at + 1 >= ld.hi) break;
        uint8_t* to = ring + off + k * row_bytes;
        const __nv_bfloat16 *h = h_src + k * sg.h_sr, *y = y_src + k * sg.y_sr;
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (at.has(j)) {
            if (y_src) cp_async16(to + j * piece_bytes, y + 256 * T * j);
            cp_async16(to + (V + j) * piece_bytes, h + 256 * T * j);
          }
      }
      h_src += 2 * p.groups * sg.h_sr;
      if (y_src) y_src += 2 * p.groups * sg.y_sr;
      ld.at += 2 * p.groups;
    }
    cp_async_commit();
  };
  for (int k = 0; k < S - 1; ++k) load(k * stage_bytes);
  uint32_t off = 0, ld_off = (S - 1) * stage_bytes;
  for (cur.hi = lo; cur.hi < hi;) {
    if (cur.hi != lo) __syncthreads();  // every group is done with the last sample's vectors
    cur.enter(p, cur.hi, hi, at.group);
    const Seg& sg = p.seg[cur.w.g];
    const int s = cur.w.s;
    if (at.group == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (!at.has(j)) continue;
        const int c = at.col(j);
        gate.put(j, at.lane_g, vec8(sg.gate ? sg.gate + s * sg.gate_ss : nullptr, c, 1.f) * vec8(sg.post_w, c, 1.f));
        mul.put(j, at.lane_g,
                (vec8(sg.scale ? sg.scale + s * sg.mod_ss : nullptr, c, 0.f) + all(1.f)) * vec8(sg.pre_w, c, 1.f));
        add.put(j, at.lane_g, vec8(sg.shift ? sg.shift + s * sg.mod_ss : nullptr, c, 0.f));
      }
    }
    __syncthreads();
    const bool has_y = sg.y != nullptr;
    const int64_t r = cur.at - cur.w.begin;
    __nv_bfloat16* h_dst = sg.h_out ? sg.h_out + s * sg.o_ss + r * sg.o_sr + at.col(0) : nullptr;
    __nv_bfloat16* x_dst = sg.x ? sg.x + s * sg.x_ss + r * sg.x_sr + at.col(0) : nullptr;
    for (; cur.at < cur.hi; cur.at += 2 * p.groups) {
      load(ld_off);
      ld_off = off;
      cp_async_wait_upto(S - 1);
      const bool second = cur.at + 1 < cur.hi;  // else the pair's second row is what the ring held
      Vec v[2][V];
      auto fetch = [&](int k, int q, int j) {
        return widen(at.has(j) ? *reinterpret_cast<const uint4*>(ring + off + k * row_bytes + (q * V + j) * piece_bytes)
                               : make_uint4(0, 0, 0, 0));
      };
      if (has_y) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int j = 0; j < V; ++j) v[k][j] = fetch(k, 0, j);
        float4 st = make_float4(0.f, 1.f, 0.f, 1.f);
        if (p.post != RA_NORM_NONE) st = row_stats<V, T>(p.post, p.post, at, ex, v[0], v[1], pieces, inv_c, p.eps);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (at.has(j)) {
            const Vec g = gate.get(j, at.lane_g);
            v[0][j] = fma((v[0][j] + all(st.x)) * all(st.y), g, all(p.alpha) * fetch(0, 1, j));
            v[1][j] = fma((v[1][j] + all(st.z)) * all(st.w), g, all(p.alpha) * fetch(1, 1, j));
          } else {
            v[0][j] = v[1][j] = all(0.f);
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int j = 0; j < V; ++j) v[k][j] = all(p.alpha) * fetch(k, 1, j);
      }
      if (h_dst) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (at.has(j)) {
            *reinterpret_cast<uint4*>(h_dst + 256 * T * j) = narrow(v[0][j]);
            if (second) *reinterpret_cast<uint4*>(h_dst + sg.o_sr + 256 * T * j) = narrow(v[1][j]);
          }
        h_dst += 2 * p.groups * sg.o_sr;
      }
      if (x_dst) {
        float4 st = make_float4(0.f, 1.f, 0.f, 1.f);
        if (p.pre != RA_NORM_NONE) st = row_stats<V, T>(p.pre, p.pre, at, ex, v[0], v[1], pieces, inv_c, p.eps);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (at.has(j)) {
            const Vec m = mul.get(j, at.lane_g), a = add.get(j, at.lane_g);
            *reinterpret_cast<uint4*>(x_dst + 256 * T * j) = narrow(fma((v[0][j] + all(st.x)) * all(st.y), m, a));
            if (second)
              *reinterpret_cast<uint4*>(x_dst + sg.x_sr + 256 * T * j) =
                  narrow(fma((v[1][j] + all(st.z)) * all(st.w), m, a));
          }
        x_dst += 2 * p.groups * sg.x_sr;
      }
      off += stage_bytes;
      if (off == S * stage_bytes) off = 0;
    }
  }
}

// ------------------------------------------------------------------ backward
template <int V, int T>
__global__ void __launch_bounds__(BWD_THREADS, 1) residual_norm_grad_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  // mul, gate of the sample; the exchange; ring[stage][piece of h, y, dx, dh_out][thread of the CTA]
  using Shared = SharedVec<V, T>;
  const Shared mul{reinterpret_cast<ulonglong2*>(smem)}, gate{reinterpret_cast<ulonglong2*>(smem + Shared::BYTES)};
  const Place<V, T> at(p.C);
  Exchange<T> ex(smem + 2 * Shared::BYTES, at.group);
  const uint32_t piece_bytes = 16 * blockDim.x, stage_bytes = 4 * V * piece_bytes;
  uint8_t* const ring = smem + 2 * Shared::BYTES + p.groups * Exchange<T>::BYTES + 16 * threadIdx.x;
  const float inv_c = 1.f / float(p.C);
  const int pieces = p.C >> 3, S = p.stages;
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
      h += p.groups * p.h_sr;
      if (has_y) y += p.groups * p.y_sr;
      if (has_dx) dx += p.groups * p.dx_sr;
      if (has_dho) dho += p.groups * p.dho_sr;
    }
    ld_i += p.groups;
    cp_async_commit();
  };
  for (int k = 0; k < S - 1; ++k) load(k * stage_bytes);
  if (at.group == 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!at.has(j)) continue;
      const int c = at.col(j);
      mul.put(j, at.lane_g,
              (vec8(p.scale ? p.scale + s * p.mod_ss : nullptr, c, 0.f) + all(1.f)) * vec8(p.pre_w, c, 1.f));
      gate.put(j, at.lane_g, vec8(p.gate ? p.gate + s * p.gate_ss : nullptr, c, 1.f) * vec8(p.post_w, c, 1.f));
    }
  }
  __syncthreads();
  Vec s0[V], s1[V], s2[V];  // column sums of the group's rows
#pragma unroll
  for (int j = 0; j < V; ++j) s0[j] = s1[j] = s2[j] = all(0.f);
  auto place = [&](__nv_bfloat16* t, int64_t ss, int64_t sr) {
    return t ? t + s * ss + first * sr + at.col(0) : nullptr;
  };
  __nv_bfloat16 *dh = place(p.dh, p.dh_ss, p.dh_sr), *dy = place(p.dy, p.dy_ss, p.dy_sr);
  uint32_t off = 0, ld_off = (S - 1) * stage_bytes;
  for (int i = first; i < hi; i += p.groups) {
    load(ld_off);
    ld_off = off;
    cp_async_wait_upto(S - 1);
    auto fetch = [&](bool given, int q, int j) {
      return widen(given && at.has(j) ? *reinterpret_cast<const uint4*>(ring + off + (q * V + j) * piece_bytes)
                                      : make_uint4(0, 0, 0, 0));
    };
    Vec a[V], b[V];  // x^, then dH and what follows from it; y^
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] = fetch(true, 0, j), b[j] = fetch(has_y, 1, j);
    float2 sa = make_float2(0.f, 1.f), sb = sa;
    if (p.pre != RA_NORM_NONE || p.post != RA_NORM_NONE) {
      const float4 st = row_stats<V, T>(p.pre, p.post, at, ex, a, b, pieces, inv_c, p.eps);
      if (p.pre != RA_NORM_NONE) sa = make_float2(st.x, st.y);
      if (p.post != RA_NORM_NONE) sb = make_float2(st.z, st.w);
    }
    // the norm before the next branch
    uint64_t e0 = both(0.f), e1 = e0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!at.has(j)) continue;
      a[j] = (a[j] + all(sa.x)) * all(sa.y);
      const Vec d = fetch(has_dx, 2, j), e = d * mul.get(j, at.lane_g);
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
      if (!at.has(j)) continue;
      // dH = dh' + r (e - m(e) - x^ m(e x^))
      const Vec e = fma(a[j], all(m.y), fma(fetch(has_dx, 2, j), mul.get(j, at.lane_g), all(m.x)));
      a[j] = fma(e, all(sa.y), fetch(has_dho, 3, j));
      b[j] = (b[j] + all(sb.x)) * all(sb.y);
      if (dh) *reinterpret_cast<uint4*>(dh + 256 * T * j) = narrow(a[j] * all(p.alpha));
      s2[j] = fma(a[j], b[j], s2[j]);
      a[j] = a[j] * gate.get(j, at.lane_g);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        e0 = f2_add(e0, a[j].p[k]);
        e1 = f2_fma(a[j].p[k], b[j].p[k], e1);
      }
    }
    if (dh) dh += p.groups * p.dh_sr;
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
      dy += p.groups * p.dy_sr;
    }
    off += stage_bytes;
    if (off == S * stage_bytes) off = 0;
  }
  // The CTA's column sums: its groups' in order, through shared memory.
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
    const ra_status as = ensure_dynamic_smem(reinterpret_cast<const void*>(fn), SMEM_MAX, who);
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

// Pieces per thread, warps of a row's group, groups of a CTA and stages of a
// group's ring: as many groups as the threads and two stages each in shared memory
// allow. stage_rows: rows (of any tensor) in a stage.
struct Shape {
  int V, warps, groups, stages, smem;
  int threads() const { return 32 * warps * groups; }
};
Shape make_shape(int C, int max_threads, int vectors, int stage_rows) {
  Shape s;
  const int units = (C + 255) / 256;  // warp-wide pieces of a row
  s.warps = (units + MAX_PIECES - 1) / MAX_PIECES;
  s.V = (units + s.warps - 1) / s.warps;
  const int piece = s.V * 32 * s.warps * 16;  // a row's, with the missing ones
  const int fixed = vectors * 2 * piece, per_group = 2 * s.warps * 16;
  s.groups = max_threads / (32 * s.warps);
  if (s.groups > 15) s.groups = 15;  // named barriers
  auto bytes = [&](int groups, int stages) { return fixed + groups * (per_group + stages * stage_rows * piece); };
  while (s.groups > 1 && bytes(s.groups, 2) > SMEM_MAX) --s.groups;
  s.stages = 2;
  while (s.stages < MAX_STAGES && bytes(s.groups, s.stages + 1) <= SMEM_MAX) ++s.stages;
  s.smem = bytes(s.groups, s.stages);
  return s;
}
Shape fwd_shape(int C) { return make_shape(C, FWD_THREADS, 3, 4); }
Shape bwd_shape(int C) {
  Shape s = make_shape(C, BWD_THREADS, 2, 4);
  const int sums = s.groups * 3 * C * 4;  // the column sums take the same memory at the end
  if (s.smem < sums) s.smem = sums;
  return s;
}
static_assert(MAX_C <= 10 * 512 && MAX_PIECES == 2, "a group has at most ten warps");
using Fwd = void (*)(Params);
using Bwd = void (*)(GradParams);
Fwd pick_fwd(const Shape& s) {
  if (s.V == 1) return residual_norm_kernel<1, 1>;
  switch (s.warps) {
#define RA_CASE(T) \
  case T: return residual_norm_kernel<2, T>;
    RA_CASE(1) RA_CASE(2) RA_CASE(3) RA_CASE(4) RA_CASE(5) RA_CASE(6) RA_CASE(7) RA_CASE(8) RA_CASE(9) RA_CASE(10)
#undef RA_CASE
    default: return nullptr;
  }
}
Bwd pick_bwd(const Shape& s) {
  if (s.V == 1) return residual_norm_grad_kernel<1, 1>;
  switch (s.warps) {
#define RA_CASE(T) \
  case T: return residual_norm_grad_kernel<2, T>;
    RA_CASE(1) RA_CASE(2) RA_CASE(3) RA_CASE(4) RA_CASE(5) RA_CASE(6) RA_CASE(7) RA_CASE(8) RA_CASE(9) RA_CASE(10)
#undef RA_CASE
    default: return nullptr;
  }
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
  const Shape sh = fwd_shape(a->C);
  p.groups = sh.groups;
  p.stages = sh.stages;
  const int64_t sms = num_sms();
  return launch(who, pick_fwd(sh), p, dim3(unsigned(rows < sms ? rows : sms)), sh.threads(), sh.smem,
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
  const Shape sh = bwd_shape(a->C);
  p.groups = sh.groups;
  p.stages = sh.stages;
  p.parts = a->rows > 0 ? grad_parts(a->B, a->rows, num_sms()) : 0;
  if (a->rows > 0) {
    const ra_status r = launch(who, pick_bwd(sh), p, dim3(unsigned(a->B * p.parts)), sh.threads(), sh.smem, st);
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
