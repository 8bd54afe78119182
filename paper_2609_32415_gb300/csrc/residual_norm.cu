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
// What holds it up is the latency of the reductions between.
// Forward, a row belongs to a group of warps, one or two pieces of eight columns a
// thread, which works on two rows of a sample at once: their reductions share
// shuffles and barriers, and their instructions fill each other's latencies. A
// thread copies its own pieces of the rows to come into a ring of its own in shared
// memory (cp.async: no barrier); what a sample's rows share (gate, scale, shift with
// the weights; 12 C bytes, more than the row) lies in shared memory. A warp reduces
// the mean and then the squares around it; the warps of a group join theirs (count,
// mean, squares) through shared memory with one barrier.
// Backward, three reductions follow one another, and columns have sums too; so the
// two directions are split (see residual_norm_grad_kernel).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstring>
#include <type_traits>

#include "api_common.h"
#include "launch_plan.h"
#include "row_walk.cuh"
#include "tc_ptx.cuh"

namespace ra {
namespace resnorm {

constexpr int MAX_C = 5120;
constexpr int MAX_PIECES = 2;                        // of a row, a thread's at most
constexpr int FWD_THREADS = 640;                     // of a CTA at most: 96 registers a thread
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
  int32_t few;             // few_pieces()
  float eps, alpha;
  const int32_t* mode;
  Seg seg[3];
};

struct GradParams {
  int32_t B, C, rows, post, pre;
  int32_t parts;                          // CTAs that share a sample's rows
  int32_t row_warps, groups, group_warps;  // of a CTA: see GradShape
  float eps, alpha;
  const __nv_bfloat16 *h, *y, *dx, *dh_out;
  int64_t h_ss, h_sr, y_ss, y_sr, dx_ss, dx_sr, dho_ss, dho_sr;
  __nv_bfloat16 *dh, *dy;
  int64_t dh_ss, dh_sr, dy_ss, dy_sr;
  const float *gate, *scale, *post_w, *pre_w;
  int64_t gate_ss, mod_ss;
  float* partial;  // [B][parts][3][C]
  int32_t* err_word;
  uint64_t budget_ns;
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

// The statistics of two rows.
template <int V, int T>
__device__ __forceinline__ float4 row_stats(int kind, const Place<V, T>& at, Exchange<T>& ex, const Vec (&v)[2][V],
                                            int pieces, float inv_c, float eps) {
  float* m = ex.entries();
  const int lane = threadIdx.x & 31;
  const bool layer = kind == RA_NORM_LAYER;
  float mean = 0.f, sq;  // of the row that the lane's parity says
  if (layer) {
    mean = warp_sum2(sum_of(v[0]), sum_of(v[1])) * at.inv_n;
    const float other = __shfl_xor_sync(0xffffffffu, mean, 1);
    sq = warp_sum2(squares_around(at, v[0], lane & 1 ? other : mean), squares_around(at, v[1], lane & 1 ? mean : other));
  } else {
    sq = warp_sum2(squares_of(v[0]), squares_of(v[1]));
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

// Shares of few pieces that none of them crosses: [lo, hi) of CTA cta, or false where
// that takes longer rounds (of `round` rows) than even shares do, by more than a
// twelfth. A CTA that goes on into another sample has its vectors to fetch, and the
// rest of the grid waits for it: 2 x (77 + 500) rows of 1280 8.3 us on even shares, 7.0
// here; 2 x (256 + 4096) of 2560 36.9 and 35.3. (The whole warp.)
__device__ __forceinline__ bool piece_share(const Params& p, int total, int round, int& lo, int& hi) {
  const int grid = int(gridDim.x), cta = int(blockIdx.x), lane = threadIdx.x & 31;
  uint32_t on[3] = {};
#pragma unroll
  for (int g = 0; g < 3; ++g)
    if (g < p.n_seg && p.seg[g].rows > 0) on[g] = __ballot_sync(0xffffffffu, lane < p.B && live(p, g, lane));
  const int even = (total + grid - 1) / grid, rounds = (even + round - 1) / round;
#pragma unroll 1
  for (int k = 0; k < 3; ++k) {
    if (k == 2 && rounds < 12) break;
    const int most = k == 0 ? even : (rounds + k - 1) * round;
    int used = 0, begin = 0;  // CTAs and rows before the segment
    lo = hi = 0;
    int part = 0, ctas = 0, n = 0;  // this CTA's part of its piece
#pragma unroll
    for (int g = 0; g < 3; ++g) {
      if (on[g] == 0) continue;
      const int rows = p.seg[g].rows, c = (rows + most - 1) / most, pieces = __popc(on[g]);
      const int mine = int(uint32_t(cta - used) / uint32_t(c));  // cta < used: past all
      if (cta >= used && mine < pieces) part = cta - used - mine * c, ctas = c, n = rows, lo = begin + mine * rows;
      used += pieces * c, begin += pieces * rows;
    }
    if (used > grid) continue;
    if (ctas > 0) {
      const int share = n / ctas, more = n - share * ctas;
      lo += share * part + min(part, more);
      hi = lo + share + (part < more ? 1 : 0);
    }
    return true;
  }
  return false;
}

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
  int lo, hi;
  if (total <= 2 * int(gridDim.x) || !p.few || !piece_share(p, total, 2 * p.groups, lo, hi)) {
    const int share = total / int(gridDim.x), more = total - share * int(gridDim.x), cta = int(blockIdx.x);
    lo = share * cta + min(cta, more), hi = lo + share + (cta < more ? 1 : 0);
  }
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
        if (p.post != RA_NORM_NONE) st = row_stats<V, T>(p.post, at, ex, v, pieces, inv_c, p.eps);
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
        if (p.pre != RA_NORM_NONE) st = row_stats<V, T>(p.pre, at, ex, v, pieces, inv_c, p.eps);
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
// A CTA takes a run of a sample's rows. A row warp has a row at a time: it copies h, y,
// dx and dh' into its slot in shared memory (bulk copies) and reduces what the whole
// row gives, in one pass over the slot. Then a group of column warps (eight columns a
// thread) takes the row from the slot: with the row's eight numbers known, dh, dy and
// the columns' sums need no further reduction, and S0, S1, S2 stay in the threads'
// registers.
// Sums are taken around K, the mean of the row's first eight values, and moved to the
// mean at the end: (mean - K)^2 is at most C / 8 times the variance, whatever the
// values, so the difference keeps the variance to (C / 8 + 1) of the sum's own
// roundings; a pass over the slot for the mean is saved.
// 8192 rows of 2560, two kinds of norms with weights, sums included: 51 us, 4.9 TB/s;
// 32,768 rows 158 us, 6.4 TB/s, where a copy of the same bytes takes 151: the pipeline
// of ten rows fills and drains once in a run of 54. (Slots filled by the row warps'
// own 16-byte copies, means in a pass of their own: 57. Teams of two or three warps a
// row and a warp of its own for the copies: 50.5, and 25 instead of 16 for rows of 256,
// where that warp cannot start copies fast enough.)
struct GradShape {
  int row_warps, groups, group_warps;  // warps that reduce rows; groups of column warps
  int smem;
  __host__ __device__ static int slot_bytes(int C) { return 4 * C * 2; }
  __host__ __device__ static int vec_bytes(int C) { return (C + 255) / 256 * 1024; }
  // [mul, gate] [numbers of a slot] [full, ready, free of a slot] [sum of gate, abort flag] [slots]
  __host__ __device__ static int off_numbers(int C) { return 2 * vec_bytes(C); }
  __host__ __device__ int off_bars(int C) const { return off_numbers(C) + row_warps * 32; }
  __host__ __device__ int off_slots(int C) const { return off_bars(C) + (row_warps * 24 + 8 + 15) / 16 * 16; }
};
constexpr int MAX_ROW_WARPS = 10;
constexpr int GRAD_THREADS = 640, GRAD_THREADS_WIDE = 768;  // of a CTA at most: 96 and 80 registers a thread

// Eight values of a sample's vector in shared memory, piece by piece, halves apart
// (a warp's 16-byte reads meet no bank conflicts).
__device__ __forceinline__ void shared_put(uint8_t* base, int piece, const Vec& v) {
  ulonglong2* m = reinterpret_cast<ulonglong2*>(base) + (piece >> 5) * 64 + (piece & 31);
  m[0] = make_ulonglong2(v.p[0], v.p[1]);
  m[32] = make_ulonglong2(v.p[2], v.p[3]);
}
__device__ __forceinline__ Vec shared_get(const uint8_t* base, int piece) {
  const ulonglong2* m = reinterpret_cast<const ulonglong2*>(base) + (piece >> 5) * 64 + (piece & 31);
  const ulonglong2 a = m[0], b = m[32];
  return {{a.x, a.y, b.x, b.y}};
}
__device__ __forceinline__ void add_up(uint64_t& acc, const Vec& v) {
  acc = f2_add(acc, f2_add(f2_add(v.p[0], v.p[1]), f2_add(v.p[2], v.p[3])));
}
__device__ __forceinline__ void dot_up(uint64_t& acc, const Vec& a, const Vec& b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) acc = f2_fma(a.p[i], b.p[i], acc);
}
// Two sums over the warp, in every lane.
__device__ __forceinline__ float2 warp_sums(uint64_t a, uint64_t b) {
  const float v = warp_sum2(sum2(a), sum2(b)), w = __shfl_xor_sync(0xffffffffu, v, 1);
  return threadIdx.x & 1 ? make_float2(w, v) : make_float2(v, w);
}

// What a row's columns need of it: 1 / deviation r and - mean r of h and y, and the
// negated means that the norms' gradients take off. (h r - mean r is off by 2^-24
// |mean| r, far below the rounding of h itself to bf16.)
struct alignas(16) RowNumbers {
  float h_r, h_b, e0, e1, y_r, y_b, f0, f1;
};

// N sums over the warp at once: lane l gets that of v[l % N].
template <int N>
__device__ __forceinline__ float warp_sums(float (&v)[N]) {
  int o = 1;
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2, o *= 2) {
    const bool up = threadIdx.x & o;
#pragma unroll
    for (int i = 0; i < n; ++i)
      v[i] = (up ? v[2 * i + 1] : v[2 * i]) + __shfl_xor_sync(0xffffffffu, up ? v[2 * i] : v[2 * i + 1], o);
  }
#pragma unroll
  for (; o < 32; o *= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
  return v[0];
}

template <int THREADS, bool PRE, bool POST>
__global__ void __launch_bounds__(THREADS, 1) residual_norm_grad_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  const GradShape shape{p.row_warps, p.groups, p.group_warps, 0};
  const int C = p.C, pieces = C >> 3, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, WR = p.row_warps;
  uint8_t *const mul_sh = smem, *const gate_sh = smem + GradShape::vec_bytes(C);
  RowNumbers* numbers = reinterpret_cast<RowNumbers*>(smem + GradShape::off_numbers(C));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + shape.off_bars(C));
  uint64_t *ready = full + WR, *free_ = full + 2 * WR;
  volatile float* gate_sum = reinterpret_cast<volatile float*>(full + 3 * WR);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(full + 3 * WR) + 1;
  uint8_t* const slots = smem + shape.off_slots(C);
  const int row_bytes = 2 * C, slot_bytes = GradShape::slot_bytes(C);
  const int s = int(blockIdx.x) / p.parts, part = int(blockIdx.x) - s * p.parts;
  const int lo = int(int64_t(p.rows) * part / p.parts), n = int(int64_t(p.rows) * (part + 1) / p.parts) - lo;
  const bool has_y = p.y != nullptr;
  pdl_launch();
  const int given = 1 + (has_y ? 1 : 0) + (p.dx ? 1 : 0) + (p.dh_out ? 1 : 0);
  auto load = [&](int r) {  // by one lane of a row warp
    mbar_arrive_expect_tx(full + warp, uint32_t(row_bytes * given));
    auto copy = [&](int q, const __nv_bfloat16* t, int64_t ss, int64_t sr) {
      if (t) bulk_load(slots + warp * slot_bytes + q * row_bytes, t + s * ss + int64_t(lo + r) * sr, row_bytes, full + warp);
    };
    copy(0, p.h, p.h_ss, p.h_sr);
    copy(1, p.y, p.y_ss, p.y_sr);
    copy(2, p.dx, p.dx_ss, p.dx_sr);
    copy(3, p.dh_out, p.dho_ss, p.dho_sr);
  };
  if (threadIdx.x == 0) *abort_flag = 0;
  if (warp < WR && lane == 0) {
    mbar_init(full + warp, 1);
    mbar_init(ready + warp, 1);
    mbar_init(free_ + warp, p.group_warps);
    fence_mbar_init();
    fence_proxy_async_smem();
    pdl_wait();
    if (warp < n) load(warp);
  }
  pdl_wait();
  if (given < 4)  // what was not given is zeros in every slot
    for (int i = threadIdx.x; i < WR * pieces; i += blockDim.x) {
      uint4* to = reinterpret_cast<uint4*>(slots + i / pieces * slot_bytes) + i % pieces;
      if (!has_y) to[pieces] = make_uint4(0, 0, 0, 0);
      if (!p.dx) to[2 * pieces] = make_uint4(0, 0, 0, 0);
      if (!p.dh_out) to[3 * pieces] = make_uint4(0, 0, 0, 0);
    }
  for (int i = threadIdx.x; i < pieces; i += blockDim.x) {
    const int c = 8 * i;
    shared_put(mul_sh, i, (vec8(p.scale ? p.scale + s * p.mod_ss : nullptr, c, 0.f) + all(1.f)) * vec8(p.pre_w, c, 1.f));
    shared_put(gate_sh, i, vec8(p.gate ? p.gate + s * p.gate_ss : nullptr, c, 1.f) * vec8(p.post_w, c, 1.f));
  }
  __syncthreads();
  const uint64_t zero = both(0.f);
  if constexpr (POST) {
    if (warp == 0) {
      uint64_t g = zero;
      for (int i = lane; i < pieces; i += 32) add_up(g, shared_get(gate_sh, i));
      const float2 sum = warp_sums(g, zero);
      if (lane == 0) *gate_sum = sum.x;
    }
    __syncthreads();
  }
  const WaitCtl ctl{abort_flag, p.err_word, p.budget_ns};
  const float inv_c = 1.f / float(C);
  Vec s0 = all(0.f), s1 = s0, s2 = s0;  // of a column thread
  const int col_warp = warp - WR, group = col_warp < 0 ? -1 : col_warp / p.group_warps;
  const int piece = 32 * (col_warp - group * p.group_warps) + lane;  // of a column thread
  if (warp < WR) {
    // ---------------------------------------------------------------- rows
    const uint8_t* const row = slots + warp * slot_bytes;
    const bool deep = p.post != RA_NORM_NONE && p.dy;
    const int mine = (pieces - lane + 31) / 32;  // pieces of this lane
    auto get = [](const uint8_t* at) { return widen(*reinterpret_cast<const uint4*>(at)); };
    auto first8 = [&](const uint8_t* at) {  // the mean of a row's first eight values
      uint64_t v = zero;
      add_up(v, get(at));
      return sum2(v) * 0.125f;
    };
    for (int k = 0, r = warp; r < n; ++k, r += WR) {
      if (!__all_sync(0xffffffffu, mbar_wait(full + warp, uint32_t(k & 1), ctl))) {
        mbar_wait_drain(full + warp, uint32_t(k & 1), p.budget_ns);  // the copies land before the CTA goes on
        break;
      }
      const float hk = PRE ? first8(row) : 0.f, yk = POST ? first8(row + row_bytes) : 0.f;
      // With h and y less K, e = dx mul, g = gate: the sums of h, y, their
      // squares, e and e h; and what sum f and f y come from, f = g dH,
      // dH = dh' + r (e - m(e) - x^ m(e x^)).
      uint64_t h0 = zero, y0 = zero, hh = zero, yy = zero, e0 = zero, eh = zero, dg = zero, eg = zero, hg = zero,
               dgy = zero, egy = zero, hgy = zero, gy = zero;
      const Vec neg_h = all(-hk), neg_y = all(-yk);
      const uint8_t *at = row + 16 * lane, *mul_at = mul_sh + 16 * lane, *gate_at = gate_sh + 16 * lane;
      auto vec = [](const uint8_t* m) -> Vec {
        const ulonglong2 a = *reinterpret_cast<const ulonglong2*>(m), b = *reinterpret_cast<const ulonglong2*>(m + 512);
        return {{a.x, a.y, b.x, b.y}};
      };
#pragma unroll 2
      for (int i = 0; i < mine; ++i, at += 512, mul_at += 1024, gate_at += 1024) {
        Vec h = get(at), y = get(at + row_bytes);
        const Vec e = get(at + 2 * row_bytes) * vec(mul_at);
        if constexpr (PRE) {
          h = h + neg_h;
          add_up(h0, h);
          add_up(e0, e);
        }
        if constexpr (POST) {
          y = y + neg_y;
          add_up(y0, y);
        }
        dot_up(hh, h, h);
        dot_up(yy, y, y);
        dot_up(eh, e, h);
        if (deep) {
          const Vec g = vec(gate_at), d = get(at + 3 * row_bytes), w = g * y;
          dot_up(dgy, d, w);
          dot_up(egy, e, w);
          dot_up(hgy, h, w);
          if constexpr (PRE || POST) add_up(gy, w);
          if constexpr (POST) {
            dot_up(dg, d, g);
            dot_up(eg, e, g);
            dot_up(hg, h, g);
          }
        }
      }
      constexpr int N = PRE || POST ? 16 : 8;
      float sums[N] = {sum2(hh), sum2(yy), sum2(eh), sum2(dgy), sum2(egy), sum2(hgy)};
      if constexpr (PRE) sums[6] = sum2(h0), sums[7] = sum2(e0);
      if constexpr (PRE || POST) sums[8] = sum2(gy);
      if constexpr (POST) sums[9] = sum2(y0), sums[10] = sum2(dg), sums[11] = sum2(eg), sums[12] = sum2(hg);
      const float one = warp_sums(sums);
      float all_of[N];
#pragma unroll
      for (int i = 0; i < N; ++i) all_of[i] = __shfl_sync(0xffffffffu, one, i);
      float mh = 0.f, my = 0.f, sum_eh = all_of[2];  // what is left to the means; sums around them
      if constexpr (PRE) mh = all_of[6] * inv_c, sum_eh = fmaf(-mh, all_of[7], sum_eh);
      if constexpr (POST) my = all_of[9] * inv_c;
      RowNumbers v = {1.f, 0.f, 0.f, 0.f, 1.f, 0.f, 0.f, 0.f};
      if (p.pre != RA_NORM_NONE) {
        v.h_r = rsqrtf(fmaxf(fmaf(all_of[0], inv_c, -mh * mh), 0.f) + p.eps), v.h_b = -(hk + mh) * v.h_r;
        if constexpr (PRE) v.e0 = -all_of[7] * inv_c;
        v.e1 = -sum_eh * v.h_r * inv_c;
      }
      if (p.post != RA_NORM_NONE) {
        v.y_r = rsqrtf(fmaxf(fmaf(all_of[1], inv_c, -my * my), 0.f) + p.eps), v.y_b = -(yk + my) * v.y_r;
        if (deep) {
          float d_gy = all_of[3], e_gy = all_of[4], h_gy = all_of[5], s_gy = 0.f;
          if constexpr (PRE || POST) s_gy = all_of[8];
          if constexpr (POST) {
            const float g = *gate_sum, d_g = all_of[10], e_g = all_of[11], h_g = all_of[12];  // h still less hk only
            const float f0 = fmaf(v.h_r, fmaf(v.h_r * v.e1, fmaf(-mh, g, h_g), fmaf(v.e0, g, e_g)), d_g);
            v.f0 = -f0 * inv_c;
            d_gy = fmaf(-my, d_g, d_gy), e_gy = fmaf(-my, e_g, e_gy);
            h_gy = fmaf(-my, h_g, h_gy), s_gy = fmaf(-my, g, s_gy);
          }
          h_gy = fmaf(-mh, s_gy, h_gy);
          v.f1 = -fmaf(v.h_r, fmaf(v.h_r * v.e1, h_gy, fmaf(v.e0, s_gy, e_gy)), d_gy) * v.y_r * inv_c;
        }
      }
      if (lane == 0) {
        numbers[warp] = v;
        mbar_arrive(ready + warp);
      }
      if (r + WR < n) {
        if (!__all_sync(0xffffffffu, mbar_wait(free_ + warp, uint32_t(k & 1), ctl))) break;
        if (lane == 0) load(r + WR);
      }
    }
  } else if (group < p.groups) {
    // ---------------------------------------------------------------- columns
    const bool in = piece < pieces;
    const Vec mul = in ? shared_get(mul_sh, piece) : all(0.f), gate = in ? shared_get(gate_sh, piece) : all(0.f);
    auto place = [&](__nv_bfloat16* t, int64_t ss, int64_t sr) {
      return t ? t + s * ss + (lo + group) * sr + 8 * piece : nullptr;
    };
    __nv_bfloat16 *dh = place(p.dh, p.dh_ss, p.dh_sr), *dy = place(p.dy, p.dy_ss, p.dy_sr);
    int w = group, k = 0;  // row r is the k-th of slot w
    for (int r = group; r < n; r += p.groups) {
      for (; w >= WR; w -= WR) ++k;
      if (!__all_sync(0xffffffffu, mbar_wait(ready + w, uint32_t(k & 1), ctl))) break;
      if (in) {
        const RowNumbers v = numbers[w];
        const uint8_t* at = slots + w * slot_bytes + 16 * piece;
        auto get = [&](int q) { return widen(*reinterpret_cast<const uint4*>(at + q * row_bytes)); };
        auto norm = [](auto centred, const Vec& h, float r, float b) {
          if constexpr (decltype(centred)::value)
            return fma(h, all(r), all(b));
          else
            return h * all(r);
        };
        const Vec x = norm(std::bool_constant<PRE>(), get(0), v.h_r, v.h_b), d = get(2);
        s0 = s0 + d;
        s1 = fma(d, x, s1);
        // dH = dh' + r (e - m(e) - x^ m(e x^))
        const Vec e = fma(d, mul, norm(std::bool_constant<PRE>(), x, v.e1, v.e0));
        const Vec t = fma(e, all(v.h_r), get(3));
        if (dh) *reinterpret_cast<uint4*>(dh) = narrow(p.alpha == 1.f ? t : t * all(p.alpha));
        if (has_y) {
          const Vec y = norm(std::bool_constant<POST>(), get(1), v.y_r, v.y_b);
          s2 = fma(t, y, s2);
          if (dy) *reinterpret_cast<uint4*>(dy) = narrow(fma(t, gate, norm(std::bool_constant<POST>(), y, v.f1, v.f0)) * all(v.y_r));
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(free_ + w);
      if (dh) dh += p.groups * p.dh_sr;
      if (dy) dy += p.groups * p.dy_sr;
      w += p.groups;
    }
  }
  // The CTA's column sums: its groups' in order, through shared memory.
  __syncthreads();
  const bool gave_up = *abort_flag;
  float* out = p.partial + int64_t(blockIdx.x) * 3 * C;
  float* sums = p.groups > 1 ? reinterpret_cast<float*>(slots) : out;  // [group][3][C]
  if (group >= 0 && group < p.groups && piece < pieces) {
    float* to = sums + group * 3 * C + 8 * piece;
    auto put = [&](float* dst, const Vec& v) {
      const Vec x = gave_up ? all(__int_as_float(0x7fffffff)) : v;
      reinterpret_cast<ulonglong2*>(dst)[0] = make_ulonglong2(x.p[0], x.p[1]);
      reinterpret_cast<ulonglong2*>(dst)[1] = make_ulonglong2(x.p[2], x.p[3]);
    };
    put(to, s0);
    put(to + C, s1);
    put(to + 2 * C, s2);
  }
  if (p.groups == 1) return;
  __syncthreads();
  for (int c = threadIdx.x; c < 3 * C; c += blockDim.x) {
    float v = 0.f;
    for (int g = 0; g < p.groups; ++g) v += sums[g * 3 * C + c];
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
  return !a || a != b || (a_ss == b_ss && a_sr == b_sr);
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
// About ten column warps, and as many row warps beside them as there is room for, a
// multiple of the groups: with a slot's rows all its own, a group cannot run a phase
// of its barrier ahead.
GradShape grad_shape(int C) {
  GradShape s;
  s.group_warps = (C + 255) / 256;
  s.groups = s.group_warps >= 10 ? 1 : 10 / s.group_warps;
  for (s.row_warps = MAX_ROW_WARPS / s.groups * s.groups;; s.row_warps -= s.groups) {
    s.smem = s.off_slots(C) + s.row_warps * GradShape::slot_bytes(C);
    if (s.smem <= SMEM_MAX) break;  // four fit at C = 5120
  }
  const int sums = s.off_slots(C) + s.groups * 3 * C * 4;
  if (s.smem < sums) s.smem = sums;
  return s;
}
static_assert(2 * 20 * 1024 + 4 * MAX_C * 2 * 4 + 2048 <= SMEM_MAX, "four slots fit");
static_assert(MAX_C <= 10 * 512 && MAX_PIECES == 2, "a group has at most ten warps");
using Fwd = void (*)(Params);
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
using Grad = void (*)(GradParams);
template <int THREADS>
Grad pick_grad(bool pre, bool post) {
  return pre ? (post ? residual_norm_grad_kernel<THREADS, true, true> : residual_norm_grad_kernel<THREADS, true, false>)
             : (post ? residual_norm_grad_kernel<THREADS, false, true> : residual_norm_grad_kernel<THREADS, false, false>);
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
  p.few = few_pieces(a->B, a->n_seg);
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
    auto in_place_ok = [&](const void* out, int64_t ss, int64_t sr) {
      return same_or_apart(out, ss, sr, a->h, a->h_stride_s, a->h_stride_r) &&
             same_or_apart(out, ss, sr, a->y, a->y_stride_s, a->y_stride_r) &&
             same_or_apart(out, ss, sr, a->dx, a->dx_stride_s, a->dx_stride_r) &&
             same_or_apart(out, ss, sr, a->dh_out, a->dh_out_stride_s, a->dh_out_stride_r);
    };
    if ((a->dy && a->dy == a->dh) || !in_place_ok(a->dh, a->dh_stride_s, a->dh_stride_r) ||
        !in_place_ok(a->dy, a->dy_stride_s, a->dy_stride_r)) {
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
  const GradShape sh = grad_shape(a->C);
  p.row_warps = sh.row_warps, p.groups = sh.groups, p.group_warps = sh.group_warps;
  p.err_word = a->err_word;
  p.budget_ns = wait_budget_ns();
  p.parts = a->rows > 0 ? grad_parts(a->B, a->rows, num_sms()) : 0;
  if (a->rows > 0) {
    const int threads = 32 * (sh.row_warps + sh.groups * sh.group_warps);
    const bool pre = a->pre == RA_NORM_LAYER, post = a->post == RA_NORM_LAYER;
    const ra_status r = launch(who, threads <= GRAD_THREADS ? pick_grad<GRAD_THREADS>(pre, post)
                                                            : pick_grad<GRAD_THREADS_WIDE>(pre, post),
                               p, dim3(unsigned(a->B * p.parts)), threads, sh.smem, st);
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
