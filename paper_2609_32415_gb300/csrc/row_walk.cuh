// The rows of a call in up to three segments (text, reference, target) of B
// samples, as row kernels walk them: a segment with gated = 1 is skipped for
// samples whose mode is REUSE. P: a kernel's parameters with B, n_seg, mode and
// seg[g].rows, seg[g].gated.
#pragma once
#include <cstdint>

#include "refadapt.h"

namespace ra {

template <class P>
__device__ __forceinline__ bool live(const P& p, int g, int s) {
  return !p.seg[g].gated || p.mode[s] != RA_MODE_REUSE;
}

// Live rows of the call (the whole warp; the modes are on the device).
template <class P>
__device__ __forceinline__ int live_rows(const P& p) {
  const int lane = threadIdx.x & 31;
  int total = 0;
  for (int g = 0; g < p.n_seg; ++g) {
    int n = p.B;
    if (p.seg[g].gated) {
      n = 0;
      for (int s0 = 0; s0 < p.B; s0 += 32)
        n += __popc(__ballot_sync(0xffffffffu, s0 + lane < p.B && live(p, g, s0 + lane)));
    }
    total += n * p.seg[g].rows;
  }
  return total;
}

// Live rows in order: segments, samples within, rows within. A piece is the
// rows of one live (segment, sample), from row `begin` of the order on.
struct Piece {
  int g = 0, s = 0, begin = 0;
  // Moves to the piece that holds row i (i at or past begin, below the total).
  template <class P>
  __device__ __forceinline__ void seek(const P& p, int i) {
    while (i - begin >= p.seg[g].rows || !live(p, g, s)) {
      if (live(p, g, s)) begin += p.seg[g].rows;
      if (++s == p.B || p.seg[g].rows == 0) {
        s = 0;
        ++g;
      }
    }
  }
  // The same over many samples (the whole warp, from a segment's first): those of
  // a segment that is not gated are counted off by a division, others 32 at a
  // time. seek() takes 0.1 us for each (256 samples of one row: 50 us).
  template <class P>
  __device__ __forceinline__ void jump(const P& p, int i) {
    for (;; ++g, s = 0) {
      const int rows = p.seg[g].rows;
      if (rows == 0) continue;
      const int k = int(uint32_t(i - begin) / uint32_t(rows));  // live samples to pass
      if (!p.seg[g].gated) {
        s = min(k, p.B);
        begin += s * rows;
        if (s < p.B) return;
        continue;
      }
      int passed = 0;
      for (; s < p.B; s += 32) {
        const int t = s + (threadIdx.x & 31);
        const int n = __popc(__ballot_sync(0xffffffffu, t < p.B && live(p, g, t)));
        if (passed + n > k) break;
        passed += n;
      }
      begin += passed * rows;
      if (s < p.B) return;  // one of the 32 samples from s on: seek() finds it
    }
  }
};

}  // namespace ra
