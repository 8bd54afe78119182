// What launches decide on the host by plain arithmetic, apart from CUDA so that it
// can be checked without a GPU.
#pragma once
#include <cstdint>
#include <mutex>

namespace ra {

// Are the (segment, sample) pairs of a row call few, and more than one? Then its
// CTAs' shares may end with them (residual_norm.cu, piece_share: a ballot of the
// samples of a segment, so no more than 32).
constexpr int FEW_PIECES = 12;
constexpr bool few_pieces(int64_t samples, int segs) {
  return samples * segs > 1 && samples * segs <= FEW_PIECES;
}

// Clusters of 1 to 8 CTAs that a device holds at once, asked once per device, kernel
// and shared memory: they lie within GPCs, which are not multiples of every size, and
// registers count too. Where a query fails (a negative answer) the call counts with one
// and nothing is kept. No allocation; past the table's end a kernel is asked on every call.
class ClusterTable {
 public:
  static constexpr int MAX_CLUSTER = 8, SLOTS = 64;
  struct Counts {
    int of[MAX_CLUSTER + 1];  // by CTAs a cluster, from 1; 0: that size does not fit
  };
  // ask(c): how many clusters of c CTAs.
  template <class Ask>
  Counts get(int device, const void* kernel, int smem, Ask ask) {
    std::lock_guard<std::mutex> lock(mu_);
    for (int i = 0; i < used_; ++i)
      if (slots_[i].device == device && slots_[i].kernel == kernel && slots_[i].smem == smem) return slots_[i].counts;
    Counts n{};
    bool known = true;
    for (int c = 1; c <= MAX_CLUSTER; ++c) {
      n.of[c] = ask(c);
      if (n.of[c] < 0) n.of[c] = 1, known = false;
    }
    if (known && used_ < SLOTS) slots_[used_++] = Slot{device, smem, kernel, n};
    return n;
  }

 private:
  struct Slot {
    int device, smem;
    const void* kernel;
    Counts counts;
  };
  std::mutex mu_;
  Slot slots_[SLOTS];
  int used_ = 0;
};

// Rows of a tensor in memory: B samples of n rows of `bytes` bytes, strides in bytes.
struct RowSpan {
  const void* ptr;  // NULL: absent
  int64_t ss, sr, B, n, bytes;
};
// Do two tensors share memory for certain: they start at one address, or both fill their
// range and the ranges meet? (Rows side by side in one buffer do not.)
inline bool surely_overlap(const RowSpan& a, const RowSpan& b) {
  if (!a.ptr || !b.ptr || a.B * a.n * a.bytes < 1 || b.B * b.n * b.bytes < 1) return false;
  if (a.ptr == b.ptr) return true;
  auto fills = [](const RowSpan& t) {  // sample after sample, or row after row of all samples
    return ((t.n == 1 || t.sr == t.bytes) && (t.B == 1 || t.ss == t.n * t.bytes)) ||
           (t.ss == t.bytes && t.sr == t.B * t.bytes);
  };
  if (!fills(a) || !fills(b)) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.ptr), pb = reinterpret_cast<uintptr_t>(b.ptr);
  return pa < pb ? pb - pa < uintptr_t(a.B * a.n * a.bytes) : pa - pb < uintptr_t(b.B * b.n * b.bytes);
}
// The first of n_out tensors that shares memory with another of them or with one of n_in
// inputs; -1: none.
inline int overlapping(const RowSpan* out, int n_out, const RowSpan* in, int n_in) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (surely_overlap(out[i], in[j])) return i;
    for (int j = 0; j < i; ++j)
      if (surely_overlap(out[i], out[j])) return i;
  }
  return -1;
}

}  // namespace ra
