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

}  // namespace ra
