// What launches decide on the host by plain arithmetic, apart from CUDA so that it
// can be checked without a GPU.
#pragma once
#include <cstdint>
#include <initializer_list>
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

// Where a tensor lies, exactly: runs of `run` bytes at `at` plus every sum of multiples of the steps (step i taken
// 0 to n[i] - 1 times; largest step first, positive). run 0: nowhere.
struct Place {
  int64_t at, run;
  int dims;
  int64_t n[3], step[3];
  int64_t extent(int from) const {
    int64_t e = run;
    for (int i = from; i < dims; ++i) e += (n[i] - 1) * step[i];
    return e;
  }
};
// Up to three dimensions of n entries, `step` bytes apart.
struct PlaceDim {
  int64_t n, step;
};
inline Place place_of(const void* ptr, int64_t run, PlaceDim a = {1, 0}, PlaceDim b = {1, 0}, PlaceDim c = {1, 0}) {
  Place p{int64_t(reinterpret_cast<uintptr_t>(ptr)), ptr && run > 0 ? run : 0, 0, {}, {}};
  for (PlaceDim d : {a, b, c}) {
    if (d.n < 1) p.run = 0;
    if (d.n <= 1 || d.step == 0) continue;
    if (d.step < 0) {
      p.at += (d.n - 1) * d.step;
      d.step = -d.step;
    }
    int i = p.dims++;
    for (; i > 0 && p.step[i - 1] < d.step; --i) p.n[i] = p.n[i - 1], p.step[i] = p.step[i - 1];
    p.n[i] = d.n;
    p.step[i] = d.step;
  }
  return p;
}
// The same bytes by fewer dimensions: runs that touch are one, steps that go on with one another too.
inline Place merged(Place p) {
  while (p.dims > 0 && p.step[p.dims - 1] <= p.run) {
    p.run += (p.n[p.dims - 1] - 1) * p.step[p.dims - 1];
    --p.dims;
  }
  for (int i = p.dims - 2; i >= 0; --i)
    if (p.step[i] == p.step[i + 1] * p.n[i + 1]) {
      p.n[i + 1] *= p.n[i];
      for (int j = i; j + 1 < p.dims; ++j) p.n[j] = p.n[j + 1], p.step[j] = p.step[j + 1];
      --p.dims;
    }
  return p;
}
// Do a's dimensions from i on, at `shift` bytes from b's from j on, share a byte with those? Only what can meet is
// looked at: parts of one buffer (equal steps) in a few steps whatever their sizes, others row by row. `left`: steps
// until it is given up, with no for an answer.
inline bool parts_meet(const Place& a, int i, int64_t shift, const Place& b, int j, int* left) {
  if (--*left < 0) return false;
  if (shift >= b.extent(j) || -shift >= a.extent(i)) return false;
  const int64_t sa = i < a.dims ? a.step[i] : 0, sb = j < b.dims ? b.step[j] : 0;
  if (sa == 0 && sb == 0) return true;
  // the smallest and largest k with shift + k step in (-e, f)
  auto from = [](int64_t shift, int64_t e, int64_t step) {
    const int64_t x = -e - shift + 1;
    return x >= 0 ? (x + step - 1) / step : -(-x / step);
  };
  auto to = [](int64_t shift, int64_t f, int64_t step) {
    const int64_t x = f - shift - 1;
    return x >= 0 ? x / step : -((-x + step - 1) / step);
  };
  auto least = [](int64_t x, int64_t y) { return x < y ? x : y; };
  auto most = [](int64_t x, int64_t y) { return x > y ? x : y; };
  if (sa == sb) {  // entry x of a and y of b: k = x - y
    const int64_t e = a.extent(i + 1), f = b.extent(j + 1);
    const int64_t end = least(to(shift, f, sa), a.n[i] - 1);
    for (int64_t k = most(from(shift, e, sa), 1 - b.n[j]); k <= end && *left >= 0; ++k)
      if (parts_meet(a, i + 1, shift + k * sa, b, j + 1, left)) return true;
  } else if (sa > sb) {
    const int64_t end = least(to(shift, b.extent(j), sa), a.n[i] - 1);
    for (int64_t k = most(from(shift, a.extent(i + 1), sa), 0); k <= end && *left >= 0; ++k)
      if (parts_meet(a, i + 1, shift + k * sa, b, j, left)) return true;
  } else {
    const int64_t end = least(to(-shift, a.extent(i), sb), b.n[j] - 1);
    for (int64_t k = most(from(-shift, b.extent(j + 1), sb), 0); k <= end && *left >= 0; ++k)
      if (parts_meet(a, i, shift - k * sb, b, j + 1, left)) return true;
  }
  return false;
}
constexpr int PLACE_STEPS = 1 << 16;
// Do two tensors share memory? (merged ones)
inline bool meet(const Place& a, const Place& b) {
  if (a.run == 0 || b.run == 0) return false;
  int left = PLACE_STEPS;
  return parts_meet(a, 0, a.at - b.at, b, 0, &left);
}
// Does a tensor have a byte twice? (as place_of gives it)
inline bool meets_itself(const Place& p) {
  int left = PLACE_STEPS;
  for (int i = 0; i < p.dims && p.run > 0; ++i) {
    const int64_t inner = p.extent(i + 1);
    for (int64_t k = 1; k < p.n[i] && k * p.step[i] < inner && left >= 0; ++k)
      if (parts_meet(p, i + 1, k * p.step[i], p, i + 1, &left)) return true;
  }
  return false;
}
// The tensors of a call. clash(): an output's byte is another tensor's too, or its own twice.
template <int OUT, int IN>
class CallPlaces {
 public:
  void reads(const Place& t) { in_[n_in_++] = merged(t); }
  void writes(const Place& t) {
    twice_ = twice_ || meets_itself(t);
    out_[n_out_++] = merged(t);
  }
  bool clash() const {
    bool yes = twice_;
    for (int i = 0; i < n_out_; ++i) {
      for (int j = 0; j < n_in_ && !yes; ++j) yes = meet(out_[i], in_[j]);
      for (int j = 0; j < i && !yes; ++j) yes = meet(out_[i], out_[j]);
    }
    return yes;
  }

 private:
  Place out_[OUT], in_[IN];
  int n_out_ = 0, n_in_ = 0;
  bool twice_ = false;
};

}  // namespace ra
