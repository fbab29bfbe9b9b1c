// Whether rows of strided tensors share memory: host checks, plain C++ (the tests compile it for the
// CPU).
#pragma once
#include <stdint.h>

#include <algorithm>

namespace mala {

// Rows of `width` bytes at base + sum i_a stride[a], 0 <= i_a < n[a] (strides in bytes, not negative,
// n > 0).
struct Rows {
  uintptr_t base;
  int64_t width;
  int64_t stride[3], n[3];

  int64_t extent() const {
    int64_t bytes = width;
    for (int a = 0; a < 3; ++a) bytes += stride[a] * (n[a] - 1);
    return bytes;
  }
};

enum Shared { kApart, kShare, kUnclear };

// Looks for d_a in [lo_a, hi_a] with first < c + sum d_a stride_a < last, axis by axis, the largest
// stride first: what the axes behind it can add leaves few values of d_a to look at where axes nest
// (a stride is not below the extent of the smaller ones), as those of a tensor do.  Others are given up
// after kSteps of them.
class Meeting {
 public:
  static constexpr int kSteps = 1 << 14;

  void axis(int64_t stride, int64_t lo, int64_t hi) {
    if (!stride || (!lo && !hi)) return;
    int a = 0;
    while (a < axes_ && stride_[a] > stride) ++a;
    if (a < axes_ && stride_[a] == stride) {
      lo_[a] += lo;
      hi_[a] += hi;
      return;
    }
    for (int i = axes_++; i > a; --i) stride_[i] = stride_[i - 1], lo_[i] = lo_[i - 1], hi_[i] = hi_[i - 1];
    stride_[a] = stride, lo_[a] = lo, hi_[a] = hi;
  }
  // other: with some d_a that is not 0
  Shared find(int64_t c, int64_t first, int64_t last, bool other) {
    constexpr int64_t kMost = (int64_t)1 << 61;      // (so that no sum below leaves 64 bits)
    first_ = first, last_ = last, steps_ = 0;
    least_[axes_] = most_[axes_] = 0;
    bool large = c < -kMost || c > kMost;
    for (int a = axes_ - 1; a >= 0 && !large; --a) {
      int64_t x, y;
      large = __builtin_mul_overflow(lo_[a], stride_[a], &x) || __builtin_mul_overflow(hi_[a], stride_[a], &y) ||
              __builtin_add_overflow(x, least_[a + 1], &least_[a]) ||
              __builtin_add_overflow(y, most_[a + 1], &most_[a]) || least_[a] < -kMost || most_[a] > kMost;
    }
    return large ? kUnclear : look(0, c, !other);
  }

 private:
  static int64_t floor_div(int64_t x, int64_t y) { return x / y - (x % y < 0); }

  Shared look(int a, int64_t c, bool fine) {
    if (a == axes_) return fine && first_ < c && c < last_ ? kShare : kApart;
    const int64_t s = stride_[a];
    const int64_t lo = std::max(lo_[a], floor_div(first_ - c - most_[a + 1], s) + 1);
    const int64_t hi = std::min(hi_[a], -floor_div(-(last_ - c - least_[a + 1]), s) - 1);
    for (int64_t d = lo; d <= hi; ++d) {
      if (++steps_ > kSteps) return kUnclear;
      const Shared x = look(a + 1, c + d * s, fine || d);
      if (x != kApart) return x;
    }
    return kApart;
  }

  int axes_ = 0, steps_ = 0;
  int64_t stride_[6], lo_[6], hi_[6], least_[7], most_[7], first_ = 0, last_ = 0;
};

// Whether two of the rows share a byte.
inline Shared rows_overlap(const Rows& r) {
  Meeting m;
  for (int a = 0; a < 3; ++a) {
    if (r.n[a] == 1) continue;
    for (int b = 0; b < a; ++b)
      if (r.n[b] > 1 && r.stride[a] == r.stride[b]) return kShare;
    if (!r.stride[a]) return kShare;
    m.axis(r.stride[a], 1 - r.n[a], r.n[a] - 1);
  }
  return m.find(0, -r.width, r.width, true);
}

// Whether a row of one and a row of the other share a byte.
inline Shared rows_meet(const Rows& x, const Rows& y) {
  if (x.base >= y.base + y.extent() || y.base >= x.base + x.extent()) return kApart;
  Meeting m;
  for (int a = 0; a < 3; ++a) {
    m.axis(x.stride[a], 0, x.n[a] - 1);
    m.axis(y.stride[a], 1 - y.n[a], 0);
  }
  return m.find((int64_t)(x.base - y.base), -x.width, y.width, false);
}

}  // namespace mala
