// Whether tensors, as their strides say, share elements: for the checks in front of a launch.  Host code.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace dash {

// Rows of d elements side by side, the one of indices (i, j, ..) at i stride[0] + j stride[1] + ..
struct Strided { const void* at; int dims; int64_t stride[3], size[3]; };

// Differences of indices a_i from lo_i to hi_i, their strides falling: whether off + sum of a_i stride_i is nearer than d to 0 for some of them.  Those alone are
// gone through that the smaller strides can make up for: one or two a stride where a tensor's dimensions lie inside of each other.  After `tries` steps: yes.
struct StridedSteps {
  typedef __int128 Place;
  struct Step { Place stride, lo, hi; };
  Step step[6];
  int n = 0, tries = 1000;
  Place d;
  explicit StridedSteps(int d) : d(d) {}
  void add(int64_t stride, int64_t lo, int64_t hi) {
    if (stride != 0 && lo < hi) step[n++] = {stride, lo, hi};
  }
  void sort() {
    for (int i = 1; i < n; i++)
      for (int k = i; k > 0 && step[k].stride > step[k - 1].stride; k--) std::swap(step[k], step[k - 1]);
  }
  static Place floor_div(Place x, Place y) { return x >= 0 ? x / y : -((y - 1 - x) / y); }
  bool near(int i, Place off) {
    if (--tries < 0) return true;
    if (i == n) return -d < off && off < d;
    Place low = off, high = off;
    for (int k = i + 1; k < n; k++) { low += step[k].stride * step[k].lo; high += step[k].stride * step[k].hi; }
    const Place last = std::min(step[i].hi, floor_div(d - 1 - low, step[i].stride));
    for (Place a = std::max(step[i].lo, -floor_div(high + d - 1, step[i].stride)); a <= last; a++)
      if (near(i + 1, off + a * step[i].stride)) return true;
    return false;
  }
};

// Whether a tensor's rows share elements among themselves.
inline bool strided_repeats(const Strided& x, int d) {
  for (int i = 0; i < x.dims; i++)
    if (x.size[i] > 1 && x.stride[i] == 0) return true;
  // the first index, by falling strides, in which two rows differ is the larger in one of them
  StridedSteps all(d);
  for (int i = 0; i < x.dims; i++) all.add(x.stride[i], 1 - x.size[i], x.size[i] - 1);
  all.sort();
  // mostly each index goes through what one step of the next larger stride holds
  StridedSteps::Place span = d;
  int inside = all.n;
  while (inside > 0 && all.step[inside - 1].stride >= span) span += all.step[inside - 1].stride * all.step[inside - 1].hi, inside--;
  if (inside == 0) return false;
  for (int i = 0; i < all.n; i++) {
    StridedSteps s = all;
    s.step[i].lo = 1;
    if (s.near(i, 0)) return true;
  }
  return false;
}

// Whether two tensors of es bytes an element and as many dimensions share elements; their addresses are multiples of es.
inline bool strided_meet(const Strided& x, const Strided& y, int d, int es) {
  const auto end = [&](const Strided& z) {
    StridedSteps::Place e = d;
    for (int i = 0; i < z.dims; i++) e += (StridedSteps::Place)z.stride[i] * (z.size[i] - 1);
    return (StridedSteps::Place)(uintptr_t)z.at + e * es;
  };
  if (end(x) <= (StridedSteps::Place)(uintptr_t)y.at || end(y) <= (StridedSteps::Place)(uintptr_t)x.at) return false;
  StridedSteps s(d);
  for (int i = 0; i < x.dims; i++) {
    if (x.stride[i] == y.stride[i]) {
      s.add(x.stride[i], 1 - x.size[i], y.size[i] - 1);
    } else {
      s.add(x.stride[i], 1 - x.size[i], 0);
      s.add(y.stride[i], 0, y.size[i] - 1);
    }
  }
  s.sort();
  return s.near(0, ((StridedSteps::Place)(uintptr_t)y.at - (StridedSteps::Place)(uintptr_t)x.at) / es);
}

}  // namespace dash
