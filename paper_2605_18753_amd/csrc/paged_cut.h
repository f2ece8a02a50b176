// Into what parts a launch of tiles of 128 rows cuts its items, as far as it is arithmetic.  Plain C++: the CPU tests compile it too.
#pragma once
#include <math.h>

#ifdef __HIP__
#define DASH_CUT __device__ __forceinline__
#else
#define DASH_CUT inline
#endif

namespace dash {

constexpr int kMinPart = 4;                                // steps a part has at least
constexpr int kUncut = 0x3fffffff;
struct PagedCut { int size, whole, items; };               // parts of at most `size` steps, of the items behind the first `whole`

// The size S of a part, no item costing more: none is cut.  For a kv-head: wgs, parts at most (above 0); slots, workgroups that are resident at once; gain, what finer
// parts must come to; items, what they cost together, the largest, and those behind the first slots / 2.
// The launch that adds the parts up has to come to the same: no products are fused with sums here.
template <bool FOUR> DASH_CUT PagedCut paged_cut(int wgs, int slots, float gain, int items, float cost, float most, float rest) {
#ifdef __clang__
#pragma clang fp contract(off)
#endif
  const auto larger = [](int x, int y) { return x > y ? x : y; };
  const auto smaller = [](int x, int y) { return x < y ? x : y; };
  if (items >= wgs) return {kUncut, 0, items};
  const int half = slots / 2;
  const auto size = [&](float c, int w) { return larger((int)fminf(c * 1.0001f / (float)(w - items), 1e9f) + 1, kMinPart); };   // the factor covers the sum's rounding
  // The time, in steps, of parts that are all resident (or of items, where more are not), and of finer ones that follow each other: what everybody
  // has on the average, half a part until the last is done (a quarter beside whole items, which run faster alone), and what a part costs besides: 4
  // steps, or 10 where it is one more than a workgroup would have.  (One item a CU whole, the others filling up: 2200 tokens against 32k, 32 / 8
  // heads, 69 items for 64 places, 1418 -> 1197 us; 1500, 47 items, 865 -> 785; against 2000, where it is not done, 54 and 64.)
  const float even = cost / (float)slots;
  PagedCut cut = {items < slots ? size(cost, slots) : kUncut, 0, items};
  float time = items <= slots ? fminf((float)cut.size, most) : fminf((float)((items + slots - 1) / slots) * most, even + 0.5f * most);
  // A cache in 4 bits, items of one length (one sequence's): as many parts each as there are places for, once or twice.  (The sum over w - n leaves places unused: 512
  // tokens against 32k, 16 items for 64 places, in three parts each 330 us, in four 296; 700, 22 items: five parts take 0.85 of the time of two.)
  bool finer = false;
  if (FOUR && items <= slots && most * (float)items <= cost) {
    const auto parts = [&](int k) { return larger((int)ceilf(most / (float)larger(k, 1)), kMinPart); };
    const int once = parts(slots / larger(items, 1)), twice = parts(smaller(2 * slots, wgs) / larger(items, 1));
    finer = 2 * twice + 6 < once;
    cut.size = finer ? twice : once;
    time = (float)once;
  } else if (wgs > slots) {
    const int fine = size(cost, wgs);
    finer = even + 0.5f * (float)fine + 4.f < gain * time;
    if (finer) cut.size = fine;
  }
  if (wgs > slots && !finer && items > half && most * (float)items < 1.2f * cost) {   // of like lengths: one item a CU stays whole, the others fill up what these leave
    const int fill = larger(size(rest, wgs), (int)(0.5f * even));
    if (even + 0.25f * (float)fill + 10.f < (gain + 0.05f) * time) cut = {fill, half, items};
  }
  if ((float)cut.size >= most) cut = {kUncut, 0, items};
  return cut;
}

}  // namespace dash
