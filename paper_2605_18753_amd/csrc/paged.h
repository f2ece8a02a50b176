// What the kernels of the paged cache share: their arguments, how a call's work is dealt to workgroups, and the
// launchers each file exports.
//
// Dealing.  The host knows the number of packed rows and sequences, not their lengths, which lie on the device.  A launch has
// a fixed grid; every workgroup finds its own work from row_start and lens (one pass over them, 64 sequences at a time).  An item of the
// attention is a tile of a sequence's rows for one kv-head; its cost is the steps of keys that it walks.
//   Tiles of 16 rows: the steps of all items of a kv-head lie one behind the other, and G workgroups take equal runs
//   [w F / G, (w + 1) F / G) of them: whatever the lengths, every CU streams as many keys.
//   Tiles of 128 rows: one item a workgroup; items that leave the chip idle are cut into parts.  With n items of costs c_i and W > n
//   workgroups, parts of S = ceil(sum c_i / (W - n)) give sum ceil(c_i / S) <= W of them.  W is what is resident at once, or n and one and a
//   half times that where the items' lengths would leave much of the chip idle; or one item a CU stays whole and the others are cut to fill up what
//   these leave (paged_part_size).  (Finer parts: 40 tokens of 40 sequences of 300 to 8000, 32 / 2 heads, 196 -> 157 us; 700 of one of 30000
//   384 -> 360; 1501 tokens beside decoding ones, where they are not taken, 305 and 326.)
//   (Equal runs for these as well: a run begins anew for every piece of an item, and most are cut.  1501 tokens beside seven decoding
//   sequences of up to 12k 305 -> 309 us and the records to add up, 2048 tokens against 32k 995 -> 1088.)
// Cut items leave records.  Of parts a second launch adds them up; of runs the workgroup whose record of an item is complete last, which
// sees the flags of all (stored past the caches, as in decode_body.h; who merges clears them, so a captured launch can be replayed), or where
// there are many in two levels.
#pragma once
#include "common.h"
#include "dash_internal.h"

namespace dash {

struct PagedArgs {
  const void* q; void* o; float* lse; const float* lse_in;
  void* k; void* v;                      // pages
  const void* k_new; const void* v_new;
  const int32_t* row_start; const int32_t* lens; const int32_t* table; const int32_t* seen;
  float* weights; int32_t* pos;
  int batch, h_q, h_kv, g, page_log, n_pages, max_pages, cap, n_rows, causal, last;
  int64_t q_t, q_h, o_t, o_h, kn_t, kn_h, vn_t, vn_h, kp_p, kp_h, kp_t, vp_p, vp_h, vp_t;
  float c1;                              // scale * log2(e)
  int wgs;                               // runs of a kv-head; 0: an item a workgroup.  Tiles of 128 rows: parts of a kv-head at most; 0: none is cut
  int whole;                             // runs: items may be left uncut; weights: two kernels share the sequences
  int slots; float gain;                 // tiles of 128 rows: workgroups of a kv-head that are resident at once; what finer parts must come to
  float* part_o; float* part_ml;         // records of cut items: two of each run (the item it begins in, the one it ends in), one of each part
  uint64_t* flags; uint64_t nonce;       // runs: two of each record, and the number that says that it is complete
};

__device__ __forceinline__ int paged_len(const PagedArgs& a, int b) { return min(max(a.lens[b], 0), a.cap); }
// first packed row of sequence b and how many it has
__device__ __forceinline__ int2 paged_rows(const PagedArgs& a, int b) {
  const int r0 = min(max(a.row_start[b], 0), a.n_rows);
  return make_int2(r0, min(max(a.row_start[b + 1], r0), a.n_rows) - r0);
}
// A lane's sequence of 64: its rows and length (none behind the batch).  The first 64 are loaded once and kept.
struct PagedLane { int2 rm; int n; };
__device__ __forceinline__ PagedLane paged_lane(const PagedArgs& a, int b) {
  PagedLane l = {make_int2(0, 0), 0};
  if (b < a.batch) {
    l.rm = paged_rows(a, b);
    l.n = paged_len(a, b);
  }
  return l;
}

// Entry i of a sequence's table, read as a scalar: the caller's index is uniform.  Reads take a page of the pool, whatever the
// entry says; writes look at it first.
__device__ __forceinline__ int paged_entry(const PagedArgs& a, int b, int i) {
  const auto* t = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.table + (int64_t)b * a.max_pages);
  return t[min(i, a.max_pages - 1)];
}
__device__ __forceinline__ int paged_clamp(const PagedArgs& a, int page) { return (int)min((uint32_t)page, (uint32_t)(a.n_pages - 1)); }
__device__ __forceinline__ int paged_page(const PagedArgs& a, int b, int i) { return paged_clamp(a, paged_entry(a, b, i)); }
// the same for an index of the lane's own
__device__ __forceinline__ int paged_page_lane(const PagedArgs& a, int b, int i) {
  return paged_clamp(a, a.table[(int64_t)b * a.max_pages + min(i, a.max_pages - 1)]);
}

// ---- parts (tiles of 128 rows) ----------------------------------------------------------------------------------------
constexpr int kMinPart = 4;                                // steps a part has at least
// The size S of a part, no item costing more: none is cut; a wave's lanes together.  shape(m, n) gives a sequence's tiles and the cost
// of one (at least 1); l0: the first 64 sequences.
constexpr int kUncut = 0x3fffffff;
struct PagedCut { int size, whole; };                      // of the items behind the first `whole`
// of sequence tiles, those among the first `whole` items; before: items before the sequence's
__device__ __forceinline__ int paged_whole(const PagedCut& cut, int before, int tiles) { return min(max(cut.whole - before, 0), tiles); }
// The launch that adds the parts up has to come to the same: no products are fused with sums here.
template <typename F> __device__ __forceinline__ PagedCut paged_part_size(const PagedArgs& a, const PagedLane& l0, F&& shape) {
#pragma clang fp contract(off)
  if (a.wgs <= 0) return {kUncut, 0};
  const int lane = lane_id(), half = a.slots / 2;
  int items = 0;
  float cost = 0.f, most = 0.f, rest = 0.f;                // rest: of the items behind the first `half`
  for (int i0 = 0; i0 < a.batch; i0 += 64) {
    const PagedLane l = i0 ? paged_lane(a, i0 + lane) : l0;
    const int2 s = shape(l.rm.y, l.n);
    const int incl = items + wave_scan(s.x);
    rest += wave_sum((float)(s.x - min(max(half - (incl - s.x), 0), s.x)) * (float)s.y);
    items = __builtin_amdgcn_readlane(incl, 63);
    cost += wave_sum((float)s.x * (float)s.y);
    most = fmaxf(most, wave_max(s.x > 0 ? (float)s.y : 0.f));
  }
  if (items >= a.wgs) return {kUncut, 0};
  const auto size = [&](float c, int w) { return max((int)fminf(c * 1.0001f / (float)(w - items), 1e9f) + 1, kMinPart); };   // the factor covers the sum's rounding
  // The time, in steps, of parts that are all resident (or of items, where more are not), and of finer ones that follow each other: what everybody
  // has on the average, half a part until the last is done (a quarter beside whole items, which run faster alone), and what a part costs besides: 4
  // steps, or 10 where it is one more than a workgroup would have.  (One item a CU whole, the others filling up: 2200 tokens against 32k, 32 / 8
  // heads, 69 items for 64 places, 1418 -> 1197 us; 1500, 47 items, 865 -> 785; against 2000, where it is not done, 54 and 64.)
  const float even = cost / (float)a.slots;
  PagedCut cut = {items < a.slots ? size(cost, a.slots) : kUncut, 0};
  float time = items <= a.slots ? fminf((float)cut.size, most) : fminf((float)((items + a.slots - 1) / a.slots) * most, even + 0.5f * most);
  if (a.wgs > a.slots) {
    const int fine = size(cost, a.wgs);
    if (even + 0.5f * (float)fine + 4.f < a.gain * time) cut = {fine, 0};
    else if (items > half && most * (float)items < 1.2f * cost) {   // of like lengths: one item a CU stays whole, the others fill up what these leave
      const int fill = max(size(rest, a.wgs), (int)(0.5f * even));
      if (even + 0.25f * (float)fill + 10.f < (a.gain + 0.05f) * time) cut = {fill, half};
    }
  }
  if ((float)cut.size >= most) cut = {kUncut, 0};
  return cut;
}

struct PagedPart { int b, tile, part, parts, rec0, r0, m, n; };   // rec0: the item's first part among those of the kv-head
// Every lane of a wave: part `idx` of a kv-head.
template <typename F> __device__ __forceinline__ bool paged_find_part(const PagedArgs& a, int idx, F&& shape, PagedPart& it) {
  const int lane = lane_id();
  const PagedLane l0 = paged_lane(a, lane);
  const PagedCut cut = paged_part_size(a, l0, shape);
  const bool whole = idx < cut.whole;
  int items = 0, base = whole ? 0 : cut.whole;
  for (int i0 = 0; i0 < a.batch; i0 += 64) {
    const PagedLane p = i0 ? paged_lane(a, i0 + lane) : l0;
    const int2 s = shape(p.rm.y, p.n);
    const int upto = items + wave_scan(s.x), uncut = paged_whole(cut, upto - s.x, s.x);
    const int parts = whole ? 1 : (s.y + cut.size - 1) / cut.size, skip = whole ? 0 : uncut, count = (s.x - skip) * parts;
    const int incl = wave_scan(count);
    const uint64_t hit = __ballot(base + incl > idx);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      it.b = i0 + l;
      it.parts = __builtin_amdgcn_readlane(parts, l);
      const int in = idx - (base + __builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(count, l));
      // the last tiles first: of a causal prompt they are the longest
      it.tile = __builtin_amdgcn_readlane(s.x, l) - 1 - __builtin_amdgcn_readlane(skip, l) - in / it.parts;
      it.part = in % it.parts;
      it.rec0 = idx - it.part;
      it.r0 = __builtin_amdgcn_readlane(p.rm.x, l);
      it.m = __builtin_amdgcn_readlane(p.rm.y, l);
      it.n = __builtin_amdgcn_readlane(p.n, l);
      return true;
    }
    items = __builtin_amdgcn_readlane(upto, 63);
    base += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// ---- runs (tiles of 16 rows) ------------------------------------------------------------------------------------------
// Steps are of 128 keys.  With m new tokens behind `old`, tile t of a causal call, T = 16 / g tokens, walks ceil((old + (t + 1) T) / 128) =
// ceil((u + t + 1) / k) steps, u = ceil(old / T), k = 128 / T, and the tiles before it H(u + t) - H(u), H(x) = sum of ceil(y / k) over
// y = 1 .. x.  Runs are used for fewer than 4096 items, of at most 2^17 steps each: 32 bits (H may wrap, its differences do not).
constexpr int kStep = 128;
// Adding up the pieces of an item takes as long as so many steps: items that are no longer than the runs would be by more than that are not cut, if there
// is a workgroup for each.  (One token of sequences of 200 to 1000, 32 / 8 heads, 16 of them: 13.6 us, cut 19.1; 32: 17.7 and 23.3; one of
// 1000: 12.2 and 9.0.)
constexpr int kJoin = 6;
struct PagedSeq { int tiles, u, flat; };                   // flat > 0: steps of every tile (no causal mask)
struct PagedItem { int b, tile, r0, m, n; PagedSeq s; };
struct PagedDeal {
  int T, k_log;                                            // tokens of a tile, log2 of k
  __device__ __forceinline__ PagedDeal(const PagedArgs& a) : T(16 / a.g), k_log(31 - __builtin_clz(kStep / (16 / a.g))) {}
  __device__ __forceinline__ PagedSeq seq(const PagedArgs& a, int m, int n) const {
    return {(m + T - 1) / T, (max(n - m, 0) + T - 1) / T, a.causal ? 0 : max((n + kStep - 1) / kStep, 1)};
  }
  __device__ __forceinline__ uint32_t h(int x) const {
    const uint32_t c = (uint32_t)x >> k_log, r = (uint32_t)x & ((1u << k_log) - 1u);
    return ((c & 1 ? c * ((c + 1) / 2) : (c / 2) * (c + 1)) << k_log) + (c + 1) * r;
  }
  __device__ __forceinline__ int before(const PagedSeq& s, int t) const { return s.flat ? s.flat * t : (int)(h(s.u + t) - h(s.u)); }
  __device__ __forceinline__ int steps(const PagedSeq& s, int t) const { return s.flat ? s.flat : ((s.u + t) >> k_log) + 1; }
  // the steps of all items of a kv-head, and if they may be left uncut how many there are, and the steps of the longest; a wave's lanes together; l0: the first 64 sequences
  __device__ __forceinline__ int total(const PagedArgs& a, const PagedLane& l0, int& items, int& most) const {
    int f = 0;
    items = most = 0;
    for (int i0 = 0; i0 < a.batch; i0 += 64) {
      const PagedLane l = i0 ? paged_lane(a, i0 + lane_id()) : l0;
      const PagedSeq s = seq(a, l.rm.y, l.n);
      f += __builtin_amdgcn_readlane(wave_scan(before(s, s.tiles)), 63);
      if (!a.whole) continue;
      items += __builtin_amdgcn_readlane(wave_scan(s.tiles), 63);
      most = max(most, (int)wave_max(s.tiles > 0 ? (float)steps(s, s.tiles - 1) : 0.f));
    }
    return f;
  }
  // the item at step f (by_steps), or item number f; returns the steps of the item before f, -1 where there is none
  __device__ __forceinline__ int find(const PagedArgs& a, const PagedLane& l0, int f, bool by_steps, PagedItem& it) const {
    const int lane = lane_id();
    for (int i0 = 0; i0 < a.batch; i0 += 64) {
      const PagedLane p = i0 ? paged_lane(a, i0 + lane) : l0;
      const PagedSeq s = seq(a, p.rm.y, p.n);
      const int v = by_steps ? before(s, s.tiles) : s.tiles, incl = wave_scan(v);
      const uint64_t hit = __ballot(incl > f);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        it.b = i0 + l;
        it.r0 = __builtin_amdgcn_readlane(p.rm.x, l);
        it.m = __builtin_amdgcn_readlane(p.rm.y, l);
        it.n = __builtin_amdgcn_readlane(p.n, l);
        it.s = {__builtin_amdgcn_readlane(s.tiles, l), __builtin_amdgcn_readlane(s.u, l), __builtin_amdgcn_readlane(s.flat, l)};
        const int in = f - __builtin_amdgcn_readlane(incl - v, l);
        if (!by_steps) {
          it.tile = it.s.tiles - 1 - in;                   // the last tiles first: of a causal prompt they are the longest
          return 0;
        }
        int lo = 0, hi = it.s.tiles;                       // before(lo) <= in < before(hi)
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (before(it.s, mid) <= in) lo = mid;
          else hi = mid;
        }
        it.tile = lo;
        return in - before(it.s, lo);
      }
      f -= __builtin_amdgcn_readlane(incl, 63);
    }
    return -1;
  }
};

// Where run w of G = min(a.wgs, F) begins: floor(w F / G), the fraction's part in floats (a numerator below 2^20 and a half, whose
// quotient is nearer than 2^-12 to exact and not nearer than 2^-11 to a whole number).  No run is empty.  I: type of a place.
template <typename I> struct PagedBounds {
  I q, total;
  uint32_t rem;
  int runs;
  float inv;
  __device__ __forceinline__ PagedBounds(const PagedArgs& a, I f) : total(f), runs((int)max(min((I)a.wgs, f), (I)1)) {
    q = f / runs;
    rem = (uint32_t)(f - q * runs);
    inv = 1.f / (float)runs;
  }
  __device__ __forceinline__ I at(int w) const {
    return w >= runs ? total : q * w + (I)(uint32_t)(((float)(rem * (uint32_t)w) + 0.5f) * inv);
  }
};

// The kernel's arguments (its first and only parameter) and thread index, asked for anew: what follows from them is not kept in registers
// from piece to piece, for which the walks have none left.
__device__ __forceinline__ PagedArgs paged_reload() {
  auto p = (const __attribute__((address_space(4))) PagedArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const PagedArgs*)p;
}
__device__ __forceinline__ int paged_thread() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// A workgroup's pieces of items, one after the other: steps [x0, x1) of item `it`.
struct PagedRun {
  PagedDeal deal;
  PagedItem it;
  int x0, x1, cost;
  int next, end, total;                                    // the step behind this piece, the run's end, the steps of the kv-head
  __device__ __forceinline__ PagedRun(const PagedArgs& a) : deal(a) {}
  __device__ __forceinline__ bool begin(const PagedArgs& a, int wg) {
    const PagedLane l0 = paged_lane(a, lane_id());
    bool cut = a.wgs > 0;
    if (cut) {
      int items, most;
      total = deal.total(a, l0, items, most);
      cut = !a.whole || items > a.wgs || (most - kJoin) * a.wgs > total;
    }
    if (!cut) {
      if (deal.find(a, l0, wg, false, it) < 0) return false;
      x0 = next = end = 0;
      x1 = cost = deal.steps(it.s, it.tile);
      return true;
    }
    const PagedBounds<int> b(a, total);
    next = __builtin_amdgcn_readfirstlane(b.at(wg));
    end = __builtin_amdgcn_readfirstlane(b.at(wg + 1));
    if (next >= end) return false;
    x0 = deal.find(a, l0, next, true, it);
    cost = deal.steps(it.s, it.tile);
    return piece();
  }
  __device__ __forceinline__ bool piece() {
    x1 = min(cost, x0 + end - next);
    next += x1 - x0;
    return true;
  }
  __device__ __forceinline__ bool advance(const PagedArgs& a) {
    if (next >= end) return false;
    x0 = 0;
    if (++it.tile >= it.s.tiles) deal.find(a, paged_lane(a, lane_id()), next, true, it);
    cost = deal.steps(it.s, it.tile);
    return piece();
  }
  __device__ __forceinline__ bool whole() const { return x0 == 0 && x1 == cost; }
};

hipError_t launch_paged_append(const PagedArgs& a, int elem, int d, hipStream_t st);
hipError_t launch_paged_attend(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st);
hipError_t launch_paged_weigh(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st);
hipError_t launch_paged_evict(const PagedArgs& a, int elem, int d, int32_t* lens, int budget, int sinks, int recent, int32_t* src,
                              char* ws, hipStream_t st);
bool paged_attend_fits(const PagedArgs& a, int dtype);
size_t paged_attend_ws(const PagedArgs& a, int dtype, int d);
size_t paged_weigh_ws(const PagedArgs& a, int dtype, int d);
size_t paged_evict_ws(const PagedArgs& a);

}  // namespace dash
