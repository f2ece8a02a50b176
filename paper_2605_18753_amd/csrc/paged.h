// What the kernels of the paged cache share: their arguments, how a call's work is dealt to workgroups, and the
// launchers each file exports.
//
// Dealing.  The host knows the number of packed rows and sequences, not their lengths, which lie on the device.  A launch has
// a fixed grid; every workgroup finds its own item from row_start and lens (one pass over them, 64 sequences at a time).  An
// item is a tile of a sequence's rows (attention) or of its keys (weights) of one kv-head; its walk over the other axis is
// cut into parts where the items alone would leave the chip idle.  With n items of costs c_i and W > n workgroups, parts of
// S = ceil(sum c_i / (W - n)) give sum ceil(c_i / S) <= W of them.
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
  int wgs;                               // workgroups of a kv-head that items may be cut for; 0: none is cut
  int min_part;                          // smallest part
  float* part_o; float* part_ml;         // records of cut items: [kv-head][part][row][d], [kv-head][part][row][2]
  int part_stride;                       // records of a kv-head
};

__device__ __forceinline__ int paged_len(const PagedArgs& a, int b) { return min(max(a.lens[b], 0), a.cap); }
// first packed row of sequence b and how many it has
__device__ __forceinline__ int2 paged_rows(const PagedArgs& a, int b) {
  const int r0 = min(max(a.row_start[b], 0), a.n_rows);
  return make_int2(r0, min(max(a.row_start[b + 1], r0), a.n_rows) - r0);
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

struct PagedItem { int b, tile, part, parts, rec0, r0, m, n; };   // rec0: the item's first part among those of the kv-head

// The size S of a part; a wave's lanes together.
template <typename F> __device__ __forceinline__ int paged_part_size(const PagedArgs& a, F&& shape) {
  if (a.wgs <= 0) return 0x3fffffff;
  const int lane = lane_id();
  int items = 0;
  float cost = 0.f;
  for (int i0 = 0; i0 < a.batch; i0 += 64) {
    int2 s = make_int2(0, 0);
    if (i0 + lane < a.batch) s = shape(paged_rows(a, i0 + lane).y, paged_len(a, i0 + lane));
    items += __builtin_amdgcn_readlane(wave_scan(s.x), 63);
    cost += wave_sum((float)s.x * (float)s.y);
  }
  if (items >= a.wgs) return 0x3fffffff;
  return max((int)fminf(cost * 1.0001f / (float)(a.wgs - items), 1e9f) + 1, a.min_part);   // the factor covers the sum's rounding
}

// Every lane of a wave: item `idx` of a kv-head.  shape(m, n) gives a sequence's tiles and the cost of one (at least 1).
template <typename F> __device__ __forceinline__ bool paged_find(const PagedArgs& a, int idx, F&& shape, PagedItem& it) {
  const int lane = lane_id();
  const int S = paged_part_size(a, shape);
  int base = 0;
  for (int i0 = 0; i0 < a.batch; i0 += 64) {
    int2 s = make_int2(0, 0), rm = make_int2(0, 0);
    int n = 0;
    if (i0 + lane < a.batch) {
      rm = paged_rows(a, i0 + lane);
      n = paged_len(a, i0 + lane);
      s = shape(rm.y, n);
    }
    const int parts = (s.y + S - 1) / S;
    const int incl = wave_scan(s.x * parts);
    const uint64_t hit = __ballot(base + incl > idx);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      it.b = i0 + l;
      it.parts = __builtin_amdgcn_readlane(parts, l);
      const int first = base + __builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(s.x, l) * it.parts;
      // the last tiles first: of a causal prompt they are the longest
      it.tile = __builtin_amdgcn_readlane(s.x, l) - 1 - (idx - first) / it.parts;
      it.part = (idx - first) % it.parts;
      it.rec0 = idx - it.part;
      it.r0 = __builtin_amdgcn_readlane(rm.x, l);
      it.m = __builtin_amdgcn_readlane(rm.y, l);
      it.n = __builtin_amdgcn_readlane(n, l);
      return true;
    }
    base += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

hipError_t launch_paged_append(const PagedArgs& a, int elem, int d, hipStream_t st);
hipError_t launch_paged_attend(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st);
hipError_t launch_paged_weigh(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st);
hipError_t launch_paged_evict(const PagedArgs& a, int elem, int d, int32_t* lens, int budget, int sinks, int recent, int32_t* src,
                              char* ws, hipStream_t st);
size_t paged_attend_ws(const PagedArgs& a, int dtype, int d);
size_t paged_weigh_ws(const PagedArgs& a, int dtype, int d);
size_t paged_evict_ws(const PagedArgs& a);

}  // namespace dash
