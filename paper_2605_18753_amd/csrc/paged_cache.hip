// The paged cache itself: new tokens into their pages, and the eviction of the tokens with the least weight.
#include "paged.h"

namespace dash {

// ---- append ----------------------------------------------------------------------------------------------------------
// A workgroup writes kAppendRows packed rows: every row's keys and values of all kv-heads, 16 bytes a thread at a time.  Bound by
// HBM: each byte is read once and written once.
constexpr int kAppendRows = 4;

template <int ES>   // bytes of an element
__global__ __launch_bounds__(256) void paged_append_kernel(PagedArgs a, int chunks) {   // chunks: 16-byte pieces of a row
  const int tid = threadIdx.x, lane = tid & 63;
  for (int i = 0; i < kAppendRows; i++) {
    const int row = blockIdx.x * kAppendRows + i;
    if (row >= a.n_rows) return;
    // the sequence the row belongs to: as many as end at or before it
    int b = 0;
    for (int i0 = 0; i0 < a.batch; i0 += 64)
      b += __popcll(__ballot(i0 + lane < a.batch && a.row_start[i0 + lane + 1] <= row));
    b = __builtin_amdgcn_readfirstlane(b);
    if (b >= a.batch) continue;
    const int2 rm = paged_rows(a, b);
    const int back = rm.x + rm.y - row, n = paged_len(a, b), slot = n - back;   // back: 1 for the newest token
    if (row < rm.x || back < 1 || slot < 0) continue;
    const uint32_t page = (uint32_t)a.table[(int64_t)b * a.max_pages + (slot >> a.page_log)];
    if (page >= (uint32_t)a.n_pages) continue;             // no page: nothing is written
    const int off = slot & ((1 << a.page_log) - 1);
    for (int x = tid; x < 2 * a.h_kv * chunks; x += 256) {
      const int c = x % chunks, y = x / chunks, h = y >> 1;
      const bool is_v = y & 1;
      const char* from = (const char*)(is_v ? a.v_new : a.k_new) + (row * (is_v ? a.vn_t : a.kn_t) + h * (is_v ? a.vn_h : a.kn_h)) * ES;
      char* to = (char*)(is_v ? a.v : a.k) + ((int64_t)page * (is_v ? a.vp_p : a.kp_p) + h * (is_v ? a.vp_h : a.kp_h) + off * (is_v ? a.vp_t : a.kp_t)) * ES;
      reinterpret_cast<u32x4*>(to)[c] = reinterpret_cast<const u32x4*>(from)[c];
    }
    if (a.weights || a.pos)
      for (int h = tid; h < a.h_kv; h += 256) {
        const int64_t at = (((int64_t)page * a.h_kv + h) << a.page_log) + off;
        if (a.weights) a.weights[at] = 0.f;
        if (a.pos) a.pos[at] = (a.seen ? a.seen[b] : n) - back;
      }
  }
}

hipError_t launch_paged_append(const PagedArgs& a, int elem, int d, hipStream_t st) {
  const dim3 grid((unsigned)((a.n_rows + kAppendRows - 1) / kAppendRows)), blk(256);
  if (elem == 2) hipLaunchKernelGGL(paged_append_kernel<2>, grid, blk, 0, st, a, d * 2 / 16);
  else hipLaunchKernelGGL(paged_append_kernel<4>, grid, blk, 0, st, a, d * 4 / 16);
  return hipGetLastError();
}

// ---- eviction --------------------------------------------------------------------------------------------------------
// Per (sequence, kv-head): the `budget` slots with the largest (key, -slot) stay, where the key orders the weights as unsigned
// numbers, with the protected tokens above every weight and NaN below.  Kept tokens behind the budget then move into the
// slots before it that were freed, both in ascending order: only those rows are read and written, and no source is a target.
struct EvictArgs {
  PagedArgs a;
  int budget, sinks, recent;
  int32_t* lens; int32_t* src;
  uint32_t* keys;      // [pair][cap]
  int32_t* moves;      // [pair][cap]: the targets from the front, the sources from the back
  int32_t* counts;     // [pair]
};

__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sinks, int first_recent) {
  if (pos < sinks || pos >= first_recent) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);             // -0 is 0
  return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kSelRows = 32;                               // keys a thread holds in registers at most: sequences of up to 32768 tokens
constexpr int kBins = 2048;                                // 11, 11 and 10 bits of a key

// sum of `v`, the same in a wave's lanes, over the waves before one's own, and over all
__device__ __forceinline__ int2 waves_before(int v, int wave, int* xch) {
  __syncthreads();
  if ((threadIdx.x & 63) == 0) xch[wave] = v;
  __syncthreads();
  int2 s = make_int2(0, 0);
#pragma unroll
  for (int w = 0; w < kSelWaves; w++) {
    const int c = xch[w];
    s.x += w < wave ? c : 0;
    s.y += c;
  }
  return s;
}

// A workgroup per pair.  Wave w owns rows of 64 slots [w rows, (w + 1) rows), so that ranks in slot order need one exchange between
// the waves.  The keys stay in registers (sequences of more than 32768 tokens: in the scratch); the budget-th largest is found by
// counting its 11 leading bits, of those that share them the next 11, then the last 10.
__global__ __launch_bounds__(kSelThreads) void paged_select_kernel(EvictArgs e) {
  const PagedArgs& a = e.a;
  __shared__ int hist[kBins];
  __shared__ int xch[kSelWaves], chosen[2];
  const int pair = blockIdx.x, h = pair % a.h_kv, b = pair / a.h_kv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = paged_len(a, b), left = min(n, e.budget);
  int32_t* src = e.src ? e.src + (int64_t)pair * e.budget : nullptr;
  if (src)
    for (int i = tid; i < e.budget; i += kSelThreads) src[i] = i < left ? i : -1;   // the moves change theirs
  if (n <= e.budget) {
    if (tid == 0) e.counts[pair] = 0;
    return;
  }
  const int first_recent = a.seen[b] - e.recent, pm = (1 << a.page_log) - 1;
  const int rows = (n + kSelThreads - 1) / kSelThreads;    // of 64 slots, a wave's
  const int slot0 = wave * rows * 64 + lane;
  uint32_t* keys = e.keys + (int64_t)pair * a.cap;
  auto key_of = [&](int i) -> uint32_t {
    const int64_t at = (((int64_t)paged_page_lane(a, b, i >> a.page_log) * a.h_kv + h) << a.page_log) + (i & pm);
    return evict_key(a.weights[at], a.pos[at], e.sinks, first_recent);
  };
  uint32_t prefix = 0, mask = 0;
  int want = e.budget;                                     // of the keys that begin with prefix
  // each(f): f(key, slot) for every row of the wave, all lanes; slots behind the end among them
  auto select = [&](auto&& each) {
    for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
    for (int step = 0; step < 3; step++) {
      const int shift = step == 0 ? 21 : step == 1 ? 10 : 0, bits = step == 2 ? 1023 : 2047;
      __syncthreads();
      each([&](uint32_t k, int i) {
        if (i < n && (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & bits], 1);
      });
      __syncthreads();
      const int b1 = hist[kBins - 1 - 2 * tid], b0 = hist[kBins - 2 - 2 * tid];      // this thread's two bins, from the largest
      hist[kBins - 1 - 2 * tid] = 0;
      hist[kBins - 2 - 2 * tid] = 0;
      const int incl = wave_scan(b1 + b0);
      const int before = waves_before(__builtin_amdgcn_readlane(incl, 63), wave, xch).x + incl - b1 - b0;
      if (before < want && before + b1 >= want) { chosen[0] = kBins - 1 - 2 * tid; chosen[1] = want - before; }
      else if (before + b1 < want && before + b1 + b0 >= want) { chosen[0] = kBins - 2 - 2 * tid; chosen[1] = want - before - b1; }
      __syncthreads();
      prefix |= (uint32_t)chosen[0] << shift;
      mask |= (uint32_t)bits << shift;
      want = chosen[1];
    }
    // of the keys equal to the last one kept, the first `want` stay
    const uint64_t below = (1ull << lane) - 1ull;
    int ties = 0;
    each([&](uint32_t k, int i) { ties += __popcll(__ballot(i < n && k == prefix)); });
    const int2 tw = waves_before(ties, wave, xch);
    const bool all_ties = tw.y == want;
    int t = tw.x, holes = 0, movers = 0;
    auto kept_of = [&](uint32_t k, int i) {
      const bool tie = i < n && k == prefix;
      bool kept = i < n && (k > prefix || tie);
      if (!all_ties) {
        const uint64_t tb = __ballot(tie);
        if (tie && t + __popcll(tb & below) >= want) kept = false;
        t += __popcll(tb);
      }
      return kept;
    };
    each([&](uint32_t k, int i) {
      const bool kept = kept_of(k, i);
      holes += __popcll(__ballot(!kept && i < left));
      movers += __popcll(__ballot(kept && i >= left));
    });
    const int2 hw = waves_before(holes, wave, xch);
    int at_hole = hw.x, at_mover = a.cap - 1 - waves_before(movers, wave, xch).x;
    int32_t* moves = e.moves + (int64_t)pair * a.cap;
    t = tw.x;
    each([&](uint32_t k, int i) {
      const bool kept = kept_of(k, i), hole = !kept && i < left, mover = kept && i >= left;
      const uint64_t hb = __ballot(hole), mb = __ballot(mover);
      if (hole) moves[at_hole + __popcll(hb & below)] = i;
      if (mover) moves[at_mover - __popcll(mb & below)] = i;
      at_hole += __popcll(hb);
      at_mover -= __popcll(mb);
    });
    if (tid == 0) e.counts[pair] = hw.y;
  };
  if (rows <= kSelRows) {
    uint32_t key[kSelRows];
#pragma unroll
    for (int j0 = 0; j0 < kSelRows; j0 += 16) {            // sixteen rows in flight
      if (j0 < rows) {
        float w[16];
        int p[16];
#pragma unroll
        for (int j = 0; j < 16; j++) {
          const int i = min(slot0 + (j0 + j) * 64, n - 1);
          const int64_t at = (((int64_t)paged_page_lane(a, b, i >> a.page_log) * a.h_kv + h) << a.page_log) + (i & pm);
          w[j] = a.weights[at];
          p[j] = a.pos[at];
        }
#pragma unroll
        for (int j = 0; j < 16; j++) key[j0 + j] = evict_key(w[j], p[j], e.sinks, first_recent);
      }
    }
    select([&](auto&& f) {
#pragma unroll
      for (int j = 0; j < kSelRows; j++) {
        if (j < rows) f(key[j], slot0 + j * 64);
      }
    });
  } else {
#pragma unroll 8
    for (int j = 0; j < rows; j++) {
      const int i = slot0 + j * 64;
      if (i < n) keys[i] = key_of(i);
    }
    select([&](auto&& f) {
#pragma unroll 8
      for (int j = 0; j < rows; j++) {
        const int i = slot0 + j * 64;
        f(i < n ? keys[i] : 0u, i);
      }
    });
  }
}

template <int ES, int D>
__global__ __launch_bounds__(256) void paged_move_kernel(EvictArgs e, int wgs) {   // wgs: workgroups of a pair
  const PagedArgs& a = e.a;
  constexpr int C = D * ES / 16, PER = 256 / (2 * C);      // 16-byte pieces of a row; moves a workgroup makes at a time
  const int pair = blockIdx.x / wgs, part = blockIdx.x % wgs, h = pair % a.h_kv, b = pair / a.h_kv;
  const int n_moves = e.counts[pair];
  if (h == 0 && part == 0 && threadIdx.x == 0) e.lens[b] = min(max(e.lens[b], 0), min(a.cap, e.budget));
  const int32_t* moves = e.moves + (int64_t)pair * a.cap;
  int32_t* src = e.src ? e.src + (int64_t)pair * e.budget : nullptr;
  const int sub = threadIdx.x / (2 * C), x = threadIdx.x % (2 * C), c = x % C;
  const bool is_v = x >= C;
  const int pm = (1 << a.page_log) - 1;
  char* base = (char*)(is_v ? a.v : a.k) + h * (is_v ? a.vp_h : a.kp_h) * ES;
  const int64_t sp = (is_v ? a.vp_p : a.kp_p) * ES, st = (is_v ? a.vp_t : a.kp_t) * ES;
  for (int j = part * PER + sub; j < n_moves; j += wgs * PER) {
    const int to = moves[j], from = moves[a.cap - 1 - j];
    const uint32_t pt = (uint32_t)a.table[(int64_t)b * a.max_pages + (to >> a.page_log)];
    const int pf = paged_page_lane(a, b, from >> a.page_log);
    if (src && x == 0) src[to] = from;
    if (pt >= (uint32_t)a.n_pages) continue;
    reinterpret_cast<u32x4*>(base + pt * sp + (to & pm) * st)[c] = reinterpret_cast<const u32x4*>(base + pf * sp + (from & pm) * st)[c];
    if (x < 2) {
      const int64_t it = (((int64_t)pt * a.h_kv + h) << a.page_log) + (to & pm), jf = (((int64_t)pf * a.h_kv + h) << a.page_log) + (from & pm);
      if (x == 0) a.weights[it] = a.weights[jf];
      else a.pos[it] = a.pos[jf];
    }
  }
}

static size_t evict_align(size_t x) { return (x + 255) & ~(size_t)255; }
size_t paged_evict_ws(const PagedArgs& a) {
  const size_t pairs = (size_t)a.batch * a.h_kv;
  return evict_align(pairs * 4) + 2 * evict_align(pairs * a.cap * 4);
}

hipError_t launch_paged_evict(const PagedArgs& a, int elem, int d, int32_t* lens, int budget, int sinks, int recent, int32_t* src,
                              char* ws, hipStream_t st) {
  EvictArgs e;
  e.a = a; e.budget = budget; e.sinks = sinks; e.recent = recent; e.lens = lens; e.src = src;
  const size_t pairs = (size_t)a.batch * a.h_kv;
  e.counts = (int32_t*)ws;
  e.keys = (uint32_t*)(ws + evict_align(pairs * 4));
  e.moves = (int32_t*)(ws + evict_align(pairs * 4) + evict_align(pairs * a.cap * 4));
  hipLaunchKernelGGL(paged_select_kernel, dim3((unsigned)pairs), dim3(kSelThreads), 0, st, e);
  if (hipError_t r = hipGetLastError(); r != hipSuccess) return r;
  // eight workgroups per CU are resident at once; how many tokens move is not known here
  const int wgs = pairs < 2048 ? (int)(2048 / pairs < 64 ? 2048 / pairs : 64) : 1;
  const dim3 grid((unsigned)(pairs * wgs)), blk(256);
  if (elem == 2 && d == 128) hipLaunchKernelGGL((paged_move_kernel<2, 128>), grid, blk, 0, st, e, wgs);
  else if (elem == 2) hipLaunchKernelGGL((paged_move_kernel<2, 64>), grid, blk, 0, st, e, wgs);
  else if (d == 128) hipLaunchKernelGGL((paged_move_kernel<4, 128>), grid, blk, 0, st, e, wgs);
  else hipLaunchKernelGGL((paged_move_kernel<4, 64>), grid, blk, 0, st, e, wgs);
  return hipGetLastError();
}

}  // namespace dash
