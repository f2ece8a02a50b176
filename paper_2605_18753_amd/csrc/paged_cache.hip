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

// sum of a value over the workgroup, to all of it (two barriers)
__device__ __forceinline__ int wg_sum(int v, int* xch) {
  const int s = __builtin_amdgcn_readlane(wave_scan(v), 63);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) xch[threadIdx.x >> 6] = s;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int i = 0; i < kSelWaves; i++) t += xch[i];
  return t;
}

__global__ __launch_bounds__(kSelThreads) void paged_select_kernel(EvictArgs e) {
  const PagedArgs& a = e.a;
  __shared__ int hist[256];
  __shared__ int xch[kSelWaves], xch2[kSelWaves], chosen[2];
  const int pair = blockIdx.x, h = pair % a.h_kv, b = pair / a.h_kv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = paged_len(a, b), left = min(n, e.budget);
  int32_t* src = e.src ? e.src + (int64_t)pair * e.budget : nullptr;
  if (src)
    for (int i = tid; i < e.budget; i += kSelThreads) src[i] = i < left ? i : -1;   // the moves change theirs
  if (n <= e.budget) {
    if (tid == 0) e.counts[pair] = 0;
    return;
  }
  uint32_t* keys = e.keys + (int64_t)pair * a.cap;
  const int first_recent = a.seen[b] - e.recent;
  for (int i = tid; i < n; i += kSelThreads) {
    const int64_t at = (((int64_t)paged_page_lane(a, b, i >> a.page_log) * a.h_kv + h) << a.page_log) + (i & ((1 << a.page_log) - 1));
    keys[i] = evict_key(a.weights[at], a.pos[at], e.sinks, first_recent);
  }
  // the budget-th largest key, eight bits at a time
  uint32_t prefix = 0, mask = 0;
  int want = e.budget;                                     // of the keys that begin with prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kSelThreads) {
      const uint32_t k = keys[i];
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {                                       // lane l: bins 255 - 4 l .. 252 - 4 l, from the largest
      int c[4], own = 0;
#pragma unroll
      for (int j = 0; j < 4; j++) own += c[j] = hist[255 - 4 * lane - j];
      int before = wave_scan(own) - own;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        if (before < want && before + c[j] >= want) { chosen[0] = 255 - 4 * lane - j; chosen[1] = want - before; }
        before += c[j];
      }
    }
    __syncthreads();
    prefix |= (uint32_t)chosen[0] << shift;
    mask |= 255u << shift;
    want = chosen[1];
  }
  // In slot order: of the keys equal to the last one kept, the first `want` stay.
  int32_t* moves = e.moves + (int64_t)pair * a.cap;
  int ties = 0, holes = 0, movers = 0;                     // before this row of 1024 slots
  for (int i0 = 0; i0 < n; i0 += kSelThreads) {
    const int i = i0 + tid;
    const uint32_t k = i < n ? keys[i] : 0u;
    const bool tie = i < n && k == prefix;
    const uint64_t tb = __ballot(tie);
    __syncthreads();
    if (lane == 0) xch[wave] = __popcll(tb);
    __syncthreads();
    int t = ties;
#pragma unroll
    for (int w = 0; w < kSelWaves; w++) { if (w < wave) t += xch[w]; ties += xch[w]; }
    const bool kept = i < n && (k > prefix || (tie && t + __popcll(tb & ((1ull << lane) - 1ull)) < want));
    const bool hole = !kept && i < left, mover = kept && i >= left;
    const uint64_t hb = __ballot(hole), mb = __ballot(mover);
    if (lane == 0) xch2[wave] = __popcll(hb) | __popcll(mb) << 16;
    __syncthreads();
    int hh = holes, mm = movers;
#pragma unroll
    for (int w = 0; w < kSelWaves; w++) {
      const int c = xch2[w];
      if (w < wave) { hh += c & 0xffff; mm += c >> 16; }
      holes += c & 0xffff; movers += c >> 16;
    }
    if (hole) moves[hh + __popcll(hb & ((1ull << lane) - 1ull))] = i;
    if (mover) moves[a.cap - 1 - (mm + __popcll(mb & ((1ull << lane) - 1ull)))] = i;
  }
  if (tid == 0) e.counts[pair] = holes;
}

constexpr int kMoveWgs = 4;   // workgroups of a pair

template <int ES, int D>
__global__ __launch_bounds__(256) void paged_move_kernel(EvictArgs e) {
  const PagedArgs& a = e.a;
  constexpr int C = D * ES / 16, PER = 256 / (2 * C);      // 16-byte pieces of a row; moves a workgroup makes at a time
  const int pair = blockIdx.x / kMoveWgs, part = blockIdx.x % kMoveWgs, h = pair % a.h_kv, b = pair / a.h_kv;
  const int n_moves = e.counts[pair];
  if (h == 0 && part == 0 && threadIdx.x == 0) e.lens[b] = min(max(e.lens[b], 0), min(a.cap, e.budget));
  const int32_t* moves = e.moves + (int64_t)pair * a.cap;
  int32_t* src = e.src ? e.src + (int64_t)pair * e.budget : nullptr;
  const int sub = threadIdx.x / (2 * C), x = threadIdx.x % (2 * C), c = x % C;
  const bool is_v = x >= C;
  const int pm = (1 << a.page_log) - 1;
  char* base = (char*)(is_v ? a.v : a.k) + h * (is_v ? a.vp_h : a.kp_h) * ES;
  const int64_t sp = (is_v ? a.vp_p : a.kp_p) * ES, st = (is_v ? a.vp_t : a.kp_t) * ES;
  for (int j = part * PER + sub; j < n_moves; j += kMoveWgs * PER) {
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
  const dim3 grid((unsigned)(pairs * kMoveWgs)), blk(256);
  if (elem == 2 && d == 128) hipLaunchKernelGGL((paged_move_kernel<2, 128>), grid, blk, 0, st, e);
  else if (elem == 2) hipLaunchKernelGGL((paged_move_kernel<2, 64>), grid, blk, 0, st, e);
  else if (d == 128) hipLaunchKernelGGL((paged_move_kernel<4, 128>), grid, blk, 0, st, e);
  else hipLaunchKernelGGL((paged_move_kernel<4, 64>), grid, blk, 0, st, e);
  return hipGetLastError();
}

}  // namespace dash
