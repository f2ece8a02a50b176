// The paged cache itself: new tokens into their pages, and the eviction of the tokens with the least weight.
#include <type_traits>

#include "paged.h"

namespace dash {

// ---- append ----------------------------------------------------------------------------------------------------------
// A wave writes a packed row: its keys and values of all kv-heads, 16 bytes a lane at a time.  Bound by HBM where there are many rows (each
// byte is read once and written once), by the chain of dependent loads where there are few: what a row holds, and the starts,
// lengths and positions of 64 sequences, are asked for together; only the page waits for them.
template <int ES, int D>   // bytes of an element
__global__ __launch_bounds__(256) void paged_append_kernel(PagedArgs a) {
  constexpr int CHUNKS = D * ES / 16, AHEAD = 4;             // 16-byte pieces of a row; pieces of a lane in flight
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.n_rows) return;
  const int pieces = 2 * a.h_kv * CHUNKS;
  const char* kn = (const char*)a.k_new + row * a.kn_t * ES;
  const char* vn = (const char*)a.v_new + row * a.vn_t * ES;
  u32x4 w[AHEAD];
  auto load = [&](int x0) {
#pragma unroll
    for (int i = 0; i < AHEAD; i++) {
      const int x = x0 + 64 * i, c = x % CHUNKS, h = x / CHUNKS >> 1;
      const char* from = x / CHUNKS & 1 ? vn + h * a.vn_h * ES : kn + h * a.kn_h * ES;
      if (x < pieces) w[i] = reinterpret_cast<const u32x4*>(from)[c];
    }
  };
  load(lane);
  // the sequence that the row belongs to: as many as end at or before it
  int b = -1, end = 0, n = 0, seen = 0;
  for (int i0 = 0; i0 < a.batch && b < 0; i0 += 64) {
    const int i = min(i0 + lane, a.batch - 1);
    const int s0 = a.row_start[i], s1 = a.row_start[i + 1], len = a.lens[i], sn = a.seen ? a.seen[i] : 0;
    const uint64_t on = __ballot(i0 + lane < a.batch && s1 > row);
    if (on) {
      const int l = __builtin_ctzll(on);
      if (__builtin_amdgcn_readlane(s0, l) > row) return;    // a row of no sequence
      b = i0 + l;
      end = min(__builtin_amdgcn_readlane(s1, l), a.n_rows);
      n = min(max(__builtin_amdgcn_readlane(len, l), 0), a.cap);
      seen = a.seen ? __builtin_amdgcn_readlane(sn, l) : n;
    }
  }
  const int back = end - row, slot = n - back;               // back: 1 for the newest token
  if (b < 0 || slot < 0) return;
  const uint32_t page = (uint32_t)paged_entry(a, b, slot >> a.page_log);
  if (page >= (uint32_t)a.n_pages) return;                   // no page: nothing is written
  const int off = slot & ((1 << a.page_log) - 1);
  char* kp = (char*)a.k + ((int64_t)page * a.kp_p + off * a.kp_t) * ES;
  char* vp = (char*)a.v + ((int64_t)page * a.vp_p + off * a.vp_t) * ES;
  for (int x0 = lane; x0 - lane < pieces; x0 += 64 * AHEAD) {
    if (x0 != lane) load(x0);
#pragma unroll
    for (int i = 0; i < AHEAD; i++) {
      const int x = x0 + 64 * i, c = x % CHUNKS, h = x / CHUNKS >> 1;
      char* to = x / CHUNKS & 1 ? vp + h * a.vp_h * ES : kp + h * a.kp_h * ES;
      if (x < pieces) reinterpret_cast<u32x4*>(to)[c] = w[i];
    }
  }
  for (int h = lane; h < a.h_kv; h += 64) {
    const int64_t at = (((int64_t)page * a.h_kv + h) << a.page_log) + off;
    if (a.weights) a.weights[at] = 0.f;
    if (a.pos) a.pos[at] = seen - back;
  }
}

hipError_t launch_paged_append(const PagedArgs& a, int elem, int d, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)a.n_rows + 3) / 4)), blk(256);
  if (elem == 2 && d == 128) hipLaunchKernelGGL((paged_append_kernel<2, 128>), grid, blk, 0, st, a);
  else if (elem == 2) hipLaunchKernelGGL((paged_append_kernel<2, 64>), grid, blk, 0, st, a);
  else if (d == 128) hipLaunchKernelGGL((paged_append_kernel<4, 128>), grid, blk, 0, st, a);
  else hipLaunchKernelGGL((paged_append_kernel<4, 64>), grid, blk, 0, st, a);
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
  // keys in registers, in blocks of four rows; a row past the wave's last counts as behind the end
  auto in_registers = [&](auto rows_tag) {
    constexpr int ROWS = decltype(rows_tag)::value, AHEAD = ROWS < 16 ? ROWS : 16;
    uint32_t key[ROWS];
#pragma unroll
    for (int j0 = 0; j0 < ROWS; j0 += AHEAD) {
      if (j0 < rows) {
        int64_t at[AHEAD];
        float w[AHEAD];
        int p[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
          const int i = min(slot0 + (j0 + j) * 64, n - 1);
          at[j] = (((int64_t)paged_page_lane(a, b, i >> a.page_log) * a.h_kv + h) << a.page_log) + (i & pm);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
          w[j] = a.weights[at[j]];
          p[j] = a.pos[at[j]];
        }
#pragma unroll
        for (int j = 0; j < AHEAD; j++) key[j0 + j] = evict_key(w[j], p[j], e.sinks, first_recent);
      }
    }
    select([&](auto&& f) {
#pragma unroll
      for (int j0 = 0; j0 < ROWS; j0 += 4) {
        if (j0 < rows) {
#pragma unroll
          for (int j = j0; j < j0 + 4; j++) f(key[j], j < rows ? slot0 + j * 64 : n);
        }
      }
    });
  };
  if (rows <= 8) {                                           // its own code: the longer one's would be fetched for nothing
    in_registers(std::integral_constant<int, 8>{});
  } else if (rows <= kSelRows) {
    in_registers(std::integral_constant<int, kSelRows>{});
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

// A wave moves kMoves tokens at a time: their places first, a lane each, then all their rows at once.
template <int ES, int D>
__global__ __launch_bounds__(256) void paged_move_kernel(EvictArgs e, int wgs) {   // wgs: workgroups of a pair
  const PagedArgs& a = e.a;
  constexpr int C = D * ES / 16, PER = 64 / C > 0 ? 64 / C : 1, MOVES = 8;        // 16-byte pieces of a row; rows a wave's load covers
  const int pair = blockIdx.x / wgs, h = pair % a.h_kv, b = pair / a.h_kv;
  const int lane = threadIdx.x & 63, wave = (blockIdx.x % wgs) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_moves = e.counts[pair];
  if (h == 0 && wave == 0 && lane == 0) e.lens[b] = min(max(e.lens[b], 0), min(a.cap, e.budget));
  const int32_t* moves = e.moves + (int64_t)pair * a.cap;
  const int pm = (1 << a.page_log) - 1, c = lane % C;
  char* kb = (char*)a.k + h * a.kp_h * ES;
  char* vb = (char*)a.v + h * a.vp_h * ES;
  for (int j0 = wave * MOVES; j0 < n_moves; j0 += wgs * 4 * MOVES) {
    const int j = min(j0 + (lane & (MOVES - 1)), n_moves - 1);
    const int to = moves[j], from = moves[a.cap - 1 - j];
    const int pt = a.table[(int64_t)b * a.max_pages + (to >> a.page_log)], pf = paged_page_lane(a, b, from >> a.page_log);
    const bool ok = (uint32_t)pt < (uint32_t)a.n_pages && j0 + (lane & (MOVES - 1)) < n_moves;
    if (lane < MOVES && j0 + lane < n_moves) {
      if (e.src) e.src[(int64_t)pair * e.budget + to] = from;
      if (ok) {
        const int64_t x = (((int64_t)pt * a.h_kv + h) << a.page_log) + (to & pm), y = (((int64_t)pf * a.h_kv + h) << a.page_log) + (from & pm);
        const float w = a.weights[y];
        const int p = a.pos[y];
        a.weights[x] = w;
        a.pos[x] = p;
      }
    }
    constexpr int N = MOVES / PER;
    u32x4 kw[N], vw[N];
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int m = i * PER + lane / C, f = __shfl(from, m), g = __shfl(pf, m);
      kw[i] = reinterpret_cast<const u32x4*>(kb + ((int64_t)g * a.kp_p + (int64_t)(f & pm) * a.kp_t) * ES)[c];
      vw[i] = reinterpret_cast<const u32x4*>(vb + ((int64_t)g * a.vp_p + (int64_t)(f & pm) * a.vp_t) * ES)[c];
    }
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int m = i * PER + lane / C, t = __shfl(to, m), g = __shfl(pt, m);
      if (__shfl((int)ok, m)) {
        reinterpret_cast<u32x4*>(kb + ((int64_t)g * a.kp_p + (int64_t)(t & pm) * a.kp_t) * ES)[c] = kw[i];
        reinterpret_cast<u32x4*>(vb + ((int64_t)g * a.vp_p + (int64_t)(t & pm) * a.vp_t) * ES)[c] = vw[i];
      }
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
