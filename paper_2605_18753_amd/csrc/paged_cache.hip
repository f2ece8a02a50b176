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
  uint32_t* keys;      // [pair][cap], caches of more than kSelKeys slots only
  int32_t* moves;      // [pair][cap]: the targets from the front, the sources from the back
  int32_t* counts;     // [pair]
};

__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sinks, int first_recent) {
  if (pos < sinks || pos >= first_recent) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);             // -0 is 0
  return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}

constexpr int kSelThreads = 1024;
constexpr int kSelKeys = 32768;                            // keys that are kept in LDS at most
constexpr int kBins = 2048;                                // 11 bits of a key
constexpr int kCands = 2048, kRanked = 256;                // keys that are picked out; that are ranked against each other

// For two counts of a thread: their sums over the threads before it (x, y) and over all (z, w).
__device__ __forceinline__ int4 threads_before(int u, int v, int2* xch) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, us = wave_scan(u), vs = wave_scan(v);
  __syncthreads();
  if (lane == 63) xch[wave] = make_int2(us, vs);
  __syncthreads();
  const int2 c = lane < kSelThreads / 64 ? xch[lane] : make_int2(0, 0);
  const int cu = wave_scan(c.x), cv = wave_scan(c.y);
  const int bu = wave ? __builtin_amdgcn_readlane(cu, wave - 1) : 0, bv = wave ? __builtin_amdgcn_readlane(cv, wave - 1) : 0;
  return make_int4(us - u + bu, vs - v + bv, __builtin_amdgcn_readlane(cu, 63), __builtin_amdgcn_readlane(cv, 63));
}

// A workgroup per pair.  The keys stay in LDS (more than 32768 of them: in the scratch, and come back in chunks).  The budget-th
// largest: the keys are counted by their 11 leading bits; those that share the ones of the key looked for are picked out and ranked
// against each other (more than 256 of them: counted by the next 11 bits, and the last 10; more than 2048 are not picked out).  Then a thread
// takes an odd number of consecutive slots, so that ranks in slot order need one scan over the threads, and its reads meet no
// other's bank.
// What bounds it: the chain of loads (lengths, pages, weights), then LDS and some fifteen barriers one after the other: 32 caches of 4352
// tokens x 8 15 us (256 threads instead of 1024: 20), two of 20 and 32k 33.
__global__ __launch_bounds__(kSelThreads) void paged_select_kernel(EvictArgs e, int room) {   // room: keys that LDS has room for
  const PagedArgs& a = e.a;
  extern __shared__ uint32_t keys[];
  __shared__ int hist[kBins];
  __shared__ int2 xch[kSelThreads / 64], rank[kRanked];
  __shared__ uint32_t cand[kCands];
  __shared__ int chosen[3], n_cand;
  const int pair = blockIdx.x, h = pair % a.h_kv, b = pair / a.h_kv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = paged_len(a, b), left = min(n, e.budget);
  for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
  if (tid < kRanked) rank[tid] = make_int2(0, 0);
  if (tid == 0) n_cand = 0;
  int32_t* src = e.src ? e.src + (int64_t)pair * e.budget : nullptr;
  if (src)
    for (int i = tid; i < e.budget; i += kSelThreads) src[i] = i < left ? i : -1;   // the moves change theirs
  if (n <= e.budget) {
    if (tid == 0) e.counts[pair] = 0;
    return;
  }
  const int first_recent = a.seen[b] - e.recent, pm = (1 << a.page_log) - 1;
  uint32_t* far = e.keys + (int64_t)pair * a.cap;
  const bool one = n <= room;                                // chunk
  __syncthreads();                                           // the counts are zero
  for (int c0 = 0; c0 < n; c0 += room) {
    // Wave w loads rows of 64 slots [w rows, (w + 1) rows) of the chunk, sixteen at a time: their pages, a lane for each 16 slots, then all
    // weights and positions.
    const int end = min(c0 + room, n), rows = (end - c0 + kSelThreads - 1) / kSelThreads, base = c0 + wave * rows * 64;
    for (int j0 = 0; j0 < rows; j0 += 16) {
      const int pages = paged_page_lane(a, b, min(base + (j0 * 4 + lane) * 16, n - 1) >> a.page_log);
      float w[16];
      int p[16];
      auto load = [&](int j) {
        const int64_t at = (((int64_t)__shfl(pages, 4 * j + (lane >> 4)) * a.h_kv + h) << a.page_log) + ((base + (j0 + j) * 64 + lane) & pm);
        w[j] = a.weights[at];
        p[j] = a.pos[at];
      };
      auto use = [&](int j) {
        const int i = base + (j0 + j) * 64 + lane;
        if (j0 + j < rows && i < end) {
          const uint32_t k = evict_key(w[j], p[j], e.sinks, first_recent);
          if (one) keys[i] = k;
          else far[i] = k;
          atomicAdd(&hist[k >> 21], 1);
        }
      };
#pragma unroll
      for (int j = 0; j < 8; j++) load(j);
      if (j0 + 8 < rows) {
#pragma unroll
        for (int j = 8; j < 16; j++) load(j);
      }
#pragma unroll
      for (int j = 0; j < 8; j++) use(j);
      if (j0 + 8 < rows) {
#pragma unroll
        for (int j = 8; j < 16; j++) use(j);
      }
    }
  }
  __syncthreads();
  // body(c0, own): the chunk that begins at slot c0 is in LDS, `own` slots a thread
  auto chunks = [&](auto&& body) {
    for (int c0 = 0; c0 < n; c0 += room) {
      const int len = min(room, n - c0);
      if (!one) {
        __syncthreads();
        for (int i = tid; i < len; i += kSelThreads) keys[i] = far[c0 + i];
        __syncthreads();
      }
      body(c0, ((len + kSelThreads - 1) / kSelThreads) | 1);
    }
  };
  // f(key, slot) for the thread's slots of a chunk
  auto each = [&](int c0, int own, auto&& f) {
    const int end = min((tid + 1) * own, min(room, n - c0));
    int i = tid * own;
    for (; i + 4 <= end; i += 4) {
      const uint32_t k0 = keys[i], k1 = keys[i + 1], k2 = keys[i + 2], k3 = keys[i + 3];
      f(k0, c0 + i); f(k1, c0 + i + 1); f(k2, c0 + i + 2); f(k3, c0 + i + 3);
    }
    for (; i < end; i++) f(keys[i], c0 + i);
  };
  // the bin that holds the want-th largest of the keys counted: how many of its keys stay, and all
  auto find_bin = [&](int want) {
    constexpr int OWN = kBins / kSelThreads;                 // bins of a thread, from the largest
    int c[OWN], sum = 0;
#pragma unroll
    for (int q = 0; q < OWN; q++) sum += c[q] = hist[kBins - 1 - OWN * tid - q];
    int before = threads_before(sum, 0, xch).x;
    if (before < want && before + sum >= want) {
#pragma unroll
      for (int q = 0; q < OWN; q++) {
        if (before < want && before + c[q] >= want) { chosen[0] = kBins - 1 - OWN * tid - q; chosen[1] = want - before; chosen[2] = c[q]; }
        before += c[q];
      }
    }
    __syncthreads();
  };
  find_bin(e.budget);
  uint32_t last = (uint32_t)chosen[0] << 21;                 // the smallest key that stays, from its leading bits on
  int want = chosen[1], ties = chosen[2];                    // of the keys that share them, those that stay, and all
  const int picked = ties <= kCands ? ties : 0;
  if (picked) {
    const uint32_t bin = last >> 21;
    chunks([&](int c0, int own) {
      int mine = 0;
      each(c0, own, [&](uint32_t k, int) { mine += k >> 21 == bin; });
      if (mine) {
        int at = atomicAdd(&n_cand, mine);
        each(c0, own, [&](uint32_t k, int) { if (k >> 21 == bin) cand[at++] = k; });
      }
    });
    __syncthreads();
  }
  if (ties <= kRanked) {
    // thread t ranks candidate t % M among a share of them
    int m_log = 0;
    while ((1 << m_log) < ties) m_log++;
    const int me = tid & ((1 << m_log) - 1), share = kSelThreads >> m_log;
    if (me < ties) {
      const uint32_t k = cand[me];
      int more = 0, same = 0;
      for (int i = tid >> m_log; i < ties; i += share) {
        const uint32_t x = cand[i];
        more += x > k;
        same += x == k;
      }
      atomicAdd(&rank[me].x, more);
      atomicAdd(&rank[me].y, same);
    }
    __syncthreads();
    if (tid < ties) {
      const int2 y = rank[tid];
      if (y.x < want && y.x + y.y >= want) {                 // those that find it are equal and write the same
        chosen[0] = (int)(cand[tid] & 0x1fffff);
        chosen[1] = want - y.x;
        chosen[2] = y.y;
      }
    }
    __syncthreads();
    last |= (uint32_t)chosen[0];
    want = chosen[1];
    ties = chosen[2];
  } else {
#pragma unroll 1
    for (int step = 0; step < 2; step++) {
      const int shift = step ? 0 : 10, known = step ? 10 : 21, bits = step ? 1023 : 2047;
      __syncthreads();
      for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      auto count = [&](uint32_t k) { if (k >> known == last >> known) atomicAdd(&hist[(k >> shift) & bits], 1); };
      if (picked) {
        for (int i = tid; i < picked; i += kSelThreads) count(cand[i]);
      } else {
        chunks([&](int c0, int own) { each(c0, own, [&](uint32_t k, int) { count(k); }); });
      }
      __syncthreads();
      find_bin(want);
      last |= (uint32_t)chosen[0] << shift;
      want = chosen[1];
      ties = chosen[2];
    }
  }
  // Of the keys equal to the last one kept, the first `want` stay.
  int32_t* moves = e.moves + (int64_t)pair * a.cap;
  int tied = 0, holes = 0, movers = 0;                       // in the chunks before
  chunks([&](int c0, int own) {
    int spare = 0x7fffffff;                                  // equal keys that stay, from the thread's first on
    if (want < ties) {
      int mine = 0;
      each(c0, own, [&](uint32_t k, int) { mine += k == last; });
      const int4 s = threads_before(mine, 0, xch);
      spare = want - tied - s.x;
      tied += s.z;
    }
    uint64_t stay = 0;                                       // of the thread's 33 slots at most
    int freed = 0, moved = 0, same = 0;
    each(c0, own, [&](uint32_t k, int i) {
      const bool kept = k > last || (k == last && same++ < spare);
      stay |= (uint64_t)kept << (i - c0 - tid * own);
      freed += !kept && i < left;
      moved += kept && i >= left;
    });
    const int4 s = threads_before(freed, moved, xch);        // (every thread has read its keys by then)
    // the lists take the keys' place, each slot of the chunk once at most, before they are written out in whole lines
    const int end = min((tid + 1) * own, min(room, n - c0));
    int at = s.x, am = s.z + s.y;
    for (int i = tid * own; i < end; i++) {
      const bool kept = (stay >> (i - tid * own)) & 1;
      if (!kept && c0 + i < left) keys[at++] = (uint32_t)(c0 + i);
      if (kept && c0 + i >= left) keys[am++] = (uint32_t)(c0 + i);
    }
    __syncthreads();
    for (int i = tid; i < s.z; i += kSelThreads) moves[holes + i] = (int)keys[i];
    for (int i = tid; i < s.w; i += kSelThreads) moves[a.cap - 1 - movers - i] = (int)keys[s.z + i];
    holes += s.z;
    movers += s.w;
  });
  if (tid == 0) e.counts[pair] = holes;
}

// A wave moves eight tokens at a time: their places first, a lane each, then all their rows at once.
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
  return evict_align(pairs * 4) + evict_align(pairs * a.cap * 4) * (a.cap > kSelKeys ? 2 : 1);
}

hipError_t launch_paged_evict(const PagedArgs& a, int elem, int d, int32_t* lens, int budget, int sinks, int recent, int32_t* src,
                              char* ws, hipStream_t st) {
  EvictArgs e;
  e.a = a; e.budget = budget; e.sinks = sinks; e.recent = recent; e.lens = lens; e.src = src;
  const size_t pairs = (size_t)a.batch * a.h_kv;
  e.counts = (int32_t*)ws;
  e.moves = (int32_t*)(ws + evict_align(pairs * 4));
  e.keys = (uint32_t*)(ws + evict_align(pairs * 4) + evict_align(pairs * a.cap * 4));   // of caches that LDS may have no room for
  const int room = a.cap < kSelKeys ? a.cap : kSelKeys;
  static LdsOptIn opt_in;
  if (hipError_t r = allow_dyn_lds((const void*)paged_select_kernel, (size_t)room * 4, opt_in); r != hipSuccess) return r;
  hipLaunchKernelGGL(paged_select_kernel, dim3((unsigned)pairs), dim3(kSelThreads), (size_t)room * 4, st, e, room);
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
