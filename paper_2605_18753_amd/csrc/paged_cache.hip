// The paged cache itself: new tokens into their pages, and the eviction of the tokens with the least weight.
#include <type_traits>

#include "paged.h"

namespace dash {

// ---- append ----------------------------------------------------------------------------------------------------------
// A wave writes a packed row: its keys and values of all kv-heads, 16 bytes a lane at a time.  Bound by HBM where there are many rows (each
// byte is read once and written once), by the chain of dependent loads where there are few: what a row holds, and the starts,
// lengths and positions of 64 sequences, are asked for together; only the page waits for them.  (2047 tokens of each of four sequences, 8 heads
// of 128: 12.3 us, 5.5 TB/s; a token of 64: 4.1 us.)
// A launch of 2^32 threads or more in a dimension loses some without an error: the workgroups lie in rows of 2^22.
constexpr int kGridLog = 22;
template <int ES, int D>   // bytes of an element
__global__ __launch_bounds__(256) void paged_append_kernel(PagedArgs a) {
  constexpr int CHUNKS = D * ES / 16, AHEAD = 4;             // 16-byte pieces of a row; pieces of a lane in flight
  const int lane = threadIdx.x & 63, row = (int)(blockIdx.y << kGridLog | blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  const int64_t wgs = ((int64_t)a.n_rows + 3) / 4, most = (int64_t)1 << kGridLog;
  const dim3 grid((unsigned)(wgs < most ? wgs : most), (unsigned)((wgs + most - 1) / most)), blk(256);
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
  int budget, sinks, recent;   // the budget is at most cap
  uint32_t src_len;    // slots of a pair in src: the caller's budget, which may be any
  int32_t* lens; int32_t* src;
  int32_t* moves;      // [pair][cap]: the targets from the front, the sources from the back
  int32_t* counts;     // [pair]
  // long caches only
  int chunks;          // chunks of a pair at most
  uint32_t* keys;      // [pair][cap]
  int2* cand;          // [pair][cap]: the keys that share their leading bits with the one looked for, and their slots
  int32_t* hists;      // [pair][chunk][kBins]
  int32_t* above;      // [pair][chunk]: keys with larger leading bits
  int32_t* heads;      // [pair][4]: the leading bits looked for, how many keys that share them stay, and all; slots picked out so far
};

__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sinks, int first_recent) {
  if (pos < sinks || pos >= first_recent) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);             // -0 is 0
  return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}

constexpr int kBins = 2048;                                // 11 bits of a key
// caches of up to so many slots: a workgroup per pair, keys in LDS (two of 8000 tokens x 8 30 us, in three launches 38; sixteen 71 and 82)
constexpr int kSelThreads = 1024, kSelKeys = 8192;
constexpr int kCands = 2048, kRanked = 256;                // keys that are picked out; that are ranked against each other
constexpr int kChunk = 4096, kChunkThreads = 256;          // longer ones: slots and threads of a workgroup
constexpr int kLongCands = 4096;                           // of those picked out, in LDS

// For two counts of a thread: their sums over the threads before it (x, y) and over all (z, w).
template <int THREADS> __device__ __forceinline__ int4 threads_before(int u, int v, int2* xch) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, us = wave_scan(u), vs = wave_scan(v);
  __syncthreads();
  if (lane == 63) xch[wave] = make_int2(us, vs);
  __syncthreads();
  const int2 c = lane < THREADS / 64 ? xch[lane] : make_int2(0, 0);
  const int cu = wave_scan(c.x), cv = wave_scan(c.y);
  const int bu = wave ? __builtin_amdgcn_readlane(cu, wave - 1) : 0, bv = wave ? __builtin_amdgcn_readlane(cv, wave - 1) : 0;
  return make_int4(us - u + bu, vs - v + bv, __builtin_amdgcn_readlane(cu, 63), __builtin_amdgcn_readlane(cv, 63));
}
// Of counts c of a thread's bins (from the largest: the thread's first is bin kBins - 1 - OWN tid): the bin that holds the want-th largest key, how
// many of its keys stay, and all, into chosen[3] (complete behind the barrier).
template <int THREADS> __device__ __forceinline__ void find_bin(const int (&c)[kBins / THREADS], int want, int2* xch, int* chosen) {
  constexpr int OWN = kBins / THREADS;
  int sum = 0;
#pragma unroll
  for (int q = 0; q < OWN; q++) sum += c[q];
  int before = threads_before<THREADS>(sum, 0, xch).x;
  if (before < want && before + sum >= want) {
#pragma unroll
    for (int q = 0; q < OWN; q++) {
      if (before < want && before + c[q] >= want) { chosen[0] = kBins - 1 - OWN * (int)threadIdx.x - q; chosen[1] = want - before; chosen[2] = c[q]; }
      before += c[q];
    }
  }
  __syncthreads();
}
template <int THREADS> __device__ __forceinline__ void find_bin_of(const int* hist, int want, int2* xch, int* chosen) {
  int c[kBins / THREADS];
#pragma unroll
  for (int q = 0; q < kBins / THREADS; q++) c[q] = hist[kBins - 1 - kBins / THREADS * (int)threadIdx.x - q];
  find_bin<THREADS>(c, want, xch, chosen);
}
// Sixteen rows of 64 slots of a wave, from slot `base` on, a multiple of 16 (those before `end`): their pages, a lane for each 16 slots, then all weights
// and positions, eight rows at least in flight; use(key, slot) of each.
template <typename F> __device__ __forceinline__ void evict_keys16(const EvictArgs& e, int b, int h, int first_recent, int base, int rows, int end, F&& use) {
  const PagedArgs& a = e.a;
  const int lane = threadIdx.x & 63, pm = (1 << a.page_log) - 1;
  const int pages = paged_page_lane(a, b, min(base + lane * 16, end - 1) >> a.page_log);
  float w[16];
  int p[16];
  auto load = [&](int j) {
    const int64_t at = (((int64_t)__shfl(pages, 4 * j + (lane >> 4)) * a.h_kv + h) << a.page_log) + ((base + j * 64 + lane) & pm);
    w[j] = a.weights[at];
    p[j] = a.pos[at];
  };
  auto take = [&](int j) {
    const int i = base + j * 64 + lane;
    if (j < rows && i < end) use(evict_key(w[j], p[j], e.sinks, first_recent), i);
  };
#pragma unroll
  for (int j = 0; j < 8; j++) load(j);
  if (8 < rows) {
#pragma unroll
    for (int j = 8; j < 16; j++) load(j);
  }
#pragma unroll
  for (int j = 0; j < 8; j++) take(j);
  if (8 < rows) {
#pragma unroll
    for (int j = 8; j < 16; j++) take(j);
  }
}
// f(key, slot) for a thread's `own` consecutive slots of the `len` whose keys are in LDS, the first of them slot c0.  An odd number of them: no
// two lanes' reads meet in a bank.
template <typename F> __device__ __forceinline__ void each_own(const uint32_t* keys, int c0, int own, int len, F&& f) {
  int i = threadIdx.x * own;
  const int end = min(i + own, len);
  for (; i + 4 <= end; i += 4) {
    const uint32_t k0 = keys[i], k1 = keys[i + 1], k2 = keys[i + 2], k3 = keys[i + 3];
    f(k0, c0 + i); f(k1, c0 + i + 1); f(k2, c0 + i + 2); f(k3, c0 + i + 3);
  }
  for (; i < end; i++) f(keys[i], c0 + i);
}
// Of the slots [c0, c0 + len) whose keys are in LDS, those that are freed before `left` and those that move from behind it, behind the
// `holes` and `movers` of the slots before them, into the lists.  Keys above `last` stay, and of those equal to it as many as
// `spare` says, in slot order; ties: whether some of them go.  Returns the counts.
template <int THREADS>
__device__ __forceinline__ int2 list_moves(uint32_t* keys, int c0, int len, int left, uint32_t last, bool ties, int spare, int holes, int movers,
                                           int32_t* moves, int cap, int2* xch) {
  const int own = ((len + THREADS - 1) / THREADS) | 1, i0 = threadIdx.x * own;
  int stays = 0x7fffffff;                                    // equal keys that stay, from the thread's first on
  if (ties) {
    int mine = 0;
    each_own(keys, c0, own, len, [&](uint32_t k, int) { mine += k == last; });
    stays = spare - threads_before<THREADS>(mine, 0, xch).x;
  }
  uint64_t stay = 0;                                         // of the thread's 17 slots at most
  int freed = 0, moved = 0, same = 0;
  each_own(keys, c0, own, len, [&](uint32_t k, int i) {
    const bool kept = k > last || (k == last && same++ < stays);
    stay |= (uint64_t)kept << (i - c0 - i0);
    freed += !kept && i < left;
    moved += kept && i >= left;
  });
  const int4 s = threads_before<THREADS>(freed, moved, xch);   // (every thread has read its keys by then)
  // the lists take the keys' place, each slot once at most, before they are written out in whole lines
  const int end = min(i0 + own, len);
  int at = s.x, am = s.z + s.y;
  for (int i = i0; i < end; i++) {
    const bool kept = (stay >> (i - i0)) & 1;
    if (!kept && c0 + i < left) keys[at++] = (uint32_t)(c0 + i);
    if (kept && c0 + i >= left) keys[am++] = (uint32_t)(c0 + i);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < s.z; i += THREADS) moves[holes + i] = (int)keys[i];
  for (int i = threadIdx.x; i < s.w; i += THREADS) moves[cap - 1 - movers - i] = (int)keys[s.z + i];
  return make_int2(s.z, s.w);
}

// Caches of up to 8192 slots: a workgroup per pair, keys in LDS.  The budget-th largest: the keys are counted by their 11 leading bits;
// those that share the ones of the key looked for are picked out and ranked against each other (more than 256 of them: counted by the next 11
// bits, and the last 10; more than 2048 are not picked out).
// What bounds it: the chain of loads (lengths, pages, weights), then LDS and some fifteen barriers one after the other: 32 caches of 4352
// tokens x 8 15 us (256 threads instead of 1024: 20).
__global__ __launch_bounds__(kSelThreads) void paged_select_kernel(EvictArgs e) {
  const PagedArgs& a = e.a;
  extern __shared__ uint32_t keys[];
  __shared__ int hist[kBins];
  __shared__ int2 xch[kSelThreads / 64], rank[kRanked];
  __shared__ uint32_t cand[kCands];
  __shared__ int chosen[3], n_cand;
  const int pair = blockIdx.x, h = pair % a.h_kv, b = pair / a.h_kv;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = paged_len(a, b), left = min(n, e.budget);
  for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
  if (tid < kRanked) rank[tid] = make_int2(0, 0);
  if (tid == 0) n_cand = 0;
  int32_t* src = e.src ? e.src + (int64_t)pair * e.src_len : nullptr;
  if (src)
    for (uint32_t i = tid; i < e.src_len; i += kSelThreads) src[i] = i < (uint32_t)left ? (int)i : -1;   // the moves change theirs
  if (n <= e.budget) {
    if (tid == 0) e.counts[pair] = 0;
    return;
  }
  const int first_recent = a.seen[b] - e.recent;
  __syncthreads();                                           // the counts are zero
  const int rows = (n + kSelThreads - 1) / kSelThreads, base = wave * rows * 64;   // rows of 64 slots, at most eight
  evict_keys16(e, b, h, first_recent, base, rows, n, [&](uint32_t k, int i) {
    keys[i] = k;
    atomicAdd(&hist[k >> 21], 1);
  });
  __syncthreads();
  find_bin_of<kSelThreads>(hist, e.budget, xch, chosen);
  uint32_t last = (uint32_t)chosen[0] << 21;                 // the smallest key that stays, from its leading bits on
  int want = chosen[1], ties = chosen[2];                    // of the keys that share them, those that stay, and all
  const int picked = ties <= kCands ? ties : 0, own = rows | 1;
  if (picked) {
    const uint32_t bin = last >> 21;
    int mine = 0;
    each_own(keys, 0, own, n, [&](uint32_t k, int) { mine += k >> 21 == bin; });
    if (mine) {
      int at = atomicAdd(&n_cand, mine);
      each_own(keys, 0, own, n, [&](uint32_t k, int) { if (k >> 21 == bin) cand[at++] = k; });
    }
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
        each_own(keys, 0, own, n, [&](uint32_t k, int) { count(k); });
      }
      __syncthreads();
      find_bin_of<kSelThreads>(hist, want, xch, chosen);
      last |= (uint32_t)chosen[0] << shift;
      want = chosen[1];
      ties = chosen[2];
    }
  }
  // Of the keys equal to the last one kept, the first `want` stay.
  const int2 s = list_moves<kSelThreads>(keys, 0, n, left, last, want < ties, want, 0, 0, e.moves + (int64_t)pair * a.cap, a.cap, xch);
  if (tid == 0) e.counts[pair] = s.x;
}

// Longer caches: a workgroup per chunk of 4096 slots, cut so that a chunk lies before the budget or behind it, in three launches.
//   1  the keys into the scratch, and the chunk's counts by their 11 leading bits
//   2  the bits of the key looked for from all chunks' counts; the slots whose keys share them into one list
//   3  that key from the list (by the next 11 bits, then the last 10), every workgroup by itself, and from the list and the chunks' counts
//      how many slots before the chunk are freed or move: then its own part of the lists
// (One workgroup per pair for these as well, the whole call: two caches of 20 and 32k tokens x 8 cut to 4096 52.5 us, one of 128k to
// 16384 214; in three launches 46 and 82.)
struct EvictChunk { int b, h, n, base, begin, len, chunks, c; };   // chunks: of the pair; len 0: none; base: begin, or the multiple of 16 before it
__device__ __forceinline__ EvictChunk evict_chunk(const EvictArgs& e) {
  const PagedArgs& a = e.a;
  EvictChunk k;
  const int pair = blockIdx.x / e.chunks;
  k.c = blockIdx.x % e.chunks;
  k.h = pair % a.h_kv;
  k.b = pair / a.h_kv;
  k.n = paged_len(a, k.b);
  const int front = (min(k.n, e.budget) + kChunk - 1) / kChunk;
  const int from = e.budget & ~15;                           // where the chunks behind the budget are counted from
  k.chunks = k.n <= e.budget ? 0 : front + (k.n - from + kChunk - 1) / kChunk;
  k.base = k.c < front ? k.c * kChunk : from + (k.c - front) * kChunk;
  k.begin = k.c < front ? k.base : max(k.base, e.budget);
  k.len = k.c >= k.chunks ? 0 : min(k.base + kChunk, k.c < front ? e.budget : k.n) - k.begin;
  return k;
}

__global__ __launch_bounds__(kChunkThreads) void paged_long_keys_kernel(EvictArgs e) {
  const PagedArgs& a = e.a;
  __shared__ int hist[kBins];
  const EvictChunk k = evict_chunk(e);
  const int pair = blockIdx.x / e.chunks, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (k.c == 0) {
    if (tid == 0) {
      e.heads[4 * pair + 3] = 0;
      if (k.chunks == 0) e.counts[pair] = 0;
    }
    if (e.src)
      for (uint32_t i = tid; i < e.src_len; i += kChunkThreads) e.src[(int64_t)pair * e.src_len + i] = i < (uint32_t)k.n ? (int)i : -1;   // the moves change theirs
  }
  if (k.len == 0) return;
  for (int i = tid; i < kBins; i += kChunkThreads) hist[i] = 0;
  __syncthreads();
  uint32_t* keys = e.keys + (int64_t)pair * a.cap;
  evict_keys16(e, k.b, k.h, a.seen[k.b] - e.recent, k.base + wave * (kChunk / 4), 16, k.begin + k.len, [&](uint32_t x, int i) {
    if (i < k.begin) return;
    keys[i] = x;
    atomicAdd(&hist[x >> 21], 1);
  });
  __syncthreads();
  int32_t* out = e.hists + ((int64_t)pair * e.chunks + k.c) * kBins;
  for (int i = tid; i < kBins; i += kChunkThreads) out[i] = hist[i];
}

// the counts of all chunks of a pair, a thread's bins from the largest, and of chunk `c` alone
__device__ __forceinline__ void sum_hists(const int32_t* hists, int chunks, int c, int (&all)[kBins / kChunkThreads], int (&own)[kBins / kChunkThreads]) {
  constexpr int OWN = kBins / kChunkThreads;
  const int4* p = reinterpret_cast<const int4*>(hists + kBins - OWN * ((int)threadIdx.x + 1));
#pragma unroll
  for (int q = 0; q < OWN; q++) all[q] = own[q] = 0;
#pragma unroll 4
  for (int i = 0; i < chunks; i++) {
    const int4 x = p[(int64_t)i * (kBins / 4)], y = p[(int64_t)i * (kBins / 4) + 1];
    const int v[OWN] = {y.w, y.z, y.y, y.x, x.w, x.z, x.y, x.x};
#pragma unroll
    for (int q = 0; q < OWN; q++) {
      all[q] += v[q];
      own[q] = i == c ? v[q] : own[q];
    }
  }
}

__global__ __launch_bounds__(kChunkThreads) void paged_long_pick_kernel(EvictArgs e) {
  const PagedArgs& a = e.a;
  constexpr int OWN = kBins / kChunkThreads;
  __shared__ int2 xch[kChunkThreads / 64];
  __shared__ int chosen[3], place;
  const EvictChunk k = evict_chunk(e);
  if (k.len == 0) return;
  const int pair = blockIdx.x / e.chunks, tid = threadIdx.x;
  const uint32_t* far = e.keys + (int64_t)pair * a.cap + k.begin;
  uint32_t key[kChunk / kChunkThreads];
#pragma unroll
  for (int j = 0; j < kChunk / kChunkThreads; j++) key[j] = far[min(j * kChunkThreads + tid, k.len - 1)];
  int all[OWN], mine[OWN];
  sum_hists(e.hists + (int64_t)pair * e.chunks * kBins, k.chunks, k.c, all, mine);
  find_bin<kChunkThreads>(all, e.budget, xch, chosen);
  const int bin = chosen[0];
  int more = 0, hits = 0;
#pragma unroll
  for (int q = 0; q < OWN; q++) more += kBins - 1 - OWN * tid - q > bin ? mine[q] : 0;
#pragma unroll
  for (int j = 0; j < kChunk / kChunkThreads; j++) hits += j * kChunkThreads + tid < k.len && (int)(key[j] >> 21) == bin;
  if (k.c == 0 && tid < 3) e.heads[4 * pair + tid] = chosen[tid];
  const int4 s = threads_before<kChunkThreads>(hits, more, xch);
  if (tid == 0) {
    e.above[(int64_t)pair * e.chunks + k.c] = s.w;
    place = s.z ? atomicAdd(&e.heads[4 * pair + 3], s.z) : 0;
  }
  __syncthreads();
  int2* to = e.cand + (int64_t)pair * a.cap + place + s.x;
#pragma unroll
  for (int j = 0; j < kChunk / kChunkThreads; j++)
    if (j * kChunkThreads + tid < k.len && (int)(key[j] >> 21) == bin) *to++ = make_int2((int)key[j], k.begin + j * kChunkThreads + tid);
}

__global__ __launch_bounds__(kChunkThreads) void paged_long_list_kernel(EvictArgs e) {
  const PagedArgs& a = e.a;
  __shared__ uint32_t keys[kChunk];
  __shared__ int2 cand[kLongCands];
  __shared__ int hist[kBins];
  __shared__ int2 xch[kChunkThreads / 64];
  __shared__ int chosen[3];
  const EvictChunk k = evict_chunk(e);
  if (k.len == 0) return;
  const int pair = blockIdx.x / e.chunks, tid = threadIdx.x, front = (e.budget + kChunk - 1) / kChunk;
  const uint32_t* far = e.keys + (int64_t)pair * a.cap;
  const int2* far_cand = e.cand + (int64_t)pair * a.cap;
  uint32_t last = (uint32_t)e.heads[4 * pair] << 21;         // the smallest key that stays, from its leading bits on
  int want = e.heads[4 * pair + 1], ties = e.heads[4 * pair + 2];   // of the keys that share them, those that stay, and all
  const int n_cand = ties;
#pragma unroll
  for (int j = 0; j < kChunk / kChunkThreads; j++) {
    const int i = j * kChunkThreads + tid;
    if (i < k.len) keys[i] = far[k.begin + i];
  }
#pragma unroll 8
  for (int i = tid; i < min(n_cand, kLongCands); i += kChunkThreads) cand[i] = far_cand[i];
  // f(key, slot) of those picked out, a thread's share; the first 4096 from LDS
  auto picked = [&](auto&& f) {
    for (int i = tid; i < min(n_cand, kLongCands); i += kChunkThreads) f((uint32_t)cand[i].x, cand[i].y);
#pragma unroll 8
    for (int i = kLongCands + tid; i < n_cand; i += kChunkThreads) {
      const int2 x = far_cand[i];
      f((uint32_t)x.x, x.y);
    }
  };
#pragma unroll 1
  for (int step = 0; step < 2; step++) {
    const int shift = step ? 0 : 10, known = step ? 10 : 21, bits = step ? 1023 : 2047;
    __syncthreads();
    for (int i = tid; i < kBins; i += kChunkThreads) hist[i] = 0;
    __syncthreads();
    picked([&](uint32_t x, int) {
      if (x >> known == last >> known) atomicAdd(&hist[(x >> shift) & bits], 1);
    });
    __syncthreads();
    find_bin_of<kChunkThreads>(hist, want, xch, chosen);
    last |= (uint32_t)chosen[0] << shift;
    want = chosen[1];
    ties = chosen[2];
  }
  // Before the chunk: keys of its side (before the budget, behind it) above `last`; equal ones of its side and of the side before it.  Of all equal
  // ones the first `want` stay.
  const bool back = k.c >= front;
  const int side = back ? e.budget : 0;
  int more = 0, same = 0, same_front = 0;
  for (int i = (back ? front : 0) + tid; i < k.c; i += kChunkThreads) more += e.above[(int64_t)pair * e.chunks + i];
  picked([&](uint32_t x, int at) {
    const bool in = at >= side && at < k.begin;
    more += in && x > last;
    same += in && x == last;
    same_front += at < side && x == last;
  });
  const int4 s = threads_before<kChunkThreads>(more, same, xch);
  const int front_ties = threads_before<kChunkThreads>(same_front, 0, xch).z;
  const int kept = s.z + min(s.w, max(want - front_ties, 0));
  const int holes = back ? 0 : k.begin - kept, movers = back ? kept : 0;
  const int2 own = list_moves<kChunkThreads>(keys, k.begin, k.len, e.budget, last, want < ties, want - front_ties - s.w, holes, movers,
                                             e.moves + (int64_t)pair * a.cap, a.cap, xch);
  if (k.c == front - 1 && tid == 0) e.counts[pair] = holes + own.x;
}

// A wave moves eight tokens at a time: their places first, a lane each, then all their rows at once.  Bound by HBM: 65536 tokens of 128, 67 MB
// read and written, 15 us.
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
      if (e.src) e.src[(int64_t)pair * e.src_len + to] = from;
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
// the scratch, dealt from `ws` on; returns its bytes
static size_t evict_scratch(EvictArgs& e, const PagedArgs& a, char* ws) {
  const size_t pairs = (size_t)a.batch * a.h_kv;
  size_t at = 0;
  const auto take = [&](size_t numbers) {
    char* p = ws ? ws + at : nullptr;
    at += evict_align(numbers * 4);
    return (int32_t*)p;
  };
  e.counts = take(pairs);
  e.moves = take(pairs * a.cap);
  if (a.cap > kSelKeys) {
    e.chunks = (a.cap + kChunk - 1) / kChunk + 1;
    e.keys = (uint32_t*)take(pairs * a.cap);
    e.cand = (int2*)take(2 * pairs * a.cap);
    e.hists = take(pairs * e.chunks * kBins);
    e.above = take(pairs * e.chunks);
    e.heads = take(pairs * 4);
  }
  return at;
}
size_t paged_evict_ws(const PagedArgs& a) {
  EvictArgs e;
  return evict_scratch(e, a, nullptr);
}

hipError_t launch_paged_evict(const PagedArgs& a, int elem, int d, int32_t* lens, int budget, int sinks, int recent, int32_t* src,
                              char* ws, hipStream_t st) {
  EvictArgs e;
  e.a = a; e.budget = budget < a.cap ? budget : a.cap; e.src_len = (uint32_t)budget; e.sinks = sinks; e.recent = recent; e.lens = lens; e.src = src;
  evict_scratch(e, a, ws);
  const size_t pairs = (size_t)a.batch * a.h_kv;
  if (a.cap <= kSelKeys) {
    hipLaunchKernelGGL(paged_select_kernel, dim3((unsigned)pairs), dim3(kSelThreads), (size_t)a.cap * 4, st, e);
  } else {
    const dim3 grid((unsigned)(pairs * e.chunks)), blk(kChunkThreads);
    hipLaunchKernelGGL(paged_long_keys_kernel, grid, blk, 0, st, e);
    hipLaunchKernelGGL(paged_long_pick_kernel, grid, blk, 0, st, e);
    hipLaunchKernelGGL(paged_long_list_kernel, grid, blk, 0, st, e);
  }
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
