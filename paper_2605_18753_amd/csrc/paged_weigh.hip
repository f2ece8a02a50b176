// The weight that the new tokens' attention gives to every cached token: w_j += sum over rows t (tokens and heads of the
// group) of e^{s_tj - lse_t}.
//
// Column sums of the softmax matrix, whose rows' log-sum-exps are known: a wave holds 64 keys (fp32: 32) as matrix operands in
// registers and walks the rows that see them, 16 at a time; a lane adds up its own pairs, and the 16 lanes of a key are added at the
// end.  Each sum is one wave's (or, for rows cut into parts, one thread's over the parts), so results do not depend on timing.
// A single token: K is read once, HBM bounds it.  Many: an exponential, an FMA and an addition per pair, 24 clocks of a SIMD for 64
// pairs, against 16 (head dimension 128; 64: 8) of matrix work: two sequences of 6000 and 16000 tokens, 1999 new ones, 16 heads of 64
// on 4: 155 us the call, which the vector units alone would take 147 for at the highest clock and the matrix products 80 at a large
// one's rate.  One of 32768, 2048 new, 32 heads of 128 on 8: 518 us, 1.03 PFLOP/s of matrix work.
//
// (block of keys, row tile) pairs of all sequences are dealt evenly to a fixed number of workgroups; blocks cut between two of them
// are added up by a second launch, in a fixed order.
// A token's weight gets one addition a call, atomic without a result: nothing waits for the old value, and pages that several sequences
// share get the weight of all of them (only then in no fixed order).
#include "f32_tiles.h"
#include "lds_copy.h"
#include "paged.h"

namespace dash {

template <typename T, int D> struct WeighTile;
template <int D> struct WeighTile<uint16_t, D> {
  static constexpr int SUBS = 4;                       // 16-key tiles of a wave
  bf16x8 v[D / 32];
  __device__ __forceinline__ void load(const uint16_t* row, int kq) {
#pragma unroll
    for (int s = 0; s < D / 32; s++) v[s] = *reinterpret_cast<const bf16x8*>(row + 32 * s + 8 * kq);
  }
  __device__ __forceinline__ void read(const uint32_t (&at)[D / 32], uint32_t by) {   // LDS
#pragma unroll
    for (int s = 0; s < D / 32; s++) v[s] = lds_read_b128(at[s] + by);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int s = 0; s < D / 32; s++) v[s] = bf16x8{};
  }
  // lane (n, kq): row n of b against rows 4 kq + i of this
  __device__ __forceinline__ f32x4 dot(const WeighTile& b) const {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < D / 32; s++) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[s], b.v[s], acc, 0, 0, 0);
    return acc;
  }
};
template <int D> struct WeighTile<float, D> {
  static constexpr int SUBS = 2;
  f32x4 v[D / 16];
  __device__ __forceinline__ void load(const float* row, int kq) { load_row<D>(row, kq, v); }
  __device__ __forceinline__ void read(const uint32_t (&at)[D / 16], uint32_t by) {
#pragma unroll
    for (int s = 0; s < D / 16; s++) v[s] = __builtin_bit_cast(f32x4, lds_read_b128(at[s] + by));
  }
  __device__ __forceinline__ f32x4 dot(const WeighTile& b) const { return mma_dot<D>(v, b.v); }
};

template <typename T> constexpr int kWeighKeys = sizeof(T) == 2 ? 256 : 128;   // keys of an item

// The work of a kv-head: items (blocks of keys) times the row tiles of their sequence, one after the other, dealt in equal runs
// [w F / G, (w + 1) F / G) to G workgroups.
struct WeighSeq { int items, tiles, x0; };                 // blocks of keys, row tiles each, the first of these
constexpr int kStreamTiles = 2;                            // row tiles of a sequence for which K is streamed
// Where the kernel that streams K and the other one both run (a.whole), each has its own sequences.
enum WeighOwn { kOwnLong, kOwnShort, kOwnAll };
template <int KEYS> __device__ __forceinline__ WeighSeq weigh_seq(const PagedArgs& a, int m, int n, WeighOwn own) {
  const int Tt = 16 / a.g, x0 = (a.last > 0 ? max(m - a.last, 0) : 0) / Tt, tiles = (m + Tt - 1) / Tt - x0;
  const bool mine = own == kOwnAll || !a.whole || (tiles <= kStreamTiles) == (own == kOwnShort);
  return {m > 0 && mine ? (n + KEYS - 1) / KEYS : 0, tiles, x0};
}
__device__ __forceinline__ int64_t scan64(int64_t v) {     // inclusive, over the lanes up to one's own
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up((long long)v, o);
    if ((int)lane_id() >= o) v += u;
  }
  return v;
}
__device__ __forceinline__ int64_t lane64(int64_t v, int l) {   // lane l's, as a scalar
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)((uint64_t)v >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, l));
}
// whole: places are items, which are not cut
template <int KEYS> __device__ __forceinline__ int64_t weigh_total(const PagedArgs& a, bool whole = false, WeighOwn own = kOwnLong) {
  const int lane = lane_id();
  int64_t total = 0;
  for (int i0 = 0; i0 < a.batch; i0 += 64) {
    int64_t v = 0;
    if (i0 + lane < a.batch) {
      const WeighSeq s = weigh_seq<KEYS>(a, paged_rows(a, i0 + lane).y, paged_len(a, i0 + lane), own);
      v = whole ? s.items : (int64_t)s.items * s.tiles;
    }
    total += lane64(scan64(v), 63);
  }
  return total;
}
struct WeighItem { int b, block, x, r0, m, n; WeighSeq s; };   // x: row tiles of the item before the place
// the item at place f < weigh_total
template <int KEYS> __device__ __forceinline__ void weigh_find(const PagedArgs& a, int64_t f, WeighItem& it, bool whole = false, WeighOwn own = kOwnLong) {
  const int lane = lane_id();
  for (int i0 = 0; i0 < a.batch; i0 += 64) {
    int2 rm = make_int2(0, 0);
    int n = 0;
    WeighSeq s = {0, 0, 0};
    if (i0 + lane < a.batch) {
      rm = paged_rows(a, i0 + lane);
      n = paged_len(a, i0 + lane);
      s = weigh_seq<KEYS>(a, rm.y, n, own);
    }
    const int64_t v = whole ? s.items : (int64_t)s.items * s.tiles, incl = scan64(v);
    const uint64_t hit = __ballot(incl > f);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      it.b = i0 + l;
      it.s = {__builtin_amdgcn_readlane(s.items, l), __builtin_amdgcn_readlane(s.tiles, l), __builtin_amdgcn_readlane(s.x0, l)};
      it.r0 = __builtin_amdgcn_readlane(rm.x, l);
      it.m = __builtin_amdgcn_readlane(rm.y, l);
      it.n = __builtin_amdgcn_readlane(n, l);
      const int64_t in = f - lane64(incl - v, l);
      it.block = whole ? (int)in : __builtin_amdgcn_readfirstlane((int)(in / it.s.tiles));
      it.x = whole ? 0 : __builtin_amdgcn_readfirstlane((int)(in - (int64_t)it.block * it.s.tiles));
      return;
    }
    f -= lane64(incl, 63);
  }
}
template <typename T, int D>
__global__ __launch_bounds__(256, (D == 128 ? 3 : 4) - (sizeof(T) == 4)) void paged_weigh_kernel(PagedArgs a) {
  constexpr int SUBS = WeighTile<T, D>::SUBS;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x % a.h_kv, wg = blockIdx.x / a.h_kv;
  const bool uncut = a.whole;                                // beside the streaming kernel: no launch adds pieces up
  const int64_t total = weigh_total<kWeighKeys<T>>(a, uncut);
  const PagedBounds<int64_t> bounds(a, total);
  const int64_t f0 = bounds.at(wg), f1 = bounds.at(wg + 1);
  int64_t todo = f1 - f0;
  if (todo <= 0) return;
  const int Tt = 16 / a.g, n = lane & 15, kq = lane >> 4, pm = (1 << a.page_log) - 1;
  const int tl = n / a.g;
  // Row tiles come through LDS, four at a time and two such stages: wave w copies tile w of a stage, all four waves read it.  A row's
  // 16-byte pieces are permuted by its number, so that the 16 rows of a piece lie in different banks.
  constexpr int ROW = D * (int)sizeof(T), PIECES = ROW / 16, TILE = 16 * ROW, COPIES = TILE / 1024;
  auto swizzle = [](int row) { return ROW == 128 ? row >> 1 : row; };
  __shared__ __attribute__((aligned(1024))) char ring[2][4 * TILE];
  __shared__ float offs[2][4][16];                           // -lse in base 2 of the rows
  const uint32_t ring0 = lds_addr_of(ring);
  uint32_t q_lane[COPIES], rd[ROW / 64];
#pragma unroll
  for (int c = 0; c < COPIES; c++) {
    const int row = (64 * c + lane) / PIECES;
    q_lane[c] = (uint32_t)(row / a.g * (int)a.q_t + row % a.g * (int)a.q_h) * (uint32_t)sizeof(T) + (((lane % PIECES) ^ swizzle(row)) << 4);
  }
#pragma unroll
  for (int s = 0; s < ROW / 64; s++) rd[s] = ring0 + n * ROW + (((4 * s + kq) ^ swizzle(n)) << 4);
  WeighItem it;
  int slot = 0;                                              // the stage to fill next
  weigh_find<kWeighKeys<T>>(a, f0, it, uncut);
  while (true) {
    const int key0 = it.block * kWeighKeys<T> + wave * SUBS * 16;
    WeighTile<T, D> kf[SUBS];
    int page[SUBS];
    f32x4 acc[SUBS];
#pragma unroll
    for (int s = 0; s < SUBS; s++) {
      // keys behind the sequence's last one repeat it
      const int k16 = min(key0 + 16 * s, (it.n - 1) & ~15), key = min(k16 + n, it.n - 1);
      page[s] = paged_entry(a, it.b, k16 >> a.page_log);
      kf[s].load((const T*)a.k + (int64_t)paged_clamp(a, page[s]) * a.kp_p + r * a.kp_h + (int64_t)(key & pm) * a.kp_t, kq);
      acc[s] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // this run's row tiles of the item, those before the first that sees one of the block's, or the wave's, keys left out
    const int take = uncut ? it.s.tiles : (int)min((int64_t)(it.s.tiles - it.x), todo), back = it.n - it.m;
    const int first = a.last > 0 ? max(it.m - a.last, 0) : 0;
    int x = it.s.x0 + it.x;
    const int xe = x + take;
    int xw = key0 < it.n ? x : xe;
    if (a.causal) {                                            // a token sees keys up to back + t
      xw = max(xw, (key0 - back) / Tt);
      x = min(max(x, (it.block * kWeighKeys<T> - back) / Tt), xe);
    }
    float l = 0.f;
    auto ask = [&](int y) {                                    // the wave's tile of a stage; rows behind the last repeat it
      if (y >= xe) return;
      const int up = it.m - 1 - y * Tt;
      const u32x4 rows = make_rsrc((const T*)a.q + (int64_t)(it.r0 + y * Tt) * a.q_t + (int64_t)(r * a.g) * a.q_h, 0xffffffff);
      const uint32_t to = ring0 + (uint32_t)((slot * 4 + wave) * TILE);
      l = a.lse_in[(int64_t)(it.r0 + y * Tt + min(tl, up)) * a.h_q + r * a.g + n % a.g];
#pragma unroll
      for (int c = 0; c < COPIES; c++) {
        const int t = (64 * c + lane) / PIECES / a.g;
        const uint32_t at = __builtin_expect(up < Tt - 1, 0) ? q_lane[c] - (uint32_t)max(t - up, 0) * (uint32_t)a.q_t * (uint32_t)sizeof(T) : q_lane[c];
        copy16_to_lds(rows, to + 1024 * c, at, 0);
      }
    };
    if (x < xe) ask(x + wave);
    for (; x < xe; x += 4) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const int y = x + wave;
      if (y < xe) {
        const int t = y * Tt + tl;
        const bool weighs = t >= first && t < it.m;            // one that does not: whatever it holds
        const float off = !weighs || l == -INFINITY ? -INFINITY : -l * kLog2e;
        if (kq == 0) offs[slot][wave][n] = off;
        if (!weighs) {
#pragma unroll
          for (int s = 0; s < ROW / 64; s++)
            *reinterpret_cast<__attribute__((address_space(3))) f32x4*>(rd[s] + (uint32_t)((slot * 4 + wave) * TILE)) = f32x4{0.f, 0.f, 0.f, 0.f};
        }
      }
      __syncthreads();
      const int had = slot;
      slot ^= 1;
      if (x + 4 < xe) ask(x + 4 + wave);
      const int i1 = min(xe - x, 4);
      WeighTile<T, D> qf;
      float off = 0.f;
      auto read = [&](int i) {
        qf.read(rd, (uint32_t)((had * 4 + i) * TILE));
        off = offs[had][i][n];
      };
      int i = max(xw - x, 0);
      if (i < i1) read(i);
      for (; i < i1; i++) {
        const int y = x + i;
        const float o = off;
        f32x4 s[SUBS];
#pragma unroll
        for (int j = 0; j < SUBS; j++) s[j] = kf[j].dot(qf);
        if (i + 1 < i1) read(i + 1);
#pragma unroll
        for (int j = 0; j < SUBS; j++)
#pragma unroll
          for (int e = 0; e < 4; e++) s[j][e] = fmaf(s[j][e], a.c1, o);         // a pair's logarithm; what is not seen weighs nothing, whatever the row holds
        if (key0 + SUBS * 16 - 1 > (a.causal ? back + y * Tt : it.n - 1)) {     // the tile's first token sees keys up to there
          const int lim = (a.causal ? min(back + y * Tt + tl, it.n - 1) : it.n - 1) - key0 - 4 * kq;
#pragma unroll
          for (int j = 0; j < SUBS; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) s[j][e] = 16 * j + e > lim ? -INFINITY : s[j][e];
        }
#pragma unroll
        for (int j = 0; j < SUBS; j++)
#pragma unroll
          for (int e = 0; e < 4; e++) acc[j][e] += __builtin_amdgcn_exp2f(s[j][e]);
      }
    }
    // over the 16 rows of a key; lane (n, kq), n < 4, takes key 4 kq + n
    const bool whole = take == it.s.tiles;
    float* rec = a.part_o + (((int64_t)r * a.wgs + wg) * 2 + (it.x == 0)) * kWeighKeys<T> + wave * SUBS * 16 + 4 * kq + n;
#pragma unroll
    for (int j = 0; j < SUBS; j++) {
#pragma unroll
      for (int e = 0; e < 4; e++) acc[j][e] = row16_sum(acc[j][e]);
      const float w = n == 0 ? acc[j][0] : n == 1 ? acc[j][1] : n == 2 ? acc[j][2] : acc[j][3];
      const int key = key0 + 16 * j + 4 * kq + n;
      if (n < 4) {
        if (!whole) rec[16 * j] = w;                           // an item cut between runs
        else if (key < it.n && (uint32_t)page[j] < (uint32_t)a.n_pages) unsafeAtomicAdd(a.weights + ((((int64_t)page[j] * a.h_kv + r) << a.page_log) + (key & pm)), w);
      }
    }
    if ((todo -= uncut ? 1 : take) <= 0) return;
    it.x = 0;
    if (++it.block >= it.s.items) weigh_find<kWeighKeys<T>>(a, f1 - todo, it, uncut);
  }
}

// Items cut between runs.  The end of run wg - 1 lies inside an item whose first piece is that run's: its last record.  Of the runs
// behind it that begin inside the item, the first records follow.  A thread per key; 16 records are asked for
// together.  (One after the other: 700 tokens of 2000, 8 heads on one, 95 records, the call 44 us instead of 23.)
template <typename T>
__global__ __launch_bounds__(kWeighKeys<T>) void paged_weigh_sum_kernel(PagedArgs a) {
  constexpr int KEYS = kWeighKeys<T>, AHEAD = 16;
  const int r = blockIdx.x % a.h_kv, wg = blockIdx.x / a.h_kv + 1, lane = threadIdx.x & 63;
  const int64_t total = weigh_total<KEYS>(a);
  const PagedBounds<int64_t> bounds(a, total);
  const int64_t f = bounds.at(wg);
  if (f >= total) return;
  WeighItem it;
  weigh_find<KEYS>(a, f, it);
  const int64_t begin = f - it.x, end = begin + it.s.tiles;
  if (it.x == 0 || bounds.at(wg - 1) > begin) return;              // not cut here, or not for the first time
  int pieces = 1;                                                  // records of the item
  for (int k0 = wg; k0 < bounds.runs; k0 += 64) {
    const int more = __popcll(__ballot(k0 + lane < bounds.runs && bounds.at(k0 + lane) < end));
    pieces += more;
    if (more < 64) break;
  }
  const float* p = a.part_o + ((int64_t)r * a.wgs + wg) * 2 * KEYS + threadIdx.x;   // of run wg; the run's before it ends in the item
  auto at = [&](int i) { return i == 0 ? p - KEYS : p + (int64_t)(i - 1) * 2 * KEYS; };
  float w = 0.f;
  for (int i0 = 0; i0 < pieces; i0 += AHEAD) {
    float x[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; k++) x[k] = *at(min(i0 + k, pieces - 1));
#pragma unroll
    for (int k = 0; k < AHEAD; k++) w += i0 + k < pieces ? x[k] : 0.f;
  }
  const int key = it.block * KEYS + threadIdx.x;
  if (key >= it.n) return;
  const uint32_t page = (uint32_t)a.table[(int64_t)it.b * a.max_pages + (key >> a.page_log)];
  if (page < (uint32_t)a.n_pages) unsafeAtomicAdd(a.weights + ((((int64_t)page * a.h_kv + r) << a.page_log) + (key & ((1 << a.page_log) - 1))), w);
}

// Few rows a sequence (decode): K is streamed once, the next block's keys asked for before the present one's are used.  Whole blocks
// only, in equal runs.
constexpr int kStreamSubs = 1;                             // 16-key tiles of a wave
// TILES: row tiles of a sequence that stay in registers from block to block
template <int D, int TILES>
__global__ __launch_bounds__(256, 4) void paged_weigh_stream_kernel(PagedArgs a) {
  using T = uint16_t;
  using Tile = WeighTile<T, D>;
  constexpr int SUBS = kStreamSubs, KEYS = 64 * SUBS;
  constexpr WeighOwn OWN = TILES > 1 ? kOwnShort : kOwnAll;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x % a.h_kv, wg = blockIdx.x / a.h_kv;
  const int Tt = 16 / a.g, n = lane & 15, kq = lane >> 4, pm = (1 << a.page_log) - 1, tl = n / a.g;
  const uint32_t q_lane = (uint32_t)(tl * (int)a.q_t + n % a.g * (int)a.q_h) * 2u + kq * 16;
  const uint32_t l_lane = (uint32_t)(tl * a.h_q + n % a.g) * 4u;
  // blocks of all sequences, and the run's
  const int64_t total = weigh_total<KEYS>(a, true, OWN);
  const PagedBounds<int64_t> bounds(a, total);
  int64_t f = bounds.at(wg);
  int todo = (int)(bounds.at(wg + 1) - f);
  if (todo <= 0) return;
  WeighItem it, next;
  weigh_find<KEYS>(a, f, it, true, OWN);
  auto advance = [&](WeighItem& x) {
    f++;
    if (++x.block >= x.s.items) weigh_find<KEYS>(a, f, x, true, OWN);
  };
  auto load_keys = [&](const WeighItem& x, Tile (&kf)[SUBS], int (&page)[SUBS]) {
    const int key0 = x.block * KEYS + wave * SUBS * 16;
#pragma unroll
    for (int s = 0; s < SUBS; s++) page[s] = paged_entry(a, x.b, min(key0 + 16 * s, (x.n - 1) & ~15) >> a.page_log);
#pragma unroll
    for (int s = 0; s < SUBS; s++) {
      const int key = min(min(key0 + 16 * s, (x.n - 1) & ~15) + n, x.n - 1);
      kf[s].load((const T*)a.k + (int64_t)paged_clamp(a, page[s]) * a.kp_p + r * a.kp_h + (int64_t)(key & pm) * a.kp_t, kq);
    }
  };
  Tile rows[TILES];
  float offs[TILES];
  int q_of = -1;                                             // the sequence whose row tiles these hold
  auto load_rows = [&](const WeighItem& x, int y, Tile& qf, float& off) {
    const int t = y * Tt + tl, up = max(t - (x.m - 1), 0);   // a lane behind the last row repeats it
    const int first = a.last > 0 ? max(x.m - a.last, 0) : 0;
    const char* q_at = (const char*)((const T*)a.q + (int64_t)(x.r0 + y * Tt) * a.q_t + (int64_t)(r * a.g) * a.q_h);
    const char* l_at = (const char*)(a.lse_in + (int64_t)(x.r0 + y * Tt) * a.h_q + r * a.g);
    qf.load((const T*)(q_at + (q_lane - (uint32_t)up * (uint32_t)a.q_t * 2u)), 0);
    const float l = *(const float*)(l_at + (l_lane - (uint32_t)(up * a.h_q) * 4u));
    off = l == -INFINITY ? -INFINITY : -l * kLog2e;
    if (t < first || t >= x.m) {                             // does not weigh, whatever it holds
      qf.clear();
      off = -INFINITY;
    }
  };
  auto work = [&](const WeighItem& x, const Tile (&kf)[SUBS], const int (&page)[SUBS]) {
    const int key0 = x.block * KEYS + wave * SUBS * 16, back = x.n - x.m;
    f32x4 acc[SUBS];
#pragma unroll
    for (int j = 0; j < SUBS; j++) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int y0 = x.s.x0; y0 < x.s.x0 + x.s.tiles; y0 += TILES) {
      const int left = x.s.x0 + x.s.tiles - y0;
      if (q_of != x.b) {
#pragma unroll
        for (int u = 0; u < TILES; u++)
          if (u < left) load_rows(x, y0 + u, rows[u], offs[u]);
      }
      q_of = x.s.tiles <= TILES ? x.b : -1;
#pragma unroll
      for (int u = 0; u < TILES; u++) {
        if (u >= left) break;
        const int y = y0 + u;
        f32x4 s[SUBS];
#pragma unroll
        for (int j = 0; j < SUBS; j++) s[j] = kf[j].dot(rows[u]);
#pragma unroll
        for (int j = 0; j < SUBS; j++)
#pragma unroll
          for (int e = 0; e < 4; e++) s[j][e] = fmaf(s[j][e], a.c1, offs[u]);
        if (key0 + SUBS * 16 - 1 > (a.causal ? back + y * Tt : x.n - 1)) {
          const int lim = (a.causal ? min(back + y * Tt + tl, x.n - 1) : x.n - 1) - key0 - 4 * kq;
#pragma unroll
          for (int j = 0; j < SUBS; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) s[j][e] = 16 * j + e > lim ? -INFINITY : s[j][e];
        }
#pragma unroll
        for (int j = 0; j < SUBS; j++)
#pragma unroll
          for (int e = 0; e < 4; e++) acc[j][e] += __builtin_amdgcn_exp2f(s[j][e]);
      }
    }
#pragma unroll
    for (int j = 0; j < SUBS; j++) {
#pragma unroll
      for (int e = 0; e < 4; e++) acc[j][e] = row16_sum(acc[j][e]);
      const float w = n == 0 ? acc[j][0] : n == 1 ? acc[j][1] : n == 2 ? acc[j][2] : acc[j][3];
      const int key = key0 + 16 * j + 4 * kq + n;
      if (n < 4 && key < x.n && (uint32_t)page[j] < (uint32_t)a.n_pages) unsafeAtomicAdd(a.weights + ((((int64_t)page[j] * a.h_kv + r) << a.page_log) + (key & pm)), w);
    }
  };
  Tile ka[SUBS], kb[SUBS];
  int pa[SUBS], pb[SUBS];
  load_keys(it, ka, pa);
  while (true) {
    next = it;
    if (todo > 1) {
      advance(next);
      load_keys(next, kb, pb);
    }
    work(it, ka, pa);
    if (--todo == 0) return;
    it = next;
    if (todo > 1) {
      advance(next);
      load_keys(next, ka, pa);
    }
    work(it, kb, pb);
    if (--todo == 0) return;
    it = next;
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------
// resident workgroups of a kv-head, by the registers of a wave: three per CU at head dimension 128, four at 64; fp32 two and three
static int weigh_wgs(const PagedArgs& a, int dtype, int d) { return max(256 * ((d == 128 ? 3 : 4) - (dtype != DASH_BF16)) / a.h_kv, 1); }

// K is streamed for sequences of up to 32 rows.  Which have more is known on the device only: calls that may have some, and bring no more than that on
// the average, launch both kernels; a call of no more tokens than sequences launches the streaming one alone, which takes whatever there is.  (32 / 8
// heads of 128.  16 sequences of 2048 to 16384 tokens, 20 rows each: 76 us with both, not streamed 86, only streamed 73.  64 sequences of 2000 to 8000,
// one with 400 new tokens, the others with one: 188, not streamed 228, only streamed 1969.  Three tokens of 8 sequences of 1000, where the second launch
// finds nothing: 17, only streamed 13.  Nobody but one of the sequences with new tokens, and fewer of them than sequences, is what the rule does not see:
// 64 of one of 64 sequences, 8000 long, 37, not streamed 22; 400 of one of 512, 195 and 56.)
enum class Weigh { kStream, kBoth, kNone };
static Weigh weigh_how(const PagedArgs& a) {
  const int64_t rows = (int64_t)a.n_rows * a.g;
  if (a.n_rows <= a.batch || rows <= 16 * kStreamTiles) return Weigh::kStream;
  return rows <= (int64_t)a.batch * 16 * kStreamTiles ? Weigh::kBoth : Weigh::kNone;
}

size_t paged_weigh_ws(const PagedArgs& a, int dtype, int d) {
  return (size_t)weigh_wgs(a, dtype, d) * a.h_kv * 2 * (dtype == DASH_BF16 ? kWeighKeys<uint16_t> : kWeighKeys<float>) * 4;
}

template <typename T, int D>
static hipError_t launch_weigh_t(PagedArgs a, char* ws, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    const Weigh how = weigh_how(a);
    if (how != Weigh::kNone) {
      a.whole = how == Weigh::kBoth;
      a.wgs = max(1024 / a.h_kv, 1);
      const dim3 grid((unsigned)(a.wgs * a.h_kv)), blk(256);
      if (a.n_rows <= a.batch) hipLaunchKernelGGL((paged_weigh_stream_kernel<D, 1>), grid, blk, 0, st, a);
      else hipLaunchKernelGGL((paged_weigh_stream_kernel<D, kStreamTiles>), grid, blk, 0, st, a);
      if (hipError_t e = hipGetLastError(); e != hipSuccess || how == Weigh::kStream) return e;
    }
  }
  a.part_o = (float*)ws;
  a.wgs = weigh_wgs(a, sizeof(T) == 2 ? DASH_BF16 : DASH_F32, D);
  hipLaunchKernelGGL((paged_weigh_kernel<T, D>), dim3((unsigned)(a.wgs * a.h_kv)), dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  // nothing is cut beside the streaming kernel, nor a single tile of rows
  if (e != hipSuccess || a.whole || a.n_rows * (int64_t)a.g <= 16 || a.wgs == 1) return e;
  hipLaunchKernelGGL(paged_weigh_sum_kernel<T>, dim3((unsigned)((a.wgs - 1) * a.h_kv)), dim3(kWeighKeys<T>), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_paged_weigh(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st) {
  if (dtype == DASH_BF16) return d == 128 ? launch_weigh_t<uint16_t, 128>(a, ws, st) : launch_weigh_t<uint16_t, 64>(a, ws, st);
  return d == 128 ? launch_weigh_t<float, 128>(a, ws, st) : launch_weigh_t<float, 64>(a, ws, st);
}

}  // namespace dash
