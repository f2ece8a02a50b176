// Attention of packed new tokens over a paged cache (one pass over the keys with the running maximum and sum of the softmax).
//
// s_tj = q_t . k_j scale over the visible tokens j of the row's sequence, o_t = sum_j softmax_j(s_t) v_j, lse_t = ln sum_j e^{s_tj}.
//
// Few rows (decode, drafted tokens): a tile is 16 (token, head) rows, the heads of a kv-head's group for 16 / g tokens.  The
// cache is read once for 4 g flops a byte, so HBM bounds it; a workgroup's four waves take 32-key tiles in turn, each through a ring of
// its own in LDS (two tiles deep, global -> LDS copies), without a barrier until the four add up at the end.  A token of each of 32 sequences of
// 4096 to 32768, 32 / 8 heads of 128: 415 us, 5.9 TB/s; one sequence of 1000: 8.6 us, a chain of round trips.
#include "paged_few.h"

namespace dash {

template <int D> struct FewCfg {
  static constexpr int NCH = D / 8, ROW_BYTES = D * 2;
  static constexpr int TILE_BYTES = 32 * ROW_BYTES;      // K or V of 32 keys
  static constexpr int COPIES = TILE_BYTES / 1024;       // copy instructions of a wave per tile and tensor
  static constexpr int RPC = 64 / NCH;                   // rows an instruction covers
  static constexpr int WAVE_BYTES = 4 * TILE_BYTES;      // two stages of K and V
  static constexpr int LDS_BYTES = 4 * WAVE_BYTES;
};

template <int D>
__global__ __launch_bounds__(256, 2) void paged_few_kernel(PagedArgs args) {
  using C = FewCfg<D>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int r = blockIdx.x % args.h_kv, wg = blockIdx.x / args.h_kv;
  PagedRun<false> run(args);
  if (!run.begin(args, wg)) return;
  const PagedItem& it = run.it;
  do {
  const PagedArgs a = paged_reload();
  const int tid = paged_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = 16 / a.g;
  const int t0 = it.tile * T;
  const int n = lane & 15, kq = lane >> 4;
  const int t = t0 + n / a.g;
  const bool row_ok = t < it.m;
  bf16x8 qf[D / 32];
  {
    const uint16_t* qp = (const uint16_t*)a.q + (it.r0 + min(t, it.m - 1)) * a.q_t + (r * a.g + n % a.g) * a.q_h + kq * 8;
#pragma unroll
    for (int s = 0; s < D / 32; s++) qf[s] = *reinterpret_cast<const bf16x8*>(qp + 32 * s);
  }
  const int last = row_ok ? paged_last_key(a, it, t) : -1;
  const int first_last = paged_last_key(a, it, t0);                              // of the tile's first token
  const int end = max(paged_last_key(a, it, min(t0 + T, it.m) - 1) + 1, 0);      // keys that a row of the tile sees
  // the wave's 32-key tiles of the piece's 128-key steps
  const int j1 = min(run.x1 * 4, (end + 31) >> 5);
  int j = run.x0 * 4 + wave;

  const uint32_t ring = lds_addr_of(lds) + wave * C::WAVE_BYTES;
  const int c_row = lane / C::NCH, c_pos = lane % C::NCH;
  // Rows of copy c: RPC c + c_row.  The part of K's permutation that depends on c is a flip of chunk bits 2 (and 3).
  const uint32_t kt2 = (uint32_t)a.kp_t * 2u, vt2 = (uint32_t)a.vp_t * 2u;
  constexpr int KV = D == 128 ? 4 : 2;
  uint32_t k_off[KV];
#pragma unroll
  for (int c = 0; c < KV; c++) k_off[c] = (uint32_t)c_row * kt2 + (uint32_t)((c_pos ^ pk_swz<D>(C::RPC * c + c_row)) << 4);
  const uint32_t v_off = (uint32_t)c_row * vt2 + (uint32_t)((c_pos ^ pv_swz<D>(c_row)) << 4);
  const char* kb = (const char*)a.k + r * a.kp_h * 2;
  const char* vb = (const char*)a.v + r * a.vp_h * 2;
  const int pm = (1 << a.page_log) - 1;
  // the pages of a tile: one, or two of 16 tokens
  auto pages_of = [&](int tile) {
    return make_int2(paged_page(a, it.b, (tile * 32) >> a.page_log), paged_page(a, it.b, (tile * 32 + 16) >> a.page_log));
  };
  // Tile -> LDS stage.  A resource ends with the sequence's last token: rows behind it read as zeros, whatever their page holds.
  auto copy = [&](int tile, int2 pg, int stage) {
    const uint32_t to = ring + stage * 2 * C::TILE_BYTES;
#pragma unroll
    for (int half = 0; half < 2; half++) {
      const int key = tile * 32 + half * 16, id = half ? pg.y : pg.x, rows = min(max(it.n - key, 0), 16);
      const char* kp = kb + ((int64_t)id * a.kp_p + (int64_t)(key & pm) * a.kp_t) * 2;
      const char* vp = vb + ((int64_t)id * a.vp_p + (int64_t)(key & pm) * a.vp_t) * 2;
      const u32x4 k_rs = make_rsrc(kp, rows ? (rows - 1) * (int64_t)kt2 + C::ROW_BYTES : 0);
      const u32x4 v_rs = make_rsrc(vp, rows ? (rows - 1) * (int64_t)vt2 + C::ROW_BYTES : 0);
#pragma unroll
      for (int i = 0; i < C::COPIES / 2; i++) {
        const int c = half * (C::COPIES / 2) + i;
        copy16_to_lds(k_rs, to + c * 1024, k_off[c % KV] + (uint32_t)(i * C::RPC) * kt2, 0);
      }
#pragma unroll
      for (int i = 0; i < C::COPIES / 2; i++) {
        const int c = half * (C::COPIES / 2) + i;
        copy16_to_lds(v_rs, to + C::TILE_BYTES + c * 1024, v_off + (uint32_t)(i * C::RPC) * vt2, 0);
      }
    }
  };
  uint32_t k_rd[D / 32];
#pragma unroll
  for (int s = 0; s < D / 32; s++) k_rd[s] = ring + (uint32_t)(n * C::ROW_BYTES + (((4 * s + kq) ^ pk_swz<D>(n)) << 4));
  // transposing read of V: lane s of a group of 16 points at row 4 kq + s / 4 (+ 16), d 4 (s % 4) of the 16-wide d-tile
  uint32_t v_rd[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; dt++)
    v_rd[dt] = ring + (uint32_t)(C::TILE_BYTES + (4 * kq + (n >> 2)) * C::ROW_BYTES +
                                 (((2 * dt + ((n & 3) >> 1)) ^ pv_swz<D>(n >> 2)) << 4) + ((n & 1) << 3));

  float m_run = -INFINITY, l_run = 0.f;
  f32x4 oacc[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; dt++) oacc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < D / 32; s++) asm volatile("" : "+v"(qf[s]));               // loaded before the copies are in flight

  int2 pg = make_int2(0, 0);
  if (j < j1) {
    copy(j, pages_of(j), 0);
    pg = pages_of(j + 4);
  }
  for (int stage = 0; j < j1; j += 4, stage ^= 1) {
    if (j + 4 < j1) {
      copy(j + 4, pg, stage ^ 1);
      pg = pages_of(j + 8);
      if constexpr (C::COPIES == 8) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
      else asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    const uint32_t at = stage * 2 * C::TILE_BYTES;
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;                                    // lane (row n, kq): keys 4 kq + i, 16 + 4 kq + i
#pragma unroll
    for (int s = 0; s < D / 32; s++) {
      s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lds_read_b128(k_rd[s] + at), qf[s], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lds_read_b128(k_rd[s] + at + 16 * C::ROW_BYTES), qf[s], s1, 0, 0, 0);
    }
    if (j * 32 + 31 > first_last || t0 + T > it.m) {
      const int lim = last - (j * 32 + 4 * kq);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        s0[i] = i > lim ? -INFINITY : s0[i];
        s1[i] = 16 + i > lim ? -INFINITY : s1[i];
      }
    }
    float mx = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
    mx = quad_rows_max(mx) * a.c1;
    if (__any(mx > m_run + kPagedLazy)) {
      const float m_new = fmaxf(m_run, mx), use = m_new == -INFINITY ? 0.f : m_new;
      const float corr = __builtin_amdgcn_exp2f(m_run - use);
      m_run = m_new;
      l_run *= corr;
#pragma unroll
      for (int dt = 0; dt < D / 16; dt++) oacc[dt] *= corr;
    }
    const float off = m_run == -INFINITY ? 0.f : -m_run;
    float p[8];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(s0[i], a.c1, off));
      p[4 + i] = __builtin_amdgcn_exp2f(fmaf(s1[i], a.c1, off));
    }
    l_run += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    // P in bf16, the operand type of the matrix cores (relative error 2^-9); the row sum takes the unrounded values
    const u32x4 pw = {cvt_bf16x2(p[0], p[1]), cvt_bf16x2(p[2], p[3]), cvt_bf16x2(p[4], p[5]), cvt_bf16x2(p[6], p[7])};
    const bf16x8 pb = __builtin_bit_cast(bf16x8, pw);
#pragma unroll
    for (int dt = 0; dt < D / 16; dt++)
      oacc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lds_read_tr_pair(v_rd[dt] + at, v_rd[dt] + at + 16 * C::ROW_BYTES), pb, oacc[dt], 0, 0, 0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                           // the stage is read before it is copied over
  }
  const float l_tot = quad_rows_sum(l_run);
  __syncthreads();
  float* x = reinterpret_cast<float*>(lds);                                      // [4][16][D + 4]
  float* ml = x + 4 * 16 * (D + 4);
  float* own = x + (wave * 16 + n) * (D + 4) + 4 * kq;
#pragma unroll
  for (int dt = 0; dt < D / 16; dt++) *reinterpret_cast<f32x4*>(own + 16 * dt) = oacc[dt];
  if (kq == 0) {
    ml[(wave * 16 + n) * 2] = m_run;
    ml[(wave * 16 + n) * 2 + 1] = l_tot;
  }
  __syncthreads();
  paged_few_finish<uint16_t, D, 4>(a, run, r, ((int64_t)r * a.wgs + wg) * 2 + (run.x0 == 0), t0, x, ml);
  if (!run.whole()) paged_few_join<uint16_t, D, 256>(a, run, r, wg, lds);
  __syncthreads();
  } while (run.advance(args));
}

// Many rows (pieces of prompts): a tile is 128 (token, head) rows, 32 of them a wave's: all heads of the group for 32 / g tokens.
// 64-key tiles of K and V are copied from their pages straight into LDS, two stages deep, and shared by the four waves.
// The first product is S^T[key, row] = K Q^T (A = K from LDS, B = Q in registers), the second O^T[d, row] += V^T P^T (A = V^T by
// transposing reads, B = P): in the 32x32 accumulator layout lane (n = lane % 32, h = lane / 32) holds, for row n, keys 8 q + 4 h + i,
// which are its slots of operand B once the contraction runs in that order, so nothing moves between the products.
// A wave pipelines its tiles: the first product of tile i runs with the exponentials of tile i - 1, the second product of
// tile i - 1 with the row maxima of tile i.  Bound by the matrix units and the card's power: 2048 tokens at the end of 32768, 32 / 8 heads of 128,
// 980 to 1080 us from card to card, 1.0 to 1.09 PFLOP/s, the matrix pipe busy for 0.58 of the clocks at 1.7 GHz.
template <int D> struct RowsCfg {
  static constexpr int NCH = D / 8, ROW_BYTES = D * 2;
  static constexpr int TILE_BYTES = 64 * ROW_BYTES;
  static constexpr int COPIES = TILE_BYTES / 4096;       // copy instructions of a wave per tile and tensor
  static constexpr int RPC = 64 / NCH;                   // rows that a copy instruction covers
  static constexpr int OUT_BYTES = 128 * (D + 4) * 4;    // a tile's rows in fp32, behind the walk
  static constexpr int LDS_BYTES = 4 * TILE_BYTES > OUT_BYTES ? 4 * TILE_BYTES : OUT_BYTES;   // K ring [2], V ring [2]
};

template <int D>
__global__ __launch_bounds__(256, 2) void paged_rows_kernel(PagedArgs a) {
  using C = RowsCfg<D>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  // kv-heads are the fast index: with 8 of them each XCD's L2 sees the pages of one
  const int r = blockIdx.x % a.h_kv;
  PagedPart it;
  if (!paged_find_part<false>(a, blockIdx.x / a.h_kv, [&](int m, int n) { return rows_shape(a, m, n); }, it)) return;
  const int T = 128 / a.g, t0 = it.tile * T, Tw = 32 / a.g, tw0 = t0 + wave * Tw;
  const int t = tw0 + n / a.g, head = r * a.g + n % a.g;
  const bool row_ok = t < it.m;
  bf16x8 qf[D / 16];
  {
    const uint16_t* qp = (const uint16_t*)a.q + (it.r0 + min(t, it.m - 1)) * a.q_t + head * a.q_h + h * 8;
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
  }
  const int last = paged_last_key(a, it, min(t, it.m - 1));
  // keys that the tile, and the wave, sees; up to where the wave's first token does
  const int end = max(paged_last_key(a, it, min(t0 + T, it.m) - 1) + 1, 0);
  const int wave_end = tw0 < it.m ? paged_last_key(a, it, min(tw0 + Tw, it.m) - 1) + 1 : 0;
  const int low = paged_last_key(a, it, min(tw0, it.m - 1));
  const int kt = (end + 63) >> 6, per = (kt + it.parts - 1) / it.parts;
  const int first = min(it.part * per, kt), n_it = min(per, kt - first);       // the part's tiles

  // ---- pages: 64 entries of the table a lane each, the next 64 behind them ----------------------------------
  const int32_t* table = a.table + (int64_t)it.b * a.max_pages;
  auto window = [&](int i) { return paged_clamp(a, table[min(i + lane, a.max_pages - 1)]); };
  int wbase = (first * 64) >> a.page_log;
  int win = window(wbase), win_next = window(wbase + 64);

  // ---- global -> LDS copies -----------------------------------------------------------------------------------
  const uint32_t kt2 = (uint32_t)a.kp_t * 2u, vt2 = (uint32_t)a.vp_t * 2u;
  const char* kb = (const char*)a.k + r * a.kp_h * 2;
  const char* vb = (const char*)a.v + r * a.vp_h * 2;
  const int64_t kp2 = a.kp_p * 2, vp2 = a.vp_p * 2;
  const int pm = (1 << a.page_log) - 1;
  const uint32_t lds0 = lds_addr_of(lds);
  // A wave copies 16 rows of a tile, which lie in one page: one resource, which ends with the sequence's last token (rows behind it
  // read as zeros, whatever the page holds).  Copy c: rows RPC c + c_row of them.  The part of K's permutation that depends on c is a
  // flip of chunk bits 2 (and 3).
  const int c_row = lane / C::NCH, c_pos = lane % C::NCH, row0 = wave * 16;
  uint32_t k_off[C::COPIES];
#pragma unroll
  for (int c = 0; c < C::COPIES; c++) k_off[c] = (uint32_t)c_row * kt2 + (uint32_t)((c_pos ^ pk_swz<D>(C::RPC * c + c_row)) << 4);
  const uint32_t v_off = (uint32_t)c_row * vt2 + (uint32_t)((c_pos ^ pv_swz<D>(c_row)) << 4);
  auto rows_from = [&](const char* base, int64_t page_bytes, uint32_t row_bytes, int id, int key, int stop) {
    const int left = min(max(stop - key, 0), 16);
    const int64_t bytes = (int64_t)left * row_bytes - (int64_t)(row_bytes - C::ROW_BYTES);
    return make_rsrc(base + (int64_t)id * page_bytes + (uint32_t)(key & pm) * row_bytes, bytes < 0 ? 0 : bytes);
  };
  int id_v = 0, id_k = 0;                                     // pages of tile i (its V is copied) and of tile i + 1 (its K)
  u32x4 k_rs = {}, v_rs = {};
  auto id_of = [&](int tile) { return __builtin_amdgcn_readlane(win, (((tile * 64 + row0) >> a.page_log) - wbase) & 63); };
  const int part_end = first + n_it;
  auto aim_k = [&](int tile) {                                // behind the part's last tile: nothing is read
    k_rs = rows_from(kb, kp2, kt2, id_k, tile * 64 + row0, tile < part_end ? it.n : 0);
  };
  auto copy_k = [&](int c, int slot) {
    copy16_to_lds(k_rs, lds0 + slot * C::TILE_BYTES + wave * (C::TILE_BYTES / 4) + c * 1024, k_off[c], (uint32_t)(c * C::RPC) * kt2);
  };
  auto copy_v = [&](int c, int slot) {
    copy16_to_lds(v_rs, lds0 + (2 + slot) * C::TILE_BYTES + wave * (C::TILE_BYTES / 4) + c * 1024, v_off, (uint32_t)(c * C::RPC) * vt2);
  };
  // ---- operand addresses in LDS, of slot 0 --------------------------------------------------------------------
  uint32_t k_rd[D / 16], v_rd[D / 32];
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) k_rd[ks] = lds0 + (uint32_t)(n * C::ROW_BYTES + (((2 * ks + h) ^ pk_swz<D>(n)) << 4));
  const int s16 = lane & 15, a16 = (lane >> 4) & 1;
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
    v_rd[dt] = lds0 + (uint32_t)((4 * h + (s16 >> 2)) * C::ROW_BYTES +
                                 ((((4 * dt) ^ pv_swz<D>(s16 >> 2)) + 2 * a16 + ((s16 & 3) >> 1)) << 4) + ((s16 & 1) << 3));

  float m_run = -INFINITY, l_run = 0.f;
  constexpr int NDT = D / 32;
  f32x16 oacc[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; dt++)
#pragma unroll
    for (int j = 0; j < 16; j++) oacc[dt][j] = 0.f;
  // all loads so far are complete, and known to be, before the copies are in flight
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) asm volatile("" : "+v"(qf[ks]));
  asm volatile("" : "+v"(win), "+v"(win_next));
  id_k = id_of(first);
  aim_k(first);
  if (n_it > 0) {
#pragma unroll
    for (int c = 0; c < C::COPIES; c++) copy_k(c, 0);
  }
  // Iteration i, LDS: tile i lives in slot i & 1 of both rings, V one iteration behind K.  At its top a wave waits for its own
  // copies (K of tile i, V of tile i - 1); the barrier makes everybody's visible and retires the reads of iteration i - 1, whose slots this
  // iteration's copies (K of tile i + 1, V of tile i) overwrite, one at a time between the MFMAs.
  int pend = 0;
  float tmax_old = 0.f;
  auto iteration = [&](auto p_tag, int i, f32x16 (&s)[2], f32x16 (&so)[2]) __attribute__((always_inline)) {
    constexpr int P = decltype(p_tag)::value;
    constexpr int NS = D / 8, KAHEAD = 4, VAHEAD = 2, EQ = 12, E0 = 2;
    const bool cur = i < n_it;
    const int tile = first + i;
    const bool on = cur && tile * 64 < wave_end;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    asm volatile("" : "+v"(win_next));                         // asked for iterations ago
    id_v = id_k;
    if (((tile + 1) * 64 >> a.page_log) - wbase >= 64) {
      wbase += 64;
      win = win_next;
      win_next = window(wbase + 64);
    }
    id_k = id_of(tile + 1);
    aim_k(tile + 1);
    v_rs = rows_from(vb, vp2, vt2, id_v, tile * 64 + row0, it.n);
    if (pend && __builtin_expect(__any(tmax_old > m_run + kPagedLazy), 0)) {
      const float m_new = fmaxf(m_run, fmaxf(tmax_old, __shfl_xor(tmax_old, 32)));
      const float use = m_new == -INFINITY ? 0.f : m_new;
      const float corr = __builtin_amdgcn_exp2f(m_run - use);
      m_run = m_new;
      l_run *= corr;
#pragma unroll
      for (int dt = 0; dt < NDT; dt++)
#pragma unroll
        for (int j = 0; j < 16; j++) oacc[dt][j] *= corr;
    }
    const float off = m_run == -INFINITY ? 0.f : -m_run;
    asm volatile("s_barrier" ::: "memory");
    auto k_read = [&](int x) -> bf16x8 {   // slot x: d slice x / 2, key half x % 2
      return lds_read_b128(k_rd[x >> 1] + (uint32_t)(P * C::TILE_BYTES + (x & 1) * 32 * C::ROW_BYTES));
    };
    auto v_read = [&](int x) -> bf16x8 {   // slot x: contraction step x / NDT, d-tile x % NDT
      const uint32_t at = v_rd[x % NDT] + (uint32_t)((2 + (P ^ 1)) * C::TILE_BYTES + 16 * (x / NDT) * C::ROW_BYTES);
      return lds_read_tr_pair(at, at + 8 * C::ROW_BYTES);
    };
    u32x4 pb[4];
    float l_tile = 0.f;
    // Pair k of tile i - 1: P^T slots 2 (k % 4), + 1 of contraction step k / 4.  P in bf16, the matrix cores' operand type; the row sum takes the
    // unrounded values.
    auto e_pair = [&](int k) {
      const int g = k >> 2, x = g >> 1, j = 8 * (g & 1) + 2 * (k & 3);
      const float p0 = __builtin_amdgcn_exp2f(fmaf(so[x][j], a.c1, off));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(so[x][j + 1], a.c1, off));
      l_tile += p0 + p1;
      uint32_t w = cvt_bf16x2(p0, p1);
      asm volatile("" : "+v"(l_tile), "+v"(w));
      pb[g][k & 3] = w;
    };
    auto copies = [&](int c) {
      if (c < C::COPIES) copy_k(c, P ^ 1);
      else if (c < 2 * C::COPIES) copy_v(c - C::COPIES, P);
    };
    bf16x8 vf[NS];
    auto first_product = [&](auto e_tag) {
      constexpr bool EXPS = decltype(e_tag)::value;
      bf16x8 kf[NS];
#pragma unroll
      for (int x = 0; x < KAHEAD; x++) kf[x] = k_read(x);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (EXPS) {
#pragma unroll
        for (int k = 0; k < E0; k++) e_pair(k);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int x = 0; x < NS; x++) {
        if (x + KAHEAD < NS) kf[x + KAHEAD] = k_read(x + KAHEAD);
        if ((x & 1) == 0) copies(x >> 1);
        const f32x16 z = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        s[x & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[x], qf[x >> 1], x < 2 ? z : s[x & 1], 0, 0, 0);
        if constexpr (EXPS) {
#pragma unroll
          for (int k = E0 + x * (EQ - E0) / NS; k < E0 + (x + 1) * (EQ - E0) / NS; k++) e_pair(k);
          if (x >= NS - VAHEAD) vf[x - (NS - VAHEAD)] = v_read(x - (NS - VAHEAD));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto mask_keys = [&]() {
      if (__builtin_expect(tile * 64 + 63 > low, 0)) {
        int lim = last - (tile * 64 + 4 * h);
        asm volatile("" : "+v"(lim));
#pragma unroll
        for (int x = 0; x < 2; x++)
#pragma unroll
          for (int j = 0; j < 16; j++) s[x][j] = x * 32 + (j >> 2) * 8 + (j & 3) > lim ? -INFINITY : s[x][j];
      }
    };
    float mloc = -INFINITY;
    auto max_quad = [&](int q) {
      const int x = q >> 2, j = 4 * (q & 3);
      mloc = fmaxf(fmaxf(mloc, s[x][j]), s[x][j + 1]);
      mloc = fmaxf(fmaxf(mloc, s[x][j + 2]), s[x][j + 3]);
    };
    auto second_product = [&]() {
#pragma unroll
      for (int x = 0; x < NS; x++) {
        if (x + VAHEAD < NS) vf[x + VAHEAD] = v_read(x + VAHEAD);
        oacc[x % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[x], __builtin_bit_cast(bf16x8, pb[x / NDT]), oacc[x % NDT], 0, 0, 0);
        if (EQ + x < 16) e_pair(EQ + x);
        if constexpr (NS == 16) { if (x >= 4 && x < 12) max_quad(x - 4); }
        else if (x >= 4) { max_quad(2 * (x - 4)); max_quad(2 * (x - 4) + 1); }
        __builtin_amdgcn_sched_barrier(0);
      }
      l_run += l_tile;
    };
    if (on) {
      if (pend) first_product(std::true_type{});
      else first_product(std::false_type{});
      mask_keys();
    } else {
      asm volatile("" : "=v"(s[0]), "=v"(s[1]));               // nobody reads them
      if (cur) {
#pragma unroll
        for (int c = 0; c < 2 * C::COPIES; c++) copies(c);
      }
      if (pend) {
#pragma unroll
        for (int x = 0; x < VAHEAD; x++) vf[x] = v_read(x);
#pragma unroll
        for (int k = 0; k < EQ; k++) e_pair(k);
      }
    }
    if (pend) {
      __builtin_amdgcn_sched_barrier(0);
      second_product();
    }
    if (!pend && on) {
#pragma unroll
      for (int q = 0; q < 8; q++) max_quad(q);
    }
    tmax_old = mloc * a.c1;                                    // this lane half's; a.c1 > 0
    pend = on;
  };
  if (n_it > 0) {
    f32x16 sa[2], sb[2];
    for (int i = 0;;) {
      iteration(std::integral_constant<int, 0>{}, i, sa, sb);
      if (++i > n_it) break;
      iteration(std::integral_constant<int, 1>{}, i, sb, sa);
      if (++i > n_it) break;
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // no copy outlives the workgroup's LDS
  const float l_tot = l_run + __shfl_xor(l_run, 32);
  // The rows go through LDS, each wave's on its own, so that they are written in whole lines: as the output, or unnormalised as a
  // record of the part.
  constexpr int LD = D + 4;
  const bool cut = it.parts > 1;
  const int64_t rec = (int64_t)r * a.wgs + it.rec0 + it.part;
  const float inv = l_tot > 0.f ? 1.f / l_tot : l_tot == 0.f ? 0.f : l_tot;    // NaN stays
  __syncthreads();                                             // nobody reads the tiles any more
  float* x = reinterpret_cast<float*>(lds) + wave * 32 * LD;
#pragma unroll
  for (int dt = 0; dt < NDT; dt++)
#pragma unroll
    for (int q4 = 0; q4 < 4; q4++)
      *reinterpret_cast<f32x4*>(x + n * LD + dt * 32 + q4 * 8 + h * 4) =
          f32x4{oacc[dt][q4 * 4], oacc[dt][q4 * 4 + 1], oacc[dt][q4 * 4 + 2], oacc[dt][q4 * 4 + 3]};
  if (h == 0) {
    x[n * LD + D] = inv;
    if (row_ok) {
      if (cut) reinterpret_cast<float2*>(a.part_ml)[rec * 128 + wave * 32 + n] = make_float2(m_run, l_tot);
      else if (a.lse) a.lse[(int64_t)(it.r0 + t) * a.h_q + head] = l_tot == 0.f ? -INFINITY : (m_run + log2f(l_tot)) * kLn2;
    }
  }
  asm volatile("" ::: "memory");                               // a wave's LDS operations complete in order
  constexpr int TPR = D / 4;
  const int c = lane % TPR, rows = min(max(it.m - tw0, 0), Tw) * a.g;
  for (int i = lane / TPR; i < rows; i += 64 / TPR) {
    const f32x4 y = *reinterpret_cast<const f32x4*>(x + i * LD + c * 4);
    if (cut) *reinterpret_cast<f32x4*>(a.part_o + (rec * 128 + wave * 32 + i) * D + c * 4) = y;
    else put_row4((uint16_t*)a.o + (it.r0 + tw0 + i / a.g) * a.o_t + (r * a.g + i % a.g) * a.o_h + c * 4, y, x[i * LD + D]);
  }
}

// Adds up the parts of tiles of 128 rows: o = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p.  A workgroup adds 256 / (D / 4) / SLICES (token, head) rows at a time, SLICES groups of threads
// each taking every SLICES-th part.
template <int D, int SLICES, bool FOUR>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedArgs a) {
  constexpr int TPR = D / 4, PER = 256 / TPR / SLICES;     // threads of a row's slice, rows of a workgroup
  __shared__ f32x4 xo[SLICES > 1 ? 256 : 1];
  __shared__ float xd[SLICES > 1 ? 2 * (256 / TPR) : 1];
  const int lane = threadIdx.x & 63, c = threadIdx.x % TPR, unit = threadIdx.x / TPR, slice = unit / PER;
  const auto shape = [&](int m, int n) { return rows_shape(a, m, n); };
  const PagedLane l0 = paged_lane<FOUR>(a, lane);
  const PagedCut cut = paged_part_size<FOUR>(a, l0, shape);
  if (cut.size == kUncut) return;
  // rows in the order kv-head, token, head of the group: neighbours lie side by side in the records
  const uint32_t per = (uint32_t)a.n_rows * (uint32_t)a.g, all = per * (uint32_t)a.h_kv, g_log = 31 - __builtin_clz(a.g);   // 2^28 at most
  for (uint32_t g0 = blockIdx.x * PER; g0 < all; g0 += gridDim.x * PER) {
    const uint32_t gr = min(g0 + unit % PER, all - 1), kv = gr / per;
    const int r = (int)kv, row = (int)((gr - kv * per) >> g_log), hg = (int)(gr - kv * per) & (a.g - 1);
    // the dealing of the launch before, for a given row
    int first = 0, parts = 0, tiles = 0, r0 = 0, items = 0, base = cut.whole;   // tiles: those that are cut
    for (int i0 = 0; i0 < a.batch; i0 += 64) {
      const PagedLane p = i0 ? paged_lane<FOUR>(a, i0 + lane) : l0;
      const int2 rm = p.rm, s = shape(rm.y, p.n);
      const int upto = items + wave_scan(s.x), nt = s.x - paged_whole(cut, upto - s.x, s.x);
      const int np = (s.y + cut.size - 1) / cut.size, incl = wave_scan(nt * np);
#pragma unroll
      for (int k = 0; k < 64 / TPR; k++) {
        const int want = __builtin_amdgcn_readlane(row, k * TPR);
        const uint64_t hit = __ballot(want >= rm.x && want < rm.x + rm.y);
        if (hit) {
          const int l = __builtin_ctzll(hit);
          const int np_l = __builtin_amdgcn_readlane(np, l), tiles_l = __builtin_amdgcn_readlane(nt, l);
          const int first_l = base + __builtin_amdgcn_readlane(incl, l) - tiles_l * np_l, r0_l = __builtin_amdgcn_readlane(rm.x, l);
          if (lane / TPR == k) { parts = np_l; tiles = tiles_l; first = first_l; r0 = r0_l; }
        }
      }
      items = __builtin_amdgcn_readlane(upto, 63);
      base += __builtin_amdgcn_readlane(incl, 63);
    }
    const int t = row - r0, tile = t >> (7 - g_log), in = ((t << g_log) & 127) + hg;   // 128 / g tokens a tile
    const bool mine = parts > 1 && tile < tiles && g0 + unit % PER < all;
    PagedSum sum;
    if (mine) {
      const int64_t rec = (int64_t)r * a.wgs + first + (tiles - 1 - tile) * parts;
      const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + rec * 128 + in;
      const f32x4* po = reinterpret_cast<const f32x4*>(a.part_o) + (rec * 128 + in) * (D / 4) + c;
#pragma unroll 8
      for (int p = slice; p < parts; p += SLICES) {
        const float2 y = ml[p * 128];
        sum.add(y.x, y.y, po[(int64_t)p * 128 * (D / 4)]);
      }
    }
    if constexpr (SLICES > 1) {
      __syncthreads();
      xo[threadIdx.x] = sum.o;
      if (c == 0) { xd[2 * unit] = sum.m; xd[2 * unit + 1] = sum.den; }
      __syncthreads();
#pragma unroll
      for (int k = 1; k < SLICES; k++) {
        if (slice > 0) break;
        sum.add(xd[2 * (unit + k * PER)], xd[2 * (unit + k * PER) + 1], xo[threadIdx.x + k * PER * TPR]);
      }
    }
    if (!mine || slice > 0) continue;
    const float M = sum.m, den = sum.den;
    const f32x4 o = sum.o;
    const float inv = den > 0.f ? 1.f / den : den == 0.f ? 0.f : den;
    const int head = r * a.g + hg;
    put_row4((uint16_t*)a.o + row * a.o_t + head * a.o_h + c * 4, o, inv);
    if (a.lse && c == 0) a.lse[(int64_t)row * a.h_q + head] = den == 0.f ? -INFINITY : (M + log2f(den)) * kLn2;
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------
// A launch of 2^32 threads or more loses some without an error.  fp32: 512 for an item (bf16: 256, and fewer than 2^22 items whatever the limits of
// n_rows h_q and batch h_kv allow).
bool paged_attend_fits(const PagedArgs& a, int dtype) { return dtype != DASH_F32 || paged_most_items(a, 16) * a.h_kv < (1 << 23); }
// The kernel for a call: tiles of 128 rows where the sequences bring more than 16 rows each on the average, tiles of 16 otherwise.  (32 / 8 heads, tiles of 128
// and of 16, sequences with like numbers of rows.  16 rows each: 64 sequences of 2000 tokens 99.6 and 97.7 us, one of 1000 14.7 and 11.0; 20 rows: 101 and 167, 8 of 16000 104 and 103; 48
// rows: 108 and 281.)  Short caches are read from the last-level cache again and again at no cost: tiles of 16 as long as each has a CU (one
// of 1000 tokens, 64 rows 15.9 and 12.4 us, 128 17.3 and 11.8).  The average hides a long piece beside many single tokens: 380 tokens of a sequence of 8000
// beside 127 sequences of 200 with one each, 507 in all, take tiles of 16 and 458 us, 400 of them tiles of 128 and 147.
static bool use_rows(const PagedArgs& a, int dtype) {
  return dtype == DASH_BF16 && (int64_t)a.n_rows * a.g > (int64_t)a.batch * 16 && !(a.cap <= 8 * kStep && paged_most_items(a, 16) * a.h_kv <= 256);
}
// Workgroups of a kv-head that are resident at once: one a CU for the 128 KB ring of 16-row tiles and the fp32 kernel, two otherwise.
static int runs_of(const PagedArgs& a, int dtype, int d, bool big) { return max((!big && (dtype == DASH_F32 || d == 128) ? 256 : 512) / a.h_kv, 1); }
static size_t ws_align(size_t x) { return (x + 255) & ~(size_t)255; }

size_t paged_attend_ws(const PagedArgs& a, int dtype, int d) {
  const size_t few = (size_t)runs_of(a, dtype, d, false) * a.h_kv * 2 * 16;    // rows of records
  const size_t rows = dtype == DASH_BF16 ? (size_t)paged_most_parts(runs_of(a, dtype, d, true)) * a.h_kv * 128 : 0, recs = few > rows ? few : rows;
  return ws_align(recs * 8) + recs * d * 4 + few / 16 * 16;   // two flags a record of 16 rows
}

template <int D, bool FOUR> static hipError_t launch_merge(const PagedArgs& a, hipStream_t st) {
  // few rows leave the chip idle unless several groups of threads share a row's parts (1280 rows, the call: 32.8 us shared, 34.0 not; 2048 59.4 and 58.0)
  const int64_t out = (int64_t)a.n_rows * a.h_q;
  constexpr int units = 256 / (D / 4);
  if (out <= 1536) hipLaunchKernelGGL((paged_merge_kernel<D, 4, FOUR>), dim3((unsigned)((out + units / 4 - 1) / (units / 4))), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((paged_merge_kernel<D, 1, FOUR>), dim3(1024), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_paged4_merge(const PagedArgs& a, int d, hipStream_t st) { return d == 128 ? launch_merge<128, true>(a, st) : launch_merge<64, true>(a, st); }

template <int D>
static hipError_t launch_attend(PagedArgs a, int dtype, char* ws, hipStream_t st) {
  const bool big = use_rows(a, dtype);
  const int runs = runs_of(a, dtype, D, big);
  const int64_t items = paged_most_items(a, big ? 128 : 16);
  // Runs of small tiles cost little (a record is 16 rows) and even out the lengths of a batch; with many items a workgroup each evens them out as well.  (A
  // token of 64 sequences of 1000 to 4000 tokens, 32 / 8 heads, 119 us in runs, 122 without; of 256, 8 items a run, 454 both ways.  Tiles of 128: 700
  // tokens against 32k 435 in parts, 641 without; two of 700 against 4k 115 and 113.)
  a.wgs = items < (big ? 2 : 8) * (int64_t)runs ? runs : 0;
  // Fine parts, if the lengths ask for them (paged_part_size).  Tiles of less than 64 rows on the average are bound by HBM, which idle workgroups hardly
  // slow down: only if they are much faster (5 tokens of 64 sequences of 300 to 4000: 122 us, in fine parts 130).
  if (big && a.wgs && items * 4 >= runs) a.wgs = (int)items + runs * 3 / 2;
  a.slots = runs;
  a.gain = (int64_t)a.n_rows * a.g < 64 * items ? 0.65f : 0.9f;
  a.whole = items * 2 >= runs;                               // fewer items: not looked into
  // Items of up to eight steps are not cut if there is one for every other CU.  (333 tokens of 1024 in fp32, 32 / 8 heads of 128: 86 us, in runs 90.)
  if (!big && a.cap <= 8 * kStep && items * a.h_kv >= 128) a.wgs = 0;
  const size_t recs = (size_t)a.wgs * a.h_kv * (big ? 128 : 2 * 16);
  a.part_ml = (float*)ws;
  a.part_o = (float*)(ws + ws_align(recs * 8));
  a.flags = (uint64_t*)((char*)a.part_o + recs * D * 4);     // runs only
  a.nonce = big ? 0 : next_nonce();
  const dim3 grid((unsigned)((a.wgs ? a.wgs : items) * a.h_kv)), blk(256);
  if (big) {
    static LdsOptIn opt_in;
    if (hipError_t e = allow_dyn_lds((const void*)paged_rows_kernel<D>, RowsCfg<D>::LDS_BYTES, opt_in); e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_rows_kernel<D>, grid, blk, RowsCfg<D>::LDS_BYTES, st, a);
  } else if (dtype == DASH_BF16) {
    static LdsOptIn opt_in;
    if (hipError_t e = allow_dyn_lds((const void*)paged_few_kernel<D>, FewCfg<D>::LDS_BYTES, opt_in); e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_few_kernel<D>, grid, blk, FewCfg<D>::LDS_BYTES, st, a);
  } else {
    constexpr int lds = 8 * 16 * (D + 6) * 4;
    static LdsOptIn opt_in;
    if (hipError_t e = allow_dyn_lds((const void*)(paged_few_f32_kernel<D, false>), lds, opt_in); e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_few_f32_kernel<D, false>), grid, dim3(512), lds, st, a);
  }
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.wgs <= 1 || !big ? e : launch_merge<D, false>(a, st);
}

hipError_t launch_paged_attend(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st) {
  return d == 128 ? launch_attend<128>(a, dtype, ws, st) : launch_attend<64>(a, dtype, ws, st);
}

}  // namespace dash
