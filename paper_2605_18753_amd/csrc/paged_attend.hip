// Attention of packed new tokens over a paged cache (one pass over the keys with the running maximum and sum of the softmax).
//
// s_tj = q_t . k_j scale over the visible tokens j of the row's sequence, o_t = sum_j softmax_j(s_t) v_j, lse_t = ln sum_j e^{s_tj}.
//
// Few rows (decode, drafted tokens): a tile is 16 (token, head) rows, the heads of a kv-head's group for 16 / g tokens.  The
// cache is read once for 4 g flops a byte, so HBM bounds it; a workgroup's four waves take 32-key tiles in turn, each through a ring of
// its own in LDS (two tiles deep, global -> LDS copies), without a barrier until the four add up at the end.
#include <math.h>

#include "f32_tiles.h"
#include "lds_copy.h"
#include "paged.h"

namespace dash {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kPagedLazy = 8.f;        // slack of the running maximum, in base-2 logit units: exponentials stay below 2^8

// chunk permutations of the LDS tiles (position of 16-byte chunk c of row `row`): 16 consecutive rows at one chunk (operand of the
// first product) and 4 rows x 4 chunks (transposing read) each spread over all banks
template <int D> __device__ __forceinline__ int pk_swz(int row) { return D == 128 ? (row & 15) : ((row >> 1) & 7); }
template <int D> __device__ __forceinline__ int pv_swz(int row) { return D == 128 ? ((row & 3) << 2) : (((row >> 1) & 1) << 2); }

// a row's last visible slot, -1: none
__device__ __forceinline__ int paged_last_key(const PagedArgs& a, const PagedItem& it, int t) {
  return a.causal ? min(it.n - it.m + t, it.n - 1) : it.n - 1;
}

template <int D> struct FewCfg {
  static constexpr int NCH = D / 8, ROW_BYTES = D * 2;
  static constexpr int TILE_BYTES = 32 * ROW_BYTES;      // K or V of 32 keys
  static constexpr int COPIES = TILE_BYTES / 1024;       // copy instructions of a wave per tile and tensor
  static constexpr int RPC = 64 / NCH;                   // rows an instruction covers
  static constexpr int WAVE_BYTES = 4 * TILE_BYTES;      // two stages of K and V
  static constexpr int LDS_BYTES = 4 * WAVE_BYTES;
};

// What the four waves hold of a tile's 16 rows is added up in LDS, and written as the output or as a record of the part.
// x: [4][16][D + 4] floats, ml: [4][16][2] behind it.  Threads 16 i .. + 15 hold row i.
template <typename T, int D>
__device__ __forceinline__ void paged_few_finish(const PagedArgs& a, const PagedItem& it, int r, int t0, const float* x, const float* ml) {
  const int row = threadIdx.x >> 4, c = threadIdx.x & 15;
  float M = -INFINITY, den = 0.f, w[4];
#pragma unroll
  for (int i = 0; i < 4; i++) M = fmaxf(M, ml[(i * 16 + row) * 2]);
  const float use = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    w[i] = __builtin_amdgcn_exp2f(ml[(i * 16 + row) * 2] - use);
    den = fmaf(w[i], ml[(i * 16 + row) * 2 + 1], den);
  }
  float o[D / 16];
#pragma unroll
  for (int j = 0; j < D / 64; j++) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(x + (i * 16 + row) * (D + 4) + j * 64 + c * 4);
#pragma unroll
      for (int e = 0; e < 4; e++) s[e] = fmaf(w[i], y[e], s[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; e++) o[j * 4 + e] = s[e];
  }
  if (it.parts > 1) {
    const int64_t rec = (int64_t)r * a.part_stride + it.rec0 + it.part;
    float* po = a.part_o + (rec * 16 + row) * D;
#pragma unroll
    for (int j = 0; j < D / 64; j++) *reinterpret_cast<f32x4*>(po + j * 64 + c * 4) = f32x4{o[j * 4], o[j * 4 + 1], o[j * 4 + 2], o[j * 4 + 3]};
    if (c == 0) reinterpret_cast<float2*>(a.part_ml)[rec * 16 + row] = make_float2(M, den);
    return;
  }
  const int t = t0 + row / a.g, head = r * a.g + row % a.g;
  if (t >= it.m) return;
  const float inv = den > 0.f ? 1.f / den : den == 0.f ? 0.f : den;     // NaN stays
  T* op = (T*)a.o + (it.r0 + t) * a.o_t + head * a.o_h;
#pragma unroll
  for (int j = 0; j < D / 64; j++) {
    if constexpr (sizeof(T) == 2) {
      uint2 y;
      y.x = cvt_bf16x2(o[j * 4] * inv, o[j * 4 + 1] * inv);
      y.y = cvt_bf16x2(o[j * 4 + 2] * inv, o[j * 4 + 3] * inv);
      *reinterpret_cast<uint2*>(op + j * 64 + c * 4) = y;
    } else {
      *reinterpret_cast<f32x4*>(op + j * 64 + c * 4) = f32x4{o[j * 4] * inv, o[j * 4 + 1] * inv, o[j * 4 + 2] * inv, o[j * 4 + 3] * inv};
    }
  }
  if (a.lse && c == 0) a.lse[(int64_t)(it.r0 + t) * a.h_q + head] = den == 0.f ? -INFINITY : (M + log2f(den)) * kLn2;
}

// tiles of 16 rows of a sequence; cost: its 128-key steps
__device__ __forceinline__ int2 few_shape(const PagedArgs& a, int m, int n) {
  const int T = 16 / a.g;
  return make_int2((m + T - 1) / T, max((n + 127) >> 7, 1));
}

template <int D>
__global__ __launch_bounds__(256, D == 128 ? 1 : 2) void paged_few_kernel(PagedArgs a) {
  using C = FewCfg<D>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x % a.h_kv;
  PagedItem it;
  if (!paged_find(a, blockIdx.x / a.h_kv, [&](int m, int n) { return few_shape(a, m, n); }, it)) return;
  const int T = 16 / a.g, t0 = it.tile * T;
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
  // this part's 128-key steps; the wave's 32-key tiles among them
  const int steps = (end + 127) >> 7, per = (steps + it.parts - 1) / it.parts;
  const int j1 = min((it.part + 1) * per * 4, (end + 31) >> 5);
  int j = it.part * per * 4 + wave;

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
  paged_few_finish<uint16_t, D>(a, it, r, t0, x, ml);
}

// fp32: the same walk with the fp32 matrix cores, operands straight from the pages, 16 keys at a time.  A token's NaN or infinity
// reaches the rows that see it and no other.
template <int D>
__global__ __launch_bounds__(256) void paged_few_f32_kernel(PagedArgs a) {
  __shared__ __attribute__((aligned(16))) float x[4 * 16 * (D + 4) + 4 * 16 * 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x % a.h_kv;
  PagedItem it;
  if (!paged_find(a, blockIdx.x / a.h_kv, [&](int m, int n) { return few_shape(a, m, n); }, it)) return;
  const int T = 16 / a.g, t0 = it.tile * T;
  const int n = lane & 15, kq = lane >> 4;
  const int t = t0 + n / a.g;
  f32x4 qv[D / 16];
  load_row<D>((const float*)a.q + (it.r0 + min(t, it.m - 1)) * a.q_t + (r * a.g + n % a.g) * a.q_h, kq, qv);
  const int last = t < it.m ? paged_last_key(a, it, t) : -1;
  const int end = max(paged_last_key(a, it, min(t0 + T, it.m) - 1) + 1, 0);
  const int steps = (end + 127) >> 7, per = (steps + it.parts - 1) / it.parts;
  const int j0 = it.part * per * 8 + wave, j1 = min((it.part + 1) * per * 8, (end + 15) >> 4);   // 16-key tiles
  const int pm = (1 << a.page_log) - 1;
  const float* kb = (const float*)a.k + r * a.kp_h;
  const float* vb = (const float*)a.v + r * a.vp_h;
  float m_run = -INFINITY, l_run = 0.f;
  f32x4 acc[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; i++) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int j = j0; j < j1; j += 4) {
    // rows behind the sequence's last token repeat it
    const int64_t id = paged_page(a, it.b, (j * 16) >> a.page_log);
    const int top = it.n - 1 - j * 16;
    const float* kp = kb + id * a.kp_p + (int64_t)(j * 16 & pm) * a.kp_t;
    const float* vp = vb + id * a.vp_p + (int64_t)(j * 16 & pm) * a.vp_t;
    f32x4 kv[D / 16], vv[1][4][D / 64];
    load_row<D>(kp + min(n, top) * a.kp_t, kq, kv);
#pragma unroll
    for (int i = 0; i < 4; i++) load_row2<D>(vp + min(4 * kq + i, top) * a.vp_t, n, vv[0][i]);
    f32x4 s[1] = {mma_dot<D>(kv, qv)};                                           // lane (row n, kq): keys 4 kq + i
    const int lim = last - (j * 16 + 4 * kq);
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      s[0][i] = i > lim ? -INFINITY : s[0][i];
      mx = fmaxf(mx, s[0][i]);
    }
    mx = quad_rows_max(mx) * a.c1;
    if (__any(mx > m_run + kPagedLazy)) {
      const float m_new = fmaxf(m_run, mx), use = m_new == -INFINITY ? 0.f : m_new;
      const float corr = __builtin_amdgcn_exp2f(m_run - use);
      m_run = m_new;
      l_run *= corr;
#pragma unroll
      for (int i = 0; i < D / 16; i++) acc[i] *= corr;
    }
    const float off = m_run == -INFINITY ? 0.f : -m_run;
#pragma unroll
    for (int i = 0; i < 4; i++) s[0][i] = __builtin_amdgcn_exp2f(fmaf(s[0][i], a.c1, off));
    l_run += (s[0][0] + s[0][1]) + (s[0][2] + s[0][3]);
    mma_outer_keys<D, 1>(vv, s, lim, min(T, it.m - t0), a.g, lane, acc);
  }
  const float l_tot = quad_rows_sum(l_run);
  float* ml = x + 4 * 16 * (D + 4);
#pragma unroll
  for (int nv = 0; nv < D / 64; nv++)
#pragma unroll
    for (int v = 0; v < 4; v++)
      *reinterpret_cast<f32x4*>(x + (wave * 16 + n) * (D + 4) + 64 * nv + 16 * kq + 4 * v) =
          f32x4{acc[4 * nv][v], acc[4 * nv + 1][v], acc[4 * nv + 2][v], acc[4 * nv + 3][v]};
  if (kq == 0) {
    ml[(wave * 16 + n) * 2] = m_run;
    ml[(wave * 16 + n) * 2 + 1] = l_tot;
  }
  __syncthreads();
  paged_few_finish<float, D>(a, it, r, t0, x, ml);
}

// Adds the parts of cut items: o = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p.  Eight packed (token, head) rows a workgroup,
// 32 threads each.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedArgs a) {
  const int lane = threadIdx.x & 63;
  const int heads = a.h_q;
  const int64_t gr0 = (int64_t)blockIdx.x * 8;
  const int sub = threadIdx.x >> 5, c = threadIdx.x & 31;
  // the rows of a workgroup may belong to several sequences: each half wave finds its own
  const int64_t gr = gr0 + sub;
  const int row = (int)min(gr / heads, (int64_t)a.n_rows - 1), head = (int)(gr % heads);
  // the dealing of the launch before, for a given row
  const auto shape = [&](int m, int n) { return few_shape(a, m, n); };
  const int S = paged_part_size(a, shape);
  int first = 0, parts = 0, tiles = 0, r0 = 0, base = 0;
  for (int i0 = 0; i0 < a.batch; i0 += 64) {
    int2 s = make_int2(0, 0), rm = make_int2(0, 0);
    if (i0 + lane < a.batch) {
      rm = paged_rows(a, i0 + lane);
      s = shape(rm.y, paged_len(a, i0 + lane));
    }
    const int np = (s.y + S - 1) / S, incl = wave_scan(s.x * np);
#pragma unroll
    for (int half = 0; half < 2; half++) {
      const int want = __builtin_amdgcn_readlane(row, half * 32);
      const uint64_t hit = __ballot(want >= rm.x && want < rm.x + rm.y);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        const int np_l = __builtin_amdgcn_readlane(np, l), tiles_l = __builtin_amdgcn_readlane(s.x, l);
        const int first_l = base + __builtin_amdgcn_readlane(incl, l) - tiles_l * np_l, r0_l = __builtin_amdgcn_readlane(rm.x, l);
        if ((lane >> 5) == half) { parts = np_l; tiles = tiles_l; first = first_l; r0 = r0_l; }
      }
    }
    base += __builtin_amdgcn_readlane(incl, 63);
  }
  if (parts <= 1 || gr >= (int64_t)a.n_rows * heads) return;
  const int Tt = 16 / a.g, t = row - r0, tile = t / Tt, in = (t % Tt) * a.g + head % a.g;
  const int64_t rec = (int64_t)(head / a.g) * a.part_stride + first + (tiles - 1 - tile) * parts;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + rec * 16 + in;
  float M = -INFINITY, den = 0.f;
  for (int p = 0; p < parts; p++) M = fmaxf(M, ml[p * 16].x);
  const float use = M == -INFINITY ? 0.f : M;
  constexpr int V = D / 32;
  float o[V];
#pragma unroll
  for (int i = 0; i < V; i++) o[i] = 0.f;
  const float* po = a.part_o + (rec * 16 + in) * D + c * V;
#pragma unroll 4
  for (int p = 0; p < parts; p++) {
    const float2 y = ml[p * 16];
    const float w = __builtin_amdgcn_exp2f(y.x - use);
    den = fmaf(w, y.y, den);
#pragma unroll
    for (int i = 0; i < V; i++) o[i] = fmaf(w, po[(int64_t)p * 16 * D + i], o[i]);
  }
  const float inv = den > 0.f ? 1.f / den : den == 0.f ? 0.f : den;
  T* op = (T*)a.o + row * a.o_t + head * a.o_h + c * V;
#pragma unroll
  for (int i = 0; i < V; i += 2) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(op + i) = cvt_bf16x2(o[i] * inv, o[i + 1] * inv);
    else { op[i] = o[i] * inv; op[i + 1] = o[i + 1] * inv; }
  }
  if (a.lse && c == 0) a.lse[(int64_t)row * heads + head] = den == 0.f ? -INFINITY : (M + log2f(den)) * kLn2;
}

// ---- host ------------------------------------------------------------------------------------------------------------
static int few_items(const PagedArgs& a) {   // most items of a kv-head
  const int T = 16 / a.g;
  const int64_t n = (int64_t)a.n_rows / T + min(a.batch, a.n_rows);
  return (int)(n < a.n_rows ? n : a.n_rows);
}
static int few_target(const PagedArgs& a) { return max(256 / a.h_kv, 1); }
static int few_wgs(const PagedArgs& a) { return few_items(a) < few_target(a) ? few_target(a) : 0; }
static size_t ws_align(size_t x) { return (x + 255) & ~(size_t)255; }

size_t paged_attend_ws(const PagedArgs& a, int dtype, int d) {
  const size_t recs = (size_t)few_target(a) * a.h_kv * 16;
  return ws_align(recs * 8) + recs * d * 4;
}

template <int D>
static hipError_t launch_few(PagedArgs a, int dtype, char* ws, hipStream_t st) {
  using C = FewCfg<D>;
  a.wgs = few_wgs(a);
  a.min_part = 1;
  a.part_stride = a.wgs;
  const size_t recs = (size_t)a.wgs * a.h_kv * 16;
  a.part_ml = (float*)ws;
  a.part_o = (float*)(ws + ws_align(recs * 8));
  const dim3 grid((unsigned)(max(a.wgs, few_items(a)) * a.h_kv)), blk(256);
  if (dtype == DASH_BF16) {
    static LdsOptIn opt_in;
    if (hipError_t e = allow_dyn_lds((const void*)paged_few_kernel<D>, C::LDS_BYTES, opt_in); e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_few_kernel<D>, grid, blk, C::LDS_BYTES, st, a);
  } else {
    hipLaunchKernelGGL(paged_few_f32_kernel<D>, grid, blk, 0, st, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.wgs == 0) return e;
  const dim3 mgrid((unsigned)(((int64_t)a.n_rows * a.h_q + 7) / 8));
  if (dtype == DASH_BF16) hipLaunchKernelGGL((paged_merge_kernel<uint16_t, D>), mgrid, blk, 0, st, a);
  else hipLaunchKernelGGL((paged_merge_kernel<float, D>), mgrid, blk, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_paged_attend(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st) {
  return d == 128 ? launch_few<128>(a, dtype, ws, st) : launch_few<64>(a, dtype, ws, st);
}

}  // namespace dash
