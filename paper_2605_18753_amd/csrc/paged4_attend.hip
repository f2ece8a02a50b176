// Attention of packed new tokens over a paged cache in 4 bits (fp4.h): the walks of paged_attend.hip, whose dealing and joining they use.
//
// Few rows: a tile is 16 (token, head) rows, or two groups of 16 that share what is read and converted.  K goes from the pages into registers: the contraction over d runs in the order in which a lane's
// codes lie, d = D / 4 kq + .., so 16 bytes of a row are one load, one scale and, converted, the lane's operands of all steps.  V is converted into LDS, from
// where transposing reads give its operands.  The next tile's loads are in flight while a tile is worked on.  Bound by HBM where the cache is long: 32 sequences
// of 4096 to 32768 tokens, 32 / 8 heads of 128, 125 to 127 us, 660 MB at 5.2 TB/s, of which 8 us are the launch's start and end (the vector units issue in 0.44 of the
// clocks); by latency where it is short: one sequence of 1000 tokens 9.2 us.
#include "fp4.h"
#include "paged_few.h"

namespace dash {

template <int D, int ROWS = 16> struct Few4Cfg {
  static constexpr int CW = D / 32;                        // words of a lane's codes: a quarter of a row
  static constexpr int ROW_BYTES = D * 2, TILE_BYTES = 32 * ROW_BYTES;   // V of 32 keys in bf16
  static constexpr int OUT_BYTES = 4 * ROWS * (D + 6) * 4;   // the waves' results, behind the walk
  static constexpr int LDS_BYTES = 4 * TILE_BYTES > OUT_BYTES ? 4 * TILE_BYTES : OUT_BYTES;
};
// Position of 16-byte chunk c of V's row: 4 rows x 2 chunks (transposing reads) and 4 rows x 4 chunks a quarter of a row apart (writes) spread over all banks.
template <int D> __device__ __forceinline__ int v4_swz(int row) { return D == 128 ? (row & 3) * 5 : ((row >> 1) & 1) * 5; }

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <int CW> struct Codes { uint32_t w[CW]; };
template <int CW> __device__ __forceinline__ Codes<CW> load_codes(__amdgpu_buffer_rsrc_t rs, uint32_t off) {
  Codes<CW> c;
  if constexpr (CW == 4) {
    const u32v4 x = __builtin_bit_cast(u32v4, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
#pragma unroll
    for (int i = 0; i < 4; i++) c.w[i] = x[i];
  } else {
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0));
    c.w[0] = x[0]; c.w[1] = x[1];
  }
  return c;
}
// bytes [0, bytes) behind p; loads past them give 0
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* p, int bytes) {
  const uint64_t at = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));   // ints: not to be widened
  return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
// Scale bytes come as the word that they lie in (bytes would be widened as soon as they arrive, which waits for them).  Block b of a row among 16 that begin
// at a multiple of 4 bytes: offset of its word, and its byte's place there.
template <int D> __device__ __forceinline__ uint32_t scale_word(int row) { return D == 128 ? row * 4 : (row >> 1) * 4; }
template <int D> __device__ __forceinline__ int scale_span(int rows) { return D == 128 ? rows * 4 : ((rows + 1) >> 1) * 4; }   // whole words
template <int D> __device__ __forceinline__ uint32_t scale_byte(uint32_t w, int row, int b) { return __builtin_amdgcn_ubfe(w, D == 128 ? 8 * b : 16 * (row & 1) + 8 * b, 8); }
// A uniform number kept within 0 .. 16.  (The compiler makes min and max a vector instruction, what follows from it too, and waits for loads whose registers it takes.)
__device__ __forceinline__ int within_16(int x) {
  int y;
  asm("s_max_i32 %0, %1, 0\n\ts_min_i32 %0, %0, 16" : "=s"(y) : "s"(x) : "scc");
  return y;
}
// Bytes of `rows` rows of codes, 0 .. 16 of them, from the first one's start.
template <int D> __device__ __forceinline__ int rows_span(int rows, uint32_t stride) {
  return max((int)((uint32_t)rows * stride - (stride - D / 2)), 0);
}
__device__ __forceinline__ void lds_write_b128(uint32_t addr, bf16x8 x) {
  *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>(addr) = x;
}

// An address with bits flipped, worked out where it is used: the registers have no room for one a chunk.
__device__ __forceinline__ uint32_t flipped(uint32_t addr, int bits) {
  uint32_t x;
  if (bits == 0) return addr;
  asm volatile("v_xor_b32 %0, %2, %1" : "=v"(x) : "v"(addr), "i"(bits));
  return x;
}

// What the walks over 32-key tiles share: where a lane's codes lie, loads and conversions.
template <int D> struct Walk4 {
  using C = Few4Cfg<D>;
  struct Raw { Codes<C::CW> k[2], v[2]; uint32_t ks[2], vs[2]; };
  const PagedArgs& a;
  int b, r, keys, j1, lane;                                // sequence, kv-head, tokens; behind the piece's last tile; all but lane uniform
  uint32_t kt, vt, k_off, v_off, ks_off, vs_off, v_wr;
  const char *kb, *vb;
  __device__ __forceinline__ Walk4(const PagedArgs& a, int b, int r, int keys, int j1, int lane, uint32_t buf) : a(a), b(b), r(r), keys(keys), j1(j1), lane(lane) {
    const int n = lane & 15, kq = lane >> 4;
    kt = (uint32_t)a.kp_t; vt = (uint32_t)a.vp_t;
    // K: row n, quarter kq; V: row lane / 4, quarter lane % 4
    k_off = (uint32_t)n * kt + kq * (D / 8); v_off = (uint32_t)(lane >> 2) * vt + (lane & 3) * (D / 8);
    ks_off = scale_word<D>(n); vs_off = scale_word<D>(lane >> 2);
    kb = (const char*)a.k + r * a.kp_h;
    vb = (const char*)a.v + r * a.vp_h;
    // of a lane's first chunk of V; chunk i lies at that address with bits 4 .. flipped by i
    v_wr = buf + (uint32_t)((lane >> 2) * C::ROW_BYTES + ((C::CW * (lane & 3)) ^ v4_swz<D>(lane >> 2)) * 16);
  }
  // the table's entries for a tile: of one page, or of two of 16 tokens; looked at a tile later, when they have arrived
  __device__ __forceinline__ int2 entries_of(int tile) const {
    return make_int2(paged_entry(a, b, (tile * 32) >> a.page_log), paged_entry(a, b, (tile * 32 + 16) >> a.page_log));
  }
  // A resource ends with the sequence's last token: rows behind it read as zeros, whatever their page holds.
  __device__ __forceinline__ void load(int tile, int2 entries, Raw& x) const {
#pragma unroll
    for (int half = 0; half < 2; half++) {
      const int key = tile * 32 + half * 16;
      const uint32_t id = paged_clamp(a, half ? entries.y : entries.x), off = key & ((1 << a.page_log) - 1);
      const int rows = within_16(min(keys - key, (j1 - tile) * 32));             // behind the piece's last tile: nothing is read
      const uint64_t at = ((((uint64_t)id * (uint32_t)a.h_kv + r) << a.page_log) + off) * (D / 32);
      x.k[half] = load_codes<C::CW>(rsrc_of(kb + (uint64_t)id * (uint64_t)a.kp_p + off * kt, rows_span<D>(rows, kt)), k_off);
      x.v[half] = load_codes<C::CW>(rsrc_of(vb + (uint64_t)id * (uint64_t)a.vp_p + off * vt, rows_span<D>(rows, vt)), v_off);
      x.ks[half] = __builtin_amdgcn_raw_buffer_load_b32(rsrc_of(a.k_sc + at, scale_span<D>(rows)), ks_off, 0, 0);
      x.vs[half] = __builtin_amdgcn_raw_buffer_load_b32(rsrc_of(a.v_sc + at, scale_span<D>(rows)), vs_off, 0, 0);
    }
  }
  __device__ __forceinline__ uint32_t k_scale(const Raw& x, int half) const { return scale_byte<D>(x.ks[half], lane & 15, (lane >> 4) * (D / 4) / 32); }
  __device__ __forceinline__ uint32_t v_scale(const Raw& x, int half) const { return scale_byte<D>(x.vs[half], lane >> 2, (lane & 3) * (D / 4) / 32); }
  // V of a tile into LDS, in bf16.  A block that is NaN goes in as numbers next to 0 (the scale's exponent 0).
  __device__ __forceinline__ void put_v(const Raw& x, const uint32_t (&vs)[2], int at) const {
#pragma unroll
    for (int half = 0; half < 2; half++) {
      const float sc = __uint_as_float(vs[half] == 255u ? 0u : vs[half] << 23);
#pragma unroll
      for (int i = 0; i < C::CW; i++) lds_write_b128(flipped(v_wr, i << 4) + at + half * 16 * C::ROW_BYTES, fp4_to_bf16(x.v[half].w[i], sc));
    }
  }
  // The rows that see the token of a block of V that is NaN: NaN there.  last: the lane's row's last key.
  __device__ __forceinline__ void spoil(const uint32_t (&vs)[2], int tile, int last, f32x4 (&oacc)[D / 16]) const {
    if (__builtin_expect(!__any(vs[0] == 255u || vs[1] == 255u), 1)) return;
#pragma unroll
    for (int half = 0; half < 2; half++)
      for (uint64_t bad = __ballot(vs[half] == 255u); bad; bad &= bad - 1) {
        const int l = __builtin_ctzll(bad), block = (l & 3) * (D / 4) / 32;
        const bool seen = tile * 32 + half * 16 + (l >> 2) <= last;
#pragma unroll
        for (int dt = 0; dt < D / 16; dt++)
          if (dt >> 1 == block && seen) oacc[dt] = f32x4{NAN, NAN, NAN, NAN};
      }
  }
};

template <int D, int G>
__global__ __launch_bounds__(256, D == 128 ? 2 : 3) void paged_few4_kernel(PagedArgs args) {
  using C = Few4Cfg<D>;
  constexpr int ROWS = 16 * G;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int r = blockIdx.x % args.h_kv, wg = blockIdx.x / args.h_kv;
  PagedRun<true> run(args, ROWS);
  if (!run.begin(args, wg)) return;
  const PagedItem& it = run.it;
  do {
  const PagedArgs a = paged_reload();
  const int tid = paged_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = ROWS / a.g;
  const int t0 = it.tile * T;
  const int n = lane & 15, kq = lane >> 4;
  // group i of rows: 16 i + n
  bf16x8 qf[G][D / 32];
  int last[G];
#pragma unroll
  for (int i = 0; i < G; i++) {
    const int row = 16 * i + n, t = t0 + row / a.g;
    const uint16_t* qp = (const uint16_t*)a.q + (it.r0 + min(t, it.m - 1)) * a.q_t + (r * a.g + row % a.g) * a.q_h + kq * (D / 4);
#pragma unroll
    for (int s = 0; s < D / 32; s++) qf[i][s] = *reinterpret_cast<const bf16x8*>(qp + 8 * s);
    last[i] = t < it.m ? paged_last_key(a, it, t) : -1;
  }
  const int first_last = paged_last_key(a, it, t0);                              // of the tile's first token
  const int end = max(paged_last_key(a, it, min(t0 + T, it.m) - 1) + 1, 0);      // keys that a row of the tile sees
  // the wave's 32-key tiles of the piece's 128-key steps
  const int j1 = __builtin_amdgcn_readfirstlane(min(run.x1 * 4, (end + 31) >> 5)), keys = __builtin_amdgcn_readfirstlane(it.n);
  int j = __builtin_amdgcn_readfirstlane(run.x0 * 4) + wave;

  const uint32_t buf = lds_addr_of(lds) + wave * C::TILE_BYTES;
  const Walk4<D> walk(a, it.b, r, keys, j1, lane, buf);
  // transposing read of V: lane s of a group of 16 points at row 4 kq + s / 4 (+ 16), d 4 (s % 4) of the 16-wide d-tile
  const uint32_t v_rd = buf + (uint32_t)((4 * kq + (n >> 2)) * C::ROW_BYTES + ((((n & 3) >> 1) ^ v4_swz<D>(n >> 2)) << 4) + ((n & 1) << 3));

  float m_run[G], l_run[G];
  f32x4 oacc[G][D / 16];
#pragma unroll
  for (int i = 0; i < G; i++) {
    m_run[i] = -INFINITY; l_run[i] = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 16; dt++) oacc[i][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Two sets of registers in turn: the next tile's loads are asked for before the present ones are waited for.  A wave's priority rises through a tile: whoever is further on
  // is served first, and the waves of a SIMD fall out of step, one's products beside another's conversions (24 sequences of 3000 to 16000 with 64 rows 109 -> 104 us, at
  // head dimension 64 32 of them 94.8 -> 85.4, 80 rows of eight 31.0 -> 28.7).
  typename Walk4<D>::Raw even, odd;
  int2 entries = make_int2(0, 0);
  if (j < j1) {
    walk.load(j, walk.entries_of(j), even);
    entries = walk.entries_of(j + 4);
  }
  auto tile = [&](const typename Walk4<D>::Raw& x, typename Walk4<D>::Raw& next) __attribute__((always_inline)) {
    walk.load(j + 4, entries, next);
    entries = walk.entries_of(j + 8);
    const uint32_t vs[2] = {walk.v_scale(x, 0), walk.v_scale(x, 1)};
    walk.put_v(x, vs, 0);
    f32x4 s0[G], s1[G];                                                          // lane (row n, kq): keys 4 kq + i, 16 + 4 kq + i
    __builtin_amdgcn_s_setprio(1);
    const float k0 = fp4_scale(walk.k_scale(x, 0)), k1 = fp4_scale(walk.k_scale(x, 1));
#pragma unroll
    for (int i = 0; i < G; i++) s0[i] = s1[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < D / 32; s++) {
      const bf16x8 x0 = fp4_to_bf16(x.k[0].w[s], k0), x1 = fp4_to_bf16(x.k[1].w[s], k1);
#pragma unroll
      for (int i = 0; i < G; i++) {
        s0[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x0, qf[i][s], s0[i], 0, 0, 0);
        s1[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x1, qf[i][s], s1[i], 0, 0, 0);
      }
    }
    if (j * 32 + 31 > first_last || t0 + T > it.m) {
#pragma unroll
      for (int g = 0; g < G; g++) {
        const int lim = last[g] - (j * 32 + 4 * kq);
#pragma unroll
        for (int i = 0; i < 4; i++) {
          s0[g][i] = i > lim ? -INFINITY : s0[g][i];
          s1[g][i] = 16 + i > lim ? -INFINITY : s1[g][i];
        }
      }
    }
    bf16x8 pb[G];
#pragma unroll
    for (int g = 0; g < G; g++) {
      float mx = fmaxf(fmaxf(fmaxf(s0[g][0], s0[g][1]), fmaxf(s0[g][2], s0[g][3])), fmaxf(fmaxf(s1[g][0], s1[g][1]), fmaxf(s1[g][2], s1[g][3])));
      mx = quad_rows_max(mx) * a.c1;
      if (__any(mx > m_run[g] + kPagedLazy)) {
        const float m_new = fmaxf(m_run[g], mx), use = m_new == -INFINITY ? 0.f : m_new;
        const float corr = __builtin_amdgcn_exp2f(m_run[g] - use);
        m_run[g] = m_new;
        l_run[g] *= corr;
#pragma unroll
        for (int dt = 0; dt < D / 16; dt++) oacc[g][dt] *= corr;
      }
      const float off = m_run[g] == -INFINITY ? 0.f : -m_run[g];
      float p[8];
#pragma unroll
      for (int i = 0; i < 4; i++) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s0[g][i], a.c1, off));
        p[4 + i] = __builtin_amdgcn_exp2f(fmaf(s1[g][i], a.c1, off));
      }
      l_run[g] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      // P in bf16, the operand type of the matrix cores (relative error 2^-9); the row sum takes the unrounded values
      const u32x4 pw = {cvt_bf16x2(p[0], p[1]), cvt_bf16x2(p[2], p[3]), cvt_bf16x2(p[4], p[5]), cvt_bf16x2(p[6], p[7])};
      pb[g] = __builtin_bit_cast(bf16x8, pw);
    }
    asm volatile("" ::: "memory");                                               // a wave's LDS operations complete in order
    __builtin_amdgcn_s_setprio(2);
    bf16x8 vf[D / 16];
#pragma unroll
    for (int dt = 0; dt < D / 16; dt++) {
      const uint32_t at = flipped(v_rd, dt << 5);
      vf[dt] = lds_read_tr_pair(at, at + 16 * C::ROW_BYTES);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int dt = 0; dt < D / 16; dt++)
#pragma unroll
      for (int g = 0; g < G; g++) oacc[g][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[dt], pb[g], oacc[g][dt], 0, 0, 0);
    asm volatile("" ::: "memory");
#pragma unroll
    for (int g = 0; g < G; g++) walk.spoil(vs, j, last[g], oacc[g]);
    __builtin_amdgcn_s_setprio(0);
  };
  while (j < j1) {
    tile(even, odd);
    if ((j += 4) >= j1) break;
    tile(odd, even);
    j += 4;
  }
  __syncthreads();
  float* x = reinterpret_cast<float*>(lds);                                      // [4][ROWS][D + 4]
  float* ml = x + 4 * ROWS * (D + 4);
#pragma unroll
  for (int g = 0; g < G; g++) {
    const float l_tot = quad_rows_sum(l_run[g]);
    const int row = wave * ROWS + 16 * g + n;
#pragma unroll
    for (int dt = 0; dt < D / 16; dt++) *reinterpret_cast<f32x4*>(x + row * (D + 4) + 4 * kq + 16 * dt) = oacc[g][dt];
    if (kq == 0) {
      ml[row * 2] = m_run[g];
      ml[row * 2 + 1] = l_tot;
    }
  }
  __syncthreads();
  paged_few_finish<uint16_t, D, 4, ROWS>(a, run, r, ((int64_t)r * a.wgs + wg) * 2 + (run.x0 == 0), t0, x, ml);
  if (!run.whole()) paged_few_join<uint16_t, D, 256, ROWS>(a, run, r, wg, lds);
  __syncthreads();
  } while (run.advance(args));
}


// Many rows: a tile is 128 (token, head) rows, as in paged_rows_kernel, whose walk this is: the two products, the exponentials and the maxima
// between their MFMAs, the order of operands.  64-key tiles of K and V are converted on their way into LDS, each by the whole workgroup once: 32 conversions a thread
// and tile, beside some 250 vector instructions and 32 MFMAs of each wave.  Bound by the vector units (0.60 of the clocks), the matrix units (0.48) and LDS (K and V, 32 KB, go to each of
// a CU's eight waves, 2050 clocks at 128 bytes a clock, and are written at 75, 850, of a step's 4000).  2048 tokens at the end of 32768, 32 / 8 heads of 128, 1000 to
// 1060 us by card (1.1 PFLOP/s; pages of bf16 967 to 1080).  Head dimension 64: three workgroups a CU (all exponentials between the first product's MFMAs, which
// spares the registers that a third one needs): the same 624 us (before waves had priorities 656, and with two workgroups a CU 741).
template <int D> struct Rows4Cfg {
  static constexpr int CW = D / 32, ROW_BYTES = D * 2;
  static constexpr int TILE_BYTES = 64 * ROW_BYTES;
  static constexpr int OUT_BYTES = 128 * (D + 4) * 4;      // a tile's rows in fp32, behind the walk
  static constexpr int LDS_BYTES = 4 * TILE_BYTES + 64 > OUT_BYTES ? 4 * TILE_BYTES + 64 : OUT_BYTES;   // K ring [2], V ring [2], blocks that are NaN
};

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void paged_rows4_kernel(PagedArgs a) {
  using C = Rows4Cfg<D>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  // kv-heads are the fast index: with 8 of them each XCD's L2 sees the pages of one
  const int r = blockIdx.x % a.h_kv;
  PagedPart it;
  if (!paged_find_part<true>(a, blockIdx.x / a.h_kv, [&](int m, int n) { return rows_shape(a, m, n); }, it)) return;
  const int T = 128 / a.g, t0 = it.tile * T, Tw = 32 / a.g, tw0 = t0 + wave * Tw;
  const int t = tw0 + n / a.g;
  bf16x8 qf[D / 16];
  {
    const uint16_t* qp = (const uint16_t*)a.q + (it.r0 + min(t, it.m - 1)) * a.q_t + (r * a.g + n % a.g) * a.q_h + h * 8;
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
  }
  // of the lane's row, worked out where it is used
  auto last_key = [&]() { return paged_last_key(a, it, min(tw0 + ((paged_thread() & 31) >> (31 - __builtin_clz(a.g))), it.m - 1)); };
  // keys that the tile, and the wave, sees; up to where the wave's first token does
  const int end = max(paged_last_key(a, it, min(t0 + T, it.m) - 1) + 1, 0);
  const int wave_end = tw0 < it.m ? paged_last_key(a, it, min(tw0 + Tw, it.m) - 1) + 1 : 0;
  const int low = paged_last_key(a, it, min(tw0, it.m - 1));
  const int kt = (end + 63) >> 6, per = (kt + it.parts - 1) / it.parts;
  const int first = min(it.part * per, kt), n_it = min(per, kt - first);       // the part's tiles

  // ---- pages: 64 entries of the table a lane each, the next 64 behind them ----------------------------------
  const int32_t* table = a.table + (int64_t)it.b * a.max_pages;
  auto window = [&](int i) { return paged_clamp(a, table[min(i + (paged_thread() & 63), a.max_pages - 1)]); };
  int wbase = (first * 64) >> a.page_log;
  int win = window(wbase), win_next = window(wbase + 64);

  // ---- pages -> registers -> LDS --------------------------------------------------------------------------------
  // A wave has 16 rows of a tile, which lie in one page: one resource, which ends with the sequence's last token (rows behind it read as
  // zeros, whatever the page holds).  A lane has a quarter of row lane / 4.
  const uint32_t k_t = (uint32_t)a.kp_t, v_t = (uint32_t)a.vp_t;
  const char* kb = (const char*)a.k + r * a.kp_h;
  const char* vb = (const char*)a.v + r * a.vp_h;
  const int pm = (1 << a.page_log) - 1, row0 = wave * 16;
  const uint32_t lds0 = lds_addr_of(lds);
  const int part_end = first + n_it;
  struct Raw { Codes<C::CW> c; uint32_t s; };
  auto scale_of = [&](const Raw& x) {
    const int l = paged_thread() & 63;
    return scale_byte<D>(x.s, l >> 2, (l & 3) * (D / 4) / 32);
  };
  auto ask = [&](Raw& x, const char* base, int64_t page_stride, uint32_t row_stride, const uint8_t* scales, int id, int tile) {
    const int l = paged_thread() & 63;
    const int key = tile * 64 + row0, rows = tile < part_end ? within_16(it.n - key) : 0;   // behind the part's last tile: nothing is read
    const uint32_t off = key & pm;
    x.c = load_codes<C::CW>(rsrc_of(base + (uint64_t)(uint32_t)id * (uint64_t)page_stride + off * row_stride, rows_span<D>(rows, row_stride)),
                           (uint32_t)(l >> 2) * row_stride + (l & 3) * (D / 8));
    x.s = __builtin_amdgcn_raw_buffer_load_b32(rsrc_of(scales + ((((uint64_t)(uint32_t)id * (uint32_t)a.h_kv + r) << a.page_log) + off) * (D / 32), scale_span<D>(rows)), scale_word<D>(l >> 2), 0, 0);
  };
  int id_v = 0, id_k = 0;                                     // pages of tile i + 1 (its V is asked for) and of tile i + 2 (its K)
  auto id_of = [&](int tile) { return __builtin_amdgcn_readlane(win, (((tile * 64 + row0) >> a.page_log) - wbase) & 63); };
  // of a lane's first chunk; chunk i lies at that address with bits 4 and 5 flipped by i (the ring begins at a multiple of 1024)
  uint32_t k_wr, v_wr;
  {
    const int row = row0 + (lane >> 2), c = C::CW * (lane & 3);
    k_wr = lds0 + (uint32_t)(row * C::ROW_BYTES + ((c ^ pk_swz<D>(row)) << 4));
    v_wr = lds0 + (uint32_t)(2 * C::TILE_BYTES + row * C::ROW_BYTES + ((c ^ v4_swz<D>(row)) << 4));
  }
  uint64_t* nan_blocks = reinterpret_cast<uint64_t*>(lds + 4 * C::TILE_BYTES);   // [slot][wave]: lanes whose block of V is NaN
  Raw kr, vr;
  float k_sc = 0.f, v_sc = 0.f;
  auto conv = [&](uint32_t to, const Raw& x, float scale, int c, int slot) {
    lds_write_b128(flipped(to, c << 4) + slot * C::TILE_BYTES, fp4_to_bf16(x.c.w[c], scale));
  };
  auto conv_k = [&](int c, int slot) { conv(k_wr, kr, k_sc, c, slot); };
  auto conv_v = [&](int c, int slot) { conv(v_wr, vr, v_sc, c, slot); };
  // ---- operand addresses in LDS, of slot 0 --------------------------------------------------------------------
  const uint32_t k_rd0 = lds0 + (uint32_t)(n * C::ROW_BYTES + ((h ^ pk_swz<D>(n)) << 4));   // d slice ks: bits 5 .. flipped by ks
  const int s16 = lane & 15, a16 = (lane >> 4) & 1;
  const uint32_t v_rd0 = lds0 + (uint32_t)((4 * h + (s16 >> 2)) * C::ROW_BYTES + (((2 * a16 + ((s16 & 3) >> 1)) ^ v4_swz<D>(s16 >> 2)) << 4) + ((s16 & 1) << 3));

  float m_run = -INFINITY, l_run = 0.f;
  constexpr int NDT = D / 32;
  f32x16 oacc[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; dt++)
#pragma unroll
    for (int j = 0; j < 16; j++) oacc[dt][j] = 0.f;
  id_k = id_of(first);
  ask(kr, kb, a.kp_p, k_t, a.k_sc, id_k, first);
  ask(vr, vb, a.vp_p, v_t, a.v_sc, id_k, first);
  k_sc = fp4_scale(scale_of(kr));
#pragma unroll
  for (int c = 0; c < C::CW; c++) conv_k(c, 0);
  id_v = id_k = id_of(first + 1);
  ask(kr, kb, a.kp_p, k_t, a.k_sc, id_k, first + 1);
  // Iteration i, LDS: tile i lives in slot i & 1 of both rings, V one iteration behind K.  The barrier at its top makes everybody's tiles visible (K of
  // tile i, V of tile i - 1) and retires the reads of iteration i - 1, whose slots this iteration writes over with what it converts: K of tile
  // i + 1 and V of tile i, a word of codes at a time between the MFMAs.  Their registers then take K of tile i + 2 and V of tile i + 1.
  // A wave's priority rises from the first product to the second: the waves of a SIMD, of several workgroups, fall out of step (2048 tokens against 32k 1060 -> 1000 us, at
  // head dimension 64 655 -> 624; raised in the second alone 1002 and 646).
  int pend = 0;
  float tmax_old = 0.f;
  auto iteration = [&](auto p_tag, int i, f32x16 (&s)[2], f32x16 (&so)[2]) __attribute__((always_inline)) {
    constexpr int P = decltype(p_tag)::value;
    constexpr int NS = D / 8, KAHEAD = D == 64 ? 3 : 4, VAHEAD = 2, EQ = D == 64 ? 16 : 12, E0 = D == 64 ? 0 : 2;
    const bool cur = i < n_it;
    const int tile = first + i;
    const bool on = cur && tile * 64 < wave_end;
    if (((tile + 2) * 64 >> a.page_log) - wbase >= 64) {
      wbase += 64;
      win = win_next;
      win_next = window(wbase + 64);
    }
    id_v = id_k;
    id_k = id_of(tile + 2);
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
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    k_sc = fp4_scale(scale_of(kr));
    const uint32_t vs = scale_of(vr);
    v_sc = __uint_as_float(vs == 255u ? 0u : vs << 23);        // a block that is NaN goes in as numbers next to 0: the rows that see it get NaN below
    if (lane == 0) nan_blocks[P * 4 + wave] = 0;
    if (const uint64_t bad = __ballot(vs == 255u); __builtin_expect(bad != 0, 0)) {
      if (lane == 0) nan_blocks[P * 4 + wave] = bad;
    }
    auto k_read = [&](int x) -> bf16x8 {   // slot x: d slice x / 2, key half x % 2
      return lds_read_b128(flipped(k_rd0, (x >> 1) << 5) + (uint32_t)(P * C::TILE_BYTES + (x & 1) * 32 * C::ROW_BYTES));
    };
    auto v_read = [&](int x) -> bf16x8 {   // slot x: contraction step x / NDT, d-tile x % NDT
      const uint32_t at = flipped(v_rd0, (x % NDT) << 6) + (uint32_t)((2 + (P ^ 1)) * C::TILE_BYTES + 16 * (x / NDT) * C::ROW_BYTES);
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
    auto next_k = [&]() { ask(kr, kb, a.kp_p, k_t, a.k_sc, id_k, tile + 2); };
    auto next_v = [&]() { ask(vr, vb, a.vp_p, v_t, a.v_sc, id_v, tile + 1); };
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
        int lim = last_key() - (tile * 64 + ((paged_thread() & 32) >> 3));
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
        if (x % 4 == 0 && x / 4 < C::CW) conv_k(x / 4, P ^ 1);
        if (x % 4 == 2 && x / 4 < C::CW) conv_v(x / 4, P);
        if constexpr (NS == 16) { if (x >= 4 && x < 12) max_quad(x - 4); }
        else if (x >= 4) { max_quad(2 * (x - 4)); max_quad(2 * (x - 4) + 1); }
        __builtin_amdgcn_sched_barrier(0);
      }
      l_run += l_tile;
      const uint64_t bad = nan_blocks[(P ^ 1) * 4 + (lane & 3)];
      if (__builtin_expect(__any(bad != 0), 0)) {              // of tile i - 1
        const int last = last_key();
        for (int w = 0; w < 4; w++)
          for (uint64_t left = nan_blocks[(P ^ 1) * 4 + w]; left; left &= left - 1) {
            const int l = __builtin_ctzll(left), block = (l & 3) * (D / 4) / 32;
            const bool sees = (tile - 1) * 64 + 16 * w + (l >> 2) <= last;
#pragma unroll
            for (int dt = 0; dt < NDT; dt++)
#pragma unroll
              for (int j = 0; j < 16; j++) oacc[dt][j] = dt == block && sees ? NAN : oacc[dt][j];
          }
      }
    };
    if (on) {
      __builtin_amdgcn_s_setprio(1);
      if (pend) first_product(std::true_type{});
      else first_product(std::false_type{});
      mask_keys();
    } else {
      asm volatile("" : "=v"(s[0]), "=v"(s[1]));               // nobody reads them
      if (pend) {
#pragma unroll
        for (int x = 0; x < VAHEAD; x++) vf[x] = v_read(x);
#pragma unroll
        for (int k = 0; k < EQ; k++) e_pair(k);
      }
    }
    if (pend) {
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(2);
      second_product();
      __builtin_amdgcn_s_setprio(0);
    } else if (cur) {
#pragma unroll
      for (int c = 0; c < C::CW; c++) { conv_k(c, P ^ 1); conv_v(c, P); }
    }
    if (cur) { next_k(); next_v(); }
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
  const float l_tot = l_run + __shfl_xor(l_run, 32);
  {
  const int lane = paged_thread() & 63, n = lane & 31, h = lane >> 5, t = tw0 + n / a.g, head = r * a.g + n % a.g;   // not kept through the walk
  const bool row_ok = t < it.m;
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
}

// ---- host ------------------------------------------------------------------------------------------------------------
// fp32: 512 threads for an item, fewer than 2^32 in all, as paged_attend_fits
bool paged4_attend_fits(const PagedArgs& a, int dtype) { return dtype != DASH_F32 || paged_most_items(a, 16) * a.h_kv < (1 << 23); }
// Workgroups of a kv-head that are resident at once: two a CU at head dimension 128, three at 64 (of 16-row tiles, of which four are, three runs a CU are as fast:
// 32 sequences of 4096 to 32768 75.7 us, four 76.3).
static int runs_of(const PagedArgs& a, int dtype, int d) { return max((dtype == DASH_F32 ? 256 : d == 128 ? 512 : 768) / a.h_kv, 1); }
// Rows of a call's tiles.  128 where the sequences bring more than 80 each on the average, but for short caches, as for pages of bf16; else 32 where they bring
// more than 16 and there are tiles for every fourth run, so that few are cut into many pieces, whose records grow with a tile's rows; else 16.
// (Tiles of 16, of 32 and of 128.  32 / 8 heads of 128, sequences of 3000 to 16000.  One of 20 rows: 19.4, 25.2, 22.8 us.  8 of 32 rows: 35.7, 37.1, 55.2; 64 rows: 56.6, 47.0,
// 59.0; 80: 68.4, 62.9, 62.6.  24 of 20: 84.8, 65.5, 173; 48: 118, 112, 182; 64: 150, 110, 183.  16 of 80: 127, 109, 121.  64 of 2000 tokens, 48 rows: 72.8, 62.4, 78.3; 80: 113,
// 89.4, 83.0.  Heads in a group of 16, two kv-heads, 8 sequences: 32 rows 22.7, 29.1, 25.9, 64 26.0, 31.7, 29.2, 96 30.6, 35.2, 31.3.  Head
// dimension 64, 8 sequences: 48 rows 34.2, 34.6, 39.8, 64 41.2, 34.6, 40.2; 32 sequences, 64 rows: 120, 88.7, 128.)
// Short caches: 16 while there are few tiles, each of which has a CU then.  (Caches of 1000 tokens.  12 of 20 rows, 192 tiles of 16, 12.3 and 16.3 us; 40 of 32, 640 of them, 24.5
// and 19.8.)
static int tile_rows(const PagedArgs& a, int dtype, int d) {
  const int64_t rows = (int64_t)a.n_rows * a.g;
  const int64_t few = a.cap <= 8 * kStep ? paged_most_items(a, 16) * a.h_kv : INT64_MAX;   // tiles of 16 rows of a short cache
  if (dtype != DASH_BF16) return 16;
  if (rows > (int64_t)a.batch * 80 && few > 256) return 128;
  return rows > (int64_t)a.batch * 16 && few > 384 && paged_most_items(a, 32) * 4 >= runs_of(a, dtype, d) ? 32 : 16;
}
static size_t ws_align(size_t x) { return (x + 255) & ~(size_t)255; }

size_t paged4_attend_ws(const PagedArgs& a, int dtype, int d) {
  const size_t few = (size_t)runs_of(a, dtype, d) * a.h_kv * 2 * 16;         // rows of records; with tiles of 32 twice as many, fewer than `rows`
  const size_t rows = dtype == DASH_BF16 ? (size_t)paged_most_parts(runs_of(a, dtype, d)) * a.h_kv * 128 : 0, recs = few > rows ? few : rows;
  return ws_align(recs * 8) + recs * d * 4 + few / 16 * 16;                      // two flags a record of 16 rows
}

template <int D, int G> static hipError_t launch_few4(const PagedArgs& a, dim3 grid, hipStream_t st) {
  constexpr int lds = Few4Cfg<D, 16 * G>::LDS_BYTES;
  static LdsOptIn opt_in;
  if (hipError_t e = allow_dyn_lds((const void*)(paged_few4_kernel<D, G>), lds, opt_in); e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_few4_kernel<D, G>), grid, dim3(256), lds, st, a);
  return hipSuccess;
}

// A launch of tiles of `tile` rows, and where they are of 128 and cut the one that adds up the parts.  items: at most so many of a kv-head.
template <int D>
static hipError_t launch_tiles4(PagedArgs a, int dtype, int tile, int64_t items, char* ws, hipStream_t st) {
  const bool big = tile == 128;
  const int runs = runs_of(a, dtype, D);
  a.wgs = items < (big ? 2 : 8) * (int64_t)runs ? runs : 0;
  if (big && a.wgs && items * 4 >= runs) a.wgs = (int)items + runs * 3 / 2;
  a.slots = runs;
  a.gain = (int64_t)a.n_rows * a.g < 64 * items ? 0.65f : 0.9f;
  // An item's start (and the end of the piece before it) takes as long as so many steps.  (0, 3, 4, 8 of them: one token of 8 sequences of 384 to 16000 25.7, 23.1, 22.3 and
  // 23.0 us, of 32 of 4096 to 32768 129.0, 127.6, 127.2 and 126.1; of 8 of one length, where all runs begin with an item, 20.3, 20.9, 21.2 and 21.2.)
  a.pad = 4;
  a.whole = items * 2 >= runs;                               // fewer items: not looked into
  if (!big && a.cap <= 8 * kStep && items * a.h_kv >= 128) a.wgs = 0;
  const size_t recs = (size_t)a.wgs * a.h_kv * (big ? 128 : 2 * tile);
  a.part_ml = (float*)ws;
  a.part_o = (float*)(ws + ws_align(recs * 8));
  a.flags = (uint64_t*)((char*)a.part_o + recs * D * 4);     // runs only
  a.nonce = big ? 0 : next_nonce();
  const dim3 grid((unsigned)((a.wgs ? a.wgs : items) * a.h_kv));
  if (big) {
    static LdsOptIn opt_in;
    if (hipError_t e = allow_dyn_lds((const void*)paged_rows4_kernel<D>, Rows4Cfg<D>::LDS_BYTES, opt_in); e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_rows4_kernel<D>, grid, dim3(256), Rows4Cfg<D>::LDS_BYTES, st, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || a.wgs <= 1 ? e : launch_paged4_merge(a, D, st);
  }
  if (dtype == DASH_BF16) {
    if (hipError_t e = tile == 32 ? launch_few4<D, 2>(a, grid, st) : launch_few4<D, 1>(a, grid, st); e != hipSuccess) return e;
  } else {
    constexpr int lds = 8 * 16 * (D + 6) * 4;
    static LdsOptIn opt_in;
    if (hipError_t e = allow_dyn_lds((const void*)(paged_few_f32_kernel<D, true>), lds, opt_in); e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_few_f32_kernel<D, true>), grid, dim3(512), lds, st, a);
  }
  return hipGetLastError();
}

// Tiles of 128 rows: in a batch, the sequences of up to 48 rows, of which such a tile would be mostly empty, have a launch of their own, of tiles of 16, in front of it.
// (32 / 8 heads of 128, a piece of a prompt beside 31 sequences of 900 to 11777 with a token each: 1000 tokens 343 us in one launch, 271 in two, 1501 578 and 393;
// beside seven: 300 107 and 100, 600 179 and 159, 1501 349 and 361, where the sequences of one token filled what the prompt's tiles leave, at head dimension 64 219 and
// 204.  Where all bring more, a launch for nothing: 8 sequences of 24 tokens 61.6 and 64.2, 16 of 32 130 and 132.)
constexpr int kFewRows = 48;
template <int D>
static hipError_t launch_attend4(PagedArgs a, int dtype, char* ws, hipStream_t st) {
  const int tile = tile_rows(a, dtype, D);
  if (tile == 128 && a.batch > 1) {
    a.few = kFewRows / a.g;
    const int64_t items = min(paged_most_items(a, 16), (int64_t)a.batch * (kFewRows / 16));
    if (hipError_t e = launch_tiles4<D>(a, dtype, 16, items, ws, st); e != hipSuccess) return e;
    a.few = -a.few;
  }
  return launch_tiles4<D>(a, dtype, tile, paged_most_items(a, tile), ws, st);
}

hipError_t launch_paged4_attend(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st) {
  return d == 128 ? launch_attend4<128>(a, dtype, ws, st) : launch_attend4<64>(a, dtype, ws, st);
}

}  // namespace dash
