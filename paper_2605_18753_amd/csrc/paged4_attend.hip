// Attention of packed new tokens over a paged cache in 4 bits (fp4.h): the walks of paged_attend.hip, whose dealing and joining they use.
//
// Few rows: a tile is 16 (token, head) rows.  K goes from the pages into registers: the contraction over d runs in the order in which a lane's
// codes lie, d = D / 4 kq + .., so 16 bytes of a row are one load, one scale and, converted, the lane's operands of all steps.  V is converted into LDS, from
// where transposing reads give its operands.  The next tile's loads are in flight while a tile is worked on.
#include "fp4.h"
#include "paged_few.h"

namespace dash {

template <int D> struct Few4Cfg {
  static constexpr int CW = D / 32;                        // words of a lane's codes: a quarter of a row
  static constexpr int ROW_BYTES = D * 2, TILE_BYTES = 32 * ROW_BYTES;   // V of 32 keys in bf16
  static constexpr int OUT_BYTES = 4 * 16 * (D + 6) * 4;   // the waves' results, behind the walk
  static constexpr int LDS_BYTES = 4 * TILE_BYTES > OUT_BYTES ? 4 * TILE_BYTES : OUT_BYTES;
};
// Position of 16-byte chunk c of V's row: 4 rows x 2 chunks (transposing reads) and 2 rows x 4 chunks a quarter of a row apart (writes) spread over
// all banks.
template <int D> __device__ __forceinline__ int v4_swz(int row) { return D == 128 ? ((row & 3) << 2) | (row & 1) : ((row >> 1) & 1) << 2; }

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32v4 __attribute__((ext_vector_type(4)));
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
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00020000);
}
__device__ __forceinline__ void lds_write_b128(uint32_t addr, bf16x8 x) {
  *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>(addr) = x;
}

template <int D>
__global__ __launch_bounds__(256, 3) void paged_few4_kernel(PagedArgs args) {
  using C = Few4Cfg<D>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int r = blockIdx.x % args.h_kv, wg = blockIdx.x / args.h_kv;
  PagedRun run(args);
  if (!run.begin(args, wg)) return;
  const PagedItem& it = run.it;
  do {
  const PagedArgs a = paged_reload();
  const int tid = paged_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = 16 / a.g;
  const int t0 = it.tile * T;
  const int n = lane & 15, kq = lane >> 4;
  const int t = t0 + n / a.g;
  bf16x8 qf[D / 32];
  {
    const uint16_t* qp = (const uint16_t*)a.q + (it.r0 + min(t, it.m - 1)) * a.q_t + (r * a.g + n % a.g) * a.q_h + kq * (D / 4);
#pragma unroll
    for (int s = 0; s < D / 32; s++) qf[s] = *reinterpret_cast<const bf16x8*>(qp + 8 * s);
  }
  const int last = t < it.m ? paged_last_key(a, it, t) : -1;
  const int first_last = paged_last_key(a, it, t0);                              // of the tile's first token
  const int end = max(paged_last_key(a, it, min(t0 + T, it.m) - 1) + 1, 0);      // keys that a row of the tile sees
  // the wave's 32-key tiles of the piece's 128-key steps
  const int j1 = min(run.x1 * 4, (end + 31) >> 5);
  int j = run.x0 * 4 + wave;

  const uint32_t buf = lds_addr_of(lds) + wave * C::TILE_BYTES;
  const uint32_t kt = (uint32_t)a.kp_t, vt = (uint32_t)a.vp_t;
  // K: row n, quarter kq; V: row lane / 4, quarter lane % 4
  const uint32_t k_off = (uint32_t)n * kt + kq * (D / 8), v_off = (uint32_t)(lane >> 2) * vt + (lane & 3) * (D / 8);
  const uint32_t ks_off = (uint32_t)(n * (D / 32) + kq * (D / 4) / 32), vs_off = (uint32_t)((lane >> 2) * (D / 32) + (lane & 3) * (D / 4) / 32);
  const char* kb = (const char*)a.k + r * a.kp_h;
  const char* vb = (const char*)a.v + r * a.vp_h;
  const int pm = (1 << a.page_log) - 1;
  // the pages of a tile: one, or two of 16 tokens
  auto pages_of = [&](int tile) {
    return make_int2(paged_page(a, it.b, (tile * 32) >> a.page_log), paged_page(a, it.b, (tile * 32 + 16) >> a.page_log));
  };
  struct Raw { Codes<C::CW> k[2], v[2]; uint32_t ks[2], vs[2]; };
  // A resource ends with the sequence's last token: rows behind it read as zeros, whatever their page holds.
  auto load = [&](int tile, int2 pg, Raw& x) {
#pragma unroll
    for (int half = 0; half < 2; half++) {
      const int key = tile * 32 + half * 16, id = half ? pg.y : pg.x, rows = min(max(it.n - key, 0), 16);
      const int64_t at = ((((int64_t)id * a.h_kv + r) << a.page_log) + (key & pm)) * (D / 32);
      x.k[half] = load_codes<C::CW>(rsrc_of(kb + (int64_t)id * a.kp_p + (int64_t)(key & pm) * a.kp_t, rows ? (rows - 1) * (int)kt + D / 2 : 0), k_off);
      x.v[half] = load_codes<C::CW>(rsrc_of(vb + (int64_t)id * a.vp_p + (int64_t)(key & pm) * a.vp_t, rows ? (rows - 1) * (int)vt + D / 2 : 0), v_off);
      x.ks[half] = __builtin_amdgcn_raw_buffer_load_b8(rsrc_of(a.k_sc + at, rows * (D / 32)), ks_off, 0, 0);
      x.vs[half] = __builtin_amdgcn_raw_buffer_load_b8(rsrc_of(a.v_sc + at, rows * (D / 32)), vs_off, 0, 0);
    }
  };
  uint32_t v_wr[C::CW];
#pragma unroll
  for (int i = 0; i < C::CW; i++) v_wr[i] = buf + (uint32_t)((lane >> 2) * C::ROW_BYTES + ((C::CW * (lane & 3) + i) ^ v4_swz<D>(lane >> 2)) * 16);
  // transposing read of V: lane s of a group of 16 points at row 4 kq + s / 4 (+ 16), d 4 (s % 4) of the 16-wide d-tile
  uint32_t v_rd[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; dt++)
    v_rd[dt] = buf + (uint32_t)((4 * kq + (n >> 2)) * C::ROW_BYTES + (((2 * dt + ((n & 3) >> 1)) ^ v4_swz<D>(n >> 2)) << 4) + ((n & 1) << 3));

  float m_run = -INFINITY, l_run = 0.f;
  f32x4 oacc[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; dt++) oacc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

  Raw next;
  int2 pg = make_int2(0, 0);
  if (j < j1) {
    load(j, pages_of(j), next);
    pg = pages_of(j + 4);
  }
  for (; j < j1; j += 4) {
    const Raw x = next;
    if (j + 4 < j1) {
      load(j + 4, pg, next);
      pg = pages_of(j + 8);
    }
    // values of a block that is NaN go in as zeros; the rows that see its token get NaN below
#pragma unroll
    for (int half = 0; half < 2; half++) {
      const float sc = x.vs[half] == 255u ? 0.f : __uint_as_float(x.vs[half] << 23);
#pragma unroll
      for (int i = 0; i < C::CW; i++)
        lds_write_b128(v_wr[i] + half * 16 * C::ROW_BYTES, fp4_to_bf16(x.vs[half] == 255u ? 0u : x.v[half].w[i], sc));
    }
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;                                    // lane (row n, kq): keys 4 kq + i, 16 + 4 kq + i
    const float k0 = fp4_scale(x.ks[0]), k1 = fp4_scale(x.ks[1]);
#pragma unroll
    for (int s = 0; s < D / 32; s++) {
      s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp4_to_bf16(x.k[0].w[s], k0), qf[s], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp4_to_bf16(x.k[1].w[s], k1), qf[s], s1, 0, 0, 0);
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
    asm volatile("" ::: "memory");                                               // a wave's LDS operations complete in order
#pragma unroll
    for (int dt = 0; dt < D / 16; dt++)
      oacc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lds_read_tr_pair(v_rd[dt], v_rd[dt] + 16 * C::ROW_BYTES), pb, oacc[dt], 0, 0, 0);
    asm volatile("" ::: "memory");
    if (__builtin_expect(__any(x.vs[0] == 255u || x.vs[1] == 255u), 0)) {
#pragma unroll
      for (int half = 0; half < 2; half++)
        for (uint64_t bad = __ballot(x.vs[half] == 255u); bad; bad &= bad - 1) {
          const int l = __builtin_ctzll(bad), block = (l & 3) * (D / 4) / 32;
          const bool seen = j * 32 + half * 16 + (l >> 2) <= last;
#pragma unroll
          for (int dt = 0; dt < D / 16; dt++)
            if (dt >> 1 == block && seen) oacc[dt] = f32x4{NAN, NAN, NAN, NAN};
        }
    }
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

// ---- host ------------------------------------------------------------------------------------------------------------
static int64_t most_items(const PagedArgs& a, int rows) {   // of a kv-head
  const int T = rows / a.g;
  return min((int64_t)a.n_rows / T + min(a.batch, a.n_rows), (int64_t)a.n_rows);
}
// fp32: 512 threads for an item, fewer than 2^32 in all, as paged_attend_fits
bool paged4_attend_fits(const PagedArgs& a, int dtype) { return dtype != DASH_F32 || most_items(a, 16) * a.h_kv < (1 << 23); }
// Workgroups of a kv-head that are resident at once.
static int runs_of(const PagedArgs& a, int dtype) { return max((dtype == DASH_F32 ? 256 : 768) / a.h_kv, 1); }
static size_t ws_align(size_t x) { return (x + 255) & ~(size_t)255; }

size_t paged4_attend_ws(const PagedArgs& a, int dtype, int d) {
  const size_t recs = (size_t)runs_of(a, dtype) * a.h_kv * 2 * 16;               // rows of records
  return ws_align(recs * 8) + recs * d * 4 + recs / 16 * 16;                     // two flags a record of 16 rows
}

template <int D>
static hipError_t launch_attend4(PagedArgs a, int dtype, char* ws, hipStream_t st) {
  const int runs = runs_of(a, dtype);
  const int64_t items = most_items(a, 16);
  a.wgs = items < 8 * (int64_t)runs ? runs : 0;
  a.slots = runs;
  a.whole = items * 2 >= runs;                               // fewer items: not looked into
  if (a.cap <= 8 * kStep && items * a.h_kv >= 128) a.wgs = 0;
  const size_t recs = (size_t)a.wgs * a.h_kv * 2 * 16;
  a.part_ml = (float*)ws;
  a.part_o = (float*)(ws + ws_align(recs * 8));
  a.flags = (uint64_t*)((char*)a.part_o + recs * D * 4);
  a.nonce = next_nonce();
  const dim3 grid((unsigned)((a.wgs ? a.wgs : items) * a.h_kv));
  if (dtype == DASH_BF16) {
    static LdsOptIn opt_in;
    if (hipError_t e = allow_dyn_lds((const void*)paged_few4_kernel<D>, Few4Cfg<D>::LDS_BYTES, opt_in); e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_few4_kernel<D>, grid, dim3(256), Few4Cfg<D>::LDS_BYTES, st, a);
  } else {
    constexpr int lds = 8 * 16 * (D + 6) * 4;
    static LdsOptIn opt_in;
    if (hipError_t e = allow_dyn_lds((const void*)(paged_few_f32_kernel<D, true>), lds, opt_in); e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_few_f32_kernel<D, true>), grid, dim3(512), lds, st, a);
  }
  return hipGetLastError();
}

hipError_t launch_paged4_attend(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st) {
  return d == 128 ? launch_attend4<128>(a, dtype, ws, st) : launch_attend4<64>(a, dtype, ws, st);
}

}  // namespace dash
