// What the attention kernels over a paged cache share, whatever its pages hold: a row's visible keys, how the waves of a workgroup and the
// pieces of a cut item are added up, and the fp32 kernel.
#pragma once
#include <math.h>

#include <type_traits>

#include "f32_tiles.h"
#include "fp4.h"
#include "lds_copy.h"
#include "paged.h"

namespace dash {

typedef uint32_t u32v4 __attribute__((ext_vector_type(4)));
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kPagedLazy = 8.f;        // slack of the running maximum, in base-2 logit units: exponentials stay below 2^8

// chunk permutations of the LDS tiles (position of 16-byte chunk c of row `row`): 16 consecutive rows at one chunk (operand of the
// first product) and 4 rows x 4 chunks (transposing read) each spread over all banks
template <int D> __device__ __forceinline__ int pk_swz(int row) { return D == 128 ? (row & 15) : ((row >> 1) & 7); }
template <int D> __device__ __forceinline__ int pv_swz(int row) { return D == 128 ? ((row & 3) << 2) : (((row >> 1) & 1) << 2); }

// a row's last visible slot, -1: none
template <typename I> __device__ __forceinline__ int paged_last_key(const PagedArgs& a, const I& it, int t) {
  return a.causal ? min(it.n - it.m + t, it.n - 1) : it.n - 1;
}

// 4 values of an output row
__device__ __forceinline__ void put_row4(uint16_t* p, f32x4 o, float inv) {
  uint2 y;
  y.x = cvt_bf16x2(o[0] * inv, o[1] * inv);
  y.y = cvt_bf16x2(o[2] * inv, o[3] * inv);
  *reinterpret_cast<uint2*>(p) = y;
}
__device__ __forceinline__ void put_row4(float* p, f32x4 o, float inv) { *reinterpret_cast<f32x4*>(p) = o * inv; }

// Records of a launch's pieces, ROWS rows of D floats each, past the caches as agent_store and agent_load, 16 bytes at a time.
template <int D, int ROWS> struct PagedRecords {
  static constexpr int AGENT = 16;                           // scope of the access: the device (sc1)
  __amdgpu_buffer_rsrc_t rs;
  __device__ __forceinline__ PagedRecords(const PagedArgs& a)
      : rs(__builtin_amdgcn_make_buffer_rsrc(a.part_o, 0, a.wgs * a.h_kv * (2 * ROWS * D * 4), 0x00020000)) {}
  __device__ __forceinline__ uint32_t place(int64_t rec, int row, int c) const { return (((uint32_t)rec * ROWS + row) * D + c) * 4; }
  __device__ __forceinline__ void store(uint32_t at, f32x4 x) const { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32v4, x), rs, at, 0, AGENT); }
  __device__ __forceinline__ f32x4 load(uint32_t at) const { return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, AGENT)); }
};

// What the waves hold of a tile's ROWS rows is added up in LDS, and written as the output or as a record of the piece.
// x: [WAVES][ROWS][D + 4] floats, ml: [WAVES][ROWS][2].  Of the first 256 threads, 16 i .. + 15 hold row i, row 16 + i ..
template <typename T, int D, int WAVES, int ROWS = 16, bool FOUR>
__device__ __forceinline__ void paged_few_finish(const PagedArgs& a, const PagedRun<FOUR>& run, int r, int64_t rec, int t0, const float* x, const float* ml) {
  const PagedItem& it = run.it;
  const int c = threadIdx.x & 15;
#pragma unroll
  for (int row = threadIdx.x >> 4, rows = 0; rows < ROWS; row += 16, rows += 16) {
  if (WAVES > 4 && row >= ROWS) return;
  float M = -INFINITY, den = 0.f, w[WAVES];
#pragma unroll
  for (int i = 0; i < WAVES; i++) M = fmaxf(M, ml[(i * ROWS + row) * 2]);
  const float use = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int i = 0; i < WAVES; i++) {
    w[i] = __builtin_amdgcn_exp2f(ml[(i * ROWS + row) * 2] - use);
    den = fmaf(w[i], ml[(i * ROWS + row) * 2 + 1], den);
  }
  float o[D / 16];
#pragma unroll
  for (int j = 0; j < D / 64; j++) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < WAVES; i++) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(x + (i * ROWS + row) * (D + 4) + j * 64 + c * 4);
#pragma unroll
      for (int e = 0; e < 4; e++) s[e] = fmaf(w[i], y[e], s[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; e++) o[j * 4 + e] = s[e];
  }
  const int t = t0 + row / a.g, head = r * a.g + row % a.g;
  if (t >= it.m) return;
  if (!run.whole()) {
    const PagedRecords<D, ROWS> recs(a);
#pragma unroll
    for (int j = 0; j < D / 64; j++) recs.store(recs.place(rec, row, j * 64 + c * 4), f32x4{o[j * 4], o[j * 4 + 1], o[j * 4 + 2], o[j * 4 + 3]});
    if (c == 0) agent_store(a.part_ml + (rec * ROWS + row) * 2, M, den);
    continue;
  }
  const float inv = den > 0.f ? 1.f / den : den == 0.f ? 0.f : den;     // NaN stays
  T* op = (T*)a.o + (it.r0 + t) * a.o_t + head * a.o_h;
#pragma unroll
  for (int j = 0; j < D / 64; j++)
    put_row4(op + j * 64 + c * 4, f32x4{o[j * 4], o[j * 4 + 1], o[j * 4 + 2], o[j * 4 + 3]}, inv);
  if (a.lse && c == 0) a.lse[(int64_t)(it.r0 + t) * a.h_q + head] = den == 0.f ? -INFINITY : (M + log2f(den)) * kLn2;
  }
}

// Partial results of a row (maximum m of the base-2 logits, sum, 4 values of the product) added one by one: what has to be loaded of
// them can be asked for together.
struct PagedSum {
  float m = -INFINITY, den = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void add(float m2, float den2, f32x4 o2) {
    const float top = fmaxf(m, m2), use = top == -INFINITY ? 0.f : top;
    const float w = __builtin_amdgcn_exp2f(m - use), w2 = __builtin_amdgcn_exp2f(m2 - use);
    m = top;
    den = fmaf(w2, den2, w * den);
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] = fmaf(w2, o2[e], w * o[e]);
  }
};

// Behind a piece of an item that is cut between runs: o = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p, by the workgroup that sees the flags
// of all its pieces.  They are those of runs w1, w1 + 1, ..; the first left its run's second record, the others their runs' first.  D / 4 threads
// a row, 4 values each, and where the item has few rows several groups of threads that take every so manieth piece.  (A launch of its
// own for this: one sequence of 1000 tokens, 32 / 8 heads, 11.1 us a step instead of 9.3.)
// Where a thread would have more than kChain records to add one after the other, two levels: groups of 8 or 16 pieces, each added up by a workgroup
// that sees its flags into a record that nobody uses (the second of a run in the middle of the item), then the groups.  More than one workgroup
// may see all flags; they write the same.  A second flag says that a piece's workgroup is done with its group: who sees all of these adds
// up the groups and clears the flags, none of which is set after that.  (16 heads on one, one sequence of 16000 tokens, 125 pieces: 92 us in one
// level, 20 in two; 32 on 8, 1000 tokens, 8 pieces: 11 in two, 9.3 in one.)
constexpr int kChain = 24;
template <typename T, int D, int THREADS, int ROWS = 16, bool FOUR>
__device__ __forceinline__ void paged_few_join(const PagedArgs& a, const PagedRun<FOUR>& run, int r, int wg, char* lds) {
  constexpr int TPR = D / 4, UNITS = THREADS / TPR;        // threads of a row; rows at a time
  const PagedItem& it = run.it;
  f32x4* xo = reinterpret_cast<f32x4*>(lds);               // [THREADS], [UNITS][2], [1]
  float* xd = reinterpret_cast<float*>(xo + THREADS);
  int* all = reinterpret_cast<int*>(xd + 2 * UNITS);
  const int lane = threadIdx.x & 63, begin = run.next - run.x1, end = begin + run.cost;
  const PagedBounds<int> bounds(a, run.total, run.deal.pad);
  int w1 = wg, pieces = 1;
  for (int k0 = wg; k0 > 0; k0 -= 64) {
    const int more = __popcll(__ballot(k0 - lane > 0 && bounds.at(max(k0 - lane, 0)) > begin));
    w1 -= more;
    pieces += more;
    if (more < 64) break;
  }
  for (int k0 = wg + 1; k0 < bounds.runs; k0 += 64) {
    const int more = __popcll(__ballot(k0 + lane < bounds.runs && bounds.at(k0 + lane) < end));
    pieces += more;
    if (more < 64) break;
  }
  const int64_t rec0 = ((int64_t)r * a.wgs + w1) * 2;
  auto record = [&](int p) { return p == 0 ? rec0 + 1 : rec0 + 2 * p; };
  uint64_t* done = a.flags + (int64_t)a.wgs * a.h_kv * 2;
  // sets the flag of this piece, behind all that the workgroup has stored, and tells whether those of pieces p0 .. p1 - 1 are set
  auto complete = [&](uint64_t* flags, int p0, int p1) -> bool {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the record is in memory ...
    __syncthreads();
    if (threadIdx.x < 64) {
      if (lane == 0) __hip_atomic_store(flags + record(wg - w1), a.nonce, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // ... before its flag, and that before the flags are read
      bool seen = true;
      for (int p = p0 + lane; p < p1; p += 64) seen &= agent_load(flags + record(p)) == a.nonce;
      const bool ok = __all(seen);
      if (lane == 0) *all = ok;
    }
    __syncthreads();
    return *all;
  };
  const int rows = min(run.deal.T, it.m - it.tile * run.deal.T) * a.g;
  const int slices = rows * 4 <= UNITS ? 4 : rows * 2 <= UNITS ? 2 : 1, per = UNITS / slices;
  const int c = threadIdx.x % TPR, unit = threadIdx.x / TPR, slice = unit / per;
  const PagedRecords<D, ROWS> recs(a);
  // adds up `count` records, place(i) the i-th; write(row, sum) by the threads that hold a row's sum
  auto add_up = [&](int count, auto&& place, auto&& write) {
    // rows of a thread, and records, asked for together; and as many records again where there are more.  (Two rows: no faster over pages of bf16, in fp32 33.3 us for 32.9.)
    constexpr int RG = FOUR ? D / 64 : 1, KP = 4;
    for (int i0 = 0; i0 < rows; i0 += per * RG) {
      PagedSum sum[RG];
      for (int p0 = 0; p0 < count; p0 += 2 * KP * slices) {
        uint64_t y[RG][2 * KP];
        f32x4 v[RG][2 * KP];
#pragma unroll
        for (int g = 0; g < RG; g++)
#pragma unroll
          for (int k0 = 0; k0 < 2 * KP; k0 += KP) {
            if ((g && i0 + per >= rows) || (k0 && p0 + KP * slices >= count)) continue;
            const int in = min(i0 + g * per + unit % per, rows - 1);
            const float* ml = a.part_ml + in * 2;
#pragma unroll
            for (int k = k0; k < k0 + KP; k++) {             // behind the last one it again
              const int64_t at = place(min(p0 + slice + k * slices, count - 1));
              y[g][k] = agent_load(ml + at * (2 * ROWS));
              v[g][k] = recs.load(recs.place(at, in, c * 4));
            }
          }
#pragma unroll
        for (int g = 0; g < RG; g++)
#pragma unroll
          for (int k = 0; k < 2 * KP; k++)
            if (p0 + slice + k * slices < count && (g == 0 || i0 + per < rows))
              sum[g].add(__uint_as_float((uint32_t)y[g][k]), __uint_as_float((uint32_t)(y[g][k] >> 32)), v[g][k]);
      }
#pragma unroll
      for (int g = 0; g < RG; g++) {
        if (g && i0 + per >= rows) break;
        if (slices > 1) {
          __syncthreads();
          xo[threadIdx.x] = sum[g].o;
          if (c == 0) { xd[2 * unit] = sum[g].m; xd[2 * unit + 1] = sum[g].den; }
          __syncthreads();
          for (int k = 1; k < slices && slice == 0; k++) sum[g].add(xd[2 * (unit + k * per)], xd[2 * (unit + k * per) + 1], xo[threadIdx.x + k * per * TPR]);
        }
        const int in = i0 + g * per + unit % per;
        if (slice == 0 && in < rows) write(in, sum[g]);
      }
    }
  };
  auto output = [&](int in, const PagedSum& sum) {
    const float inv = sum.den > 0.f ? 1.f / sum.den : sum.den == 0.f ? 0.f : sum.den;
    const int row = it.r0 + it.tile * run.deal.T + in / a.g, head = r * a.g + in % a.g;
    put_row4((T*)a.o + row * a.o_t + head * a.o_h + c * 4, sum.o, inv);
    if (a.lse && c == 0) a.lse[(int64_t)row * a.h_q + head] = sum.den == 0.f ? -INFINITY : (sum.m + log2f(sum.den)) * kLn2;
  };
  const bool levels = ((rows + per - 1) / per) * pieces > kChain * slices && pieces > 8;
  if (levels) {
    const int size = pieces > 128 ? 16 : 8, me = wg - w1, first = me / size * size, members = min(size, pieces - first);
    // group's record: a last piece on its own is one already
    auto group = [&](int i) { return i * size == pieces - 1 ? record(i * size) : rec0 + 2 * max(i * size, 1) + 1; };
    if (complete(a.flags, first, first + members) && members > 1) {
      const int64_t to = group(first / size);
      add_up(members, [&](int p) { return record(first + p); }, [&](int in, const PagedSum& sum) {
        recs.store(recs.place(to, in, c * 4), sum.o);
        if (c == 0) agent_store(a.part_ml + (to * ROWS + in) * 2, sum.m, sum.den);
      });
    }
    if (!complete(done, 0, pieces)) return;
    add_up((pieces + size - 1) / size, group, output);
  } else {
    if (!complete(a.flags, 0, pieces)) return;
    add_up(pieces, record, output);
  }
  for (int p = threadIdx.x; p < pieces; p += THREADS) {
    __hip_atomic_store(a.flags + record(p), (uint64_t)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (levels) __hip_atomic_store(done + record(p), (uint64_t)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// fp32: the same walk with the fp32 matrix cores, operands straight from the pages, 16 keys at a time.  A token's NaN or infinity
// reaches the rows that see it and no other.  Eight waves, one of each step's eight tiles each: the matrix cores' fp32 rate
// bounds a wave (1024 clocks a tile at head dimension 64), and items are few.  (Four waves, 333 tokens of two sequences of up to 1024, 4 / 2
// heads of 64: 19.0 us; eight: 17.4.)
// A wave's priority rises from the first product to the second: the two of a SIMD fall out of step (4 bits, 17.7 -> 17.0; 500 tokens of each of four sequences of 2000, 32 / 8
// heads of 128, 682 -> 672).
// FOUR: the cache holds 4 bits a number; the same values come out of their conversion.
template <int D, bool FOUR>
__global__ __launch_bounds__(512) void paged_few_f32_kernel(PagedArgs args) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  float* x = reinterpret_cast<float*>(lds);                                      // [8][16][D + 4], [8][16][2]
  const int r = blockIdx.x % args.h_kv, wg = blockIdx.x / args.h_kv;
  PagedRun<FOUR> run(args);
  if (!run.begin(args, wg)) return;
  const PagedItem& it = run.it;
  do {
  const PagedArgs a = paged_reload();
  const int tid = paged_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = 16 / a.g;
  const int t0 = it.tile * T;
  const int n = lane & 15, kq = lane >> 4;
  const int t = t0 + n / a.g;
  f32x4 qv[D / 16];
  const float* qp = (const float*)a.q + (it.r0 + min(t, it.m - 1)) * a.q_t + (r * a.g + n % a.g) * a.q_h;
  if constexpr (FOUR) load_quarter<D>(qp, kq, qv);
  else load_row<D>(qp, kq, qv);
  const int last = t < it.m ? paged_last_key(a, it, t) : -1;
  const int end = max(paged_last_key(a, it, min(t0 + T, it.m) - 1) + 1, 0);
  const int j0 = run.x0 * 8 + wave, j1 = min(run.x1 * 8, (end + 15) >> 4);       // 16-key tiles
  const int pm = (1 << a.page_log) - 1;
  using E = typename std::conditional<FOUR, uint8_t, float>::type;
  const E* kb = (const E*)a.k + r * a.kp_h;
  const E* vb = (const E*)a.v + r * a.vp_h;
  float m_run = -INFINITY, l_run = 0.f;
  f32x4 acc[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; i++) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  // the next tile's rows are asked for before the present one's are used; rows behind the sequence's last token repeat it
  f32x4 kv[D / 16], vv[1][4][D / 64], kn[D / 16], vn[4][D / 64];
  auto ask = [&](int j) {
    const int64_t id = paged_page(a, it.b, (j * 16) >> a.page_log);
    const int top = it.n - 1 - j * 16;
    const E* kp = kb + id * a.kp_p + (int64_t)(j * 16 & pm) * a.kp_t;
    const E* vp = vb + id * a.vp_p + (int64_t)(j * 16 & pm) * a.vp_t;
    if constexpr (FOUR) {
      const int64_t at = ((id * a.h_kv + r) << a.page_log) + (j * 16 & pm);
      load_quarter4<D>(kp + min(n, top) * a.kp_t, a.k_sc + (at + min(n, top)) * (D / 32), kq, kn);
#pragma unroll
      for (int i = 0; i < 4; i++) load_row2_4<D>(vp + min(4 * kq + i, top) * a.vp_t, a.v_sc + (at + min(4 * kq + i, top)) * (D / 32), n, vn[i]);
    } else {
      load_row<D>(kp + min(n, top) * a.kp_t, kq, kn);
#pragma unroll
      for (int i = 0; i < 4; i++) load_row2<D>(vp + min(4 * kq + i, top) * a.vp_t, n, vn[i]);
    }
  };
  if (j0 < j1) ask(j0);
  for (int j = j0; j < j1; j += 8) {
#pragma unroll
    for (int i = 0; i < D / 16; i++) kv[i] = kn[i];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int e = 0; e < D / 64; e++) vv[0][i][e] = vn[i][e];
    if (j + 8 < j1) ask(j + 8);
    __builtin_amdgcn_s_setprio(1);
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
    __builtin_amdgcn_s_setprio(2);
    mma_outer_keys<D, 1>(vv, s, lim, min(T, it.m - t0), a.g, lane, acc);
    __builtin_amdgcn_s_setprio(0);
  }
  const float l_tot = quad_rows_sum(l_run);
  float* ml = x + 8 * 16 * (D + 4);
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
  paged_few_finish<float, D, 8>(a, run, r, ((int64_t)r * a.wgs + wg) * 2 + (run.x0 == 0), t0, x, ml);
  if (!run.whole()) paged_few_join<float, D, 512>(a, run, r, wg, lds);
  __syncthreads();
  } while (run.advance(args));
}

// tiles of 128 rows of a sequence; cost: their steps of 64 keys
__device__ __forceinline__ int2 rows_shape(const PagedArgs& a, int m, int n) {
  const int T = 128 / a.g;
  return make_int2((m + T - 1) / T, max((n + 63) >> 6, 1));
}

inline int64_t paged_most_items(const PagedArgs& a, int rows) {   // of a kv-head
  const int T = rows / a.g;
  return min((int64_t)a.n_rows / T + min(a.batch, a.n_rows), (int64_t)a.n_rows);
}
inline int paged_most_parts(int runs) { return runs * 7 / 2; }   // of a kv-head: fewer than two items a resident workgroup, and one and a half
hipError_t launch_paged4_merge(const PagedArgs& a, int d, hipStream_t st);

}  // namespace dash
