// The weight that the new tokens' attention gives to every cached token: w_j += sum over rows t (tokens and heads of the
// group) of e^{s_tj - lse_t}.
//
// Column sums of the softmax matrix, whose rows' log-sum-exps are known: a wave holds 64 keys (fp32: 32) as matrix operands in
// registers and walks the rows that see them, 16 at a time; a lane adds up its own pairs, and the 16 lanes of a key are added at the
// end.  Each sum is one wave's (or, for rows cut into parts, one thread's over the parts), so results do not depend on timing.
// A single token: K is read once, HBM bounds it.  Many: an exponential, an FMA and an addition per pair, 24 clocks of a SIMD for 64
// pairs, against 16 (head dimension 128; 64: 8) of matrix work.
//
// The keys of all sequences are dealt evenly: items of 4 waves' keys, a contiguous run of them to each of a fixed number of
// workgroups; fewer items than workgroups have their rows cut into parts instead, added up by a second launch.
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
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int s = 0; s < D / 16; s++) v[s] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ f32x4 dot(const WeighTile& b) const { return mma_dot<D>(v, b.v); }
};

template <typename T> constexpr int kWeighKeys = sizeof(T) == 2 ? 256 : 128;   // keys of an item

// rows of a sequence that weigh, from t0 on
__device__ __forceinline__ int weigh_first(const PagedArgs& a, int m) { return a.last > 0 ? max(m - a.last, 0) : 0; }

// items of a sequence; none without rows
template <typename T> __device__ __forceinline__ int weigh_items(int m, int n) { return m > 0 ? (n + kWeighKeys<T> - 1) / kWeighKeys<T> : 0; }

template <typename T> __device__ __forceinline__ int weigh_total(const PagedArgs& a) {
  const int lane = lane_id();
  int total = 0;
  for (int i0 = 0; i0 < a.batch; i0 += 64)
    total += __builtin_amdgcn_readlane(
        wave_scan(i0 + lane < a.batch ? weigh_items<T>(paged_rows(a, i0 + lane).y, paged_len(a, i0 + lane)) : 0), 63);
  return total;
}
struct WeighItem { int b, block, blocks, r0, m, n; };
template <typename T> __device__ __forceinline__ void weigh_find(const PagedArgs& a, int idx, WeighItem& it) {
  const int lane = lane_id();
  int base = 0;
  for (int i0 = 0; i0 < a.batch; i0 += 64) {
    int2 rm = make_int2(0, 0);
    int n = 0;
    if (i0 + lane < a.batch) {
      rm = paged_rows(a, i0 + lane);
      n = paged_len(a, i0 + lane);
    }
    const int x = weigh_items<T>(rm.y, n), incl = wave_scan(x);
    const uint64_t hit = __ballot(base + incl > idx);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      it.b = i0 + l;
      it.blocks = __builtin_amdgcn_readlane(x, l);
      it.block = idx - (base + __builtin_amdgcn_readlane(incl, l) - it.blocks);
      it.r0 = __builtin_amdgcn_readlane(rm.x, l);
      it.m = __builtin_amdgcn_readlane(rm.y, l);
      it.n = __builtin_amdgcn_readlane(n, l);
      return;
    }
    base += __builtin_amdgcn_readlane(incl, 63);
  }
}

// parts that an item's rows are cut into; one where the host gave no room for records
__device__ __forceinline__ int weigh_parts(const PagedArgs& a, int total) { return a.part_o ? min(max(a.wgs / total, 1), 64) : 1; }

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_weigh_kernel(PagedArgs a) {
  constexpr int SUBS = WeighTile<T, D>::SUBS;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x % a.h_kv, wg = blockIdx.x / a.h_kv;
  const int total = weigh_total<T>(a);
  if (total == 0) return;
  // parts > 1: one item each, its rows cut; else a run of whole items
  const int parts = weigh_parts(a, total);
  int i0, i1, part = 0;
  if (parts > 1) {
    i0 = wg / parts; part = wg % parts; i1 = min(i0 + 1, total);
  } else {
    i0 = (int)((int64_t)wg * total / a.wgs); i1 = (int)((int64_t)(wg + 1) * total / a.wgs);
  }
  const int Tt = 16 / a.g, n = lane & 15, kq = lane >> 4, pm = (1 << a.page_log) - 1;
  const int head = r * a.g + n % a.g;
  WeighItem it;
  it.block = it.blocks = 0;
  for (int i = i0; i < i1; i++) {
    if (++it.block >= it.blocks) weigh_find<T>(a, i, it);
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
    // row tiles: from the first that sees one of the wave's keys
    const int first = weigh_first(a, it.m), back = it.n - it.m;
    const int x0 = first / Tt, x1 = (it.m + Tt - 1) / Tt, per = (x1 - x0 + parts - 1) / parts;
    int x = x0 + part * per;
    const int xe = min(x + per, x1);
    if (a.causal) x = max(x, (key0 - back) / Tt);              // its token sees keys up to back + t
    if (key0 >= it.n) x = xe;
    WeighTile<T, D> qf;
    float off = -INFINITY;
    auto ask = [&](int y) {
      const int t = y * Tt + n / a.g, tc = min(t, it.m - 1);
      qf.load((const T*)a.q + (it.r0 + tc) * a.q_t + head * a.q_h, kq);
      const float l = a.lse_in[(int64_t)(it.r0 + tc) * a.h_q + head];
      const bool live = t < it.m && t >= first && l != -INFINITY;
      off = live ? -l * kLog2e : -INFINITY;
      if (!live) qf.clear();                                   // whatever the row holds
    };
    if (x < xe) ask(x);
    for (; x < xe; x++) {
      f32x4 s[SUBS];
#pragma unroll
      for (int j = 0; j < SUBS; j++) s[j] = kf[j].dot(qf);
      const float o = off;
      const int t0 = x * Tt;
      if (x + 1 < xe) ask(x + 1);
      const int low = a.causal ? back + t0 : it.n - 1;         // the tile's first token sees keys up to here
      if (key0 + SUBS * 16 - 1 > low) {
        const int lim = (a.causal ? min(back + t0 + n / a.g, it.n - 1) : it.n - 1) - key0 - 4 * kq;
#pragma unroll
        for (int j = 0; j < SUBS; j++)
#pragma unroll
          for (int e = 0; e < 4; e++) s[j][e] = 16 * j + e > lim ? -INFINITY : s[j][e];
      }
#pragma unroll
      for (int j = 0; j < SUBS; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) acc[j][e] += __builtin_amdgcn_exp2f(fmaf(s[j][e], a.c1, o));
    }
    // over the 16 rows of a key; lane (n, kq), n < 4, takes key 4 kq + n
#pragma unroll
    for (int j = 0; j < SUBS; j++) {
#pragma unroll
      for (int e = 0; e < 4; e++) acc[j][e] = row16_sum(acc[j][e]);
      const float w = n == 0 ? acc[j][0] : n == 1 ? acc[j][1] : n == 2 ? acc[j][2] : acc[j][3];
      const int key = key0 + 16 * j + 4 * kq + n;
      if (n < 4) {
        if (parts > 1) a.part_o[((int64_t)r * a.wgs + wg) * kWeighKeys<T> + wave * SUBS * 16 + 16 * j + 4 * kq + n] = w;
        else if (key < it.n && (uint32_t)page[j] < (uint32_t)a.n_pages) a.weights[(((int64_t)page[j] * a.h_kv + r) << a.page_log) + (key & pm)] += w;
      }
    }
  }
}

// the parts of items whose rows were cut: a thread per key
template <typename T>
__global__ __launch_bounds__(kWeighKeys<T>) void paged_weigh_sum_kernel(PagedArgs a) {
  const int r = blockIdx.x % a.h_kv, i = blockIdx.x / a.h_kv;
  const int total = weigh_total<T>(a);
  if (i >= total) return;
  const int parts = weigh_parts(a, total);
  if (parts <= 1) return;
  WeighItem it;
  weigh_find<T>(a, i, it);
  const int key = it.block * kWeighKeys<T> + threadIdx.x;
  if (key >= it.n) return;
  const float* p = a.part_o + ((int64_t)r * a.wgs + (int64_t)i * parts) * kWeighKeys<T> + threadIdx.x;
  float w = 0.f;
#pragma unroll 4
  for (int j = 0; j < parts; j++) w += p[(int64_t)j * kWeighKeys<T>];
  const uint32_t page = (uint32_t)a.table[(int64_t)it.b * a.max_pages + (key >> a.page_log)];
  if (page >= (uint32_t)a.n_pages) return;
  a.weights[(((int64_t)page * a.h_kv + r) << a.page_log) + (key & ((1 << a.page_log) - 1))] += w;
}

// ---- host ------------------------------------------------------------------------------------------------------------
static int weigh_wgs(const PagedArgs& a) { return max(768 / a.h_kv, 1); }
// whether cutting rows into parts can pay: more than two tiles of them
static bool weigh_may_cut(const PagedArgs& a) { return (int64_t)a.n_rows * a.g > 32; }

size_t paged_weigh_ws(const PagedArgs& a, int dtype, int) {
  return (size_t)weigh_wgs(a) * a.h_kv * (dtype == DASH_BF16 ? kWeighKeys<uint16_t> : kWeighKeys<float>) * 4;
}

template <typename T, int D>
static hipError_t launch_weigh_t(PagedArgs a, char* ws, hipStream_t st) {
  a.part_o = weigh_may_cut(a) ? (float*)ws : nullptr;
  a.wgs = weigh_wgs(a);
  hipLaunchKernelGGL((paged_weigh_kernel<T, D>), dim3((unsigned)(a.wgs * a.h_kv)), dim3(256), 0, st, a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || !a.part_o) return e;
  hipLaunchKernelGGL(paged_weigh_sum_kernel<T>, dim3((unsigned)((a.wgs / 2 + 1) * a.h_kv)), dim3(kWeighKeys<T>), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_paged_weigh(const PagedArgs& a, int dtype, int d, char* ws, hipStream_t st) {
  if (dtype == DASH_BF16) return d == 128 ? launch_weigh_t<uint16_t, 128>(a, ws, st) : launch_weigh_t<uint16_t, 64>(a, ws, st);
  return d == 128 ? launch_weigh_t<float, 128>(a, ws, st) : launch_weigh_t<float, 64>(a, ws, st);
}

}  // namespace dash
