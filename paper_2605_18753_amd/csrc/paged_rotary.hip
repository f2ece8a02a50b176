// New tokens into a paged cache, their keys turned by their positions on the way; the same into a cache in 4 bits; and that cache read back.
#include "fp4.h"
#include "paged.h"
#include "rotary.h"

namespace dash {

constexpr int kGridLog = 22;                                 // workgroups of a launch's row: below 2^32 threads in a dimension
static dim3 rows_grid(int n_rows) {
  const int64_t wgs = ((int64_t)n_rows + 3) / 4, most = (int64_t)1 << kGridLog;
  return dim3((unsigned)(wgs < most ? wgs : most), (unsigned)((wgs + most - 1) / most));
}

// A row's heads h0, h0 + step, .., turned: the first N asked for before anything is known about the row.
template <typename T, int D, int N> struct Heads {
  using U = Unit<T, D>;
  typename U::Data x[N];
  __device__ __forceinline__ void ask(const U& unit, const T* row, int64_t stride, int h0, int step, int heads) {
#pragma unroll
    for (int i = 0; i < N; i++)
      if (h0 + i * step < heads) x[i] = unit.load(row + (h0 + i * step) * stride);
  }
  __device__ __forceinline__ void turn(const U& unit, const typename U::Pairs& cs, bool adjacent, const T* row, int64_t stride, int h0, int step, int heads,
                                       T* to, int64_t to_stride) {
    for (int h = h0; h < heads; h += N * step) {
      if (h != h0) ask(unit, row, stride, h, step, heads);
#pragma unroll
      for (int i = 0; i < N; i++)
        if (h + i * step < heads) unit.store(to + (h + i * step) * to_stride, x[i], cs, adjacent);
    }
  }
};

// A wave has a packed row.  What the row holds is asked for first, with the turns; then the row's place is found, a lane works out the cosine and sine of a
// pair, into LDS, and takes those of its unit's eight pairs from there.
// Bound by HBM: 2047 tokens of each of four sequences, 32 / 8 heads of 128, 42.6 us, 101 MB in and 102 out at 4.8 TB/s; by latency where there are few: 64
// tokens 5.3 us.  (Of that many, two heads asked for ahead; four, which costs registers and waves, 3 us more.)
template <typename T, int D>
__global__ __launch_bounds__(256, 4) void paged_append_rotary_kernel(PagedArgs a, RotaryArgs r) {
  using U = Unit<T, D>;
  constexpr int HEADS = 64 / U::COUNT, CHUNK = 16 / sizeof(T), CHUNKS = D / CHUNK, NV = 2;
  __shared__ float2 table[4][rotary_place(D / 2)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(blockIdx.y << kGridLog | blockIdx.x) * 4 + wave;
  if (row >= a.n_rows) return;
  const int h0 = lane / U::COUNT;
  const U unit(r, lane % U::COUNT);
  const T* kn = (const T*)a.k_new + row * a.kn_t;
  const T* vn = (const T*)a.v_new + row * a.vn_t;
  const T* qn = (const T*)a.q + row * a.q_t;
  const uint64_t turns = r.turns[min(lane, r.half - 1)];
  Heads<T, D, 1> k;
  Heads<T, D, 2> q;
  u32x4 v[NV];
  k.ask(unit, kn, a.kn_h, h0, HEADS, a.h_kv);
  auto ask_v = [&](int x0) {
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int x = x0 + 64 * i;
      if (x < a.h_kv * CHUNKS) v[i] = *reinterpret_cast<const u32x4*>(vn + x / CHUNKS * a.vn_h + x % CHUNKS * CHUNK);
    }
  };
  ask_v(lane);
  if (a.q) q.ask(unit, qn, a.q_h, h0, HEADS, a.h_q);
  PagedPlace at;
  if (!paged_place(a, row, at)) return;
  const uint32_t page = (uint32_t)paged_entry(a, at.b, at.slot >> a.page_log);
  const double2 t = rotary_cos_sin(r, turns, at.position);
  table[wave][rotary_place(min(lane, D / 2 - 1))] = make_float2((float)t.x, (float)t.y);       // lanes behind the last pair: no one's
  asm volatile("" ::: "memory");                             // a wave's LDS operations complete in order
  const typename U::Pairs cs = unit.pairs(table[wave]);
  if (a.q) q.turn(unit, cs, r.adjacent, qn, a.q_h, h0, HEADS, a.h_q, (T*)a.o + row * a.o_t, a.o_h);
  if (page >= (uint32_t)a.n_pages) return;                   // no page: nothing is written
  const int off = at.slot & ((1 << a.page_log) - 1);
  k.turn(unit, cs, r.adjacent, kn, a.kn_h, h0, HEADS, a.h_kv, (T*)a.k + (int64_t)page * a.kp_p + off * a.kp_t, a.kp_h);
  T* vp = (T*)a.v + (int64_t)page * a.vp_p + off * a.vp_t;
  for (int x0 = lane; x0 < a.h_kv * CHUNKS; x0 += 64 * NV) {
    if (x0 != lane) ask_v(x0);
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int x = x0 + 64 * i;
      if (x < a.h_kv * CHUNKS) *reinterpret_cast<u32x4*>(vp + x / CHUNKS * a.vp_h + x % CHUNKS * CHUNK) = v[i];
    }
  }
  for (int h = lane; h < a.h_kv; h += 64) {
    const int64_t x = (((int64_t)page * a.h_kv + h) << a.page_log) + off;
    if (a.weights) a.weights[x] = 0.f;
    if (a.pos) a.pos[x] = at.position;
  }
}

// 4 bits: a lane has 8 elements of a head, a word of codes; four lanes a scale.  Keys are turned in 64 bits, cosines and sines included, and rounded once,
// so that a number next to the border between two codes falls on the side that it lies on.  The same 2047 tokens of four sequences 40 us, 101 MB in and 77 out at
// 4.4 TB/s; the vector units issue in 0.44 of the clocks, half of it the 64-bit products.
template <typename T, int D, bool ROTARY>
__global__ __launch_bounds__(256) void paged4_append_kernel(PagedArgs a, RotaryArgs r) {
  using U = Unit<T, D>;
  constexpr int HEADS = 64 / U::COUNT, LANES = D / 8, STEP = 64 / LANES, NK = 2;
  __shared__ double2 table[ROTARY ? 4 : 1][rotary_place(D / 2)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(blockIdx.y << kGridLog | blockIdx.x) * 4 + wave;
  if (row >= a.n_rows) return;
  const int h0 = lane / U::COUNT, c = lane % LANES, k0 = lane / LANES;
  const T* kn = (const T*)a.k_new + row * a.kn_t;
  const T* vn = (const T*)a.v_new + row * a.vn_t;
  const T* qn = (const T*)a.q + row * a.q_t;
  // the piece of 8 that holds the other elements of this one's pairs, and the first pair
  const bool turned = ROTARY && 8 * c < 2 * r.half, second = ROTARY && !r.adjacent && 8 * c >= r.half;
  const int other = !ROTARY || r.adjacent || !turned ? c : second ? c - r.half / 8 : c + r.half / 8, pair = ROTARY && r.adjacent ? 4 * c : 8 * min(c, other);
  uint64_t turns = 0;
  if constexpr (ROTARY) turns = r.turns[min(lane, r.half - 1)];
  Piece<T> k[NK], ko[NK], v[NK];
  auto ask = [&](int h) {
#pragma unroll
    for (int i = 0; i < NK; i++)
      if (h + i * STEP < a.h_kv) {
        k[i] = load_piece(kn + (h + i * STEP) * a.kn_h + 8 * c);
        if constexpr (ROTARY) ko[i] = load_piece(kn + (h + i * STEP) * a.kn_h + 8 * other);
        v[i] = load_piece(vn + (h + i * STEP) * a.vn_h + 8 * c);
      }
  };
  ask(k0);
  const U unit(r, lane % U::COUNT);
  Heads<T, D, 4> q;
  if constexpr (ROTARY) {
    if (a.q) q.ask(unit, qn, a.q_h, h0, HEADS, a.h_q);
  }
  PagedPlace at;
  if (!paged_place(a, row, at)) return;
  const uint32_t page = (uint32_t)paged_entry(a, at.b, at.slot >> a.page_log);
  if constexpr (ROTARY) {
    table[wave][rotary_place(min(lane, D / 2 - 1))] = rotary_cos_sin(r, turns, at.position);   // lanes behind the last pair: no one's
    asm volatile("" ::: "memory");                           // a wave's LDS operations complete in order
    if (a.q) q.turn(unit, unit.pairs(table[wave]), r.adjacent, qn, a.q_h, h0, HEADS, a.h_q, (T*)a.o + row * a.o_t, a.o_h);
  }
  if (page >= (uint32_t)a.n_pages) return;                   // no page: nothing is written
  const int off = at.slot & ((1 << a.page_log) - 1);
  auto put = [&](const Eight& e, int h, char* codes, int64_t codes_h, uint8_t* scales) {
    uint32_t scale;
    const uint32_t w = fp4_of_eight(e.x, scale);
    *reinterpret_cast<uint32_t*>(codes + h * codes_h + c * 4) = w;
    if ((lane & 3) == 0) scales[((((int64_t)page * a.h_kv + h) << a.page_log) + off) * (D / 32) + c / 4] = (uint8_t)scale;
  };
  char* kp = (char*)a.k + (int64_t)page * a.kp_p + off * a.kp_t;
  char* vp = (char*)a.v + (int64_t)page * a.vp_p + off * a.vp_t;
  for (int hb = k0; hb < a.h_kv; hb += NK * STEP) {
    if (hb != k0) ask(hb);
#pragma unroll
    for (int i = 0; i < NK; i++) {
      const int h = hb + i * STEP;
      if (h >= a.h_kv) break;
      Eight x = eight_of(k[i]);
      if constexpr (ROTARY) {
        if (turned && r.adjacent) {
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const double2 t = table[wave][rotary_place(pair) + e];
            const double p = x.x[2 * e], y = x.x[2 * e + 1];
            x.x[2 * e] = sticky_float(__builtin_fma(p, t.x, -(y * t.y)));
            x.x[2 * e + 1] = sticky_float(__builtin_fma(p, t.y, y * t.x));
          }
        } else if (turned) {
          const Eight y = eight_of(ko[i]);
#pragma unroll
          for (int e = 0; e < 8; e++) {
            const double2 t = table[wave][rotary_place(pair) + e];
            const double z = (double)y.x[e] * t.y;
            x.x[e] = sticky_float(__builtin_fma((double)x.x[e], t.x, second ? z : -z));
          }
        }
      }
      put(x, h, kp, a.kp_h, const_cast<uint8_t*>(a.k_sc));
      put(eight_of(v[i]), h, vp, a.vp_h, const_cast<uint8_t*>(a.v_sc));
    }
  }
}

// A thread has words of eight codes, one of every so many rows, and writes what they stand for; the rows of K of a head of a page, and those of V, are a
// workgroup's at a time.  Bound by HBM and the last-level cache: 10 MB of codes in and 38 MB out in 12 us.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged4_unpack_kernel(PagedArgs a, T* k_pages, T* v_pages) {
  constexpr int WORDS = D / 8, ROWS = 256 / WORDS, AHEAD = 4;                  // rows at a time
  const int heads = a.n_pages * a.h_kv, P = 1 << a.page_log, w = threadIdx.x % WORDS, row0 = threadIdx.x / WORDS;
  for (int head = blockIdx.x; head < heads; head += gridDim.x) {
    const int page = head / a.h_kv, h = head - page * a.h_kv;
#pragma unroll
    for (int x = 0; x < 2; x++) {
      const char* codes = (x ? (const char*)a.v + page * a.vp_p + h * a.vp_h : (const char*)a.k + page * a.kp_p + h * a.kp_h) + w * 4;
      const uint32_t stride = x ? (uint32_t)a.vp_t : (uint32_t)a.kp_t;         // a page's rows span less than 2 GiB
      const uint8_t* scales = (x ? a.v_sc : a.k_sc) + ((int64_t)head << a.page_log) * (D / 32) + w / 4;
      T* to = (x ? v_pages : k_pages) + ((int64_t)head << a.page_log) * D + w * 8;
      for (int r0 = row0; r0 < P; r0 += ROWS * AHEAD) {
        uint32_t word[AHEAD], scale[AHEAD];                                    // asked for together
#pragma unroll
        for (int i = 0; i < AHEAD; i++) {
          const int r = min(r0 + i * ROWS, P - 1);
          word[i] = *reinterpret_cast<const uint32_t*>(codes + r * stride);
          scale[i] = scales[r * (D / 32)];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; i++) {
          const int r = r0 + i * ROWS;
          if (r >= P) break;
          const float s = fp4_scale(scale[i]);
          if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<bf16x8*>(to + r * D) = fp4_to_bf16(word[i], s);
          } else {
            reinterpret_cast<f32x4*>(to + r * D)[0] = fp4_to_f32<0>(word[i], s);
            reinterpret_cast<f32x4*>(to + r * D)[1] = fp4_to_f32<1>(word[i], s);
          }
        }
      }
    }
  }
}

hipError_t launch_paged_append_rotary(const PagedArgs& a, const RotaryArgs& r, int elem, int d, hipStream_t st) {
  const dim3 grid = rows_grid(a.n_rows), blk(256);
  if (elem == 2 && d == 128) hipLaunchKernelGGL((paged_append_rotary_kernel<uint16_t, 128>), grid, blk, 0, st, a, r);
  else if (elem == 2) hipLaunchKernelGGL((paged_append_rotary_kernel<uint16_t, 64>), grid, blk, 0, st, a, r);
  else if (d == 128) hipLaunchKernelGGL((paged_append_rotary_kernel<float, 128>), grid, blk, 0, st, a, r);
  else hipLaunchKernelGGL((paged_append_rotary_kernel<float, 64>), grid, blk, 0, st, a, r);
  return hipGetLastError();
}

template <typename T, int D> static void launch_append4(const PagedArgs& a, const RotaryArgs* r, hipStream_t st) {
  if (r) hipLaunchKernelGGL((paged4_append_kernel<T, D, true>), rows_grid(a.n_rows), dim3(256), 0, st, a, *r);
  else hipLaunchKernelGGL((paged4_append_kernel<T, D, false>), rows_grid(a.n_rows), dim3(256), 0, st, a, RotaryArgs{});
}
hipError_t launch_paged4_append(const PagedArgs& a, const RotaryArgs* r, int elem, int d, hipStream_t st) {
  if (elem == 2 && d == 128) launch_append4<uint16_t, 128>(a, r, st);
  else if (elem == 2) launch_append4<uint16_t, 64>(a, r, st);
  else if (d == 128) launch_append4<float, 128>(a, r, st);
  else launch_append4<float, 64>(a, r, st);
  return hipGetLastError();
}

hipError_t launch_paged4_unpack(const PagedArgs& a, void* k_pages, void* v_pages, int elem, int d, hipStream_t st) {
  const int64_t heads = (int64_t)a.n_pages * a.h_kv;
  const dim3 grid((unsigned)(heads < 1 << 20 ? heads : 1 << 20)), blk(256);
  if (elem == 2 && d == 128) hipLaunchKernelGGL((paged4_unpack_kernel<uint16_t, 128>), grid, blk, 0, st, a, (uint16_t*)k_pages, (uint16_t*)v_pages);
  else if (elem == 2) hipLaunchKernelGGL((paged4_unpack_kernel<uint16_t, 64>), grid, blk, 0, st, a, (uint16_t*)k_pages, (uint16_t*)v_pages);
  else if (d == 128) hipLaunchKernelGGL((paged4_unpack_kernel<float, 128>), grid, blk, 0, st, a, (float*)k_pages, (float*)v_pages);
  else hipLaunchKernelGGL((paged4_unpack_kernel<float, 64>), grid, blk, 0, st, a, (float*)k_pages, (float*)v_pages);
  return hipGetLastError();
}

}  // namespace dash
