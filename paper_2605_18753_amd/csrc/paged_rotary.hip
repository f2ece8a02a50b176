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

// Turns the row's heads h0, h0 + step, .. (units of 16 elements, rotary_unit), from and to rows of heads.
template <typename T>
__device__ __forceinline__ void turn_heads(const RotaryArgs& r, const float2 (&cs)[8], int u, const T* from, int64_t from_h, T* to, int64_t to_h,
                                           int h0, int step, int heads) {
  const int2 at = rotary_unit(r, u);
  const bool turns = 8 * u < r.half;
  for (int h = h0; h < heads; h += step) {
    Eight p = load_eight(from + h * from_h + at.x), q = load_eight(from + h * from_h + at.y);
    if (turns) turn_unit(p, q, cs, r.adjacent);
    store_eight(to + h * to_h + at.x, p);
    store_eight(to + h * to_h + at.y, q);
  }
}

// A wave has a packed row: a lane works out the cosine and sine of a pair, into LDS, and takes those of its unit's eight pairs from there.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_append_rotary_kernel(PagedArgs a, RotaryArgs r) {
  constexpr int UNITS = D / 16, HEADS = 64 / UNITS, CHUNK = 16 / sizeof(T), CHUNKS = D / CHUNK;
  __shared__ float2 table[4][D / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(blockIdx.y << kGridLog | blockIdx.x) * 4 + wave;
  if (row >= a.n_rows) return;
  PagedPlace at;
  if (!paged_place(a, row, at)) return;
  const uint32_t page = (uint32_t)paged_entry(a, at.b, at.slot >> a.page_log);
  if (lane < r.half) {
    const double2 t = rotary_cos_sin(r, lane, at.position);
    table[wave][lane] = make_float2((float)t.x, (float)t.y);
  }
  asm volatile("" ::: "memory");                             // a wave's LDS operations complete in order
  const int u = lane % UNITS, h0 = lane / UNITS;
  float2 cs[8];
#pragma unroll
  for (int i = 0; i < 8; i++) cs[i] = table[wave][min(8 * u, r.half - 8) + i];
  if (a.q) turn_heads(r, cs, u, (const T*)a.q + row * a.q_t, a.q_h, (T*)a.o + row * a.o_t, a.o_h, h0, HEADS, a.h_q);
  if (page >= (uint32_t)a.n_pages) return;                   // no page: nothing is written
  const int off = at.slot & ((1 << a.page_log) - 1);
  turn_heads(r, cs, u, (const T*)a.k_new + row * a.kn_t, a.kn_h, (T*)a.k + (int64_t)page * a.kp_p + off * a.kp_t, a.kp_h, h0, HEADS, a.h_kv);
  const T* vn = (const T*)a.v_new + row * a.vn_t;
  T* vp = (T*)a.v + (int64_t)page * a.vp_p + off * a.vp_t;
  for (int x = lane; x < a.h_kv * CHUNKS; x += 64) {
    const int h = x / CHUNKS, c = x % CHUNKS * CHUNK;
    *reinterpret_cast<u32x4*>(vp + h * a.vp_h + c) = *reinterpret_cast<const u32x4*>(vn + h * a.vn_h + c);
  }
  for (int h = lane; h < a.h_kv; h += 64) {
    const int64_t x = (((int64_t)page * a.h_kv + h) << a.page_log) + off;
    if (a.weights) a.weights[x] = 0.f;
    if (a.pos) a.pos[x] = at.position;
  }
}

// 4 bits: a lane has 8 elements of a head, a word of codes; four lanes a scale.  Keys are turned in 64 bits, cosines and sines included, and rounded once,
// so that a number next to the border between two codes falls on the side that it lies on.
template <typename T, int D, bool ROTARY>
__global__ __launch_bounds__(256) void paged4_append_kernel(PagedArgs a, RotaryArgs r) {
  constexpr int UNITS = D / 16, HEADS = 64 / UNITS, LANES = D / 8;
  __shared__ double2 table[ROTARY ? 4 : 1][D / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(blockIdx.y << kGridLog | blockIdx.x) * 4 + wave;
  if (row >= a.n_rows) return;
  PagedPlace at;
  if (!paged_place(a, row, at)) return;
  const uint32_t page = (uint32_t)paged_entry(a, at.b, at.slot >> a.page_log);
  if constexpr (ROTARY) {
    if (lane < r.half) table[wave][lane] = rotary_cos_sin(r, lane, at.position);
    asm volatile("" ::: "memory");                           // a wave's LDS operations complete in order
    if (a.q) {
      const int u = lane % UNITS;
      float2 cs[8];
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const double2 t = table[wave][min(8 * u, r.half - 8) + i];
        cs[i] = make_float2((float)t.x, (float)t.y);
      }
      turn_heads(r, cs, u, (const T*)a.q + row * a.q_t, a.q_h, (T*)a.o + row * a.o_t, a.o_h, lane / UNITS, HEADS, a.h_q);
    }
  }
  if (page >= (uint32_t)a.n_pages) return;                   // no page: nothing is written
  const int off = at.slot & ((1 << a.page_log) - 1), c = lane % LANES;
  auto put = [&](const float (&v)[8], int h, char* codes, int64_t codes_h, uint8_t* scales) {
    uint32_t scale;
    const uint32_t w = fp4_of_eight(v, scale);
    *reinterpret_cast<uint32_t*>(codes + h * codes_h + c * 4) = w;
    if ((lane & 3) == 0) scales[((((int64_t)page * a.h_kv + h) << a.page_log) + off) * (D / 32) + c / 4] = (uint8_t)scale;
  };
  const T* kn = (const T*)a.k_new + row * a.kn_t;
  const T* vn = (const T*)a.v_new + row * a.vn_t;
  char* kp = (char*)a.k + (int64_t)page * a.kp_p + off * a.kp_t;
  char* vp = (char*)a.v + (int64_t)page * a.vp_p + off * a.vp_t;
  const bool turns = ROTARY && 8 * c < 2 * r.half;
  // the pieces of 8 that hold the other elements of this one's pairs, and its first pair
  const bool second = !r.adjacent && 8 * c >= r.half;
  const int other = r.adjacent ? c : second ? c - r.half / 8 : c + r.half / 8, pair = r.adjacent ? 4 * c : 8 * min(c, other);
  for (int h = lane / LANES; h < a.h_kv; h += 64 / LANES) {
    Eight x = load_eight(kn + h * a.kn_h + 8 * c);
    if constexpr (ROTARY) {
      if (turns) {
        const Eight y = r.adjacent ? x : load_eight(kn + h * a.kn_h + 8 * other);
        if (r.adjacent) {
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const double2 t = table[wave][pair + i];
            const double p = x.x[2 * i], q = x.x[2 * i + 1];
            x.x[2 * i] = sticky_float(__builtin_fma(p, t.x, -(q * t.y)));
            x.x[2 * i + 1] = sticky_float(__builtin_fma(p, t.y, q * t.x));
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; i++) {
            const double2 t = table[wave][pair + i];
            const double q = (double)y.x[i] * t.y;
            x.x[i] = sticky_float(__builtin_fma((double)x.x[i], t.x, second ? q : -q));
          }
        }
      }
    }
    put(x.x, h, kp, a.kp_h, const_cast<uint8_t*>(a.k_sc));
    put(load_eight(vn + h * a.vn_h + 8 * c).x, h, vp, a.vp_h, const_cast<uint8_t*>(a.v_sc));
  }
}

// A thread has a word of codes, the eight values of which it writes; rows of the pool one after the other, those of V behind those of K.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged4_unpack_kernel(PagedArgs a, T* k_pages, T* v_pages) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES;
  const int64_t rows = ((int64_t)a.n_pages * a.h_kv) << a.page_log;
  const int c = threadIdx.x % LANES;
  for (int64_t i = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; i < 2 * rows; i += (int64_t)gridDim.x * ROWS) {
    const bool v = i >= rows;
    const int64_t row = v ? i - rows : i, head = row >> a.page_log;
    const int64_t page = head / a.h_kv, h = head - page * a.h_kv, off = row & ((1 << a.page_log) - 1);
    const char* codes = v ? (const char*)a.v + page * a.vp_p + h * a.vp_h + off * a.vp_t : (const char*)a.k + page * a.kp_p + h * a.kp_h + off * a.kp_t;
    const uint32_t w = reinterpret_cast<const uint32_t*>(codes)[c];
    const float s = fp4_scale((v ? a.v_sc : a.k_sc)[row * (D / 32) + c / 4]);
    T* to = (v ? v_pages : k_pages) + row * D + 8 * c;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<bf16x8*>(to) = fp4_to_bf16(w, s);
    } else {
      reinterpret_cast<f32x4*>(to)[0] = fp4_to_f32<0>(w, s);
      reinterpret_cast<f32x4*>(to)[1] = fp4_to_f32<1>(w, s);
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
  const int64_t wgs = ((((int64_t)a.n_pages * a.h_kv) << a.page_log) * 2 + 2048 / d - 1) / (2048 / d);
  const dim3 grid((unsigned)(wgs < 1 << 16 ? wgs : 1 << 16)), blk(256);
  if (elem == 2 && d == 128) hipLaunchKernelGGL((paged4_unpack_kernel<uint16_t, 128>), grid, blk, 0, st, a, (uint16_t*)k_pages, (uint16_t*)v_pages);
  else if (elem == 2) hipLaunchKernelGGL((paged4_unpack_kernel<uint16_t, 64>), grid, blk, 0, st, a, (uint16_t*)k_pages, (uint16_t*)v_pages);
  else if (d == 128) hipLaunchKernelGGL((paged4_unpack_kernel<float, 128>), grid, blk, 0, st, a, (float*)k_pages, (float*)v_pages);
  else hipLaunchKernelGGL((paged4_unpack_kernel<float, 64>), grid, blk, 0, st, a, (float*)k_pages, (float*)v_pages);
  return hipGetLastError();
}

}  // namespace dash
