// Rotary positions: what the kernels that turn queries and keys share.
//
// Pair i, (x, y), becomes mscale (x cos a - y sin a, x sin a + y cos a), a = position theta_i.  theta_i comes as the 64-bit fraction of a whole turn that
// it makes, so position * fraction modulo 2^64 is the angle's own fraction: off by position * 2^-65 turns, 4e-13 radians at a million, where
// a product in fp32 is off by 0.06.  The nearest quarter turn is taken off in whole numbers, and the rest, at most pi / 4, goes into the Taylor series of
// sine and cosine in 64 bits (terms up to y^17 and y^16: what follows is below 1e-17).
#pragma once
#include "common.h"
#include "dash_internal.h"

namespace dash {

struct RotaryArgs {
  const uint64_t* turns;
  int half;        // pairs: rot_dim / 2, a multiple of 8
  int adjacent;    // pairs of neighbours; otherwise of elements half a rotated part apart
  double mscale;
};

// (cos, sin) of 2 pi x / 2^64
__device__ __forceinline__ double2 cos_sin_of_turn(uint64_t x) {
  const uint32_t quarter = (uint32_t)((x + (1ull << 61)) >> 62);               // modulo 4, as the whole angle is
  const double y = (double)(int64_t)(x - ((uint64_t)quarter << 62)) * (6.283185307179586477 / 18446744073709551616.0);
  const double z = y * y;
  double s = __builtin_fma(z, 1.0 / 355687428096000.0, -1.0 / 1307674368000.0);
  s = __builtin_fma(z, s, 1.0 / 6227020800.0);
  s = __builtin_fma(z, s, -1.0 / 39916800.0);
  s = __builtin_fma(z, s, 1.0 / 362880.0);
  s = __builtin_fma(z, s, -1.0 / 5040.0);
  s = __builtin_fma(z, s, 1.0 / 120.0);
  s = __builtin_fma(z, s, -1.0 / 6.0);
  s = __builtin_fma(y * z, s, y);
  double c = __builtin_fma(z, 1.0 / 20922789888000.0, -1.0 / 87178291200.0);
  c = __builtin_fma(z, c, 1.0 / 479001600.0);
  c = __builtin_fma(z, c, -1.0 / 3628800.0);
  c = __builtin_fma(z, c, 1.0 / 40320.0);
  c = __builtin_fma(z, c, -1.0 / 720.0);
  c = __builtin_fma(z, c, 1.0 / 24.0);
  c = __builtin_fma(z, c, -0.5);
  c = __builtin_fma(z, c, 1.0);
  const double a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;               // |cos|, |sin| of the whole angle up to signs
  return make_double2(quarter == 1 || quarter == 2 ? -a : a, quarter >= 2 ? -b : b);
}

// of pair i at a position, times mscale
__device__ __forceinline__ double2 rotary_cos_sin(const RotaryArgs& r, int i, int position) {
  const double2 t = cos_sin_of_turn((uint64_t)(int64_t)position * r.turns[i]);
  return make_double2(t.x * r.mscale, t.y * r.mscale);
}

// A unit is 16 elements of a head, two pieces of 8 that hold the pairs 8 u .. 8 u + 7 (or, behind the rotated part, none): their offsets.
__device__ __forceinline__ int2 rotary_unit(const RotaryArgs& r, int u) {
  return r.adjacent || 8 * u >= r.half ? make_int2(16 * u, 16 * u + 8) : make_int2(8 * u, r.half + 8 * u);
}

// 8 elements of a tensor as floats, and back (rounded to nearest)
struct Eight { float x[8]; };
template <typename T> __device__ __forceinline__ Eight load_eight(const T* p);
template <> __device__ __forceinline__ Eight load_eight<uint16_t>(const uint16_t* p) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; i++) { e.x[2 * i] = bf16_lo(w[i]); e.x[2 * i + 1] = bf16_hi(w[i]); }
  return e;
}
template <> __device__ __forceinline__ Eight load_eight<float>(const float* p) {
  const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
  return {{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
__device__ __forceinline__ void store_eight(uint16_t* p, const Eight& e) {
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; i++) w[i] = __builtin_bit_cast(uint32_t, pair{(__bf16)e.x[2 * i], (__bf16)e.x[2 * i + 1]});
  *reinterpret_cast<u32x4*>(p) = w;
}
__device__ __forceinline__ void store_eight(float* p, const Eight& e) {
  reinterpret_cast<f32x4*>(p)[0] = f32x4{e.x[0], e.x[1], e.x[2], e.x[3]};
  reinterpret_cast<f32x4*>(p)[1] = f32x4{e.x[4], e.x[5], e.x[6], e.x[7]};
}

// Turns the pairs of a unit's two pieces; cs: (cos, sin) of its eight pairs.  Products and sums in fp32, of which each result has two roundings.
__device__ __forceinline__ void turn_unit(Eight& a, Eight& b, const float2 (&cs)[8], bool adjacent) {
  if (adjacent) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      Eight& e = i < 4 ? a : b;
      const float x = e.x[2 * (i & 3)], y = e.x[2 * (i & 3) + 1];
      e.x[2 * (i & 3)] = fmaf(x, cs[i].x, -(y * cs[i].y));
      e.x[2 * (i & 3) + 1] = fmaf(x, cs[i].y, y * cs[i].x);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float x = a.x[i], y = b.x[i];
      a.x[i] = fmaf(x, cs[i].x, -(y * cs[i].y));
      b.x[i] = fmaf(x, cs[i].y, y * cs[i].x);
    }
  }
}

// Validates r for heads of head_dim and fills out: a dash_status.
int rotary_args(const dash_rotary* r, int head_dim, RotaryArgs* out);

}  // namespace dash
