// Rotary positions: what the kernels that turn queries and keys share.
//
// Pair i, (x, y), becomes mscale (x cos a - y sin a, x sin a + y cos a), a = position theta_i.  theta_i comes as the 64-bit fraction of a whole turn that
// it makes, so position * fraction modulo 2^64 is the angle's own fraction: off by position * 2^-65 turns, 1.7e-13 radians at a million, where
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

// of a pair's turns at a position, times mscale
__device__ __forceinline__ double2 rotary_cos_sin(const RotaryArgs& r, uint64_t turns, int position) {
  const double2 t = cos_sin_of_turn((uint64_t)(int64_t)position * turns);
  return make_double2(t.x * r.mscale, t.y * r.mscale);
}

// Where a pair's cosine and sine lie in LDS: a gap behind every eight, so that lanes that read eight each do not meet in the banks.  Four pairs that begin at a
// multiple of 4 lie together.
__host__ __device__ constexpr int rotary_place(int pair) { return pair + pair / 8; }

// Eight elements of a tensor as they lie in memory: asked for early, made floats when they are used.
template <typename T> struct Piece { u32x4 w[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ Piece<T> load_piece(const T* p) {
  Piece<T> x;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; i++) x.w[i] = reinterpret_cast<const u32x4*>(p)[i];
  return x;
}
template <typename T> __device__ __forceinline__ void store_piece(T* p, const Piece<T>& x) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; i++) reinterpret_cast<u32x4*>(p)[i] = x.w[i];
}
struct Eight { float x[8]; };
__device__ __forceinline__ Eight eight_of(const Piece<uint16_t>& p) {
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; i++) { e.x[2 * i] = bf16_lo(p.w[0][i]); e.x[2 * i + 1] = bf16_hi(p.w[0][i]); }
  return e;
}
__device__ __forceinline__ Eight eight_of(const Piece<float>& p) {
  Eight e;
#pragma unroll
  for (int i = 0; i < 8; i++) e.x[i] = __uint_as_float(p.w[i >> 2][i & 3]);
  return e;
}

// A unit is two 16-byte pieces of a head, of V elements each, and V pairs (or none, behind the rotated part): of pairs that lie apart, piece a has
// the first elements and b the second ones; neighbours lie in a piece, V / 2 pairs, and b is half a head behind a.  Neighbouring units are neighbours in memory.
// (Pieces one behind the other in a thread: 2 x 20 heads of 64 x 3001 tokens in fp32 17.2 us; as here 11.5 to 11.9 by card.)
template <typename T, int D> struct Unit {
  static constexpr int V = 16 / sizeof(T), COUNT = D / (2 * V);                // units of a head
  int a, b, pa, pb;              // elements where the pieces begin; first pairs of the lower and the upper half of cs
  bool ta, tb;                   // whether they turn
  __device__ __forceinline__ Unit(const RotaryArgs& r, int u) {
    if (r.adjacent) {
      a = V * u; b = V * (u + COUNT);
      ta = a < 2 * r.half; tb = b < 2 * r.half;
      pa = a / 2; pb = b / 2;
    } else {
      ta = tb = V * u < r.half;
      a = ta ? V * u : 2 * V * u; b = ta ? r.half + V * u : 2 * V * u + V;
      pa = V * u; pb = pa + V / 2;
    }
    pa = min(pa, r.half - V / 2);                            // that no one uses
    pb = min(pb, r.half - V / 2);
  }
  struct Pairs { float2 cs[V]; };
  template <typename C> __device__ __forceinline__ Pairs pairs(const C* cs) const {   // cs as rotary_place has them
    Pairs p;
#pragma unroll
    for (int i = 0; i < V; i++) {
      const C c = cs[i < V / 2 ? rotary_place(pa) + i : rotary_place(pb) + i - V / 2];
      p.cs[i] = make_float2((float)c.x, (float)c.y);
    }
    return p;
  }
  struct Data { u32x4 a, b; };
  __device__ __forceinline__ Data load(const T* head) const { return {*reinterpret_cast<const u32x4*>(head + a), *reinterpret_cast<const u32x4*>(head + b)}; }
  __device__ __forceinline__ static float get(const u32x4& w, int i) {
    if constexpr (V == 4) return __uint_as_float(w[i]);
    else return i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
  }
  __device__ __forceinline__ static u32x4 put(const float (&x)[V]) {           // rounded to nearest
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if constexpr (V == 4) w[i] = __float_as_uint(x[i]);
      else w[i] = __builtin_bit_cast(uint32_t, pair{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
    }
    return w;
  }
  // Products and sums in fp32, of which each result has two roundings.
  __device__ __forceinline__ static u32x4 neighbours(const u32x4& w, const float2* cs) {
    float y[V];
#pragma unroll
    for (int i = 0; i < V / 2; i++) {
      const float p = get(w, 2 * i), q = get(w, 2 * i + 1);
      y[2 * i] = fmaf(p, cs[i].x, -(q * cs[i].y));
      y[2 * i + 1] = fmaf(p, cs[i].y, q * cs[i].x);
    }
    return put(y);
  }
  __device__ __forceinline__ void store(T* head, Data x, const Pairs& p, bool adjacent) const {
    if (adjacent) {
      if (ta) x.a = neighbours(x.a, p.cs);
      if (tb) x.b = neighbours(x.b, p.cs + V / 2);
    } else if (ta) {
      float y[V], z[V];
#pragma unroll
      for (int i = 0; i < V; i++) {
        const float m = get(x.a, i), n = get(x.b, i);
        y[i] = fmaf(m, p.cs[i].x, -(n * p.cs[i].y));
        z[i] = fmaf(m, p.cs[i].y, n * p.cs[i].x);
      }
      x.a = put(y);
      x.b = put(z);
    }
    *reinterpret_cast<u32x4*>(head + a) = x.a;
    *reinterpret_cast<u32x4*>(head + b) = x.b;
  }
};

// Validates r for heads of head_dim and fills out: a dash_status.
int rotary_args(const dash_rotary* r, int head_dim, RotaryArgs* out);

}  // namespace dash
