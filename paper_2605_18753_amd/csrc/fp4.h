// Numbers in 4 bits: a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (E2M1), 32 of a row times a power of two of their own (a byte e + 127, E8M0; 255: all
// of them are NaN).  Eight codes are a word, the first in its low bits.  The hardware converts two at a time, scale included, and exactly: a level has two
// bits and e lies within -120 .. 125, so bf16 holds every value.
//
// Why not the matrix cores' own 4-bit operands: q as two 8-bit operands beside K in 4 bits needs no conversion, but v_mfma_scale_f32_16x16x128_f8f6f4 drops
// what lies more than 13 to 14 bits below the largest product of a sum (measured against 64 bits: 0.4 to 2.4e-4 of the largest product, where the bf16
// instruction is off by 1e-7).  Logits are held in 32 bits here.
#pragma once
#include "common.h"

namespace dash {

// A scale byte as a float: 2^e, or NaN.
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte == 255u ? 0x7fc00000u : byte << 23); }

// Eight codes as bf16; a NaN scale gives NaN.
__device__ __forceinline__ bf16x8 fp4_to_bf16(uint32_t w, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return __builtin_bit_cast(bf16x8, r);
}
// Four codes as floats: those of the low (HALF 0) or high 16 bits.
template <int HALF> __device__ __forceinline__ f32x4 fp4_to_f32(uint32_t w, float scale) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2 * HALF), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2 * HALF + 1);
  return f32x4{a[0], a[1], b[0], b[1]};
}

// The code of each of eight numbers that share their scale with the lanes of the same quad, and the scale.  Ties go to the even code (the hardware's
// rounding); v is finite or the scale 255.
__device__ __forceinline__ uint32_t fp4_of_eight(const float (&v)[8], uint32_t& scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true));   // quad_perm [1,0,3,2]
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true));   // quad_perm [2,3,0,1]
  if (top >= 0x7f800000u) {
    scale = 255u;
    return 0u;
  }
  // one more above 7.25: a fraction of more than 0.8125
  const int e = min(max((int)(top >> 23) - 129 + ((top & 0x7fffffu) > 0x680000u), -120), 125);
  scale = (uint32_t)(e + 127);
  const float s = __uint_as_float(scale << 23);
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
}

// A double as a float that rounds on as the double would: truncated, and its last bit set if anything was cut off.  Below 2^-126: 0.
__device__ __forceinline__ float sticky_float(double x) {
  const uint64_t b = __double_as_longlong(x);
  const uint32_t hi = (uint32_t)(b >> 32), lo = (uint32_t)b, mag = hi & 0x7fffffffu;
  uint32_t w = (uint32_t)(b >> 29) - (896u << 23);         // the exponent's bias: 1023 - 127
  w = (w | ((lo & 0x1fffffffu) != 0u)) & 0x7fffffffu;
  if (mag < 0x38100000u) w = 0u;
  if (mag >= 0x47f00000u) w = 0x7f800000u;                 // 2^128 and more, and what is not finite
  return __uint_as_float(w | (hi & 0x80000000u));
}

// Operands of the fp32 kernel from rows in 4 bits (f32_tiles.h has those from rows of floats).  First kind, contraction in an order of its own: lane (m, kq) has
// d = D / 4 kq + 4 s + e of its row m, for both operands: a lane's codes lie together.
template <int D> __device__ __forceinline__ void load_quarter(const float* row, int kq, f32x4 (&v)[D / 16]) {
#pragma unroll
  for (int s = 0; s < D / 16; s++) v[s] = *reinterpret_cast<const f32x4*>(row + D / 4 * kq + 4 * s);
}
template <int D> __device__ __forceinline__ void load_quarter4(const uint8_t* row, const uint8_t* scales, int kq, f32x4 (&v)[D / 16]) {
  const uint2* p = reinterpret_cast<const uint2*>(row + D / 8 * kq);
  const float sc = fp4_scale(scales[D / 4 * kq / 32]);
#pragma unroll
  for (int i = 0; i < D / 64; i++) {
    const uint2 w = p[i];
    v[4 * i] = fp4_to_f32<0>(w.x, sc);
    v[4 * i + 1] = fp4_to_f32<1>(w.x, sc);
    v[4 * i + 2] = fp4_to_f32<0>(w.y, sc);
    v[4 * i + 3] = fp4_to_f32<1>(w.y, sc);
  }
}
// second kind
template <int D> __device__ __forceinline__ void load_row2_4(const uint8_t* row, const uint8_t* scales, int m, f32x4 (&v)[D / 64]) {
#pragma unroll
  for (int nv = 0; nv < D / 64; nv++)
    v[nv] = fp4_to_f32<0>(reinterpret_cast<const uint16_t*>(row + 32 * nv)[m], fp4_scale(scales[2 * nv + (m >> 3)]));
}

}  // namespace dash
