// Rows held in microscaled 4-bit floating point (MX, E2M1 elements with an E8M0 scale per 32 of them), on the device: the
// conversion instructions of gfx950 take a packed word of eight codes and the block's scale.  Compared with every code under every
// scale, and with the numbers between codes and their neighbours under scales from 2^-127 to 2^125, they are exact: halves go to the
// even code, what is beyond 6 to 6, subnormal scales and results are kept.
#pragma once

#include "tb_device.h"

namespace tb {
namespace {

constexpr int kMxBlock = 32;       // elements that share a scale
constexpr int kMxCodeBytes = 16;   // ... their codes

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));

// A scale byte as the number whose exponent the conversions read: 2^(byte - 127) (byte 0: its exponent field counts as 2^-127),
// 255 as infinity, which they turn into NaN.
__device__ __forceinline__ float mx_scale(const uint32_t byte) { return __uint_as_float(byte << 23); }

// Elements 2 PAIR and 2 PAIR + 1 of a word of eight codes.
template <int PAIR>
__device__ __forceinline__ void mx_to_f32(const uint32_t word, const float scale, float& lo, float& hi) {
  const mx_f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, PAIR);
  lo = v.x;
  hi = v.y;
}
// ... as two bf16 numbers (exact: two significant bits, the exponent range of fp32; what is beyond it, under bytes 253 and 254, is an infinity).
template <int PAIR>
__device__ __forceinline__ uint32_t mx_to_bf16(const uint32_t word, const float scale) {
  const mx_bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, PAIR);
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  return u;
}
__device__ __forceinline__ void mx_to_f32(const uint32_t word, const float scale, float (&f)[8]) {
  mx_to_f32<0>(word, scale, f[0], f[1]);
  mx_to_f32<1>(word, scale, f[2], f[3]);
  mx_to_f32<2>(word, scale, f[4], f[5]);
  mx_to_f32<3>(word, scale, f[6], f[7]);
}
__device__ __forceinline__ void mx_to_bf16(const uint32_t word, const float scale, uint32_t (&u)[4]) {
  u[0] = mx_to_bf16<0>(word, scale);
  u[1] = mx_to_bf16<1>(word, scale);
  u[2] = mx_to_bf16<2>(word, scale);
  u[3] = mx_to_bf16<3>(word, scale);
}

// A number as the exact sum of P bf16 numbers, 8 bits each (one: it is a bf16 number; three: any); an infinity or a NaN has them
// once and zeros behind.
template <int P>
__device__ __forceinline__ void mx_split_bf16(const float x, uint32_t (&part)[P]) {
  if constexpr (P == 1) {
    part[0] = __float_as_uint(x) >> 16;
  } else {
    const bool finite = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
    float rest = x;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      uint32_t top = __float_as_uint(rest) & 0xFFFF0000u;
      if (p == 0 && x != x) top |= 0x00400000u;  // (a NaN whose upper half alone would be an infinity)
      part[p] = top >> 16;
      rest = finite ? rest - __uint_as_float(top) : 0.f;  // exact
    }
  }
}

// Eight numbers as a word of codes under a scale byte below 255.
__device__ __forceinline__ uint32_t mx_from_f32(const float (&f)[8], const uint32_t byte) {
  const float scale = mx_scale(byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], scale, 3);
  return w;
}

}  // namespace
}  // namespace tb
