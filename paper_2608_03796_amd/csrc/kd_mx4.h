// 4-bit microscaled numbers: blocks of 32 consecutive columns, each element as
// e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; code = sign << 3 | place in
// this list; two codes a byte, the even column in the low half), each block with a
// power of two 2^(s - 127) as scale (one byte s; 255 = not a number). The scale is
// the least power of two, at least 2^-127, that brings the block's largest
// magnitude to 6 or less, so nothing saturates. An element times its scale has 2
// significant bits: exact in bf16 and fp32. Elements are off by at most a fifth of
// themselves (2.5 reads as 2), or by a quarter of the scale where they are below it.
//
// The conversions are gfx950's own, which divide and multiply by the exponent
// of their scale operand (0x00400000 = 2^-127 included) and round to the nearest,
// ties to even; a scale with exponent 255 gives not-a-number.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kd_device.h"

namespace kd {

constexpr int kMx4Block = 32;
constexpr int kMx4NaN = 255;
// At the largest scale (2^126, of magnitudes over 3 * 2^126) an element over 3.5
// would round to 4, which stands for 2^128: it is held as 3.
constexpr int kMx4TopScale = 253;

typedef __attribute__((ext_vector_type(8))) int i32x8_t;

// scale byte of a block whose largest magnitude has these bits (infinities and
// what is not a number from 0x7f800000 on)
__device__ __forceinline__ int mx4_scale(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return kMx4NaN;
  // 6 = 1.5 * 2^2: one more where the significand is over 1.5
  const int s = (int)(amax_bits >> 23) - 2 + ((amax_bits & 0x7fffffu) > 0x400000u);
  return s < 0 ? 0 : s;
}
__device__ __forceinline__ float mx4_scale_f(int s) {
  return __builtin_bit_cast(float, s == 0 ? 0x00400000u : (uint32_t)s << 23);
}

// eight values -> a dword of codes
__device__ __forceinline__ uint32_t mx4_pack8(const float (&v)[8], int s) {
  if (s == kMx4NaN) return 0u;
  const float sc = mx4_scale_f(s);
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = v[i];
    if (s == kMx4TopScale) {
      const float lim = 3.f * 0x1p126f;
      x[i] = fminf(fmaxf(x[i], -lim), lim);
    }
  }
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], sc, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], sc, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], sc, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], sc, 3);
  return r;
}

// a dword of codes -> eight bf16 (exact). `sc` is the scale's byte in the exponent
// (mx4_scale_f without the case of 0, whose exponent field reads as 2^-127)
__device__ __forceinline__ u32x4_t mx4_unpack8(uint32_t w, float sc) {
  return u32x4_t{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3))};
}

// One 16x16x128 step of two 4-bit operands: lane l holds row l % 16, columns
// 32 (l / 16) .. + 31 of each (16 bytes of codes, one block) and that block's
// scale byte in bits 0..7 of sa and sb.
__device__ __forceinline__ f32x4_t mfma_mx4(u32x4_t a, u32x4_t b, f32x4_t c, int sa, int sb) {
  const i32x8_t x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8_t y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, sa, 0, sb);
}

// eight floats -> the three bf16 terms whose sum they are: each term is the
// magnitude cut off after 8 bits (never rounded up, so the largest numbers do not
// overflow), the rests are exact. An infinity or what is not a number is its first
// term alone.
__device__ __forceinline__ void cut8(const float (&x)[8], u32x4_t (&t)[3]) {
  uint32_t w[3][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x[i]);
    const bool fin = (b & 0x7f800000u) != 0x7f800000u;
    const uint32_t h = b & 0xffff0000u;
    const float r = fin ? x[i] - __builtin_bit_cast(float, h) : 0.f;
    const uint32_t m = __builtin_bit_cast(uint32_t, r) & 0xffff0000u;
    w[0][i] = fin ? h : (b & 0x7fffffu) != 0u ? 0x7fc00000u : h;
    w[1][i] = m;
    w[2][i] = __builtin_bit_cast(uint32_t, r - __builtin_bit_cast(float, m));
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
    t[k] = u32x4_t{(w[k][0] >> 16) | (w[k][1] & 0xffff0000u), (w[k][2] >> 16) | (w[k][3] & 0xffff0000u),
                   (w[k][4] >> 16) | (w[k][5] & 0xffff0000u), (w[k][6] >> 16) | (w[k][7] & 0xffff0000u)};
}

}  // namespace kd
