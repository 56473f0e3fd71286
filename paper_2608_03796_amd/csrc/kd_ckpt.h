// Hidden states held in 8 bits: blocks of 32 consecutive columns, each element
// as e4m3 (4 significant bits, largest value 448, subnormals below 2^-6), each
// block with a power of two 2^(s - 127) as scale (one byte s; 255 = not a
// number). The scale is the least power of two, at least 2^-127, that brings
// the block's largest magnitude to 448 or less, so nothing saturates, and a
// stored element times its scale has 4 significant bits: exact in bf16 and
// fp32 down to 2^-133, where bf16's subnormals end. Elements are off by at most 2^-4 of
// themselves, or 2^-10 of the scale where they are e4m3 subnormals.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kd_device.h"

namespace kd {

constexpr int kCkptBlock = 32;
constexpr int kCkptNaN = 255;

// scale byte of a block whose largest magnitude is amax (not a number and
// infinities as bit patterns of at least 0x7f800000)
__device__ __forceinline__ int ckpt_scale(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return kCkptNaN;
  // 448 = 1.75 * 2^8: one more where the significand is over 1.75
  const int s = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u);
  return s < 0 ? 0 : s;
}

// v_cvt_pk_fp8_f32 rounds to the nearest e4m3, ties to even. At the largest scale
// (2^120) an element of 248 and more would round to 256, which stands for 2^128:
// such elements (the last 1/32 of the types' range) are held as 240.
constexpr int kCkptTopScale = 247;
__device__ __forceinline__ uint32_t ckpt_pack4(float a, float b, float c, float d, int s) {
  if (s == kCkptNaN) return 0x7f7f7f7fu;
  const int e = 127 - s;
  const float lim = s == kCkptTopScale ? 240.f : 448.f;
  auto scaled = [&](float x) { return fminf(fmaxf(__builtin_amdgcn_ldexpf(x, e), -lim), lim); };
  int r = 0;
  r = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(a), scaled(b), r, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(c), scaled(d), r, true);
  return (uint32_t)r;
}

// the four values of a dword of codes (every value is exact in fp32)
__device__ __forceinline__ void ckpt_unpack4(uint32_t w, int s, float* v) {
  typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;
  const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  const int e = s == kCkptNaN ? 0 : s - 127;  // such a block's codes are not numbers
  v[0] = __builtin_amdgcn_ldexpf(lo[0], e);
  v[1] = __builtin_amdgcn_ldexpf(lo[1], e);
  v[2] = __builtin_amdgcn_ldexpf(hi[0], e);
  v[3] = __builtin_amdgcn_ldexpf(hi[1], e);
}

// 16 bytes of a row of T from column d on (d a multiple of 16 / sizeof(T)), as
// the checkpoint of rows of D columns holds them
template <typename T>
__device__ __forceinline__ u32x4_t ckpt_load16(const uint8_t* codes, const uint8_t* scales,
                                               int64_t row, int D, int d) {
  const int64_t at = row * D + d;
  const int s = scales[at / kCkptBlock];
  if constexpr (sizeof(T) == 2) {
    const u32x2_t w = *reinterpret_cast<const u32x2_t*>(codes + at);
    float v[8];
    ckpt_unpack4(w[0], s, v);
    ckpt_unpack4(w[1], s, v + 4);
    return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                   pack_bf16x2(v[6], v[7])};
  } else {
    float v[4];
    ckpt_unpack4(*reinterpret_cast<const uint32_t*>(codes + at), s, v);
    return __builtin_bit_cast(u32x4_t, f32x4_t{v[0], v[1], v[2], v[3]});
  }
}

}  // namespace kd
