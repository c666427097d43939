// The 8-bit cache format: e4m3 codes with one power of two (an e8m0 byte c, for
// 2^(c - 127)) for each block of kQ8Block tokens, KV head, and of K and V.
//
//   value = code * 2^(c - 127)
//   c     = the smallest byte with amax <= 448 * 2^(c - 127), amax the largest
//           finite magnitude of the block's tokens (448: the largest e4m3 value)
//   code  = x * 2^(127 - c) rounded to the nearest e4m3 value, ties to even;
//           an infinity or NaN is stored as NaN
//
// A power of two costs no accuracy against amax / 448 (e4m3 has three mantissa
// bits at any scale, and 2^15 between its largest and its smallest normal value)
// and buys two things: scaling is exact, so a code depends on nothing but x and
// c, and codes are re-scaled exactly when a block's power of two changes, but for
// those that fall below 2^-6, where e4m3's steps stop shrinking.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "cmc_internal.cuh"

namespace cmc {

constexpr int kQ8Block = 32;

// Bytes of one (unit, K or V) row of powers of two for T tokens: one a block,
// padded so that each 128-token tile's four lie in one aligned word.
__host__ __device__ inline int q8_scale_bytes(int T) { return (T + 127) / 128 * 4; }

// 2^(c - 127); 255 is NaN.
__device__ __forceinline__ float e8m0_to_f32(int c) {
  return __uint_as_float(c == 0 ? 0x00400000u : c == 255 ? 0x7FFFFFFFu : static_cast<uint32_t>(c) << 23);
}
// 2^(127 - c), what values are multiplied by to give codes.
__device__ __forceinline__ float code_factor(int c) { return e8m0_to_f32(c == 255 ? 255 : 254 - c); }
// 2^(c_old - c), what a block's codes are multiplied by when its byte goes from
// c_old to c.  Limited to fp32's normal powers: below them every code gives 0.
__device__ __forceinline__ float recode_factor(int c_old, int c) {
  return c_old == 255 ? e8m0_to_f32(255)
                      : __uint_as_float(static_cast<uint32_t>(min(max(127 + c_old - c, 1), 254)) << 23);
}
// The byte of a block from the bits of its largest finite magnitude (fp32):
// 448 = 1.75 * 2^8.
__device__ __forceinline__ int block_code(uint32_t amax_bits) {
  return max(0, static_cast<int>(amax_bits >> 23) - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}
// |x| as bits, 0 for an infinity or NaN.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}

// Two values to e4m3 (round to nearest even; `lo` in the low byte).
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// x * f, NaN for an infinite x (which the conversion would store as 448).
__device__ __forceinline__ float scaled(float x, float f) { return fmaf(x, 0.f, x * f); }
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float f) {
  return e4m3_pair(scaled(a, f), scaled(b, f)) | (e4m3_pair(scaled(c, f), scaled(d, f)) << 16);
}
// Four codes to fp32.
__device__ __forceinline__ void decode4(uint32_t w, float (&v)[4]) {
  uint32_t lo, hi;
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n"
      " cvt.rn.f16x2.e4m3x2 %1, b;\n}\n"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}\n"
      : "=f"(v[0]), "=f"(v[1])
      : "r"(lo));
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}\n"
      : "=f"(v[2]), "=f"(v[3])
      : "r"(hi));
}

// 16 codes multiplied by f and rounded again.
__device__ __forceinline__ uint32_t recode4(uint32_t w, float f) {
  float v[4];
  decode4(w, v);
  return e4m3_pair(v[0] * f, v[1] * f) | (e4m3_pair(v[2] * f, v[3] * f) << 16);
}
__device__ __forceinline__ uint4 recode16(const uint4& x, float f) {
  return make_uint4(recode4(x.x, f), recode4(x.y, f), recode4(x.z, f), recode4(x.w, f));
}
// The largest magnitude code of 16 that are no NaN, bytewise in the result's
// four bytes with `m`'s (e4m3 magnitudes are ordered as their bits).
__device__ __forceinline__ uint32_t max_codes4(uint32_t m, uint32_t w) {
  w &= 0x7F7F7F7Fu;
  return __vmaxu4(m, w & ~__vcmpeq4(w, 0x7F7F7F7Fu));
}
__device__ __forceinline__ uint32_t max_codes16(uint32_t m, const uint4& x) {
  return max_codes4(max_codes4(max_codes4(max_codes4(m, x.x), x.y), x.z), x.w);
}
// The fp32 bits of the value of a largest magnitude code (see max_codes4) of a block with byte c,
// 0 if the byte is NaN.
__device__ __forceinline__ uint32_t held_bits(uint32_t m, int c) {
  m = __vmaxu4(m, m >> 16);
  m = max(m & 0xFFu, (m >> 8) & 0xFFu);
  float v[4];
  decode4(m, v);
  return c == 255 ? 0u : finite_bits(v[0] * e8m0_to_f32(c));
}

}  // namespace cmc
