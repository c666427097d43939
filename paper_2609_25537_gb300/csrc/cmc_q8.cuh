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
// The byte of a block from the bits of its largest finite magnitude (fp32, or with an exponent beyond:
// held_bits): 448 = 1.75 * 2^8.
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
// Four codes to fp16, exactly (lo: bytes 0 and 1).
__device__ __forceinline__ void codes_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n"
      " cvt.rn.f16x2.e4m3x2 %1, b;\n}\n"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
// Two fp16 values to fp32.
__device__ __forceinline__ void f16x2_f32(uint32_t h, float& a, float& b) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}\n"
      : "=f"(a), "=f"(b)
      : "r"(h));
}
// Four codes to fp32.
__device__ __forceinline__ void decode4(uint32_t w, float (&v)[4]) {
  uint32_t lo, hi;
  codes_f16(w, lo, hi);
  f16x2_f32(lo, v[0], v[1]);
  f16x2_f32(hi, v[2], v[3]);
}

// Codes for another power of two are the old ones multiplied by 2^(c_old - c) and rounded again, in
// fp16 and two steps (2^17, from the least code to the largest, is above fp16's largest).  Nothing is
// lost on the way: codes are multiples of 2^-9, so a product below fp16's 2^-24 a step has no bits that
// count, being below 2^-20, which e4m3 rounds to 0 (as it does all below 2^-10).
struct Recode {
  uint32_t first, second;  // fp16 factors, in both halves
};
__device__ __forceinline__ Recode recode_by(int c_old, int c) {
  const int n = c_old - c, a = min(max(n, -14), 9), b = min(max(n - a, -14), 9);
  return {c_old == 255 ? 0x7FFF7FFFu : static_cast<uint32_t>(15 + a) * 0x04000400u,
          static_cast<uint32_t>(15 + b) * 0x04000400u};
}
__device__ __forceinline__ uint32_t recode4(uint32_t w, const Recode& f) {
  uint32_t lo, hi, r;
  codes_f16(w, lo, hi);
  asm("mul.rn.f16x2 %0, %0, %1;\n" : "+r"(lo) : "r"(f.first));
  asm("mul.rn.f16x2 %0, %0, %1;\n" : "+r"(hi) : "r"(f.first));
  asm("mul.rn.f16x2 %0, %0, %1;\n" : "+r"(lo) : "r"(f.second));
  asm("mul.rn.f16x2 %0, %0, %1;\n" : "+r"(hi) : "r"(f.second));
  asm("{\n .reg .b16 a, b;\n cvt.rn.satfinite.e4m3x2.f16x2 a, %1;\n cvt.rn.satfinite.e4m3x2.f16x2 b, %2;\n"
      " mov.b32 %0, {a, b};\n}\n"
      : "=r"(r)
      : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ uint4 recode16(const uint4& x, const Recode& f) {
  return make_uint4(recode4(x.x, f), recode4(x.y, f), recode4(x.z, f), recode4(x.w, f));
}
// The largest magnitudes of 16 codes that are no NaN and of `m`, in fp16, two at a time.  (In bytes, the
// codes' bits being ordered as their magnitudes, it takes four times the instructions.)
__device__ __forceinline__ uint32_t max_codes4(uint32_t m, uint32_t w) {
  uint32_t lo, hi;
  codes_f16(w, lo, hi);
  asm("{\n .reg .b32 a, b;\n abs.f16x2 a, %1;\n abs.f16x2 b, %2;\n max.f16x2 %0, %0, a;\n max.f16x2 %0, %0, b;\n}\n"
      : "+r"(m)
      : "r"(lo), "r"(hi));
  return m;
}
__device__ __forceinline__ uint32_t max_codes16(uint32_t m, const uint4& x) {
  return max_codes4(max_codes4(max_codes4(max_codes4(m, x.x), x.y), x.z), x.w);
}
// The value of the larger of two largest magnitudes (max_codes16) of a block with byte c as fp32 bits, 0 if the
// byte is NaN.  The code's bits get the byte's exponent in whole numbers, which goes past fp32's largest (bf16's
// is stored as 2^128, and a byte may say up to 448 * 2^127); what falls below its smallest normal
// value comes out too small, and gives the byte 0 as it should.
__device__ __forceinline__ uint32_t held_bits(uint32_t m, int c) {
  float a, b;
  f16x2_f32(m, a, b);
  const uint32_t bits = __float_as_uint(fmaxf(a, b)), down = static_cast<uint32_t>(max(127 - c, 0)) << 23;
  if (c == 255 || bits <= down) return 0u;
  return c >= 127 ? bits + (static_cast<uint32_t>(c - 127) << 23) : bits - down;
}

}  // namespace cmc
