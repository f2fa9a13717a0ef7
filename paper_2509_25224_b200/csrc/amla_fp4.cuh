// The 4-bit cache: what a page holds and how its numbers are read.
//
// A page is 64 keys: 64 rows of 288 bytes, E2M1 numbers (sign, 2 exponent bits with bias 1, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4,
// 6), two to a byte with the lower column in the low half, then 64 rows of 36 E4M3 scales, one for 16 neighbouring columns.
// value = e2m1 * e4m3 * kv_scale.  The product of an E2M1 and an E4M3 number has at most six significant bits and lies
// between 2^-10 and 2688 in magnitude: f16 and bf16 hold it exactly.
#pragma once

#include <stdint.h>

#include "amla_common.cuh"

namespace amla {

constexpr int kGroup = 16;                                       // columns that share a scale
constexpr int kCodeRow = kDqk / 2, kScaleRow = kDqk / kGroup;    // 288 and 36 bytes a key
constexpr int kCodeBytes = kPage * kCodeRow;                     // the scales begin here
constexpr int kPageBytes4 = kCodeBytes + kPage * kScaleRow;      // 20 736

// Factors with which every step of the format (2^-9 .. 448 times kv_scale) stays a normal FP32 number.
inline bool fp4_scale_ok(float kv_scale) { return kv_scale >= 0x1p-100f && kv_scale <= 0x1p100f; }

// Two E4M3 bytes (low 16 bits) -> two f16, exact (NaN stays NaN).
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t pair) {
  uint32_t h2;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(static_cast<unsigned short>(pair)));
  return h2;
}
// Four bytes of two E2M1 numbers each -> four pairs of f16, exact; the low half of a byte becomes the low half of a pair.
__device__ __forceinline__ void e2m1x8_to_f16x2(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}


// What a store makes of numbers: the larger of two (NaN if one is), the quotient by a group's step, two E2M1 numbers to a byte.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// x / step, inv = fl(1 / step) (0 for a group of zeros).  What is beyond E2M1's 6 by far saturates whatever its last bits are (and the
// remainder of an infinity is a NaN).  The sign is x's, of a zero too (the remainder of -0 is +0).
__device__ __forceinline__ float quotient(float x, float step, float inv) {
  const float y = x * inv;
  return copysignf(fabsf(y) < 16.f ? fmaf(fmaf(-y, step, x), inv, y) : y, x);
}
// low half: a, high half: b
__device__ __forceinline__ uint32_t e2m1_byte(float a, float b) {
  uint32_t r;
  asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

}  // namespace amla
