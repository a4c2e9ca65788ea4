// vd_q4.cuh -- the 4-bit row format of vd_q4_cache (include/vd.h): 16 values along
// the head share an unsigned 8-bit scale of 5 exponent and 3 mantissa bits, and a
// value is a 4-bit code (sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6) times it.
//
// A scale byte shifted left by 7 is the scale in fp16, subnormals included.  Code
// and scale have 2 and 4 significant bits, so their product is exact in fp16 and in
// bf16: what a kernel multiplies is what the format stands for, without a rounding.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace vd {

constexpr int kQ4Group = 16;
constexpr uint32_t kQ4MaxScale = 226;  // 10240: 6 times it is below fp16's largest
constexpr uint32_t kQ4NanScale = 255;

// Four packed code pairs (the low nibble first) to fp16 pairs.
__device__ __forceinline__ void q4_unpack4(uint32_t w, uint32_t (&o)[4]) {
  asm("{ .reg .b8 a, b, c, d; mov.b32 {a, b, c, d}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, a; cvt.rn.f16x2.e2m1x2 %1, b;\n"
      "cvt.rn.f16x2.e2m1x2 %2, c; cvt.rn.f16x2.e2m1x2 %3, d; }"
      : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
      : "r"(w));
}

// Eight fp32 values to codes, rounded to nearest, ties to the even code, at most 6.
__device__ __forceinline__ uint32_t q4_pack8(const float (&y)[8]) {
  uint32_t r;
  asm("{ .reg .b8 a, b, c, d;\n"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1; cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5; cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
      "mov.b32 %0, {a, b, c, d}; }"
      : "=r"(r)
      : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return r;
}

// The scale byte for a group's largest magnitude (finite): amax / 6 rounded to
// nearest even.  The quotient's own rounding does not matter: amax has 8 significant
// bits, so a quotient that is no tie of the 4-bit grid is at least 2^-8 of itself away
// from one, and one that is a tie is exact.
__device__ __forceinline__ uint32_t q4_scale_byte(float amax) {
  const float t = __fdiv_rn(amax, 6.f);
  uint32_t b;
  if (t < 0x1p-14f) {  // subnormal: multiples of 2^-17
    b = (uint32_t)__float2int_rn(t * 0x1p17f);
  } else {
    const uint32_t u = __float_as_uint(t);
    b = ((u + 0x7ffffu + ((u >> 20) & 1u)) >> 20) - ((127 - 15) << 3);
  }
  return b < kQ4MaxScale ? b : kQ4MaxScale;
}

__device__ __forceinline__ float q4_scale_value(uint32_t byte) {
  float f;
  asm("{ .reg .b16 h; cvt.u16.u32 h, %1; cvt.f32.f16 %0, h; }" : "=f"(f) : "r"(byte << 7));
  return f;
}

__device__ __forceinline__ uint32_t h2_mul(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

}  // namespace vd
