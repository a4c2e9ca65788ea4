// vd_attend.cuh -- what the attention kernels share: conversions, the warp's matrix products,
// the scaling of query rows.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "vd_device.cuh"

namespace vd {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Two weights in bf16, and in `low` what that leaves of them: together within 2^-16 of a weight.
__device__ __forceinline__ uint32_t split_bf16(float x, float y, uint32_t& low) {
  const uint32_t high = pack_bf16(x, y);
  low = pack_bf16(x - __uint_as_float(high << 16), y - __uint_as_float(high & 0xffff0000u));
  return high;
}

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// c = a b in fp16, and c += a b.
__device__ __forceinline__ void mma_16816_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                                uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

template <bool BF16>
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                          uint32_t b1) {
  if (BF16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A query row's power of two: its largest magnitude goes to [2^-9, 2^-8), exact in bf16, so
// that no finite key row makes a score overflow.  The factor is 2^-126 at least: a row whose
// largest magnitude is 2^118 or more goes to something below 4, and 256 products with new keys
// below 2^118 stay finite.  For fp16 kTo16 more, at most 2^15: the 8 bits of a bf16 value fit
// down to 2^-17, 2^-21 of the row's largest; what is smaller is off by at most 2^-29 of the
// largest (the fp32 sum of a score's products is bound by 2^-23 of their magnitudes).
constexpr float kTo16 = 0x1p13f, kFrom16 = 0x1p-13f;

struct QueryScale {
  uint32_t up;  // the factor in bf16, twice
  float down;   // its inverse
};

// top: the row's largest magnitude as bf16 bits
__device__ __forceinline__ QueryScale scale_of(uint32_t top) {
  const uint32_t ex = top ? min(244u, max(1u, top >> 7)) : 118u;
  return {((245u - ex) << 7) * 0x00010001u, __uint_as_float((ex + 9u) << 23)};
}

// What a row's scores are multiplied by for log2 units.  Finite, so that a score of 0 stays one,
// and not 0, so that a masked score stays masked.  Subnormal factors count: new keys of 2^127
// make scores of up to 2^128 before it.
__device__ __forceinline__ float score_factor(float down, float scale) {
  return fminf(fmaxf(down * scale * kLog2e, 0x1p-149f), 3.40282347e38f);
}

// The same for cached tokens, whose queries are kTo16 larger.
__device__ __forceinline__ float cached_factor(float factor) {
  return fmaxf(factor * kFrom16, 0x1p-149f);
}

}  // namespace vd
