// vd_paged.cuh -- a paged cache (vd_paged_cache in include/vd.h): where its rows lie, what
// every call checks of it.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "vd_host.cuh"

namespace vd {

constexpr unsigned kStDevicePage = 11;

// One layer of a paged cache, for kernels.  Offsets and strides are in bytes.
struct Pages {
  char *k, *v;
  const float *k_scale, *v_scale;  // of the layer's heads (nullable)
  const int32_t* table;
  const int32_t* len;
  unsigned* status;
  long long page_stride, head_stride, slot_stride;
  int page_size, n_page, max_pages;
  uint32_t per_page;  // 2^(30 + page_shift) / page_size, rounded up
  int page_shift;

  // The place of a slot's page in the table, slot / page_size: exact for slots below 2^30.
  __device__ __forceinline__ int place_of(int slot) const {
    return (int)(__umulhi((uint32_t)slot << 2, per_page) >> page_shift);
  }
  __device__ __forceinline__ int capacity() const { return page_size * max_pages; }
  // The page that holds a slot, -1 (recorded) if the table names none.
  __device__ __forceinline__ int page_of(int seq, int slot) const {
    const int p = __ldcg(table + (size_t)seq * max_pages + place_of(slot));
    if ((unsigned)p < (unsigned)n_page) return p;
    record_status(status, kStDevicePage);
    return -1;
  }
  // Offset of a slot's row of the first KV head.
  __device__ __forceinline__ long long row(int page, int slot) const {
    return page * page_stride + (slot - place_of(slot) * page_size) * slot_stride;
  }
};

// Sums over the lanes up to this one.
__device__ __forceinline__ long long warp_scan_i64(long long x) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long y = __shfl_up_sync(kFull, x, off);
    if (lane >= off) x += y;
  }
  return x;
}

vd_status validate_paged(const vd_paged_cache* c);

inline Pages pages_of(const vd_paged_cache* c, int layer, unsigned* status) {
  const int size = c->type == VD_PAGED_E4M3 ? 1 : 2;
  Pages p;
  p.k = static_cast<char*>(c->k) + layer * c->layer_stride * size;
  p.v = static_cast<char*>(c->v) + layer * c->layer_stride * size;
  p.k_scale = c->k_scale ? c->k_scale + (size_t)layer * c->n_kv_head : nullptr;
  p.v_scale = c->v_scale ? c->v_scale + (size_t)layer * c->n_kv_head : nullptr;
  p.table = c->page_table;
  p.len = c->len;
  p.status = status;
  p.page_stride = c->page_stride * size;
  p.head_stride = c->head_stride * size;
  p.slot_stride = c->slot_stride * size;
  p.page_size = c->page_size;
  p.n_page = c->n_page;
  p.max_pages = c->max_pages;
  // for slots n < 2^30: n / page_size = n per_page >> 30 + page_shift, as per_page page_size
  // exceeds 2^(30 + page_shift) by less than page_size <= 2^page_shift
  p.page_shift = 0;
  while ((1LL << p.page_shift) < c->page_size) ++p.page_shift;
  p.per_page = (uint32_t)(((1ull << (30 + p.page_shift)) + c->page_size - 1) / c->page_size);
  return p;
}

// Four fp32 values to e4m3, the first in the lowest byte: to nearest, ties to even,
// magnitudes above 448 to 448, NaN to NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  uint32_t r;
  asm("{ .reg .b16 l, h;\n"
      "cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n"
      "cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n"
      "mov.b32 %0, {l, h}; }"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}

// y / s for the rounding to e4m3 that follows: the fp32 quotient, correctly rounded, wherever it is
// between 2^-11 and 2^9 (smaller ones become 0, larger ones 448, whatever their last bits).
// From y times the rounded inverse, which is off by 1.5 units in the last place, by two steps
// q + (y - q s) inverse with one rounding each: the first leaves one unit, and the second rounds
// correctly (Markstein's theorem on quotients from a correctly rounded inverse, which excepts a
// divisor whose significand is all ones).  Divisors that the steps do not suit are divided by.
struct Divisor {
  float s, inverse;
  bool plain;
  __device__ __forceinline__ explicit Divisor(float scale) : s(scale), inverse(1.f / scale) {
    plain = !(scale >= 0x1p-60f && scale <= 0x1p60f) ||
            (__float_as_uint(scale) & 0x7fffffu) == 0x7fffffu;
  }
  __device__ __forceinline__ void operator()(float& x, float& y) const {
    const unsigned long long xy = f2_pack(x, y), inv = f2_pack(inverse, inverse),
                             minus = f2_pack(-s, -s), first = f2_mul(xy, inv);
    const unsigned long long second = f2_fma(f2_fma(first, minus, xy), inv, first);
    const unsigned long long third = f2_fma(f2_fma(second, minus, xy), inv, second);
    float x0, y0, x1, y1;
    f2_unpack(first, x0, y0);
    f2_unpack(third, x1, y1);
    x = fabsf(x0) < 0x1p10f && fabsf(x0) > 0x1p-12f ? x1 : x0;
    y = fabsf(y0) < 0x1p10f && fabsf(y0) > 0x1p-12f ? y1 : y0;
  }
};

// Eight values to e4m3.
__device__ __forceinline__ uint2 pack_quotients(const Divisor& by, const float (&v)[8]) {
  float x[8];
  if (by.plain) {  // the same for the threads of a head
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i] / by.s;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      x[i] = v[i];
      x[i + 1] = v[i + 1];
      by(x[i], x[i + 1]);
    }
  }
  return make_uint2(pack_e4m3(x[0], x[1], x[2], x[3]), pack_e4m3(x[4], x[5], x[6], x[7]));
}

// Two e4m3 values (the low or the high half of w) to two fp16 ones, exactly.
__device__ __forceinline__ uint32_t e4m3_to_h2(uint32_t w, bool high) {
  uint32_t r;
  if (high)
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %1; cvt.rn.f16x2.e4m3x2 %0, h; }" : "=r"(r) : "r"(w));
  else
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %1; cvt.rn.f16x2.e4m3x2 %0, l; }" : "=r"(r) : "r"(w));
  return r;
}

}  // namespace vd
