// vd_q4_rows.cu -- rows into a cache held in 4 bits and back: vd_q4_append,
// vd_q4_pack, vd_q4_unpack (include/vd.h; the row format is in vd_q4.cuh).
//
// Bound by DRAM: 288 units of 4096 rows of 128 values into 4 bits and back 228 us for 1.55
// GB, the copy peak (two lanes a group, 16-byte accesses: 417).
#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "vd_host.cuh"
#include "vd_q4.cuh"

namespace vd {

vd_status validate_q4(const vd_q4_cache* c) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->len) return VD_ERR_INVALID_ARG;
  if (c->n_seq < 1 || c->n_layer < 1 || c->n_kv_head < 1 || c->capacity < 1 || c->head_dim < 1)
    return VD_ERR_INVALID_ARG;
  if (c->head_dim % 32 != 0 || c->capacity % 8 != 0) return VD_ERR_ALIGNMENT;
  if (c->head_dim > 256 || c->capacity > (1 << 30)) return VD_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v) |
       reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale)) & 15u)
    return VD_ERR_ALIGNMENT;
  const long long units = (long long)c->n_seq * c->n_layer * c->n_kv_head;
  if (units * 16 > INT_MAX) return VD_ERR_UNSUPPORTED;
  return VD_OK;
}

namespace {

// A thread takes a group of 16 values of K and the same one of V: a 32-byte access to each
// bf16 row, so that a warp's accesses are contiguous, and a group's scale is its own affair.
// kGroups such pairs are loaded before the first is turned, for loads in flight, in CTAs of
// kRowThreads, small ones for an even end.  us for (groups, threads) = (2, 256), (4, 256),
// (2, 128), (4, 128), (8, 128), (4, 64): pack_odd of perf/operators.py 38.6, 33.1, 38.0, 31.7, 35.6,
// 36.7; append_decode_ragged 39.4, 38.5, 39.2, 37.5, 41.7, 36.9; pack_cache 233, 230, 228, 228,
// 248, 232.  Looked at for these three alone: 432 units of up to 1100 rows of 96 values, 1792 of
// one row, 288 of 4096 rows of 128.
constexpr int kGroups = 4, kRowThreads = 128;

enum RowsOp { kAppend, kPack, kUnpack };

struct RowsArgs {
  uint8_t* q[2];         // codes of K and V
  uint8_t* scale[2];     // their scale bytes
  uint16_t* rows[2];     // bf16 rows
  const int32_t* len_in; // lengths that say which rows
  int32_t* len_out;      // pack, unpack: where they are copied to (nullable)
  unsigned* status;
  int layers, heads;     // of the call
  int q_layers, layer0;  // layers of the 4-bit cache, the first one of the call
  int q_cap, row_cap;    // rows per unit of either side (append: the new rows)
  long long items;       // append: groups of all units
  unsigned blocks;       // pack, unpack: CTAs per unit
  bool wide;             // the bf16 buffers are 32-byte aligned
};

struct Row16 {  // 16 bf16 values
  uint32_t w[8];
};

// wide: at a 32-byte boundary (buffers are only known to be 16-byte aligned)
__device__ __forceinline__ Row16 load_row16(const uint16_t* p, bool wide) {
  Row16 r;
  if (!wide) {
    const uint4 x = ld_cg16(p), y = ld_cg16(p + 8);
    return {{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w}};
  }
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]),
                 "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
               : "l"(p));
  return r;
}

__device__ __forceinline__ void store_row16(uint16_t* p, const Row16& r, bool wide) {
  if (!wide) {
    st16(p, make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]));
    st16(p + 8, make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]));
    return;
  }
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r.w[0]),
               "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]),
               "r"(r.w[7])
               : "memory");
}

// Larger magnitude of two pairs of bf16 without their signs, as integers: the order of
// magnitudes, infinities and NaN above all.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }

// A group to its code bytes (the return value) and its scale byte.
__device__ __forceinline__ uint2 quantise(const Row16& r, uint32_t& scale, unsigned* status) {
  uint32_t top = r.w[0] & 0x7fff7fffu;
#pragma unroll
  for (int i = 1; i < 8; ++i) top = max_u16x2(top, r.w[i] & 0x7fff7fffu);
  top = max(top & 0xffffu, top >> 16);
  if (top >= 0x7f80u) {
    record_status(status, kStNonfinite);
    scale = kQ4NanScale;
    return make_uint2(0u, 0u);
  }
  scale = q4_scale_byte(__uint_as_float(top << 16));
  // x / s by the reciprocal, snapped to multiples of 2^-13: x has 8 significant bits and s
  // 4, so a quotient is either a tie of the code grid, which the snap restores, or at least
  // 2^-10 away from one.  The sum takes the sign of a quotient that it rounds to 0: put back.
  const float inv = scale ? __frcp_rn(q4_scale_value(scale)) : 0.f;
  const unsigned long long inv2 = f2_pack(inv, inv), snap = f2_pack(1536.f, 1536.f);
  uint32_t code[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t w = r.w[4 * h + e];
      float lo, hi;
      f2_unpack(f2_sub(f2_fma(bf16x2_to_f2(w), inv2, snap), snap), lo, hi);
      y[2 * e] = __uint_as_float(__float_as_uint(lo) | ((w << 16) & 0x80000000u));
      y[2 * e + 1] = __uint_as_float(__float_as_uint(hi) | (w & 0x80000000u));
    }
    code[h] = q4_pack8(y);
  }
  return make_uint2(code[0], code[1]);
}

__device__ __forceinline__ Row16 values(const uint2& code, uint32_t scale) {
  Row16 r;
  const uint32_t s2 = scale * 0x00800080u;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t p[4];
    q4_unpack4(h ? code.y : code.x, p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t v = h2_mul(p[e], s2);  // exact
      float lo, hi;
      asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b; }"
          : "=f"(lo), "=f"(hi)
          : "r"(v));
      // exact in bf16 too: the upper halves (a NaN keeps its quiet bit)
      r.w[4 * h + e] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
    }
  }
  return r;
}

// append: bf16 rows [0, B) of the source to slots [len, len + B); pack: rows [0, len);
// unpack: the way back.  G: groups of a row.
template <int OP, int G>
__global__ void __launch_bounds__(kRowThreads) q4_rows_kernel(RowsArgs a) {
  grid_dependency_wait();
  grid_launch_dependents();
  bool on[kGroups];
  size_t row[kGroups], qrow[kGroups];  // group indices of both sides
  if (OP == kAppend) {
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const long long i = ((long long)blockIdx.x * kGroups + k) * kRowThreads + threadIdx.x;
      on[k] = i < a.items;
      if (!on[k]) continue;
      const long long r = i / G;
      const int g = (int)(i % G), b = (int)(r % a.row_cap);
      const long long unit = r / a.row_cap;
      const int n = __ldcg(a.len_in + unit / (a.layers * a.heads));
      if (n < 0 || n > a.q_cap - a.row_cap) {
        if (g == 0 && b == 0 && unit % (a.layers * a.heads) == 0)
          record_status(a.status, kStDeviceLen);
        on[k] = false;
        continue;
      }
      row[k] = (size_t)i;
      qrow[k] = ((size_t)unit * a.q_cap + n + b) * G + g;
    }
  } else {
    const unsigned unit = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
    const unsigned seq = unit / (a.layers * a.heads), inner = unit % (a.layers * a.heads);
    const int n = __ldcg(a.len_in + seq);
    const bool leader = threadIdx.x == 0 && block == 0 && inner == 0;
    if (n < 0 || n > a.row_cap || n > a.q_cap) {
      if (leader) record_status(a.status, kStDeviceLen);
      return;
    }
    if (leader && a.len_out) a.len_out[seq] = n;
    const size_t q0 = (((size_t)seq * a.q_layers + a.layer0 + inner / a.heads) * a.heads +
                       inner % a.heads) * a.q_cap * G;
    const size_t row0 = (size_t)unit * a.row_cap * G;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const size_t i = ((size_t)block * kGroups + k) * kRowThreads + threadIdx.x;
      on[k] = i < (size_t)n * G;
      row[k] = row0 + i;
      qrow[k] = q0 + i;
    }
  }
  if (OP == kUnpack) {
    uint2 code[kGroups][2];
    uint32_t scale[kGroups][2];
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (on[k]) {
          code[k][t] = __ldcg(reinterpret_cast<const uint2*>(a.q[t] + qrow[k] * 8));
          scale[k][t] = __ldcg(a.scale[t] + qrow[k]);
        }
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (on[k]) store_row16(a.rows[t] + row[k] * 16, values(code[k][t], scale[k][t]), a.wide);
  } else {
    Row16 x[kGroups][2];
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (on[k]) x[k][t] = load_row16(a.rows[t] + row[k] * 16, a.wide);
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (on[k]) {
          uint32_t scale;
          const uint2 code = quantise(x[k][t], scale, a.status);
          *reinterpret_cast<uint2*>(a.q[t] + qrow[k] * 8) = code;
          a.scale[t][qrow[k]] = (uint8_t)scale;
        }
  }
}

using RowsKernel = void (*)(RowsArgs);

template <int G>
constexpr RowsKernel rows_kernel_of(int op) {
  return op == kAppend ? q4_rows_kernel<kAppend, G>
         : op == kPack ? q4_rows_kernel<kPack, G>
                       : q4_rows_kernel<kUnpack, G>;
}

RowsKernel rows_kernel(int op, int d) {
  switch (d / 32) {
    case 1: return rows_kernel_of<2>(op);
    case 2: return rows_kernel_of<4>(op);
    case 3: return rows_kernel_of<6>(op);
    case 4: return rows_kernel_of<8>(op);
    case 5: return rows_kernel_of<10>(op);
    case 6: return rows_kernel_of<12>(op);
    case 7: return rows_kernel_of<14>(op);
    default: return rows_kernel_of<16>(op);
  }
}

// units of `most` rows each at most.  pack and unpack take CTAs for all of them, as the lengths
// are on the device: 288 units of 100 rows of 128 values 7.7 us at a capacity of 128, 24 at
// 4096, 592 at 131072.
vd_status launch_rows(int op, RowsArgs& a, long long units, int most, int d, cudaStream_t s) {
  a.wide = ((reinterpret_cast<uintptr_t>(a.rows[0]) | reinterpret_cast<uintptr_t>(a.rows[1])) & 31u) == 0;
  const long long per = (long long)kGroups * kRowThreads, groups = (long long)most * (d / 16);
  long long grid;
  if (op == kAppend) {
    a.items = units * groups;
    grid = (a.items + per - 1) / per;
  } else {
    a.blocks = (unsigned)((groups + per - 1) / per);
    grid = units * a.blocks;
  }
  if (grid > INT_MAX) return VD_ERR_UNSUPPORTED;
  return launch_clusters((unsigned)grid, kRowThreads, 1, 0, s, rows_kernel(op, d), a);
}

RowsArgs rows_args(const vd_q4_cache* c, int layers, int layer0, unsigned* status) {
  RowsArgs a = {};
  a.q[0] = static_cast<uint8_t*>(c->k);
  a.q[1] = static_cast<uint8_t*>(c->v);
  a.scale[0] = static_cast<uint8_t*>(c->k_scale);
  a.scale[1] = static_cast<uint8_t*>(c->v_scale);
  a.status = status;
  a.layers = layers;
  a.heads = c->n_kv_head;
  a.q_layers = c->n_layer;
  a.layer0 = layer0;
  a.q_cap = c->capacity;
  return a;
}

// pack and unpack: layers [layer0, layer0 + b->n_layer) of c against all of b
vd_status run_copy(bool pack, const vd_q4_cache* c, int32_t layer0, const vd_cache* b,
                   cudaStream_t s) {
  vd_status r = validate_q4(c);
  if (r != VD_OK) return r;
  if (!b || !b->k || !b->v || !b->len) return VD_ERR_INVALID_ARG;
  if (b->n_seq != c->n_seq || b->n_kv_head != c->n_kv_head || b->head_dim != c->head_dim ||
      b->n_layer < 1 || b->capacity < 1 || layer0 < 0 || layer0 > c->n_layer - b->n_layer)
    return VD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(b->k) | reinterpret_cast<uintptr_t>(b->v)) & 15u)
    return VD_ERR_ALIGNMENT;
  DeviceInfo dev;
  r = device_info(&dev);
  if (r != VD_OK) return r;
  RowsArgs a = rows_args(c, b->n_layer, layer0, dev.status);
  a.rows[0] = static_cast<uint16_t*>(b->k);
  a.rows[1] = static_cast<uint16_t*>(b->v);
  a.row_cap = b->capacity;
  a.len_in = pack ? b->len : c->len;
  if (pack)
    a.len_out = layer0 + b->n_layer == c->n_layer ? c->len : nullptr;
  else
    a.len_out = b->len;
  const int most = c->capacity < b->capacity ? c->capacity : b->capacity;
  return launch_rows(pack ? kPack : kUnpack, a, (long long)b->n_seq * b->n_layer * b->n_kv_head,
                     most, c->head_dim, s);
}

}  // namespace

}  // namespace vd

extern "C" {

vd_status vd_q4_append(const vd_q4_cache* c, const void* k_new, const void* v_new, int32_t B,
                       vd_stream_t stream) {
  vd_status r = vd::validate_q4(c);
  if (r != VD_OK) return r;
  if (!k_new || !v_new || B < 0 || B > c->capacity) return VD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new)) & 15u)
    return VD_ERR_ALIGNMENT;
  if (B == 0) return VD_OK;
  vd::DeviceInfo dev;
  r = vd::device_info(&dev);
  if (r != VD_OK) return r;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  vd::RowsArgs a = vd::rows_args(c, c->n_layer, 0, dev.status);
  a.rows[0] = static_cast<uint16_t*>(const_cast<void*>(k_new));  // read only
  a.rows[1] = static_cast<uint16_t*>(const_cast<void*>(v_new));
  a.row_cap = B;
  a.len_in = c->len;
  r = vd::launch_rows(vd::kAppend, a, (long long)c->n_seq * c->n_layer * c->n_kv_head, B,
                      c->head_dim, s);
  return r != VD_OK ? r : vd::launch_len_add(c->len, c->n_seq, c->capacity, B, s);
}

vd_status vd_q4_pack(const vd_q4_cache* dst, int32_t layer0, const vd_cache* src,
                     vd_stream_t stream) {
  return vd::run_copy(true, dst, layer0, src, reinterpret_cast<cudaStream_t>(stream));
}

vd_status vd_q4_unpack(const vd_q4_cache* src, int32_t layer0, const vd_cache* dst,
                       vd_stream_t stream) {
  return vd::run_copy(false, src, layer0, dst, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
