// vd_q4_rows.cu -- rows into a cache held in 4 bits and back: vd_q4_append,
// vd_q4_pack, vd_q4_unpack (include/vd.h; the row format is in vd_q4.cuh).
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
  if (c->head_dim > 256) return VD_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v) |
       reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale)) & 15u)
    return VD_ERR_ALIGNMENT;
  const long long units = (long long)c->n_seq * c->n_layer * c->n_kv_head;
  if (units * 16 > INT_MAX) return VD_ERR_UNSUPPORTED;
  return VD_OK;
}

namespace {

// One CTA per block of kRowsPerCta rows of one unit and both its tensors.  A thread
// takes 8 values: a 16-byte access to the bf16 row, so that a warp's accesses are
// contiguous, and the two lanes of a group share its largest magnitude.
constexpr int kRowsPerCta = 32;

struct RowsArgs {
  uint8_t* q[2];         // codes of K and V
  uint8_t* scale[2];     // their scale bytes
  uint16_t* rows[2];     // bf16 rows
  const int32_t* len_in; // lengths that say which rows
  int32_t* len_out;      // pack, unpack: where they are copied to (nullable)
  unsigned* status;
  int layers, heads;     // of the call
  int q_layers, layer0;  // layers of the 4-bit cache, the first one of the call
  int q_cap, row_cap;    // rows per unit of either side
  int count;             // rows of the call per unit (append), -1: the length
  int d;
  unsigned blocks;       // CTAs per unit
};

__device__ __forceinline__ float abs_max8(const uint4& w, float (&x)[8]) {
  unpack8(w, x);
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
  return m;
}

__device__ __forceinline__ bool any_nonfinite(const uint4& w) {
  const uint32_t a[4] = {w.x, w.y, w.z, w.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= (a[i] & 0x7f80u) == 0x7f80u || (a[i] & 0x7f800000u) == 0x7f800000u;
  return bad;
}

// PACK: bf16 rows to 4 bits (append: rows [0, count) of the source to slots
// [len, len + count); pack: rows [0, len)); else 4 bits to bf16, rows [0, len).
template <bool PACK>
__global__ void __launch_bounds__(kThreads) q4_rows_kernel(RowsArgs a) {
  grid_dependency_wait();
  grid_launch_dependents();
  const unsigned unit = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
  const unsigned seq = unit / (a.layers * a.heads);
  const unsigned inner = unit % (a.layers * a.heads);
  const int n = __ldcg(a.len_in + seq);
  const bool append = a.count >= 0;
  const int rows = append ? a.count : n;
  const int first = append ? n : 0;
  const bool leader = threadIdx.x == 0 && block == 0 && inner == 0;
  if (n < 0 || rows > a.row_cap || first > a.q_cap - rows) {
    if (leader) record_status(a.status, kStDeviceLen);
    return;
  }
  if (leader && a.len_out) a.len_out[seq] = n;
  const unsigned layer = inner / a.heads, head = inner % a.heads;
  const size_t qrow0 =
      (((size_t)seq * a.q_layers + a.layer0 + layer) * a.heads + head) * a.q_cap + first;
  const size_t row0 = (size_t)unit * a.row_cap;
  const int d8 = a.d >> 3, per = kRowsPerCta * d8;
  const int r0 = (int)block * kRowsPerCta;
  // a row's lanes are even in number (d is a multiple of 32), so the two lanes of a
  // group are neighbours and leave the loop together
  for (int i = threadIdx.x; i < 2 * per; i += kThreads) {
    const int t = i >= per;
    const int j = t ? i - per : i;
    const int row = r0 + j / d8, c = j % d8;
    if (row < rows) {
      uint16_t* src = (t ? a.rows[1] : a.rows[0]) + (row0 + row) * a.d + c * 8;
      uint8_t* q = (t ? a.q[1] : a.q[0]) + (qrow0 + row) * (a.d >> 1) + c * 4;
      uint8_t* scale = (t ? a.scale[1] : a.scale[0]) + (qrow0 + row) * (a.d >> 4) + (c >> 1);
      if (PACK) {
        const uint4 w = ld_cg16(src);
        float x[8], y[8];
        float m = abs_max8(w, x);
        const unsigned pair = 3u << (threadIdx.x & 30);
        bool bad = any_nonfinite(w);
        m = fmaxf(m, __shfl_xor_sync(pair, m, 1));
        bad |= __shfl_xor_sync(pair, (int)bad, 1) != 0;
        uint32_t sb = bad ? kQ4NanScale : q4_scale_byte(m);
        if (bad) record_status(a.status, kStNonfinite);
        // x / s by the reciprocal, snapped to 16 bits: x has 8 significant bits and s 4,
        // so a quotient is either a tie of the code grid with at most 3 bits, which the
        // snap restores, or at least 2^-8 of itself away from one
        const float s = q4_scale_value(sb);
        const float inv = sb ? __frcp_rn(s) : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          y[e] = __uint_as_float((__float_as_uint(x[e] * inv) + 0x80u) & 0xffffff00u);
        *reinterpret_cast<uint32_t*>(q) = bad ? 0u : q4_pack8(y);
        if ((c & 1) == 0) *scale = (uint8_t)sb;
      } else {
        uint32_t h[4];
        q4_unpack4(__ldcg(reinterpret_cast<const uint32_t*>(q)), h);
        const uint32_t s2 = (uint32_t)__ldcg(scale) * 0x00800080u;
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t p = h2_mul(h[e], s2);  // exact
          float lo, hi;
          asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b; }"
              : "=f"(lo), "=f"(hi)
              : "r"(p));
          // exact in bf16 too: the upper halves (a NaN keeps its quiet bit)
          o[e] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
        }
        st16(src, make_uint4(o[0], o[1], o[2], o[3]));
      }
    }
  }
}

vd_status launch_rows(bool pack, RowsArgs& a, long long units, int most, cudaStream_t s) {
  a.blocks = (unsigned)((most + kRowsPerCta - 1) / kRowsPerCta);
  const long long grid = units * a.blocks;
  if (grid > INT_MAX) return VD_ERR_UNSUPPORTED;
  return launch_dependent((unsigned)grid, s, pack ? q4_rows_kernel<true> : q4_rows_kernel<false>, a);
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
  a.d = c->head_dim;
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
  a.count = -1;
  a.len_in = pack ? b->len : c->len;
  if (pack)
    a.len_out = layer0 + b->n_layer == c->n_layer ? c->len : nullptr;
  else
    a.len_out = b->len;
  const int most = c->capacity < b->capacity ? c->capacity : b->capacity;
  return launch_rows(pack, a, (long long)b->n_seq * b->n_layer * b->n_kv_head, most, s);
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
  a.count = B;
  a.len_in = c->len;
  r = vd::launch_rows(true, a, (long long)c->n_seq * c->n_layer * c->n_kv_head, B, s);
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
