// vd_paged_rows.cu -- rows into a paged cache and back (include/vd.h): vd_paged_append, from
// projections with norms and rotation on the way (vd_qkv.cuh), vd_paged_pack and
// vd_paged_unpack, from and to the contiguous layout, and vd_paged_advance.
//
// One read and one write of every value: bound by DRAM for prompts and whole caches, by launch
// and latency for single tokens.
#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "vd_host.cuh"
#include "vd_paged.cuh"
#include "vd_qkv.cuh"

namespace vd {

vd_status validate_paged(const vd_paged_cache* c) {
  if (!c || !c->k || !c->v || !c->page_table || !c->len) return VD_ERR_INVALID_ARG;
  if (c->type != VD_PAGED_BF16 && c->type != VD_PAGED_E4M3) return VD_ERR_INVALID_ARG;
  if (c->type == VD_PAGED_BF16 && (c->k_scale || c->v_scale)) return VD_ERR_INVALID_ARG;
  if (c->n_seq < 1 || c->n_layer < 1 || c->n_kv_head < 1 || c->head_dim < 1 || c->page_size < 1 ||
      c->n_page < 1 || c->max_pages < 1)
    return VD_ERR_INVALID_ARG;
  const int64_t stride[4] = {c->layer_stride, c->page_stride, c->head_stride, c->slot_stride};
  const int extent[4] = {c->n_layer, c->n_page, c->n_kv_head, c->page_size};
  const int unit = c->type == VD_PAGED_E4M3 ? 16 : 8;  // values of 16 bytes
  bool aligned = c->head_dim % unit == 0 && !misaligned16(c->k) && !misaligned16(c->v);
  for (int i = 0; i < 4; ++i) {
    if (extent[i] > 1 && stride[i] < c->head_dim) return VD_ERR_INVALID_ARG;
    if (extent[i] > 1 && stride[i] % unit != 0) aligned = false;
  }
  if (!aligned) return VD_ERR_ALIGNMENT;
  // where a layer's rows lie is counted in 32 bits, 16 bytes each
  double span = 0;
  for (int i = 1; i < 4; ++i) span += (double)(extent[i] - 1) * (double)stride[i];
  if (span / unit >= 4294967040.0) return VD_ERR_UNSUPPORTED;
  if (c->head_dim > 256 || (long long)c->page_size * c->max_pages > (1LL << 30) ||
      c->n_seq > (1 << 20) || c->n_kv_head > 65536 ||
      (long long)c->n_seq * c->n_kv_head > INT_MAX / c->n_layer)
    return VD_ERR_UNSUPPORTED;
  return VD_OK;
}

namespace {

// ---------------------------------------------------------------------------
// rows of new tokens
// ---------------------------------------------------------------------------
struct PagedRowsArgs {
  Pages pages;
  const int32_t* n_new;          // nullable
  const int32_t* pos_first_new;  // nullable
};

// The bytes of a new token's row in its page, at the first KV head.
constexpr long long kNoRow = -1;   // its page is not one
constexpr long long kNoToken = -2; // padding, or a sequence that gets nothing

template <bool E4M3>
struct PagedRows {
  const QkvArgs& a;
  const PagedRowsArgs& p;
  long long* rows;

  __device__ void place(int t, int tok) const {
    const int seq = tok / a.B, b = tok - seq * a.B;
    const int n = __ldcg(p.pages.len + seq), add = p.n_new ? __ldcg(p.n_new + seq) : a.B;
    long long at = kNoToken;
    if (add < 0 || add > a.B || n < 0 || n > p.pages.capacity() - add) {
      record_status(p.pages.status, kStDeviceLen);
    } else if (b < add) {
      const int page = p.pages.page_of(seq, n + b);
      at = page < 0 ? kNoRow : p.pages.row(page, n + b);
    }
    rows[t] = at;
  }
  __device__ long long position(int tok) const {
    const int seq = tok / a.B, b = tok - seq * a.B;
    return (long long)(p.pos_first_new ? p.pos_first_new[seq] : __ldcg(p.pages.len + seq)) + b;
  }
  __device__ bool on(int t) const { return rows[t] != kNoToken; }
  __device__ void put(char* base, const float* scale, int t, int kh, int c,
                      const float (&x)[8]) const {
    if (rows[t] == kNoRow) return;
    char* dst = base + rows[t] + kh * p.pages.head_stride + c * (E4M3 ? 8 : 16);
    if (E4M3) {
      const float s = scale ? scale[kh] : 1.f;
      *reinterpret_cast<uint2*>(dst) =
          make_uint2(pack_e4m3(x[0] / s, x[1] / s, x[2] / s, x[3] / s),
                     pack_e4m3(x[4] / s, x[5] / s, x[6] / s, x[7] / s));
    } else {
      st16(dst, pack8(x));
    }
  }
  __device__ void key(int t, int kh, int c, const float (&x)[8]) const {
    put(p.pages.k, p.pages.k_scale, t, kh, c, x);
  }
  __device__ void value(int t, int kh, int c, const uint4& w) const {
    if (E4M3) {
      float x[8];
      unpack8(w, x);
      put(p.pages.v, p.pages.v_scale, t, kh, c, x);
    } else if (rows[t] != kNoRow) {
      st16(p.pages.v + rows[t] + kh * p.pages.head_stride + c * 16, w);
    }
  }
};

template <bool INTERLEAVED, bool E4M3>
__global__ void __launch_bounds__(kThreads) paged_append_kernel(QkvArgs a, PagedRowsArgs p) {
  extern __shared__ __align__(16) float table[];
  __shared__ long long rows[kMaxTokens];
  norm_rope_tokens<INTERLEAVED>(a, table, PagedRows<E4M3>{a, p, rows});
}

__global__ void __launch_bounds__(kThreads)
    paged_advance_kernel(int32_t* len, const int32_t* n_new, int n_seq, int cap, int B,
                         unsigned* status) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int s = blockIdx.x * kThreads + threadIdx.x;
  if (s >= n_seq) return;
  const int n = len[s], add = n_new ? n_new[s] : B;
  if (add < 0 || add > B || n < 0 || n > cap - add)
    record_status(status, kStDeviceLen);
  else
    len[s] = n + add;
}

// ---------------------------------------------------------------------------
// whole caches: pages to contiguous rows and back
// ---------------------------------------------------------------------------
struct CopyArgs {
  Pages pages;           // layer layer0; its len is not used
  long long layer_stride;  // bytes
  uint16_t *k, *v;       // the contiguous side
  const int32_t* len_in; // lengths that say which rows
  int32_t* len_out;      // where they are copied to (nullable)
  int layers, heads, cap, d;
  unsigned blocks;       // CTAs of a unit
};

constexpr int kRowsInFlight = 4;  // of K and of V, a thread

struct Values16 {  // 8 bf16 values, or 16 that are e4m3 in the pages
  uint4 w[2];
};

// A thread takes 16 bytes of a page's row of K and of V, or what becomes them; the threads of a
// CTA take whole rows, one after the other, kRowsInFlight of them at a time.
template <bool PACK, bool E4M3>
__global__ void __launch_bounds__(kThreads) paged_copy_kernel(CopyArgs a) {
  grid_dependency_wait();
  grid_launch_dependents();
  const unsigned unit = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
  const unsigned per = a.layers * a.heads;
  const int seq = unit / per, inner = unit % per, layer = inner / a.heads, head = inner % a.heads;
  const int n = __ldcg(a.len_in + seq);
  const bool leader = threadIdx.x == 0 && block == 0 && inner == 0;
  if (n < 0 || n > a.cap || n > a.pages.capacity()) {
    if (leader) record_status(a.pages.status, kStDeviceLen);
    return;
  }
  if (leader && a.len_out) a.len_out[seq] = n;
  constexpr int kValues = E4M3 ? 16 : 8;
  const int chunks = a.d / kValues, rows = kThreads / chunks;
  const int r = threadIdx.x / chunks, c = threadIdx.x % chunks;
  if (r >= rows) return;
  const long long in_page = layer * a.layer_stride + head * a.pages.head_stride + c * 16;
  const size_t in_rows = (size_t)unit * a.cap * a.d + c * kValues;
  float ks = 1.f, vs = 1.f;
  if (E4M3) {
    if (a.pages.k_scale) ks = a.pages.k_scale[inner];
    if (a.pages.v_scale) vs = a.pages.v_scale[inner];
  }
  const long long step = (long long)a.blocks * rows * kRowsInFlight;
  for (long long t0 = (long long)block * rows * kRowsInFlight + r; t0 < n; t0 += step) {
    long long at[kRowsInFlight];
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
      const long long t = t0 + i * rows;
      at[i] = -1;
      if (t < n) {
        const int page = a.pages.page_of(seq, (int)t);
        if (page >= 0) at[i] = in_page + a.pages.row(page, (int)t);
      }
    }
    Values16 x[kRowsInFlight][2];
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
      if (at[i] < 0) continue;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint16_t* row = (t ? a.v : a.k) + in_rows + (t0 + i * rows) * a.d;
        if (PACK) {
          x[i][t].w[0] = ld_cg16(row);
          if (E4M3) x[i][t].w[1] = ld_cg16(row + 8);
        } else {
          x[i][t].w[0] = ld_cg16((t ? a.pages.v : a.pages.k) + at[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
      if (at[i] < 0) continue;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        uint16_t* row = (t ? a.v : a.k) + in_rows + (t0 + i * rows) * a.d;
        char* page = (t ? a.pages.v : a.pages.k) + at[i];
        const float s = t ? vs : ks;
        if (PACK) {
          if (E4M3) {
            float y[8], z[8];
            unpack8(x[i][t].w[0], y);
            unpack8(x[i][t].w[1], z);
            st16(page, make_uint4(pack_e4m3(y[0] / s, y[1] / s, y[2] / s, y[3] / s),
                                  pack_e4m3(y[4] / s, y[5] / s, y[6] / s, y[7] / s),
                                  pack_e4m3(z[0] / s, z[1] / s, z[2] / s, z[3] / s),
                                  pack_e4m3(z[4] / s, z[5] / s, z[6] / s, z[7] / s)));
          } else {
            st16(page, x[i][t].w[0]);
          }
        } else if (E4M3) {
          const uint32_t w[4] = {x[i][t].w[0].x, x[i][t].w[0].y, x[i][t].w[0].z, x[i][t].w[0].w};
          uint32_t o[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float lo, hi;
            asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b; }"
                : "=f"(lo), "=f"(hi)
                : "r"(e4m3_to_h2(w[e >> 1], e & 1)));
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[e]) : "f"(hi * s), "f"(lo * s));
          }
          st16(row, make_uint4(o[0], o[1], o[2], o[3]));
          st16(row + 8, make_uint4(o[4], o[5], o[6], o[7]));
        } else {
          st16(row, x[i][t].w[0]);
        }
      }
    }
  }
}

vd_status run_paged_copy(bool pack, const vd_paged_cache* c, int32_t layer0, const vd_cache* b,
                         cudaStream_t s) {
  vd_status r = validate_paged(c);
  if (r != VD_OK) return r;
  if (!b || !b->k || !b->v || !b->len) return VD_ERR_INVALID_ARG;
  if (b->n_seq != c->n_seq || b->n_kv_head != c->n_kv_head || b->head_dim != c->head_dim ||
      b->n_layer < 1 || b->capacity < 1 || layer0 < 0 || layer0 > c->n_layer - b->n_layer)
    return VD_ERR_INVALID_ARG;
  if (misaligned16(b->k) || misaligned16(b->v)) return VD_ERR_ALIGNMENT;
  DeviceInfo dev;
  r = device_info(&dev);
  if (r != VD_OK) return r;
  const bool e4m3 = c->type == VD_PAGED_E4M3;
  CopyArgs a;
  a.pages = pages_of(c, layer0, dev.status);
  a.layer_stride = c->layer_stride * (e4m3 ? 1 : 2);
  a.k = static_cast<uint16_t*>(b->k);
  a.v = static_cast<uint16_t*>(b->v);
  a.layers = b->n_layer;
  a.heads = b->n_kv_head;
  a.cap = b->capacity;
  a.d = b->head_dim;
  a.len_in = pack ? b->len : c->len;
  a.len_out = !pack ? b->len : layer0 + b->n_layer == c->n_layer ? c->len : nullptr;
  // CTAs for a few waves at most, each going on over its unit's rows: the lengths are on the
  // device, and a large capacity costs nothing beyond them
  const long long units = (long long)b->n_seq * b->n_layer * b->n_kv_head;
  const long long most = (long long)c->page_size * c->max_pages < b->capacity
                             ? (long long)c->page_size * c->max_pages
                             : b->capacity;
  const int rows = kThreads / (b->head_dim / (e4m3 ? 16 : 8)) * kRowsInFlight;
  long long blocks = (most + rows - 1) / rows, want = (32LL * dev.sms + units - 1) / units;
  if (blocks > want) blocks = want;
  a.blocks = (unsigned)blocks;
  if (units * blocks > INT_MAX) return VD_ERR_UNSUPPORTED;
  void (*kern)(CopyArgs) = pack ? (e4m3 ? paged_copy_kernel<true, true> : paged_copy_kernel<true, false>)
                                : (e4m3 ? paged_copy_kernel<false, true> : paged_copy_kernel<false, false>);
  return launch_clusters((unsigned)(units * blocks), kThreads, 1, 0, s, kern, a);
}

}  // namespace

}  // namespace vd

extern "C" {

vd_status vd_paged_append(const vd_paged_cache* c, int32_t layer, const void* qkv, int32_t B,
                          int32_t n_q_head, const int32_t* n_new, const void* q_weight,
                          const void* k_weight, float eps, const float* inv_freq,
                          int32_t rotary_dim, int32_t interleaved, const int32_t* pos_first_new,
                          void* q_out, vd_stream_t stream) {
  using namespace vd;
  vd_status r = validate_paged(c);
  if (r != VD_OK) return r;
  if (layer < 0 || layer >= c->n_layer) return VD_ERR_INVALID_ARG;
  r = validate_qkv(qkv, c->n_seq, B, n_q_head, c->n_kv_head, c->head_dim, q_weight, k_weight, eps,
                   inv_freq, rotary_dim, q_out);
  if (r != VD_OK) return r;
  DeviceInfo dev;
  r = device_info(&dev);
  if (r != VD_OK) return r;
  const QkvArgs a = qkv_args(qkv, c->n_seq, B, n_q_head, c->n_kv_head, c->head_dim, q_weight,
                             k_weight, eps, inv_freq, rotary_dim, q_out, dev.sms);
  const PagedRowsArgs p = {pages_of(c, layer, dev.status), n_new, pos_first_new};
  const bool e4m3 = c->type == VD_PAGED_E4M3;
  void (*kern)(QkvArgs, PagedRowsArgs) =
      interleaved ? (e4m3 ? paged_append_kernel<true, true> : paged_append_kernel<true, false>)
                  : (e4m3 ? paged_append_kernel<false, true> : paged_append_kernel<false, false>);
  return launch_clusters(qkv_grid(a), kThreads, 1, qkv_smem(a),
                         reinterpret_cast<cudaStream_t>(stream), kern, a, p);
}

vd_status vd_paged_advance(const vd_paged_cache* c, const int32_t* n_new, int32_t B,
                           vd_stream_t stream) {
  using namespace vd;
  vd_status r = validate_paged(c);
  if (r != VD_OK) return r;
  if (B < 0) return VD_ERR_INVALID_ARG;
  DeviceInfo dev;
  r = device_info(&dev);
  if (r != VD_OK) return r;
  return launch_dependent((unsigned)((c->n_seq + kThreads - 1) / kThreads),
                          reinterpret_cast<cudaStream_t>(stream), paged_advance_kernel, c->len,
                          n_new, c->n_seq, c->page_size * c->max_pages, B, dev.status);
}

vd_status vd_paged_pack(const vd_paged_cache* dst, int32_t layer0, const vd_cache* src,
                        vd_stream_t stream) {
  return vd::run_paged_copy(true, dst, layer0, src, reinterpret_cast<cudaStream_t>(stream));
}

vd_status vd_paged_unpack(const vd_paged_cache* src, int32_t layer0, const vd_cache* dst,
                          vd_stream_t stream) {
  return vd::run_paged_copy(false, src, layer0, dst, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
