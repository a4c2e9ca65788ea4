// vd_paged_rows.cu -- rows into a paged cache and back (include/vd.h): vd_paged_append, from
// projections with norms and rotation on the way (vd_qkv.cuh), vd_paged_pack and
// vd_paged_unpack, from and to the contiguous layout, and vd_paged_advance.
//
// One read and one write of every value.  Whole caches are bound by DRAM (36 layers of 8 heads and
// 4096 slots out of pages and back 364 us, 98 % of the copy peak); prompts by the issue of the norms'
// and the rotation's instructions (16384 tokens of 48 heads 78 us, 5.1 TB/s); ragged 8-bit pages (183 MB
// 52 us) by neither, 0.46 instructions a cycle and scheduler: their CTAs are short, each with a chain of
// latencies before its first row (lengths, scan, page), and come in 1.6 to 2.4 waves, as the grid goes by
// capacities; single tokens by launch and latency (5.3 us in a graph).
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
  static constexpr bool kRows = false;
  __device__ bool on(int t) const { return rows[t] != kNoToken; }
  __device__ void put(char* base, const float* scale, int t, int kh, int c,
                      const float (&x)[8]) const {
    if (rows[t] == kNoRow) return;
    char* dst = base + rows[t] + kh * p.pages.head_stride + c * (E4M3 ? 8 : 16);
    if (E4M3) {
      const Divisor by(scale ? __ldcg(scale + kh) : 1.f);
      *reinterpret_cast<uint2*>(dst) = pack_quotients(by, x);
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

template <bool INTERLEAVED, bool E4M3, bool FEW>
__global__ void __launch_bounds__(kThreads, FEW ? 2 : E4M3 ? 3 : 5) paged_append_kernel(QkvArgs a, PagedRowsArgs p) {
  extern __shared__ __align__(16) float table[];
  __shared__ long long rows[kMaxTokens];
  norm_rope_tokens<INTERLEAVED, FEW>(a, table, PagedRows<E4M3>{a, p, rows});
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
  Pages pages;             // layer layer0; its len is not used
  long long layer_stride;  // bytes
  uint16_t *k, *v;         // the contiguous side
  const int32_t* len_in;   // lengths that say which rows
  int32_t* len_out;        // where they are copied to (nullable)
  int n_seq, units, heads, cap, d;  // units: layers x heads
};

constexpr int kRowsInFlight = 2;  // of K and of V, a thread, twice

// The copies of all sequences make a line: a block of rows of the first one in unit (layer and
// head) after unit, the next block, and so on.  Each CTA takes an equal piece of it, whatever the
// lengths are.  A thread takes 8 values of some rows of K and of V.  A block's pages are looked up once for its units, for which they are the same, and the
// loads of the next unit are under way while one is stored.
template <bool PACK, bool E4M3>
__global__ void __launch_bounds__(kThreads, PACK && E4M3 ? 2 : 3) paged_copy_kernel(CopyArgs a) {
  __shared__ long long sums[kWarps];
  __shared__ long long found[2];
  grid_dependency_wait();
  grid_launch_dependents();
  const int chunks = a.d / 8, rows = kThreads / chunks, per_block = rows * kRowsInFlight;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // Rows of a sequence, none where either side is too short for its length: what the line is cut by,
  // and what the walk along it goes by, which passes over refused sequences too.
  auto rows_of = [&](int s, bool report) {
    if (s >= a.n_seq) return 0;
    const int n = __ldcg(a.len_in + s);
    if (n >= 0 && n <= a.cap && n <= a.pages.capacity()) return n;
    if (report) record_status(a.pages.status, kStDeviceLen);
    return 0;
  };
  auto blocks_of = [&](int n) { return (n + per_block - 1) / per_block; };
  // sum over the CTA's threads up to this one, and over all
  auto scan = [&](long long x, long long& all) {
    const long long upto = warp_scan_i64(x);
    __syncthreads();
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    long long before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += sums[w];
      all += sums[w];
    }
    return before + upto;
  };
  long long all = 0, upto = 0, mine = 0;
  if (a.n_seq > kThreads) {
    long long x = 0;
    for (int s = threadIdx.x; s < a.n_seq; s += kThreads) x += blocks_of(rows_of(s, blockIdx.x == 0));
    scan(x, all);
  } else {
    mine = blocks_of(rows_of(threadIdx.x, blockIdx.x == 0));
    upto = scan(mine, all);
  }
  if (a.len_out)
    for (int s = blockIdx.x * kThreads + threadIdx.x; s < a.n_seq; s += gridDim.x * kThreads) {
      const int n = __ldcg(a.len_in + s);
      if (n >= 0 && n <= a.cap && n <= a.pages.capacity()) a.len_out[s] = n;
    }
  // this CTA's piece, the block and the sequence of its first position
  const long long line = all * a.units;
  const long long per = line / gridDim.x, more = line - per * gridDim.x;
  long long at = per * blockIdx.x + min((long long)blockIdx.x, more);
  const long long end = at + per + (blockIdx.x < more ? 1 : 0);
  if (at >= end) return;
  long long block = at / a.units;
  int u = (int)(at - block * a.units);
  long long base = 0;  // of a chunk of sequences
  for (int chunk = 0;; chunk += kThreads) {
    if (a.n_seq > kThreads) {
      mine = blocks_of(rows_of(chunk + threadIdx.x, false));
      long long here;
      upto = base + scan(mine, here);
      all = base + here;
    }
    if (block < upto && block >= upto - mine) {
      found[0] = chunk + threadIdx.x;
      found[1] = block - (upto - mine);
    }
    __syncthreads();
    if (block < all) break;
    if (chunk + kThreads >= a.n_seq) return;  // the lengths have changed since the line was cut
    base = all;
  }
  int seq = (int)found[0];
  block = found[1];
  const int r = threadIdx.x / chunks, c = threadIdx.x - r * chunks;

  struct Data {
    uint4 w[kRowsInFlight][2];  // of an e4m3 row the first two words
    float scale[2];
  };
  // Where a unit lies on both sides
  struct Place {
    long long page, row;  // bytes, values
    int u, head;
  };
  auto place = [&](int unit) {
    const int layer = unit / a.heads, head = unit - layer * a.heads;
    return Place{layer * a.layer_stride + head * a.pages.head_stride,
                 ((long long)seq * a.units + unit) * a.cap * a.d, unit, head};
  };
  const long long to_layer = a.layer_stride - (a.heads - 1) * a.pages.head_stride,
                  to_unit = (long long)a.cap * a.d;
  auto step = [&](Place& p) {
    p.row += to_unit;
    ++p.u;
    if (++p.head == a.heads) {
      p.head = 0;
      p.page += to_layer;
    } else {
      p.page += a.pages.head_stride;
    }
  };
  while (at < end && seq < a.n_seq) {
    const int n = rows_of(seq, false);
    if (block >= blocks_of(n)) {
      ++seq;
      block = 0;
      continue;
    }
    const int u1 = (int)min((long long)a.units, u + (end - at));
    const long long t0 = block * per_block + r;
    constexpr uint32_t kNoRow = 0xffffffffu;
    uint32_t in_pages[kRowsInFlight];  // rows, in 16 bytes
#pragma unroll
    for (int i = 0; i < kRowsInFlight; ++i) {
      const long long t = t0 + i * rows;
      const int page = r < rows && t < n ? a.pages.page_of(seq, (int)t) : -1;
      in_pages[i] = page < 0 ? kNoRow : (uint32_t)(a.pages.row(page, (int)t) >> 4);
    }
    const long long in_rows = t0 * a.d + c * 8, in_page = c * (E4M3 ? 8 : 16);
    auto load = [&](const Place& p, Data& x) {
      if (E4M3) {
        x.scale[0] = a.pages.k_scale ? __ldcg(a.pages.k_scale + p.u) : 1.f;
        x.scale[1] = a.pages.v_scale ? __ldcg(a.pages.v_scale + p.u) : 1.f;
      }
#pragma unroll
      for (int i = 0; i < kRowsInFlight; ++i) {
        if (in_pages[i] == kNoRow) continue;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const char* page =
              (t ? a.pages.v : a.pages.k) + (p.page + in_page) + (size_t)in_pages[i] * 16;
          if (PACK) {
            x.w[i][t] = ld_cg16((t ? a.v : a.k) + (p.row + in_rows) + i * rows * a.d);
          } else if (E4M3) {
            const uint2 w = __ldcg(reinterpret_cast<const uint2*>(page));
            x.w[i][t].x = w.x;
            x.w[i][t].y = w.y;
          } else {
            x.w[i][t] = ld_cg16(page);
          }
        }
      }
    };
    auto store = [&](const Place& p, const Data& x) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const Divisor by(PACK && E4M3 ? x.scale[t] : 1.f);
#pragma unroll
        for (int i = 0; i < kRowsInFlight; ++i) {
          if (in_pages[i] == kNoRow) continue;
          uint16_t* row = (t ? a.v : a.k) + (p.row + in_rows) + i * rows * a.d;
          char* page =
              (t ? a.pages.v : a.pages.k) + (p.page + in_page) + (size_t)in_pages[i] * 16;
          const uint4& w = x.w[i][t];
          if (PACK && E4M3) {
            float y[8];
            unpack8(w, y);
            *reinterpret_cast<uint2*>(page) = pack_quotients(by, y);
          } else if (PACK) {
            st16(page, w);
          } else if (E4M3) {
            const uint32_t in[2] = {w.x, w.y};
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float lo, hi;
              asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b; }"
                  : "=f"(lo), "=f"(hi)
                  : "r"(e4m3_to_h2(in[e >> 1], e & 1)));
              asm("cvt.rn.bf16x2.f32 %0, %1, %2;"
                  : "=r"(o[e])
                  : "f"(hi * x.scale[t]), "f"(lo * x.scale[t]));
            }
            st16(row, make_uint4(o[0], o[1], o[2], o[3]));
          } else {
            st16(row, w);
          }
        }
      }
    };
    Data x, y;
    Place from = place(u), to = from;
    load(from, x);
    for (int i = u; i < u1; i += 2) {
      if (i + 1 < u1) {
        step(from);
        load(from, y);
      }
      store(to, x);
      step(to);
      if (i + 2 < u1) {
        step(from);
        load(from, x);
      }
      if (i + 1 < u1) {
        store(to, y);
        step(to);
      }
    }
    at += u1 - u;
    u = 0;
    ++block;
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
  a.n_seq = b->n_seq;
  a.units = b->n_layer * b->n_kv_head;
  a.heads = b->n_kv_head;
  a.cap = b->capacity;
  a.d = b->head_dim;
  a.len_in = pack ? b->len : c->len;
  a.len_out = !pack ? b->len : layer0 + b->n_layer == c->n_layer ? c->len : nullptr;
  const long long most = (long long)c->page_size * c->max_pages < b->capacity
                             ? (long long)c->page_size * c->max_pages
                             : b->capacity;
  // Pieces for many waves, so that none lasts long, of 16 units at least (the length's look-up and
  // the pages' have to pay)
  const int per_block = kThreads / (b->head_dim / 8) * kRowsInFlight;
  const long long line = (most + per_block - 1) / per_block * b->n_seq * a.units;
  const long long pieces = (line + 15) / 16, some = 32LL * dev.sms;
  const long long ctas = pieces < some ? pieces : some;
  void (*kern)(CopyArgs) = pack ? (e4m3 ? paged_copy_kernel<true, true> : paged_copy_kernel<true, false>)
                                : (e4m3 ? paged_copy_kernel<false, true> : paged_copy_kernel<false, false>);
  return launch_clusters((unsigned)ctas, kThreads, 1, 0, s, kern, a);
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
  using Kernel = void (*)(QkvArgs, PagedRowsArgs);
  static const Kernel kernels[2][2][2] = {  // [interleaved][e4m3][few tokens]
      {{paged_append_kernel<false, false, false>, paged_append_kernel<false, false, true>},
       {paged_append_kernel<false, true, false>, paged_append_kernel<false, true, true>}},
      {{paged_append_kernel<true, false, false>, paged_append_kernel<true, false, true>},
       {paged_append_kernel<true, true, false>, paged_append_kernel<true, true, true>}}};
  const Kernel kern = kernels[interleaved != 0][e4m3][a.tokens_per_cta == 1];
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
