// vd_paged_attend.cu -- vd_paged_attend (include/vd.h): the kernel, the join of its parts, the
// host side.
//
//   s_j = scale * q . k_j,  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
//
// in one pass over the slots with a running maximum m and sum.
#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "vd_host.cuh"
#include "vd_paged.cuh"
#include "vd_paged_attend.cuh"

namespace vd {

namespace {

constexpr int kTileRows = 4;
constexpr int kMaxDim = 256;

struct Row8 {
  float x[8];
};

template <bool E4M3>
__device__ __forceinline__ Row8 load8(const char* p, float scale) {
  Row8 r;
  if (E4M3) {
    const uint2 w = __ldcg(reinterpret_cast<const uint2*>(p));
    const uint32_t h[4] = {e4m3_to_h2(w.x, false), e4m3_to_h2(w.x, true), e4m3_to_h2(w.y, false),
                           e4m3_to_h2(w.y, true)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b; }"
          : "=f"(r.x[2 * i]), "=f"(r.x[2 * i + 1])
          : "r"(h[i]));
      r.x[2 * i] *= scale;
      r.x[2 * i + 1] *= scale;
    }
  } else {
    unpack8(ld_cg16(p), r.x);
  }
  return r;
}

// A lane has 8 of the head's values (head_dim 256 fills a warp), a warp a token at a time.
template <bool E4M3>
__global__ void __launch_bounds__(kThreads, 1) paged_attend_kernel(PagedAttendArgs a) {
  __shared__ long long sh[kWarps + 1 + kThreads];
  __shared__ float part[kWarps][kTileRows][kMaxDim / 8][8];
  __shared__ float stat[kWarps][kTileRows][2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dependency_wait();
  grid_launch_dependents();
  write_empty(a);
  Walk walk(a, sh, kWarps);
  if (threadIdx.x == 0) a.split[blockIdx.x] = make_int4(-1, 0, 0, 0);
  const bool on = lane < a.d / 8;
  const Row8 zero = {};
  Share s;
  while (walk.next(s)) {
    Row8 q[kTileRows], o[kTileRows];
    float m[kTileRows], l[kTileRows];
    int sees[kTileRows];
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
      const long long row = out_row(a, s, i);
      q[i] = on && row >= 0 ? load8<false>(reinterpret_cast<const char*>(a.q + row * a.d + lane * 8), 1.f)
                            : zero;
      o[i] = zero;
      m[i] = -INFINITY;
      l[i] = 0.f;
      sees[i] = a.causal ? s.w.len + (s.tile * kTileRows + i) / a.group + 1 : s.w.len;
    }
    const float ks = a.pages.k_scale ? a.pages.k_scale[s.head] : 1.f;
    const float vs = a.pages.v_scale ? a.pages.v_scale[s.head] : 1.f;
    const long long in = s.head * a.pages.head_stride + lane * (E4M3 ? 8 : 16);
    for (int stage = s.s0 + warp; stage < s.s1; stage += kWarps) {
      const int last = min(s.w.total, (stage + 1) * kStageKeys);
      for (int t = stage * kStageKeys; t < last; ++t) {
        const int page = a.pages.page_of(s.seq, t);
        if (page < 0) continue;
        const long long at = a.pages.row(page, t) + in;
        const Row8 k = on ? load8<E4M3>(a.pages.k + at, ks) : zero;
        const Row8 v = on ? load8<E4M3>(a.pages.v + at, vs) : zero;
#pragma unroll
        for (int i = 0; i < kTileRows; ++i) {
          float x = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) x = fmaf(q[i].x[e], k.x[e], x);
#pragma unroll
          for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(kFull, x, off);
          x *= a.scale;
          x = x * kLog2e;
          if (t >= sees[i] || x == -INFINITY) continue;
          const float top = fmaxf(m[i], x), f = exp2f(m[i] - top), p = exp2f(x - top);
          m[i] = top;
          l[i] = l[i] * f + p;
#pragma unroll
          for (int e = 0; e < 8; ++e) o[i].x[e] = o[i].x[e] * f + p * v.x[e];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
      if (l[i] != l[i] && m[i] == -INFINITY) m[i] = 0.f;  // all scores NaN: so is the output
      if (on)
#pragma unroll
        for (int e = 0; e < 8; ++e) part[warp][i][lane][e] = o[i].x[e];
      if (lane == 0) {
        stat[warp][i][0] = m[i];
        stat[warp][i][1] = l[i];
      }
    }
    __syncthreads();
    // warp i joins row i
    if (warp < kTileRows) {
    float top = -INFINITY, sum = 0.f;
    Row8 y = zero;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stat[w][warp][0]);
    for (int w = 0; w < kWarps; ++w) {
      const float f = stat[w][warp][0] == -INFINITY ? 0.f : exp2f(stat[w][warp][0] - top);
      if (f == 0.f) continue;
      sum += f * stat[w][warp][1];
      if (on)
#pragma unroll
        for (int e = 0; e < 8; ++e) y.x[e] += f * part[w][warp][lane][e];
    }
    const long long row = out_row(a, s, warp);
    if (s.whole) {
      if (row >= 0) {
        const float r = top == -INFINITY ? 0.f : 1.f / sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) y.x[e] *= r;
        if (on) st16(a.out + row * a.d + lane * 8, pack8(y.x));
        if (a.lse && lane == 0) a.lse[row] = (top + log2f(sum)) * kLn2;
      }
    } else {
      const size_t at = (size_t)s.slot * kTileRows + warp;
      if (on) {
        float4* dst = reinterpret_cast<float4*>(a.parts + at * a.d + lane * 8);
        dst[0] = make_float4(y.x[0], y.x[1], y.x[2], y.x[3]);
        dst[1] = make_float4(y.x[4], y.x[5], y.x[6], y.x[7]);
      }
      if (lane == 0) a.stats[at] = make_float2(top, sum);
      if (threadIdx.x == 0 && s.s0 == 0) a.split[blockIdx.x] = walk.split_of(s);
    }
    }
    __syncthreads();
  }
}

// A CTA puts together one row of the unit that CTA `first` of the kernel before begins and
// does not end.
__global__ void __launch_bounds__(kThreads) paged_join_kernel(PagedAttendArgs a) {
  __shared__ float part[kWarps][kMaxDim];
  __shared__ float stat[kWarps][2];
  grid_dependency_wait();
  grid_launch_dependents();
  const int first = blockIdx.x / a.rows, i = blockIdx.x % a.rows;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int4 unit = __ldcg(a.split + first);
  if (unit.x < 0) return;
  Share s;
  s.seq = unit.x;
  s.head = unit.y;
  s.tile = unit.z;
  s.w = seq_work(a, s.seq, false);
  const long long row = out_row(a, s, i);
  if (row < 0) return;
  const int n = unit.w - first + 1;
  auto at = [&](int p) { return (size_t)(2 * (first + p) + (p == 0 ? 1 : 0)) * a.rows + i; };
  float top = -INFINITY, sum = 0.f, y[kMaxDim / 32];
#pragma unroll
  for (int e = 0; e < kMaxDim / 32; ++e) y[e] = 0.f;
  for (int p = warp; p < n; p += kWarps) {
    const float2 st = __ldcg(a.stats + at(p));
    const float m = fmaxf(top, st.x);
    const float f = top == -INFINITY ? 0.f : exp2f(top - m), g = st.x == -INFINITY ? 0.f : exp2f(st.x - m);
    top = m;
    sum = sum * f + (g == 0.f ? 0.f : g * st.y);
#pragma unroll
    for (int e = 0; e < kMaxDim / 32; ++e)
      if (e * 32 + lane < a.d) {
        const float v = __ldcg(a.parts + at(p) * a.d + e * 32 + lane);
        y[e] = y[e] * f + (g == 0.f ? 0.f : g * v);
      }
  }
#pragma unroll
  for (int e = 0; e < kMaxDim / 32; ++e) part[warp][e * 32 + lane] = y[e];
  if (lane == 0) {
    stat[warp][0] = top;
    stat[warp][1] = sum;
  }
  __syncthreads();
  top = -INFINITY;
  sum = 0.f;
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stat[w][0]);
  float z = 0.f;
  for (int w = 0; w < kWarps; ++w) {
    const float f = stat[w][0] == -INFINITY ? 0.f : exp2f(stat[w][0] - top);
    if (f == 0.f) continue;
    sum += f * stat[w][1];
    z += f * part[w][threadIdx.x];
  }
  if (threadIdx.x < a.d) {
    z = top == -INFINITY ? 0.f : z / sum;
    uint16_t h;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(z));
    a.out[row * a.d + threadIdx.x] = h;
  }
  if (threadIdx.x == 0 && a.lse) a.lse[row] = (top + log2f(sum)) * kLn2;
}

struct Plan {
  int rows, ctas;
  size_t split, stats, parts;  // bytes of the workspace's three parts
};

// Refuses what the call refuses of its sizes.
vd_status plan_of(const vd_paged_cache* c, int n_q_head, int B, Plan* plan) {
  vd_status r = validate_paged(c);
  if (r != VD_OK) return r;
  if (B < 1 || n_q_head < 1 || n_q_head % c->n_kv_head != 0) return VD_ERR_INVALID_ARG;
  const long long rows = (long long)B * (n_q_head / c->n_kv_head);
  if (rows > (1 << 24) || c->n_seq * (long long)c->n_kv_head > INT_MAX / rows)
    return VD_ERR_UNSUPPORTED;
  DeviceInfo dev;
  r = device_info(&dev);
  if (r != VD_OK) return r;
  plan->rows = kTileRows;
  plan->ctas = 2 * dev.sms;
  const size_t parts = 2 * (size_t)plan->ctas * plan->rows;
  plan->split = (size_t)plan->ctas * sizeof(int4);
  plan->stats = parts * sizeof(float2);
  plan->parts = parts * c->head_dim * sizeof(float);
  return VD_OK;
}

}  // namespace

}  // namespace vd

extern "C" {

size_t vd_paged_attend_workspace(const vd_paged_cache* c, int32_t n_q_head, int32_t B) {
  vd::Plan p;
  return vd::plan_of(c, n_q_head, B, &p) == VD_OK ? p.split + p.stats + p.parts : 0;
}

vd_status vd_paged_attend(const vd_paged_cache* c, int32_t layer, const void* q, int32_t B,
                          int32_t n_q_head, const int32_t* n_new, int32_t causal, float scale,
                          void* out, float* lse_out, void* workspace, size_t workspace_bytes,
                          vd_stream_t stream) {
  using namespace vd;
  vd_status r = validate_paged(c);
  if (r != VD_OK) return r;
  if (!q || !out || !workspace || layer < 0 || layer >= c->n_layer || !(scale > 0.f) ||
      scale > 3.4e38f || B < 1 || n_q_head < 1 || n_q_head % c->n_kv_head != 0)
    return VD_ERR_INVALID_ARG;
  if (misaligned16(q) || misaligned16(out) || misaligned16(workspace)) return VD_ERR_ALIGNMENT;
  Plan p;
  r = plan_of(c, n_q_head, B, &p);
  if (r != VD_OK) return r;
  if (workspace_bytes < p.split + p.stats + p.parts) return VD_ERR_INVALID_ARG;
  DeviceInfo dev;
  r = device_info(&dev);
  if (r != VD_OK) return r;
  PagedAttendArgs a;
  a.pages = pages_of(c, layer, dev.status);
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse_out;
  a.n_new = n_new;
  char* w = static_cast<char*>(workspace);
  a.split = reinterpret_cast<int4*>(w);
  a.stats = reinterpret_cast<float2*>(w + p.split);
  a.parts = reinterpret_cast<float*>(w + p.split + p.stats);
  a.n_seq = c->n_seq;
  a.heads = c->n_kv_head;
  a.group = n_q_head / c->n_kv_head;
  a.B = B;
  a.d = c->head_dim;
  a.rows = p.rows;
  a.causal = causal != 0;
  a.scale = scale;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  r = launch_dependent((unsigned)p.ctas, s,
                       c->type == VD_PAGED_E4M3 ? paged_attend_kernel<true>
                                                : paged_attend_kernel<false>,
                       a);
  if (r != VD_OK) return r;
  return launch_dependent((unsigned)(p.ctas * p.rows), s, paged_join_kernel, a);
}

}  // extern "C"
