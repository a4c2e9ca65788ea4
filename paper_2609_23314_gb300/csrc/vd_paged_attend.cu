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
#include "vd_paged_stream.cuh"

namespace vd {

namespace {

constexpr int kMaxDim = 256;

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
  const int2 size = seq_size(a, s.seq, false);
  s.w = seq_work(a, size.x, size.y);
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
  const PagedKernel* kernel;
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
  const auto& kernels = c->type == VD_PAGED_E4M3 ? kPagedE4m3 : kPagedBf16;
  plan->kernel = &kernels[(c->head_dim + 31) / 32 - 1][rows > 8];
  plan->rows = plan->kernel->rows;
  plan->ctas = dev.sms;
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
  const PagedKernel& k = *p.kernel;
  if (cudaFuncSetAttribute(k.kern, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem) !=
      cudaSuccess) {
    cudaGetLastError();
    return VD_ERR_CUDA;
  }
  r = launch_clusters((unsigned)p.ctas, (unsigned)k.threads, 1, k.smem, s, k.kern, a);
  if (r != VD_OK) return r;
  return launch_dependent((unsigned)(p.ctas * p.rows), s, paged_join_kernel, a);
}

}  // extern "C"
