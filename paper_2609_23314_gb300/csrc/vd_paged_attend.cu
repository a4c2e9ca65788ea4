// vd_paged_attend.cu -- vd_paged_attend (include/vd.h): the kernel, the join of its parts, the
// host side.
//
//   s_j = scale * q . k_j,  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
//
// in one pass over the slots with a running maximum m and sum.
#include <cuda_runtime.h>

#include <climits>
#include <cstdint>
#include <mutex>

#include "vd_host.cuh"
#include "vd_paged.cuh"
#include "vd_paged_attend.cuh"
#include "vd_paged_stream.cuh"
#include "vd_qkv.cuh"

namespace vd {

namespace {

constexpr int kMaxDim = 256;

// Puts together the rows of units that a CTA of the kernel before begins and another one ends.  A block
// for every kWarps rows of each of those CTAs.  A unit of up to kWarps parts: the blocks of the CTA that
// begins it, a warp a row, without a meeting.  Of more: the CTAs after that one are in the unit too and
// begin none, so that their blocks help: a block a row, its warps take the parts in turn (one unit over
// all CTAs would be 150 parts for a warp).  A lane has 4 of the row's values, or 8.  Against a block a
// row everywhere: 32 sequences of 4000 tokens, 8 heads, 131.1 us (132.5), 40 of 300 tokens with one of
// 100000 35.2 (36.6), 100 of 200 with one of 50000 28.4 (26.9).
constexpr int kTogether = 4;  // parts that a warp loads at once

__global__ void __launch_bounds__(kThreads)
    paged_join_kernel(const __grid_constant__ PagedAttendArgs a) {
  __shared__ float4 part[kWarps][kMaxDim / 4];
  __shared__ float2 stat[kWarps];
  grid_dependency_wait();
  grid_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int at = blockIdx.x * kWarps >> a.row_shift, sub = blockIdx.x * kWarps & (a.rows - 1);
  // the last unit begun by one of the kWarps CTAs up to `at`
  int4 unit = make_int4(-1, 0, 0, 0);
  if (lane < kWarps && lane <= at) unit = __ldcg(a.split + (at - lane));
  const uint32_t begun = __ballot_sync(0xffffffffu, unit.x >= 0);
  if (begun == 0) return;
  const int back = __ffs(begun) - 1, first = at - back;
  unit = make_int4(__shfl_sync(0xffffffffu, unit.x, back), __shfl_sync(0xffffffffu, unit.y, back),
                   __shfl_sync(0xffffffffu, unit.z, back), __shfl_sync(0xffffffffu, unit.w, back));
  const int n = unit.w - first + 1;
  const bool many = n > kWarps;
  if (!many && back > 0) return;
  const int i = many ? ((back << a.row_shift) + sub) / kWarps : sub + warp;
  if (i >= unit.z) return;
  const int begin = many ? warp : 0, step = many ? kWarps : 1;
  const int tok = (unit.y + i) / a.group, g = unit.y + i - tok * a.group;
  const long long row = unit.x + (long long)tok * a.heads * a.group + g;
  float2 total = make_float2(-INFINITY, 0.f);
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = 0.f;
  for (int p0 = begin; p0 < n; p0 += kTogether * step) {
    float2 st[kTogether];
    float4 v[kTogether][2];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const int p = p0 + j * step;
      const size_t from = (size_t)(2 * (first + p) + (p == 0 ? 1 : 0)) * a.rows + i;
      st[j] = make_float2(-INFINITY, 0.f);
      if (p < n) {
        st[j] = __ldcg(a.stats + from);
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (128 * h + 4 * lane < a.d)
            v[j][h] = __ldcg(reinterpret_cast<const float4*>(a.parts + from * a.d + 128 * h + 4 * lane));
      }
    }
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      if (st[j].x == -INFINITY) continue;  // nothing seen
      const float m = fmaxf(total.x, st[j].x);
      const float f = total.x == -INFINITY ? 0.f : exp2_approx(total.x - m);
      const float w = exp2_approx(st[j].x - m);
      total = make_float2(m, total.y * f + w * st[j].y);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (128 * h + 4 * lane < a.d) {
          y[4 * h] = y[4 * h] * f + w * v[j][h].x;
          y[4 * h + 1] = y[4 * h + 1] * f + w * v[j][h].y;
          y[4 * h + 2] = y[4 * h + 2] * f + w * v[j][h].z;
          y[4 * h + 3] = y[4 * h + 3] * f + w * v[j][h].w;
        }
    }
  }
  if (!many) {
    const float inverse = total.x == -INFINITY ? 0.f : 1.f / total.y;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (128 * h + 4 * lane < a.d)
        *reinterpret_cast<uint2*>(a.out + row * a.d + 128 * h + 4 * lane) =
            make_uint2(pack_bf16(y[4 * h] * inverse, y[4 * h + 1] * inverse),
                       pack_bf16(y[4 * h + 2] * inverse, y[4 * h + 3] * inverse));
    if (lane == 0 && a.lse) a.lse[row] = (total.x + log2f(total.y)) * kLn2;
    return;
  }
  part[warp][lane] = make_float4(y[0], y[1], y[2], y[3]);
  part[warp][32 + lane] = make_float4(y[4], y[5], y[6], y[7]);
  if (lane == 0) stat[warp] = total;
  __syncthreads();
  float top = -INFINITY, sum = 0.f, z = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stat[w].x);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const float f = stat[w].x == -INFINITY ? 0.f : exp2_approx(stat[w].x - top);
    if (stat[w].x == -INFINITY) continue;
    sum += f * stat[w].y;
    z += f * reinterpret_cast<const float*>(part[w])[threadIdx.x];
  }
  if (threadIdx.x < a.d) {
    z = top == -INFINITY ? 0.f : z / sum;
    uint16_t h;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(z));
    a.out[row * a.d + threadIdx.x] = h;
  }
  if (threadIdx.x == 0 && a.lse) a.lse[row] = (top + log2f(sum)) * kLn2;
}

// Clusters of 1 to 16 CTAs of a kernel that run at once on a device; asked for once per device and
// kernel.  They do not go by powers of two: 152 SMs hold 15 of 8 or of 9, 8 of 12, 7 of 16.
constexpr int kMaxCluster = 16;

struct Slots {
  bool ready;
  int at[kMaxCluster + 1];
};
std::mutex g_slots_mu;
Slots g_slots[64][2][8][kKinds];

vd_status slots_of(const DeviceInfo& dev, const PagedKernel& k, Slots& s) {
  std::lock_guard<std::mutex> lk(g_slots_mu);
  if (s.ready) return VD_OK;
  if (cudaFuncSetAttribute(k.kern, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem) !=
          cudaSuccess ||
      cudaFuncSetAttribute(k.kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) !=
          cudaSuccess) {
    cudaGetLastError();
    return VD_ERR_CUDA;
  }
  for (int n = 1; n <= kMaxCluster; ++n) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n * dev.sms);
    cfg.blockDim = dim3(k.threads);
    cfg.dynamicSmemBytes = k.smem;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)n;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int active = 0;
    if (cudaOccupancyMaxActiveClusters(&active, k.kern, &cfg) != cudaSuccess) {
      cudaGetLastError();
      active = 0;
    }
    s.at[n] = active;
  }
  if (s.at[1] < 1) return VD_ERR_CUDA;
  s.ready = true;
  return VD_OK;
}

// 0, 1: the streaming kernel with tiles of 8 or of 16 query rows, 2: the block kernel.  By the
// capacity, which the host knows, not by the lengths.  Up to 8 rows stream.  More: tiles of 8, which
// go over the slots once each (from L2 mostly), while they are few; us with tiles of 8 / tiles of
// 16 / block at 8 KV heads, head_dim 128, bf16:
//   one sequence of 4000 tokens, 32 rows 16.1 / 23.6 / 18.8, 48 rows 22.9 / 24.3 / 19.5; of 500, 48
//   rows 11.3 / 15.1 / 14.0; 4 of 1000, 16 rows 13.4 / 16.8 / 15.4, 24 rows 20.2 / 18.8 / 15.4; 8 of
//   500, 16 rows 19.1 / 17.4 / 14.7.
// Long sequences in a batch are bound by reading the slots: bf16 ones take tiles of 16 up to 16 rows
// (32 of 2000, 12 rows 90.5 / 62.5 / 68.7), e4m3 ones tiles of 8 up to 24, as the block kernel turns
// them to fp16 on the way (32 of 2000, 24 rows 70.0 / 83.7 / 80.9, 32 rows 88.4 / 88.5 / 81.3).
int choose_kernel(long long rows, long long units, long long capacity, bool e4m3, int sms) {
  const long long tiles8 = units * ((rows + 7) / 8);
  if (rows <= 8 || tiles8 <= (rows <= 16 || e4m3 ? 64 : 47)) return 0;
  if (capacity >= 1500) {
    if (e4m3 && rows <= 24) return 0;
    if (!e4m3 && rows <= 16 && units > sms) return 1;
  }
  return 2;
}

struct Plan {
  const PagedKernel* kernel;
  int rows, tiles, cluster, ctas;
  bool one_launch;             // no parts to join
  size_t split, stats;         // bytes of the workspace's first two parts
  size_t workspace;            // of all that a call may take
  unsigned* status;
};

// What a call over a cache of this type and head_dim takes at most: pieces of the line on all SMs (the
// streaming kernel's shared memory leaves room for one CTA on each), in the larger of its tiles.  By
// neither tokens nor sequences: a single token may go in pieces where a block of tokens takes
// clusters, and a workspace that fits the one call has to fit the other.
size_t workspace_of(const PagedKernel* kernels, int sms, int d) {
  const size_t rows = kernels[0].rows > kernels[1].rows ? kernels[0].rows : kernels[1].rows;
  return 16 + sms * (sizeof(int4) + 2 * rows * (sizeof(float2) + d * sizeof(float)));
}

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
  const bool e4m3 = c->type == VD_PAGED_E4M3;
  const int m = (c->head_dim + 31) / 32 - 1;
  const int want_kind = env_int("VD_PAGED_KERNEL", -1);
  const long long capacity = (long long)c->page_size * c->max_pages;
  const int kind = want_kind >= 0 && want_kind < kKinds
                       ? want_kind
                       : choose_kernel(rows, (long long)c->n_seq * c->n_kv_head, capacity, e4m3, dev.sms);
  const PagedKernel* kernels = (e4m3 ? kPagedE4m3 : kPagedBf16)[m];
  const PagedKernel& k = kernels[kind];
  Slots& slots = g_slots[dev.id][e4m3][m][kind];
  r = slots_of(dev, k, slots);
  if (r != VD_OK) return r;
  plan->kernel = &k;
  plan->status = dev.status;
  plan->rows = k.rows;
  plan->tiles = (int)((rows + k.rows - 1) / k.rows);
  // A cluster for each unit: the largest with which they run at once and whose CTAs have slots enough
  // to pay for the join, large clusters more of them.  us, 8 KV heads, clusters of 8 / 12: 4096 slots
  // 11.2 / 11.7, 16000 25.0 / 20.2.
  const long long units = (long long)c->n_seq * c->n_kv_head * plan->tiles;
  int n = kMaxCluster;
  while (n > 1 && (units > slots.at[n] || capacity < (n > 8 ? 512 : 128) * n)) --n;
  // Streaming: unless equal pieces are ahead, whose look at all lengths and whose join cost what 600
  // slots of a CTA do.  us, clusters / pieces, one sequence, head_dim 128: 8 KV heads of 1024 slots
  // 11.3 / 15.1, 8000 16.1 / 18.1, 16000 20.2 / 25.0; one KV head of 16000 17.4 / 15.4.
  if (kind < 2 && capacity / n > units * capacity / dev.sms + 600) n = 1;
  const int want = env_int("VD_PAGED_CLUSTER", -1);
  if (want >= 1 && want <= kMaxCluster && slots.at[want] > 0) n = want;
  plan->cluster = n;
  plan->one_launch = n > 1 || kind == 2;
  if (units * n > INT_MAX) return VD_ERR_UNSUPPORTED;
  plan->ctas = plan->one_launch ? (int)(units * n) : slots.at[1] < dev.sms ? slots.at[1] : dev.sms;
  plan->split = plan->one_launch ? 0 : (size_t)plan->ctas * sizeof(int4);
  plan->stats = plan->one_launch ? 0 : 2 * (size_t)plan->ctas * plan->rows * sizeof(float2);
  plan->workspace = workspace_of(kernels, dev.sms, c->head_dim);
  return VD_OK;
}

}  // namespace

}  // namespace vd

extern "C" {

size_t vd_paged_attend_workspace(const vd_paged_cache* c, int32_t n_q_head, int32_t B) {
  vd::Plan p;
  return vd::plan_of(c, n_q_head, B, &p) == VD_OK ? p.workspace : 0;
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
  if (workspace_bytes < p.workspace) return VD_ERR_INVALID_ARG;
  PagedAttendArgs a;
  a.pages = pages_of(c, layer, p.status);
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
  auto log2 = [](int x) {
    int e = 0;
    while (1 << e < x) ++e;
    return e;
  };
  a.page16 = (uint32_t)(a.pages.page_stride >> 4);
  a.slot16 = (uint32_t)(a.pages.slot_stride >> 4);
  a.wait_limit = wait_limit();
  a.row_shift = log2(p.rows);
  a.stage_shift = log2(p.kernel->stage_keys);
  a.causal = causal != 0;
  a.scale = scale;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  a.tiles = p.tiles;
  a.cluster = p.cluster;
  const PagedKernel& k = *p.kernel;
  r = launch_clusters((unsigned)p.ctas, (unsigned)k.threads, (unsigned)p.cluster, k.smem, s, k.kern,
                      a);
  if (r != VD_OK || p.one_launch) return r;
  // rows are 8 or 16, kWarps or twice that
  return launch_dependent((unsigned)(p.ctas * p.rows / kWarps), s, paged_join_kernel, a);
}

}  // extern "C"
