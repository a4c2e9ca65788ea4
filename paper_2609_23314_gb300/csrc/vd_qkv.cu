// vd_qkv.cu -- vd_qkv_norm_rope (include/vd.h): from the projection rows of new
// tokens to the queries and to the new rows of one layer, in one pass.
//
// Per head of a query or key,  y = x * w / sqrt(mean(x^2) + eps),  and its first
// rotary_dim values turn in pairs (a, b) -> (a cos t - b sin t, b cos t + a sin t) by
// t = position * inv_freq.  Values are copied.  One read and one write of every value:
// bound by DRAM for prompts (16384 tokens of 48 heads of 128 values 69.7 us, 85 % of the copy
// peak; 82.5 without the early load of the next head), by launch and latency for single
// tokens (4.1 us in a graph).
#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "vd_host.cuh"

namespace vd {

namespace {

struct QkvArgs {
  const uint16_t* qkv;
  const uint16_t *q_weight, *k_weight;
  const float* inv_freq;
  const int32_t* pos_first_new;
  uint16_t *q_out, *k_new, *v_new;
  int tokens, B, n_q, n_kv, d, rd, layer, n_layer;
  int items, lanes;  // chunk pairs of a head, lanes that share a head (a power of two)
  int tokens_per_cta;
  float eps;
};

constexpr int kMaxTokens = 8;  // of a CTA

// Angle over pi, reduced to [-1, 1].  The product and its reduction are in fp64:
// in fp32 a position of 10^6 would leave an error of 0.06.
__device__ __forceinline__ float half_turns(double pos, float inv_freq) {
  const double t = pos * (double)inv_freq * 0.31830988618379067154;
  return (float)(t - 2.0 * rint(0.5 * t));
}

__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// A thread holds two 8-value chunks of a head that turn together: chunks j and
// j + rotary_dim / 16 (pairs (i, i + rotary_dim / 2)), or, interleaved, 2 j and 2 j + 1;
// behind rotary_dim, neighbours.  `lanes` threads hold a head and share the sum of its
// squares; the cosines of the CTA's tokens are made once, in shared memory, for all heads.
template <bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) qkv_norm_rope_kernel(QkvArgs a) {
  extern __shared__ __align__(16) float table[];  // [token][cos half | sin half]
  __shared__ size_t new_row[kMaxTokens];          // a token's row of the new rows' first head
  const int half = a.rd >> 1;
  const int tok0 = (int)blockIdx.x * a.tokens_per_cta;
  const int n_tok = min(a.tokens - tok0, a.tokens_per_cta);
  const int heads = a.n_q + 2 * a.n_kv;
  const int j = threadIdx.x % a.lanes, slots = kThreads / a.lanes;
  const int rot8 = a.rd >> 3, d8 = a.d >> 3;  // chunks that turn, chunks
  int c0, c1;
  if (INTERLEAVED || j >= rot8 / 2) {
    c0 = 2 * j;
    c1 = 2 * j + 1;
  } else {
    c0 = j;
    c1 = j + rot8 / 2;
  }
  const bool active = j < a.items, second = active && c1 < d8;
  const int items = n_tok * heads;
  grid_dependency_wait();
  grid_launch_dependents();
  const uint16_t* src = a.qkv + (size_t)tok0 * heads * a.d;
  uint4 n0 = make_uint4(0, 0, 0, 0), n1 = n0;  // the next item's chunks
  auto fetch = [&](int it) {
    const uint16_t* p = src + (size_t)it * a.d;
    if (active && it < items) n0 = ld_cg16(p + c0 * 8);
    if (second && it < items) n1 = ld_cg16(p + c1 * 8);
  };
  fetch(threadIdx.x / a.lanes);
  if (threadIdx.x < n_tok) {
    const int tok = tok0 + threadIdx.x;
    new_row[threadIdx.x] = ((size_t)(tok / a.B) * a.n_layer + a.layer) * a.n_kv * a.B + tok % a.B;
  }
  for (int i = threadIdx.x; i < n_tok * half; i += kThreads) {
    const int t = i / half, f = i % half, tok = tok0 + t;
    const double pos = (double)((long long)a.pos_first_new[tok / a.B] + tok % a.B);
    float sn, cs;
    sincospif(half_turns(pos, a.inv_freq[f]), &sn, &cs);
    table[t * a.rd + f] = cs;
    table[t * a.rd + half + f] = sn;
  }
  __syncthreads();
  for (int it = threadIdx.x / a.lanes; it < items; it += slots) {
    const int t = it / heads, h = it % heads;
    uint4 w0 = n0, w1 = n1;
    fetch(it + slots);
    uint16_t* dst;
    if (h < a.n_q) {
      dst = a.q_out + ((size_t)(tok0 + t) * a.n_q + h) * a.d;
    } else {
      const int kh = h < a.n_q + a.n_kv ? h - a.n_q : h - a.n_q - a.n_kv;
      dst = (h < a.n_q + a.n_kv ? a.k_new : a.v_new) + (new_row[t] + (size_t)kh * a.B) * a.d;
    }
    if (h < a.n_q + a.n_kv) {
      float x[8], y[8];
      unpack8(w0, x);
      unpack8(w1, y);
      const uint16_t* wt = h < a.n_q ? a.q_weight : a.k_weight;
      if (wt) {  // the same for the lanes of a head
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], fmaf(y[e], y[e], ss));
        const unsigned lane = threadIdx.x & 31;
        const unsigned mask = ((1u << a.lanes) - 1u) << (lane & ~(a.lanes - 1u));  // <= 16 lanes
        for (int off = a.lanes >> 1; off > 0; off >>= 1) ss += __shfl_xor_sync(mask, ss, off);
        const float r = 1.f / sqrtf(ss / (float)a.d + a.eps);
        float g[8];
        if (active) {
          unpack8(*reinterpret_cast<const uint4*>(wt + c0 * 8), g);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = x[e] * r * g[e];
        }
        if (second) {
          unpack8(*reinterpret_cast<const uint4*>(wt + c1 * 8), g);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = y[e] * r * g[e];
        }
      }
      if (j < rot8 / 2) {
        const float* tb = table + t * a.rd;
        const int f0 = 8 * j;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float cs = tb[f0 + e], sn = tb[half + f0 + e];
          if (INTERLEAVED) {  // frequency 8 j + e: values 2 e, 2 e + 1 of the 16
            float* z = e < 4 ? x : y;
            const int p = 2 * (e & 3);
            const float u = z[p], v = z[p + 1];
            z[p] = u * cs - v * sn;
            z[p + 1] = v * cs + u * sn;
          } else {
            const float u = x[e], v = y[e];
            x[e] = u * cs - v * sn;
            y[e] = v * cs + u * sn;
          }
        }
      }
      w0 = pack8(x);
      w1 = pack8(y);
    }
    if (active) st16(dst + c0 * 8, w0);
    if (second) st16(dst + c1 * 8, w1);
  }
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace

}  // namespace vd

extern "C" vd_status vd_qkv_norm_rope(const void* qkv, int32_t n_seq, int32_t B, int32_t n_q_head,
                                      int32_t n_kv_head, int32_t head_dim, const void* q_weight,
                                      const void* k_weight, float eps, const float* inv_freq,
                                      int32_t rotary_dim, int32_t interleaved,
                                      const int32_t* pos_first_new, void* q_out, void* k_new,
                                      void* v_new, int32_t layer, int32_t n_layer,
                                      vd_stream_t stream) {
  using namespace vd;
  if (!qkv || !q_out || !k_new || !v_new) return VD_ERR_INVALID_ARG;
  if (n_seq < 1 || B < 1 || n_q_head < 1 || n_kv_head < 1 || head_dim < 1 || n_layer < 1 ||
      layer < 0 || layer >= n_layer || rotary_dim < 0 || rotary_dim > head_dim)
    return VD_ERR_INVALID_ARG;
  if (rotary_dim > 0 && (!inv_freq || !pos_first_new)) return VD_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || eps > 1.f) return VD_ERR_INVALID_ARG;
  if (head_dim % 8 != 0) return VD_ERR_ALIGNMENT;
  if (head_dim > 256 || rotary_dim % 16 != 0) return VD_ERR_UNSUPPORTED;
  if (misaligned(qkv) || misaligned(q_weight) || misaligned(k_weight) || misaligned(q_out) ||
      misaligned(k_new) || misaligned(v_new))
    return VD_ERR_ALIGNMENT;
  const long long tokens = (long long)n_seq * B;
  if (tokens > INT_MAX - kMaxTokens || (long long)n_q_head + 2LL * n_kv_head > 65536)
    return VD_ERR_UNSUPPORTED;
  DeviceInfo dev;
  const vd_status r = device_info(&dev);
  if (r != VD_OK) return r;
  QkvArgs a;
  a.qkv = static_cast<const uint16_t*>(qkv);
  a.q_weight = static_cast<const uint16_t*>(q_weight);
  a.k_weight = static_cast<const uint16_t*>(k_weight);
  a.inv_freq = inv_freq;
  a.pos_first_new = pos_first_new;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_new = static_cast<uint16_t*>(k_new);
  a.v_new = static_cast<uint16_t*>(v_new);
  a.tokens = (int)tokens;
  a.B = B;
  a.n_q = n_q_head;
  a.n_kv = n_kv_head;
  a.d = head_dim;
  a.rd = rotary_dim;
  a.layer = layer;
  a.n_layer = n_layer;
  a.items = (head_dim / 8 + 1) / 2;
  a.lanes = 1;
  while (a.lanes < a.items) a.lanes <<= 1;
  a.eps = eps;
  // four tokens share a CTA's sines where there are enough (us at 16384 tokens: 2 tokens 74.4,
  // 4 69.7, 8 72.6)
  a.tokens_per_cta = tokens >= 8LL * dev.sms ? 4 : 1;
  const long long grid = (tokens + a.tokens_per_cta - 1) / a.tokens_per_cta;
  const size_t smem = (size_t)a.tokens_per_cta * rotary_dim * sizeof(float);
  return launch_clusters((unsigned)grid, kThreads, 1, smem, reinterpret_cast<cudaStream_t>(stream),
                         interleaved ? qkv_norm_rope_kernel<true> : qkv_norm_rope_kernel<false>,
                         a);
}
