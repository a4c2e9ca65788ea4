// vd_qkv.cuh -- the pass from the projection rows of new tokens to queries, keys and values,
// shared by vd_qkv_norm_rope (new rows of a contiguous cache, vd_qkv.cu) and vd_paged_append
// (pages, vd_paged_rows.cu).
//
// Per head of a query or key,  y = x * w / sqrt(mean(x^2) + eps),  and its first
// rotary_dim values turn in pairs (a, b) -> (a cos t - b sin t, b cos t + a sin t) by
// t = position * inv_freq.  Values are copied.  One read and one write of every value.
#pragma once

#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "vd_host.cuh"

namespace vd {

struct QkvArgs {
  const uint16_t* qkv;
  const uint16_t *q_weight, *k_weight;
  const float* inv_freq;
  uint16_t* q_out;
  int tokens, B, n_q, n_kv, d, rd;
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

// x times r times w, rounded after each.
__device__ __forceinline__ void scale8(float (&x)[8], float r, const uint4& w) {
  const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    f2_unpack(f2_mul(f2_mul(f2_pack(x[2 * e], x[2 * e + 1]), f2_pack(r, r)), bf16x2_to_f2(in[e])),
              x[2 * e], x[2 * e + 1]);
}

// A thread holds two 8-value chunks of a head that turn together: chunks j and
// j + rotary_dim / 16 (pairs (i, i + rotary_dim / 2)), or, interleaved, 2 j and 2 j + 1;
// behind rotary_dim, neighbours.  `lanes` threads hold a head and share the sum of its
// squares; the cosines of the CTA's tokens are made once, in shared memory, for all heads.
// table: [token][cos half | sin half].  Sink: where keys and values go,
//   place(t, tok)  by one thread for each token t of the CTA, before the others are called
//   position(tok)  of a token (any thread)
//   kRows          every head goes to a bf16 row, which
//     row(t, kh, key)  names (of the keys, or of the values); else
//     on(t)            whether the token's heads are written at all
//     key(t, kh, c, x), value(t, kh, c, w)  chunk c of a KV head, in fp32 and as it came
// Rows have one store for all heads and their place by a quotient, the others by steps: 16384 tokens
// into rows 69.4 us (72.0 the other way), into 8-bit pages 97.1 (101.7), where what is live around the
// conversions leaves no registers for it.
// FEW (a token a CTA, and all CTAs run at once or nearly): the norm weights are loaded with the first
// values, not where they are wanted: one token 4.9 us in a graph for 6.4; with many tokens their
// registers cost CTAs of the SM (16384 tokens 91 us for 81 into pages; 608 into rows 9.5 for 7.5).
template <bool INTERLEAVED, bool FEW, class Sink>
__device__ __forceinline__ void norm_rope_tokens(const QkvArgs& a, float* table, const Sink& sink) {
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
  uint4 early[2][2];  // FEW: of queries, of keys
  if (FEW) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint16_t* w = k ? a.k_weight : a.q_weight;
      early[k][0] = early[k][1] = make_uint4(0, 0, 0, 0);
      if (w && active) early[k][0] = *reinterpret_cast<const uint4*>(w + c0 * 8);
      if (w && second) early[k][1] = *reinterpret_cast<const uint4*>(w + c1 * 8);
    }
  }
  if (threadIdx.x < n_tok) sink.place(threadIdx.x, tok0 + threadIdx.x);
  for (int i = threadIdx.x; i < n_tok * half; i += kThreads) {
    const int t = i / half, f = i % half, tok = tok0 + t;
    const double pos = (double)sink.position(tok);
    float sn, cs;
    sincospif(half_turns(pos, a.inv_freq[f]), &sn, &cs);
    table[t * a.rd + f] = cs;
    table[t * a.rd + half + f] = sn;
  }
  __syncthreads();
  const int dt = slots / heads, dh = slots - dt * heads;  // of a round
  int step_t = (int)(threadIdx.x / a.lanes) / heads,
      step_h = (int)(threadIdx.x / a.lanes) - step_t * heads;
  auto advance = [&] {
    step_t += dt;
    step_h += dh;
    if (step_h >= heads) {
      step_h -= heads;
      ++step_t;
    }
  };
  for (int it = threadIdx.x / a.lanes; it < items; it += slots, advance()) {
    const int t = Sink::kRows ? it / heads : step_t, h = Sink::kRows ? it % heads : step_h;
    uint4 w0 = n0, w1 = n1;
    fetch(it + slots);
    uint16_t* dst = nullptr;  // kRows: of the head
    if constexpr (Sink::kRows) {
      if (h < a.n_q) {
        dst = a.q_out + ((size_t)(tok0 + t) * a.n_q + h) * a.d;
      } else {
        const bool key = h < a.n_q + a.n_kv;
        dst = sink.row(t, key ? h - a.n_q : h - a.n_q - a.n_kv, key);
      }
    } else {
      if (!sink.on(t)) continue;
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
        if (active) {
          scale8(x, r, FEW ? (h < a.n_q ? early[0][0] : early[1][0])
                           : *reinterpret_cast<const uint4*>(wt + c0 * 8));
        }
        if (second) {
          scale8(y, r, FEW ? (h < a.n_q ? early[0][1] : early[1][1])
                           : *reinterpret_cast<const uint4*>(wt + c1 * 8));
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
      if constexpr (Sink::kRows) {
        w0 = pack8(x);
        w1 = pack8(y);
      } else if (h >= a.n_q) {
        if (active) sink.key(t, h - a.n_q, c0, x);
        if (second) sink.key(t, h - a.n_q, c1, y);
      } else {
        dst = a.q_out + ((size_t)(tok0 + t) * a.n_q + h) * a.d;
        if (active) st16(dst + c0 * 8, pack8(x));
        if (second) st16(dst + c1 * 8, pack8(y));
      }
    } else if constexpr (!Sink::kRows) {
      if (active) sink.value(t, h - a.n_q - a.n_kv, c0, w0);
      if (second) sink.value(t, h - a.n_q - a.n_kv, c1, w1);
    }
    if constexpr (Sink::kRows) {
      if (active) st16(dst + c0 * 8, w0);
      if (second) st16(dst + c1 * 8, w1);
    }
  }
}

inline bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// What both calls check of the arguments that they share, before any launch.
inline vd_status validate_qkv(const void* qkv, int n_seq, int B, int n_q, int n_kv, int d,
                              const void* q_weight, const void* k_weight, float eps,
                              const float* inv_freq, int rd, const void* q_out,
                              const void* k_new = nullptr, const void* v_new = nullptr) {
  if (!qkv || !q_out) return VD_ERR_INVALID_ARG;
  if (n_seq < 1 || B < 1 || n_q < 1 || n_kv < 1 || d < 1 || rd < 0 || rd > d)
    return VD_ERR_INVALID_ARG;
  if (rd > 0 && !inv_freq) return VD_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || eps > 1.f) return VD_ERR_INVALID_ARG;
  if (d % 8 != 0) return VD_ERR_ALIGNMENT;
  if (d > 256 || rd % 16 != 0) return VD_ERR_UNSUPPORTED;
  if (misaligned16(qkv) || misaligned16(q_weight) || misaligned16(k_weight) ||
      misaligned16(q_out) || misaligned16(k_new) || misaligned16(v_new))
    return VD_ERR_ALIGNMENT;
  if ((long long)n_seq * B > INT_MAX - kMaxTokens || (long long)n_q + 2LL * n_kv > 65536)
    return VD_ERR_UNSUPPORTED;
  return VD_OK;
}

inline QkvArgs qkv_args(const void* qkv, int n_seq, int B, int n_q, int n_kv, int d,
                        const void* q_weight, const void* k_weight, float eps,
                        const float* inv_freq, int rd, void* q_out, int sms) {
  QkvArgs a;
  a.qkv = static_cast<const uint16_t*>(qkv);
  a.q_weight = static_cast<const uint16_t*>(q_weight);
  a.k_weight = static_cast<const uint16_t*>(k_weight);
  a.inv_freq = inv_freq;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.tokens = n_seq * B;
  a.B = B;
  a.n_q = n_q;
  a.n_kv = n_kv;
  a.d = d;
  a.rd = rd;
  a.items = (d / 8 + 1) / 2;
  a.lanes = 1;
  while (a.lanes < a.items) a.lanes <<= 1;
  a.eps = eps;
  // four tokens share a CTA's sines where there are enough (us at 16384 tokens: 2 tokens 74.4,
  // 4 69.7, 8 72.6)
  a.tokens_per_cta = a.tokens >= 8LL * sms ? 4 : 1;
  return a;
}

inline unsigned qkv_grid(const QkvArgs& a) {
  return (unsigned)((a.tokens + (long long)a.tokens_per_cta - 1) / a.tokens_per_cta);
}

inline size_t qkv_smem(const QkvArgs& a) {
  return (size_t)a.tokens_per_cta * a.rd * sizeof(float);
}

}  // namespace vd
