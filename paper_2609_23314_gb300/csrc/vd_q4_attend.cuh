// vd_q4_attend.cuh -- attention over one layer of a 4-bit cache (vd_q4_attend in
// include/vd.h): the streaming kernel, for few query rows per KV head.
//
//   s_ij = scale * q_i . k_j,  o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i)
//
// over the cached tokens of a sequence (4-bit rows, vd_q4.cuh) and the call's new
// tokens (bf16, causal).  One pass over the cache with a running maximum and sum.
//
// A cluster of C CTAs takes one (sequence, KV head) and a tile of 8 * NT query rows;
// its CTAs split the cached tokens, their warps take stages of kStageKeys tokens in
// turn, each with its own ring of bulk copies and its own running state, so that warps
// wait for nothing but their copies.  The partial results meet once, at the end: in the
// CTA's shared memory, then across the cluster through distributed shared memory.
//
// Per 16 tokens a warp computes  S^T = K Q^T  and  O^T += V^T P^T  with tokens and
// head dims on the 16-row side of m16n8k16, so that 8 query rows fill a tile: decode
// has 1 to 8 rows (the query heads that share a KV head) per token.  K and V go from
// codes to fp16 in registers (exact), Q goes to fp16 with each row scaled by a power of
// two (QueryScale), sums are fp32, and P is rounded to fp16: 2^-11 of a weight, its error
// averaged over the tokens (for the new rows, in bf16, to two parts).  Weights are relative to a
// point 2^15 below the running maximum (kLift), so that those far below it keep their bits: the
// smallest that does not become 0 is 2^-40 of the largest, 27 nats down (17 without the lift).
// About 21 warp instructions a token at head_dim 128, 128 of them in 16 tokens on half-rate
// pipes (conversions and fp16 products).  While an SM is active it issues 2.4 instructions a
// cycle of 4 and the ALU pipe is at 52 %: half-rate pipes and latency bound it, not the issue;
// 5.3 ns a token and SM (its 144 bytes take 3.2 at the copy peak).  And SMs idle: a quarter of
// the time where 512 KV heads are 1.7 waves of CTAs.  us: 512 KV heads around 4096 tokens 62.1
// (3.7 TB/s), 16 heads of 131000 tokens 107.4 (2.8 TB/s; 256 CTAs on 304 places; the copies
// alone 48), 8 heads of 4096 tokens 7.8.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "vd_device.cuh"
#include "vd_q4.cuh"

namespace vd {

struct AttendArgs {
  const uint8_t *k, *v, *ks, *vs;  // the layer's first unit of sequence 0
  const uint16_t *q, *k_new, *v_new;  // k_new, v_new: of the layer, null without new rows
  uint16_t* out;
  float* lse;  // nullable
  const int32_t* len;
  unsigned* status;
  size_t seq_rows;      // rows between two sequences of the cache
  size_t seq_new_rows;  // and of the new rows
  int heads, group, B, cap;
  int rows;    // query rows per KV head: B * group
  int tiles;   // row tiles of a KV head
  int cluster;
  float scale;
  uint32_t wait_limit;
};

constexpr int kStageKeys = 32;
constexpr float kLift = 15.f;  // fp16's largest power of two
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Two weights in bf16, and in `low` what that leaves of them: together within 2^-16 of a weight.
__device__ __forceinline__ uint32_t split_bf16(float x, float y, uint32_t& low) {
  const uint32_t high = pack_bf16(x, y);
  low = pack_bf16(x - __uint_as_float(high << 16), y - __uint_as_float(high & 0xffff0000u));
  return high;
}

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// c = a b in fp16, and c += a b.
__device__ __forceinline__ void mma_16816_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                                uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

template <bool BF16>
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                          uint32_t b1) {
  if (BF16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A query row's power of two: its largest magnitude goes to [2^-9, 2^-8), exact in bf16, so
// that no finite key row makes a score overflow.  The factor is 2^-126 at least: a row whose
// largest magnitude is 2^118 or more goes to something below 4, and 256 products with new keys
// below 2^118 stay finite.  For fp16 kTo16 more, at most 2^15: the 8 bits of a bf16 value fit
// down to 2^-17, 2^-21 of the row's largest; what is smaller is off by at most 2^-29 of the
// largest (the fp32 sum of a score's products is bound by 2^-23 of their magnitudes).
constexpr float kTo16 = 0x1p13f, kFrom16 = 0x1p-13f;

struct QueryScale {
  uint32_t up;  // the factor in bf16, twice
  float down;   // its inverse
};

// top: the row's largest magnitude as bf16 bits
__device__ __forceinline__ QueryScale scale_of(uint32_t top) {
  const uint32_t ex = top ? min(244u, max(1u, top >> 7)) : 118u;
  return {((245u - ex) << 7) * 0x00010001u, __uint_as_float((ex + 9u) << 23)};
}

// What a row's scores are multiplied by for log2 units.  Finite, so that a score of 0 stays one,
// and not 0, so that a masked score stays masked.  Subnormal factors count: new keys of 2^127
// make scores of up to 2^128 before it.
__device__ __forceinline__ float score_factor(float down, float scale) {
  return fminf(fmaxf(down * scale * kLog2e, 0x1p-149f), 3.40282347e38f);
}

// The same for cached tokens, whose queries are kTo16 larger.
__device__ __forceinline__ float cached_factor(float factor) {
  return fmaxf(factor * kFrom16, 0x1p-149f);
}

__device__ __forceinline__ uint32_t ld_shared_u8(uint32_t addr) {
  uint32_t r;
  asm volatile("{ .reg .u16 t; ld.shared.u8 t, [%1]; cvt.u32.u16 %0, t; }" : "=r"(r) : "r"(addr));
  return r;
}

__device__ __forceinline__ uint32_t ld_shared_u16(uint32_t addr) {
  uint32_t r;
  asm volatile("{ .reg .u16 t; ld.shared.u16 t, [%1]; cvt.u32.u16 %0, t; }" : "=r"(r) : "r"(addr));
  return r;
}

__device__ __forceinline__ uint32_t ld_shared_b32(uint32_t addr) {
  uint32_t r;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(addr));
  return r;
}

// Shared memory of a CTA: the warps' rings, which the partial results reuse, then the
// warps' maxima and sums, the CTA's, and the ring barriers.
template <int M, int NT>
struct AttendShape {
  static constexpr int kD = 32 * M;
  static constexpr int kRows = 8 * NT;
  static constexpr int kStages = M <= 2 ? 4 : M <= 4 ? 3 : 2;
  static constexpr int kCodeBytes = kStageKeys * 16 * M;
  static constexpr int kScaleBytes = kStageKeys * 2 * M;
  static constexpr int kStageBytes = 2 * (kCodeBytes + kScaleBytes);
  static constexpr int kRing = kWarps * kStages * kStageBytes;
  static constexpr int kPart = kD + 4;  // floats of a partial row
  static constexpr int kPartBytes = (kWarps + 1) * kRows * kPart * 4;
  static constexpr int kMain = kRing > kPartBytes ? kRing : kPartBytes;
  static constexpr int kStats = kMain;                                 // [warp][row] max, sum
  static constexpr int kBars = kStats + 2 * (kWarps + 1) * kRows * 4;  // [warp][stage]
  static constexpr int kTotal = kBars + kWarps * kStages * 8;
};

// Where a lane's V dims lie: the two dims of m-tile t for lane row r, and the bytes.
// M a multiple of 4: 2 M bytes in a row; even: words of 8 dims, 64 dims apart; odd:
// half words of 4 dims, 32 apart.  A byte is the two dims of one tile.
template <int M>
__device__ __forceinline__ int v_dim(int t, int r) {
  if (M % 4 == 0) return 4 * M * r + 2 * t;
  if (M % 2 == 0) return 64 * (t >> 2) + 8 * r + 2 * (t & 3);
  return 32 * (t >> 1) + 4 * r + 2 * (t & 1);
}

// First dim of word w (8 dims, two k16 steps) of a lane's K row: contiguous words, or
// words 32 dims apart.
template <int M>
__device__ __forceinline__ int k_dim(int w, int c) {
  return M % 4 == 0 ? 8 * M * c + 8 * w : 32 * w + 8 * c;
}

template <int M, int NT>
__global__ void __launch_bounds__(kThreads, M * NT <= 4 ? 2 : 1) q4_attend_kernel(AttendArgs a) {
  using Sh = AttendShape<M, NT>;
  constexpr int kD = Sh::kD;
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t base = smem_addr(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = lane >> 2, c = lane & 3;
  const unsigned rank = blockIdx.x % a.cluster;
  const unsigned item = blockIdx.x / a.cluster;
  const int tile = item % a.tiles;
  const unsigned unit = item / a.tiles;
  const int seq = unit / a.heads, head = unit % a.heads;
  const uint32_t bars = base + Sh::kBars + warp * Sh::kStages * 8;
  if (lane == 0) {
    for (int i = 0; i < Sh::kStages; ++i) mbar_init(bars + 8 * i, 1);
    fence_mbar_init();
  }
  __syncwarp();
  grid_dependency_wait();
  grid_launch_dependents();

  // Q: lane (r, c) holds row r of each n-tile, dims k_dim(w, c) .. + 7 for every w.  Loaded
  // before the length is waited for
  const int row0 = tile * Sh::kRows;
  uint32_t qf[NT][M][4];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = row0 + 8 * t + r;
    const bool valid = row < a.rows;
    const size_t at = (((size_t)seq * a.B + row / a.group) * a.heads + head) * a.group +
                      row % a.group;
#pragma unroll
    for (int w = 0; w < M; ++w) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (valid) x = ld_cg16(a.q + at * kD + k_dim<M>(w, c));
      qf[t][w][0] = x.x;
      qf[t][w][1] = x.y;
      qf[t][w][2] = x.z;
      qf[t][w][3] = x.w;
    }
  }
  const int n = __ldcg(a.len + seq);
  if (n < 0 || n > a.cap) {  // the whole cluster leaves
    if (rank == 0 && tile == 0 && head == 0 && threadIdx.x == 0)
      record_status(a.status, kStDeviceLen);
    return;
  }
  const size_t unit_row = (size_t)seq * a.seq_rows + (size_t)head * a.cap;

  // this warp's stages: first, first + kWarps, ... below `last`
  const int stages = (n + kStageKeys - 1) / kStageKeys;
  const int begin = (int)((long long)stages * rank / a.cluster);
  const int last = (int)((long long)stages * (rank + 1) / a.cluster);
  const uint32_t ring = base + warp * Sh::kStages * Sh::kStageBytes;
  // Copy `what` of a stage (codes of K and V, scales of K and V): four lanes issue a stage's
  // copies together, and in the beginning 4 * kStages lanes those of all stages
  auto fetch = [&](int stage, int slot, int what) {
    const int key0 = stage * kStageKeys;
    const int keys = min(kStageKeys, n - key0);
    const uint32_t codes = (uint32_t)keys * (kD / 2);
    const uint32_t scales = (uint32_t)((keys + 7) & ~7) * (kD / 16);  // within the capacity
    const uint32_t dst = ring + slot * Sh::kStageBytes + (what & 1) * (what < 2 ? Sh::kCodeBytes
                                                                               : Sh::kScaleBytes) +
                         (what < 2 ? 0 : 2 * Sh::kCodeBytes);
    const uint32_t bar = bars + 8 * slot;
    const uint8_t* src = what == 0 ? a.k : what == 1 ? a.v : what == 2 ? a.ks : a.vs;
    if (what == 0) mbar_expect_tx(bar, 2 * (codes + scales));
    bulk_g2s(dst, src + (unit_row + key0) * (what < 2 ? kD / 2 : kD / 16),
             what < 2 ? codes : scales, bar);
  };
  if (lane < 4 * Sh::kStages) {
    const int stage = begin + warp + (lane >> 2) * kWarps;
    if (stage < last) fetch(stage, lane >> 2, lane & 3);
  }

  float o[NT][2 * M][4];
  float mx[NT][2], sum[NT][2];  // references and sums of columns (query rows) 2 c and 2 c + 1
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    mx[t][0] = mx[t][1] = -INFINITY;
    sum[t][0] = sum[t][1] = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * M; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[t][i][e] = 0.f;
  }
  // Takes the scores of 16 or 32 tokens (qs times them: log2 units) into the running state and
  // turns them into weights.  The reference mx, the maximum less kLift, is renewed only where
  // a score exceeds it by more.  It is rounded up: no weight exceeds 2^kLift.  Scores
  // are rounded before the maximum is taken off them: a difference of the unrounded product
  // would be off by half a unit of the maximum, 2^8 at 2^33.  (Both the maximum and the
  // difference use the product, which keeps it rounded.)
  auto soften = [&](auto& s, const unsigned long long (&qs)[NT]) {
    constexpr int kChunks = sizeof(s) / sizeof(s[0]);
    float top[NT][2];
    bool above = false;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int g = 0; g < kChunks; ++g)
#pragma unroll
        for (int e = 0; e < 4; e += 2)
          f2_unpack(f2_mul(f2_pack(s[g][t][e], s[g][t][e + 1]), qs[t]), s[g][t][e], s[g][t][e + 1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float m = fmaxf(s[0][t][e], s[0][t][e + 2]);
#pragma unroll
        for (int g = 1; g < kChunks; ++g) m = fmaxf(m, fmaxf(s[g][t][e], s[g][t][e + 2]));
        top[t][e] = __fadd_ru(m, -kLift);
        above |= top[t][e] > mx[t][e];
      }
    }
    if (__any_sync(kFull, above)) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float m = fmaxf(mx[t][e], top[t][e]);
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, off));
          const float f = m == -INFINITY ? 1.f : exp2_approx(mx[t][e] - m);
          mx[t][e] = m;
          sum[t][e] *= f;
#pragma unroll
          for (int i = 0; i < 2 * M; ++i) {
            o[t][i][e] *= f;
            o[t][i][e + 2] *= f;
          }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const unsigned long long shift = f2_pack(mx[t][0] == -INFINITY ? 0.f : -mx[t][0],
                                               mx[t][1] == -INFINITY ? 0.f : -mx[t][1]);
#pragma unroll
      for (int g = 0; g < kChunks; ++g) {
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          float lo, hi;
          f2_unpack(f2_add(f2_pack(s[g][t][e], s[g][t][e + 1]), shift), lo, hi);
          s[g][t][e] = exp2_approx(lo);
          s[g][t][e + 1] = exp2_approx(hi);
        }
        sum[t][0] += s[g][t][0] + s[g][t][2];
        sum[t][1] += s[g][t][1] + s[g][t][3];
      }
    }
  };

  // Each row of Q times its power of two; qs: what the scores of columns 2 c and 2 c + 1
  // have to be multiplied by for log2 units
  unsigned long long qs[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    uint32_t top = 0;  // largest magnitude, as bits
#pragma unroll
    for (int w = 0; w < M; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t x = qf[t][w][e];
        top = max(top, max(x & 0x7fffu, (x >> 16) & 0x7fffu));
      }
    top = max(top, __shfl_xor_sync(kFull, top, 1));
    top = max(top, __shfl_xor_sync(kFull, top, 2));
    const QueryScale f = scale_of(top);
    const uint32_t up = f.up;
#pragma unroll
    for (int w = 0; w < M; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(qf[t][w][e]) : "r"(up));
    const float factor = score_factor(f.down, a.scale);
    qs[t] = f2_pack(__shfl_sync(kFull, factor, 8 * c), __shfl_sync(kFull, factor, 8 * c + 4));
  }
  // the new rows, 16 at a time, in bf16: few, so a warp reads them straight from memory.
  // They go to the cluster's warps from the last one on.
  if (a.k_new) {
    const int seen = min(a.rows, row0 + Sh::kRows);  // query rows up to the tile's last
    const int keys = (seen - 1) / a.group + 1;
    const size_t new_row = (size_t)seq * a.seq_new_rows + (size_t)head * a.B;
    for (int k0 = 16 * (int)((a.cluster - 1 - rank) * kWarps + (kWarps - 1 - warp)); k0 < keys;
         k0 += 16 * kWarps * a.cluster) {
      float s[1][NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[0][t][e] = 0.f;
      const bool in0 = k0 + r < a.B, in1 = k0 + r + 8 < a.B;
      const uint16_t* kr = a.k_new + (new_row + k0 + r) * kD;
      const uint16_t* vr = a.v_new + (new_row + k0) * kD;
      uint4 kx[M], ky[M];
#pragma unroll
      for (int w = 0; w < M; ++w) {
        kx[w] = ky[w] = make_uint4(0, 0, 0, 0);
        if (in0) kx[w] = ld_cg16(kr + k_dim<M>(w, c));
        if (in1) ky[w] = ld_cg16(kr + 8 * kD + k_dim<M>(w, c));
      }
      uint32_t vx[2 * M][4];  // of every m-tile two dims of tokens 2c, 2c + 1, 2c + 8, 2c + 9
      // A value that is not finite must not reach the tokens before its own, whose weight
      // for it is 0: then the products are made one by one, for those that see it.
      bool odd = false;
#pragma unroll
      for (int i = 0; i < 2 * M; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = 2 * c + (e & 1) + (e >> 1) * 8;
          vx[i][e] = k0 + key < keys ? __ldcg(reinterpret_cast<const uint32_t*>(
                                           vr + (size_t)key * kD + v_dim<M>(i, r)))
                                     : 0u;
        }
#pragma unroll
      for (int w = 0; w < M; ++w) {
        const uint4 x = kx[w], y = ky[w];
        const uint32_t f0[4] = {x.x, y.x, x.y, y.y}, f1[4] = {x.z, y.z, x.w, y.w};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          mma_16816<true>(s[0][t], f0, qf[t][w][0], qf[t][w][1]);
          mma_16816<true>(s[0][t], f1, qf[t][w][2], qf[t][w][3]);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = row0 + 8 * t + 2 * c + (e & 1), key = k0 + r + (e >> 1) * 8;
          // rows behind the last see what the last one sees
          const int token = min(row, a.rows - 1) / a.group;
          if (key > token) s[0][t][e] = -INFINITY;
        }
      soften(s, qs);
#pragma unroll
      for (int i = 0; i < 2 * M; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          odd |= (vx[i][e] & 0x7f80u) == 0x7f80u || (vx[i][e] & 0x7f800000u) == 0x7f800000u;
      if (__any_sync(kFull, odd)) {
        for (int key = 0; key < 16 && k0 + key < keys; ++key) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const float lo0 = __shfl_sync(kFull, s[0][t][0], 4 * (key & 7) + c);
            const float lo1 = __shfl_sync(kFull, s[0][t][1], 4 * (key & 7) + c);
            const float hi0 = __shfl_sync(kFull, s[0][t][2], 4 * (key & 7) + c);
            const float hi1 = __shfl_sync(kFull, s[0][t][3], 4 * (key & 7) + c);
            const float p0 = key < 8 ? lo0 : hi0, p1 = key < 8 ? lo1 : hi1;
            const int row = row0 + 8 * t + 2 * c;
            const bool see0 = k0 + key <= min(row, a.rows - 1) / a.group;
            const bool see1 = k0 + key <= min(row + 1, a.rows - 1) / a.group;
#pragma unroll
            for (int i = 0; i < 2 * M; ++i) {
              const uint32_t x = __ldcg(
                  reinterpret_cast<const uint32_t*>(vr + (size_t)key * kD + v_dim<M>(i, r)));
              const float v0 = __uint_as_float(x << 16), v1 = __uint_as_float(x & 0xffff0000u);
              if (see0) o[t][i][0] = fmaf(p0, v0, o[t][i][0]), o[t][i][2] = fmaf(p0, v1, o[t][i][2]);
              if (see1) o[t][i][1] = fmaf(p1, v0, o[t][i][1]), o[t][i][3] = fmaf(p1, v1, o[t][i][3]);
            }
          }
        }
        continue;
      }
      uint32_t p[NT][2], rest[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          uint32_t low;
          const uint32_t high = split_bf16(s[0][t][2 * e], s[0][t][2 * e + 1], low);
          p[t][e] = transpose_8x8(high);
          rest[t][e] = transpose_8x8(low);
        }
#pragma unroll
      for (int i = 0; i < 2 * M; ++i) {
        const uint32_t(&x)[4] = vx[i];
        const uint32_t f[4] = {__byte_perm(x[0], x[1], 0x5410), __byte_perm(x[0], x[1], 0x7632),
                               __byte_perm(x[2], x[3], 0x5410), __byte_perm(x[2], x[3], 0x7632)};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          mma_16816<true>(o[t][i], f, p[t][0], p[t][1]);
          mma_16816<true>(o[t][i], f, rest[t][0], rest[t][1]);
        }
      }
    }
  }

  // Q to fp16
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float qs0, qs1;
    f2_unpack(qs[t], qs0, qs1);
    qs[t] = f2_pack(cached_factor(qs0), cached_factor(qs1));
#pragma unroll
    for (int w = 0; w < M; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t x = qf[t][w][e];
        qf[t][w][e] = pack_f16(__uint_as_float(x << 16) * kTo16,
                               __uint_as_float(x & 0xffff0000u) * kTo16);
      }
  }

  // the cached tokens.  Token index k of a 16-token chunk sits in row
  // phys(k) = 8 (k >> 3) + 2 ((k >> 1) & 3) + ((k ^ (k >> 1)) & 1): a quarter warp's K
  // loads then cover two neighbouring rows, and V's token pairs differ in row parity.
  int slot = 0, issued = begin + warp + Sh::kStages * kWarps;
  uint32_t phase = 0;
  bool alive = true;
  for (int stage = begin + warp; stage < last; stage += kWarps) {
    const uint32_t at = ring + slot * Sh::kStageBytes;
    alive = mbar_wait(bars + 8 * slot, phase, a.status, a.wait_limit);
    if (!__all_sync(kFull, alive)) {
      alive = false;
      break;
    }
    const int left = n - stage * kStageKeys;  // tokens of this stage, at least 1
    if (left < kStageKeys) {  // whatever lies behind the last token counts as zero
      const uint32_t scales = at + 2 * Sh::kCodeBytes + Sh::kScaleBytes;
      for (int i = left * 2 * M + 2 * lane; i < Sh::kScaleBytes; i += 64)
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(scales + i), "h"((unsigned short)0)
                     : "memory");
      __syncwarp();
    }
    float s[2][NT][4];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int pr = 16 * g + (r & 6) + ((r ^ (r >> 1)) & 1);  // rows pr and pr + 8
      uint32_t w0[M], w1[M], sc0[M], sc1[M];
      const uint32_t k0 = at + pr * (16 * M), k1 = k0 + 8 * 16 * M;
      if (M % 4 == 0) {
#pragma unroll
        for (int w = 0; w < M; w += 4) {
          const uint4 x = ld_shared16(k0 + 4 * M * c + 4 * w);
          const uint4 y = ld_shared16(k1 + 4 * M * c + 4 * w);
          w0[w] = x.x, w0[w + 1] = x.y, w0[w + 2] = x.z, w0[w + 3] = x.w;
          w1[w] = y.x, w1[w + 1] = y.y, w1[w + 2] = y.z, w1[w + 3] = y.w;
        }
      } else {
#pragma unroll
        for (int w = 0; w < M; ++w) {
          w0[w] = ld_shared_b32(k0 + 16 * w + 4 * c);
          w1[w] = ld_shared_b32(k1 + 16 * w + 4 * c);
        }
      }
      const uint32_t ks0 = at + 2 * Sh::kCodeBytes + pr * (2 * M), ks1 = ks0 + 8 * 2 * M;
      if (M % 4 == 0) {  // groups M / 2 * c + (w >> 1)
#pragma unroll
        for (int w = 0; w < M; w += 4) {
          const uint32_t x = ld_shared_u16(ks0 + M / 2 * c + (w >> 1));
          const uint32_t y = ld_shared_u16(ks1 + M / 2 * c + (w >> 1));
          sc0[w] = sc0[w + 1] = (x & 255u) * 0x00800080u;
          sc0[w + 2] = sc0[w + 3] = (x >> 8) * 0x00800080u;
          sc1[w] = sc1[w + 1] = (y & 255u) * 0x00800080u;
          sc1[w + 2] = sc1[w + 3] = (y >> 8) * 0x00800080u;
        }
      } else {  // group 2 w + (c >> 1)
#pragma unroll
        for (int w = 0; w < M; ++w) {
          sc0[w] = ld_shared_u8(ks0 + 2 * w + (c >> 1)) * 0x00800080u;
          sc1[w] = ld_shared_u8(ks1 + 2 * w + (c >> 1)) * 0x00800080u;
        }
      }
#pragma unroll
      for (int w = 0; w < M; ++w) {
        uint32_t x[4], y[4];
        q4_unpack4(w0[w], x);
        q4_unpack4(w1[w], y);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = h2_mul(x[e], sc0[w]);
          y[e] = h2_mul(y[e], sc1[w]);
        }
        const uint32_t f0[4] = {x[0], y[0], x[1], y[1]}, f1[4] = {x[2], y[2], x[3], y[3]};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (w == 0)
            mma_16816_first(s[g][t], f0, qf[t][w][0], qf[t][w][1]);
          else
            mma_16816<false>(s[g][t], f0, qf[t][w][0], qf[t][w][1]);
          mma_16816<false>(s[g][t], f1, qf[t][w][2], qf[t][w][3]);
        }
      }
      if (left < kStageKeys) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (pr + (e >> 1) * 8 >= left) s[g][t][e] = -INFINITY;
      }
    }
    soften(s, qs);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t p[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        p[t][0] = transpose_8x8(pack_f16(s[g][t][0], s[g][t][1]));
        p[t][1] = transpose_8x8(pack_f16(s[g][t][2], s[g][t][3]));
      }
      // rows of tokens 2c, 2c + 1, 2c + 8, 2c + 9
      const int p0 = 16 * g + 2 * c + (c & 1), p1 = 16 * g + 2 * c + ((c & 1) ^ 1);
      const int prow[4] = {p0, p1, p0 + 8, p1 + 8};
      constexpr int kWords = M % 2 == 0 ? M / 2 : (M + 1) / 2;
      uint32_t x[4][kWords];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t row = at + Sh::kCodeBytes + prow[e] * (16 * M);
        if (M == 4) {
          const unsigned long long q = ld_shared_b64(row + 8 * r);
          x[e][0] = (uint32_t)q;
          x[e][kWords - 1] = (uint32_t)(q >> 32);
        } else if (M % 4 == 0) {
          const uint4 q = ld_shared16(row + 16 * r);
          x[e][0] = q.x, x[e][1 % kWords] = q.y, x[e][2 % kWords] = q.z, x[e][3 % kWords] = q.w;
        } else if (M % 2 == 0) {
#pragma unroll
          for (int w = 0; w < kWords; ++w) x[e][w] = ld_shared_b32(row + 32 * w + 4 * r);
        } else {
#pragma unroll
          for (int w = 0; w < kWords; ++w) {
            x[e][w] = ld_shared_u16(row + 32 * w + 2 * r);
            if (2 * w + 1 < M) x[e][w] |= ld_shared_u16(row + 32 * w + 16 + 2 * r) << 16;
          }
        }
      }
      // scale of the group of byte b (word w, tiles 4 w + b), token by token, in fp16
      auto scales = [&](int group, uint32_t& s01, uint32_t& s23) {
        uint32_t sb[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sb[e] = ld_shared_u8(at + 2 * Sh::kCodeBytes + Sh::kScaleBytes + prow[e] * (2 * M) +
                               group);
        }
        s01 = sb[0] * 0x80u + sb[1] * 0x800000u;
        s23 = sb[2] * 0x80u + sb[3] * 0x800000u;
      };
      uint32_t s01 = 0, s23 = 0;
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        // even M: one group per word; odd: one per half word
        if (M % 4 == 0 && (w & 1) == 0) scales((M / 4) * r + (w >> 1), s01, s23);
        if (M % 4 == 2) scales(4 * w + (r >> 1), s01, s23);
        if (M % 2 == 1) scales(4 * w + (r >> 2), s01, s23);
        const uint32_t m4 = 0x0f0f0f0fu;
        uint32_t f[4][4];  // [fragment register][tile of the word]
        q4_unpack4((x[0][w] & m4) | ((x[1][w] << 4) & ~m4), f[0]);
        q4_unpack4(((x[0][w] >> 4) & m4) | (x[1][w] & ~m4), f[1]);
        q4_unpack4((x[2][w] & m4) | ((x[3][w] << 4) & ~m4), f[2]);
        q4_unpack4(((x[2][w] >> 4) & m4) | (x[3][w] & ~m4), f[3]);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int i = 4 * w + b;
          if (i >= 2 * M) break;
          if (M % 2 == 1 && b == 2) scales(4 * w + 2 + (r >> 2), s01, s23);
          const uint32_t fr[4] = {h2_mul(f[0][b], s01), h2_mul(f[1][b], s01),
                                  h2_mul(f[2][b], s23), h2_mul(f[3][b], s23)};
#pragma unroll
          for (int t = 0; t < NT; ++t) mma_16816<false>(o[t][i], fr, p[t][0], p[t][1]);
        }
      }
    }
    __syncwarp();
    if (lane < 4 && issued < last) {
      fence_proxy_async_smem();
      fetch(issued, slot, lane);
    }
    issued += kWarps;
    if (++slot == Sh::kStages) {
      slot = 0;
      phase ^= 1;
    }
  }
  if (!alive) {  // a copy gave up: wait for this warp's others before their memory is reused
    if (lane == 0) {
      for (int i = 0; i < Sh::kStages; ++i, ++slot) {
        if (slot == Sh::kStages) slot = 0, phase ^= 1;
        if (issued - (Sh::kStages - i) * kWarps < last)
          mbar_wait(bars + 8 * slot, phase, a.status, kWaitLimit);
      }
    }
    __syncwarp();
  }

  // the warps' results to shared memory, [warp][row][dim], once every ring is idle
  __syncthreads();
  float* part = reinterpret_cast<float*>(smem);
  float* stat_m = reinterpret_cast<float*>(smem + Sh::kStats);
  float* stat_l = stat_m + (kWarps + 1) * Sh::kRows;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float l = sum[t][e];
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(kFull, l, off);
      const int row = 8 * t + 2 * c + e;
      if (r == 0) {
        stat_m[warp * Sh::kRows + row] = mx[t][e];
        stat_l[warp * Sh::kRows + row] = l;
      }
      float* dst = part + ((size_t)warp * Sh::kRows + row) * Sh::kPart;
#pragma unroll
      for (int i = 0; i < 2 * M; ++i)
        *reinterpret_cast<float2*>(dst + v_dim<M>(i, r)) = make_float2(o[t][i][e], o[t][i][e + 2]);
    }
  __syncthreads();
  // the CTA's: behind the warps'
  float* cta = part + (size_t)kWarps * Sh::kRows * Sh::kPart;
  for (int i = threadIdx.x; i < Sh::kRows * (kD / 4); i += kThreads) {
    const int row = i / (kD / 4), dim = i % (kD / 4) * 4;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, stat_m[w * Sh::kRows + row]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float mw = stat_m[w * Sh::kRows + row];
      // a warp without tokens has sums of zero; one whose scores were all NaN has NaN sums
      const float f = mw == -INFINITY ? 1.f : exp2_approx(mw - m);
      const float4 x =
          *reinterpret_cast<const float4*>(part + ((size_t)w * Sh::kRows + row) * Sh::kPart + dim);
      acc.x = fmaf(x.x, f, acc.x);
      acc.y = fmaf(x.y, f, acc.y);
      acc.z = fmaf(x.z, f, acc.z);
      acc.w = fmaf(x.w, f, acc.w);
      l = fmaf(stat_l[w * Sh::kRows + row], f, l);
    }
    *reinterpret_cast<float4*>(cta + row * Sh::kPart + dim) = acc;
    if (dim == 0) {
      stat_m[kWarps * Sh::kRows + row] = m;
      stat_l[kWarps * Sh::kRows + row] = l;
    }
  }
  if (a.cluster > 1)
    cluster_sync();
  else
    __syncthreads();
  // Each CTA writes its share of the tile, from all CTAs' results in rank order: first every
  // CTA's factor for every row, then the sums.
  const uint32_t cta_addr = smem_addr(cta);
  const uint32_t m_addr = smem_addr(stat_m + kWarps * Sh::kRows);
  const uint32_t l_addr = smem_addr(stat_l + kWarps * Sh::kRows);
  const bool none = n == 0 && !a.k_new;  // no token to attend to
  float* all_m = part;                   // [cluster][row], over the warps' results
  float* all_l = all_m + 16 * Sh::kRows;
  if ((int)threadIdx.x < a.cluster * Sh::kRows) {
    const int q = threadIdx.x / Sh::kRows, row = threadIdx.x % Sh::kRows;
    all_m[threadIdx.x] = ld_cluster_f32(mapa(m_addr + 4 * row, q));
    all_l[threadIdx.x] = ld_cluster_f32(mapa(l_addr + 4 * row, q));
  }
  __syncthreads();
  if ((int)threadIdx.x < Sh::kRows) {
    const int row = threadIdx.x;
    float m = -INFINITY, l = 0.f;
    for (int q = 0; q < a.cluster; ++q) m = fmaxf(m, all_m[q * Sh::kRows + row]);
    for (int q = 0; q < a.cluster; ++q) {
      const float mq = all_m[q * Sh::kRows + row];
      // a CTA without tokens has sums of zero; one whose scores were all NaN has NaN sums
      const float f = mq == -INFINITY ? 1.f : exp2_approx(mq - m);
      l = fmaf(all_l[q * Sh::kRows + row], f, l);
      all_m[q * Sh::kRows + row] = f;
    }
    all_l[row] = none ? 0.f : 1.f / l;  // q == 0's, which is read above by this thread alone
    const int gr = row0 + row;
    if (a.lse && rank == 0 && gr < a.rows)
      a.lse[(((size_t)seq * a.B + gr / a.group) * a.heads + head) * a.group + gr % a.group] =
          none ? -INFINITY : (m + kLift) / kLog2e + logf(l * 0x1p-15f);
  }
  __syncthreads();
  const int total = min(Sh::kRows, a.rows - row0) * (kD / 4);
  for (int i = (int)rank * kThreads + threadIdx.x; i < total; i += kThreads * a.cluster) {
    const int row = i / (kD / 4), dim = i % (kD / 4) * 4;
    const uint32_t x_addr = cta_addr + 4 * (row * Sh::kPart + dim);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int q0 = 0; q0 < a.cluster; q0 += 8) {
      float4 x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (q0 + q < a.cluster) x[q] = ld_cluster_f32x4(mapa(x_addr, q0 + q));
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (q0 + q < a.cluster) {
          const float f = all_m[(q0 + q) * Sh::kRows + row];
          acc.x = fmaf(x[q].x, f, acc.x);
          acc.y = fmaf(x[q].y, f, acc.y);
          acc.z = fmaf(x[q].z, f, acc.z);
          acc.w = fmaf(x[q].w, f, acc.w);
        }
    }
    const int gr = row0 + row;
    const size_t at =
        (((size_t)seq * a.B + gr / a.group) * a.heads + head) * a.group + gr % a.group;
    const float inv = all_l[row];
    *reinterpret_cast<uint2*>(a.out + at * kD + dim) =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  }
  if (a.cluster > 1) cluster_sync();  // no CTA leaves while its results are read
}

}  // namespace vd
