// vd_q4_tile.cuh -- attention over one layer of a 4-bit cache (vd_q4_attend in
// include/vd.h): the block kernel, for many query rows per KV head (blocks of block
// prompt processing, prompts).
//
// The formula is vd_q4_attend.cuh's.  128 query rows of a KV head are one CTA's (a row per
// thread of four warps and per lane of tensor memory), the tokens come in tiles of kKeys,
// and the two products run on tcgen05 with Q, the weights P and both results in tensor
// memory, so that shared memory carries K and V only:
//   S = Q K^T   (128 x kKeys, K's rows along the depth)
//   O += P V    (128 x head_dim, V's rows along the columns)
// Roles of the warps, which meet only at mbarriers:
//   0-7   softmax, a row per pair of threads with half the columns each: maximum, weights,
//         their sum.  Weights are relative to a point kTileLift below the maximum (as in the
//         streaming kernel), and O is rescaled where the maximum has risen kLift above it (a
//         smaller rise only makes the weights larger);
//   8-11  K's tiles, a slice of the tokens each: cached codes, which come by bulk copies into
//         the warp's own ring, to fp16 in the swizzled layout of the products (exact), or
//         copies of the new tokens' bf16 rows;
//   12-14 V's tiles, the same;
//   15    one thread issues the products: S of tile i + 1 before O takes tile i, so that the
//         softmax of one tile runs beside the products of its neighbours.
// The new tokens' tiles come first, in bf16, then Q is rewritten in fp16 (rows scaled by
// powers of two, as in the streaming kernel) for the cached ones.  A cluster splits the
// tiles of a unit and joins the results through distributed shared memory.
//
// Per tile of 128 tokens at head_dim 128: the products take 1024 cycles at 4096
// multiply-adds a cycle, the roles issue 6400 warp instructions (their polls among them), 1600
// a scheduler, at 2.5 a cycle of 4, and the tensor pipe is at 40 % while an SM is active: the
// chain from scores to weights to product, its latencies and half-rate conversions bound it.  K
// and V are unpacked once for every 128 query rows.  K's and V's warps share their code, as the
// roles' code does not fit the instruction cache (385 us with one each, 343 shared, in one run).
// us: 512 new tokens over 32768 cached ones, 8 KV heads of 4 query heads, 356 (277 GFLOP, 780
// TFLOP/s; 128 CTAs on 152 SMs); of a 352 us form, without the softmax 280, without the unpacking
// 263, without the products 330; 128 new tokens over 2048 18.6; 8192 over themselves 1970.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "vd_device.cuh"
#include "vd_q4.cuh"
#include "vd_q4_attend.cuh"
#include "vd_tcgen05.cuh"

namespace vd {

constexpr int kTileRows = 128;  // rows of a block

// A rise of the maximum by 2^4 rescales O; the smallest weight that does not become 0 is 2^-36
// of the largest, 25 nats down.
constexpr float kTileLift = 11.f, kTileUnlift = 0x1p-11f;

constexpr int kTileThreads = 512;
constexpr int kSoftWarps = 8, kKeyWarps = 4, kValueWarps = 3, kProductWarp = 15;

template <int M>
struct TileShape {
  static constexpr int kD = 32 * M;
  static constexpr int kKeys = M <= 4 ? 128 : 64;   // tokens of a tile
  static constexpr int kBlocks = (kD + 63) / 64;    // 64-column blocks of a row
  static constexpr int kTileBytes = kBlocks * kKeys * 128;
  static constexpr int kKeyBufs = 2, kValueBufs = 3;
  static constexpr int kRaw = 3;                    // tiles of codes and scales on their way
  static constexpr int kRawCodes = kKeys * 16 * M, kRawScales = kKeys * 2 * M;
  static constexpr int kRawBytes = 2 * (kRawCodes + kRawScales);
  static constexpr int kRing = (kKeyBufs + kValueBufs) * kTileBytes;
  static constexpr int kUsed = kRing + kRaw * kRawBytes;
  static constexpr int kPartBytes = kTileRows * kD * 4;
  static constexpr int kStats = kUsed > kPartBytes ? kUsed : kPartBytes;  // row maxima, sums
  static constexpr int kFactors = kStats + 3 * kTileRows * 4;  // two sums a row
  static constexpr int kSwap = kFactors + kTileRows * 4;  // [2][2][row]: halves' maxima
  static constexpr int kBars = kSwap + 4 * kTileRows * 4;
  static constexpr int kNumBars = 18 + (kKeyWarps + kValueWarps) * kRaw;
  static constexpr int kMisc = kBars + kNumBars * 8;  // tensor memory address, flags
  // The base is rounded up to 1024.  So much that no other CTA with tensor memory fits on the
  // SM: it would wait for this one's, and, in one cluster with it, this one for it.
  static constexpr int kNeed = kMisc + 16 + 1024;
  static constexpr int kTotal = kNeed > 200 * 1024 ? kNeed : 200 * 1024;
  // columns of tensor memory: two S, P, O, Q (P and Q 16-bit pairs).  At head_dim 256 there
  // is no room for P, which then takes the lower half of its S.  The low parts of the new rows'
  // weights take the upper half at any head_dim
  static constexpr bool kAlias = M == 8;
  static constexpr int kColP = 2 * kKeys;
  static constexpr int kColO = kColP + (kAlias ? 0 : kKeys / 2);
  static constexpr int kColQ = kColO + kD;
  static_assert(kColQ + kD / 2 <= 512, "tensor memory");
};

__device__ __forceinline__ bool mbar_done(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; "
      "selp.u32 %0, 1, 0, p; }"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}

// Waits like mbar_wait, and gives up as well once another role has.  Short: the roles' loops
// share the instruction cache, and unrolled polls cost the product thread 250 cycles a wait.
__device__ __forceinline__ bool tile_wait(uint32_t bar, uint32_t parity, unsigned* status,
                                          uint32_t limit, volatile int* dead) {
  if (mbar_done(bar, parity)) return true;
#pragma unroll 1
  for (uint32_t i = 0; i < limit; ++i) {
    if (mbar_done(bar, parity)) return true;
    if (*dead) return false;
  }
  *dead = 1;
  record_status(status, kStTimeout);
  return false;
}

// The same for a whole warp, which goes on together.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, unsigned* status,
                                          uint32_t limit, volatile int* dead) {
  const bool ok = __all_sync(kFull, tile_wait(bar, parity, status, limit, dead));
  __syncwarp();
  return ok;
}

// The largest of three, NaN left aside like fmaxf.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// One arrival for a warp: 128 single ones would take the barrier's word in turn.
__device__ __forceinline__ void warp_arrive(uint32_t bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0)
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
  __syncwarp();
}

// The tokens of a tile that a warp of `warps` takes: multiples of 8, as scales are copied.
template <int KEYS>
struct Slice {
  int first, count;
  __device__ __forceinline__ Slice(int warp, int warps) {
    const int a = (KEYS / 8 * warp + warps - 1) / warps;
    const int b = (KEYS / 8 * (warp + 1) + warps - 1) / warps;
    first = 8 * a;
    count = 8 * (b - a);
  }
};

// Swizzled place of a row's 16-byte chunk.
template <int M>
__device__ __forceinline__ uint32_t tile_at(uint32_t dst, int key, int chunk) {
  return dst + (chunk >> 3) * (TileShape<M>::kKeys * 128) + key * 128 +
         (((chunk & 7) ^ (key & 7)) << 4);
}

// New tokens' rows of a slice: bf16 as they are, zeros behind the last one (left: rows that
// are there).  finite: what is not finite becomes zero too; returns whether there was any.
template <int M>
__device__ __forceinline__ bool copy_rows(const uint16_t* src, int left, uint32_t dst, int first,
                                          int count, int lane, bool finite) {
  constexpr int kD = 32 * M;
  constexpr int kAhead = M <= 4 ? 4 : 2;  // chunks of 16 bytes loaded together
  bool found = false;
#pragma unroll 1
  for (int j0 = lane; j0 < count * (kD / 8); j0 += 32 * kAhead) {
    uint4 x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + 32 * u, key = first + j / (kD / 8), chunk = j % (kD / 8);
      x[u] = make_uint4(0, 0, 0, 0);
      if (j < count * (kD / 8) && key < left) x[u] = ld_cg16(src + (size_t)key * kD + 8 * chunk);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + 32 * u, key = first + j / (kD / 8), chunk = j % (kD / 8);
      if (j >= count * (kD / 8)) break;
      if (finite) {
        uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u, found = true;
          if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0xffffu, found = true;
        }
        x[u] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      st_shared16(tile_at<M>(dst, key, chunk), x[u]);
    }
  }
  return found;
}

// A slice of cached codes to fp16.  32 values, 16 bytes of codes, are a unit.
template <int M, int UNITS>
struct CodeSlice {
  uint4 x[UNITS];
  uint32_t sb[UNITS];

  // there: the slice's tokens that are there; what lies behind them reads as zero
  __device__ __forceinline__ void load(uint32_t codes, uint32_t scales, int there, int lane) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int j = lane + 32 * u;
      x[u] = make_uint4(0, 0, 0, 0);
      sb[u] = 0;
      if (j < there * M) {
        x[u] = ld_shared16(codes + 16 * j);
        sb[u] = ld_shared_u16(scales + 2 * j);
      }
    }
  }

  // The order of a unit's four 16-byte stores, so that 8 neighbouring lanes meet 8 chunk
  // positions: the unit's e-th store is its chunk e ^ turn.
  static __device__ __forceinline__ int turn_of(int blk) {
    return M == 4 ? (blk & 2) : M == 8 ? (blk >> 1) & 3 : 0;
  }

  __device__ __forceinline__ void unpack(uint32_t dst, int first, int count, int lane) const {
    // where 32 lanes are a multiple of 8 tokens, a lane's units differ by a constant
    constexpr bool kRegular = M == 1 || M == 2 || M == 4;
    uint32_t place[4];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int j = lane + 32 * u;
      if (j >= count * M) break;
      const int key = first + j / M, blk = j % M, turn = turn_of(blk);
      if (u == 0 || !kRegular)
#pragma unroll
        for (int e = 0; e < 4; ++e) place[e] = tile_at<M>(dst, key, 4 * blk + (e ^ turn));
      uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      uint32_t sc[2] = {(sb[u] & 255u) * 0x00800080u, (sb[u] >> 8) * 0x00800080u};
      if (M == 8 && (turn & 1)) {
        uint32_t y = w[0];
        w[0] = w[1], w[1] = y;
        y = w[2], w[2] = w[3], w[3] = y;
      }
      if (M % 4 == 0 && (turn & 2)) {
        uint32_t y = w[0];
        w[0] = w[2], w[2] = y;
        y = w[1], w[1] = w[3], w[3] = y;
        y = sc[0], sc[0] = sc[1], sc[1] = y;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t h[4];
        q4_unpack4(w[e], h);
        st_shared16(place[e] + (kRegular ? u * (32 / M) * 128 : 0),
                    make_uint4(h2_mul(h[0], sc[e >> 1]), h2_mul(h[1], sc[e >> 1]),
                               h2_mul(h[2], sc[e >> 1]), h2_mul(h[3], sc[e >> 1])));
      }
    }
  }
};

template <int M>
__global__ void __launch_bounds__(kTileThreads, 1) q4_tile_kernel(AttendArgs a) {
  using Sh = TileShape<M>;
  constexpr int kD = Sh::kD, kKeys = Sh::kKeys;
  constexpr int kKeyBufs = Sh::kKeyBufs, kValueBufs = Sh::kValueBufs, kRaw = Sh::kRaw;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw_base = smem_addr(smem_raw);
  const uint32_t base = (raw_base + 1023u) & ~1023u;
  unsigned char* smem = smem_raw + (base - raw_base);
  const int warp = threadIdx.x >> 5;
  const unsigned rank = blockIdx.x % a.cluster;
  const unsigned item = blockIdx.x / a.cluster;
  const int tile = item % a.tiles;
  const unsigned unit = item / a.tiles;
  const int seq = unit / a.heads, head = unit % a.heads;

  // full[i % 4]: K of tile i and V of the tile before it are there (V's warps may be three
  // tiles ahead of K's: with fewer barriers they would arrive for a tile to come); s_done[i % 2]: the tile's
  // scores are, and its K buffer is free; o_done[i % 3]: it is added to O, and its V buffer
  // free; p_full[i % 2]: its weights are there; swap: a pair of softmax warps has exchanged its
  // rows' maxima; Q written; all products complete; a warp's codes are there
  const uint32_t full = base + Sh::kBars, s_done = full + 32, o_done = s_done + 16;
  const uint32_t p_full = o_done + 24, swap = p_full + 16, q_full = swap + 32;
  const uint32_t drain = q_full + 8, raw_full = drain + 8;
  volatile int* dead = reinterpret_cast<volatile int*>(smem + Sh::kMisc + 4);
  volatile int* odd = dead + 1;  // a new row of V holds a value that is not finite
  if (threadIdx.x == 0) {
    for (int i = 0; i < 4; ++i) mbar_init(full + 8 * i, kKeyWarps + kValueWarps);
    for (int i = 0; i < 3; ++i) mbar_init(o_done + 8 * i, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_done + 8 * i, 1);
      mbar_init(p_full + 8 * i, kSoftWarps);
    }
    for (int i = 0; i < (kKeyWarps + kValueWarps) * kRaw; ++i) mbar_init(raw_full + 8 * i, 1);
    for (int i = 0; i < 4; ++i) mbar_init(swap + 8 * i, 2);
    mbar_init(q_full, kSoftWarps);
    mbar_init(drain, 1);
    fence_mbar_init();
    *dead = 0;
    *odd = 0;
  }
  if (warp == kProductWarp) tmem_alloc(base + Sh::kMisc);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = *reinterpret_cast<volatile uint32_t*>(smem + Sh::kMisc);
  grid_dependency_wait();
  grid_launch_dependents();

  const int len = __ldcg(a.len + seq);
  const bool bad_len = len < 0 || len > a.cap;
  const int n = bad_len ? 0 : len;
  if (bad_len && rank == 0 && tile == 0 && head == 0 && threadIdx.x == 0)
    record_status(a.status, kStDeviceLen);
  const int row0 = tile * kTileRows;
  // this CTA's token tiles: of the new tokens [t0, t0 + fresh), then of the cached ones
  const int keys_new = a.k_new ? (min(a.rows, row0 + kTileRows) - 1) / a.group + 1 : 0;
  const int tiles_new = (keys_new + kKeys - 1) / kKeys;
  const int tiles_all = bad_len ? 0 : tiles_new + (n + kKeys - 1) / kKeys;
  const int t0 = (int)((long long)tiles_all * rank / a.cluster);
  const int count = (int)((long long)tiles_all * (rank + 1) / a.cluster) - t0;
  const int fresh = min(count, max(0, tiles_new - t0));
  const int cached0 = t0 + fresh - tiles_new;  // its first cached tile
  const size_t new_row = (size_t)seq * a.seq_new_rows + (size_t)head * a.B;

  const int half = (warp >> 2) & 1, lane_row = threadIdx.x & 127;  // of the softmax threads
  const int row = row0 + lane_row;
  const uint32_t lanes = tm + ((uint32_t)(warp & 3) << 21);  // their warp's 32 lanes
  const int token = min(row, a.rows - 1) / a.group;
  // in log2 units; the reference of the weights, at least kTileLift below the maximum when it
  // is set; the sum: of this half
  float row_max = -INFINITY, row_sum = 0.f;
  if (warp < kSoftWarps) {
    constexpr int kHalf = kKeys / 2;
    float* swapped = reinterpret_cast<float*>(smem + Sh::kSwap) + lane_row;
    // the larger of both halves' m; `turn` counts the calls
    auto exchange = [&](float& m, int turn) {
      float* at = swapped + (turn & 1) * 2 * kTileRows;
      at[half * kTileRows] = m;
      warp_arrive(swap + 8 * (warp & 3));
      if (!warp_wait(swap + 8 * (warp & 3), turn & 1, a.status, a.wait_limit, dead)) return false;
      m = fmaxf(m, at[(half ^ 1) * kTileRows]);
      return true;
    };
    if (count > 0) {
      const uint32_t q_col = lanes + Sh::kColQ + half * 8 * M;
      // Q as in the streaming kernel (scale_of)
      float factor;
      bool ok;
      {
        const uint16_t* q = a.q + ((((size_t)seq * a.B + token) * a.heads + head) * a.group +
                                   row % a.group) * kD + half * 16 * M;
        uint32_t w[8 * M];
#pragma unroll
        for (int i = 0; i < 2 * M; ++i) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (row < a.rows) x = ld_cg16(q + 8 * i);
          w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8 * M; ++i)
          top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
        float both = (float)top;
        ok = exchange(both, 0);
        top = (uint32_t)both;
        const QueryScale qs = scale_of(top);
        const uint32_t up = qs.up;
        factor = score_factor(qs.down, a.scale);
#pragma unroll
        for (int i = 0; i < 8 * M; ++i) {
          asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(w[i]) : "r"(up));
          if (fresh == 0)
            w[i] = pack_f16(__uint_as_float(w[i] << 16) * kTo16,
                            __uint_as_float(w[i] & 0xffff0000u) * kTo16);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < M; ++i) tmem_st8(q_col + 8 * i, w + 8 * i);
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(q_full);
      }
      bool large = false;  // a reference of the warp's rows beyond 2^20
      for (int i = 0; ok && i < count; ++i) {
        const uint32_t s_col = lanes + (i & 1) * kKeys;
        ok = warp_wait(s_done + 8 * (i & 1), (i >> 1) & 1, a.status, a.wait_limit, dead);
        if (!ok) break;
        tc_fence_after();
        if (i == fresh - 1 && fresh < count) {  // the last product with Q in bf16
#pragma unroll 1
          for (int j = 0; j < M; ++j) {
            uint32_t w[8];
            tmem_ld(q_col + 8 * j, w);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              w[e] = pack_f16(__uint_as_float(w[e] << 16) * kTo16,
                              __uint_as_float(w[e] & 0xffff0000u) * kTo16);
            tmem_st8(q_col + 8 * j, w);
          }
          tmem_wait_st();
          tc_fence_before();
          warp_arrive(q_full);
        }
        const bool is_new = i < fresh;
        const float c = is_new ? factor : cached_factor(factor);
        uint32_t s[kHalf];
        tmem_ld(s_col + half * kHalf, s);
        // tokens behind this row's last one do not count
        const int seen = (is_new ? token - (t0 + i) * kKeys
                                 : n - 1 - (cached0 + i - fresh) * kKeys) - half * kHalf;
        if (__any_sync(kFull, seen < kHalf - 1)) {
#pragma unroll
          for (int j = 0; j < kHalf; ++j)
            if (j > seen) s[j] = 0xff800000u;
        }
        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < kHalf; j += 2)
          m4[(j >> 1) & 3] =
              max3(m4[(j >> 1) & 3], __uint_as_float(s[j]), __uint_as_float(s[j + 1]));
        float m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * c;
        // where weights lie over S: both halves have read their scores before either writes some
        if (Sh::kAlias || is_new) tc_fence_before();
        ok = exchange(m, i + 1);
        if (!ok) break;
        if (Sh::kAlias || is_new) tc_fence_after();
        bool added = i == 0;  // the tile before is in O, and P is free
        auto wait_added = [&] {
          if (!added)
            added = warp_wait(o_done + 8 * ((i - 1) % 3), ((i - 1) / 3) & 1, a.status,
                              a.wait_limit, dead);
          if (added) tc_fence_after();
          return added;
        };
        // the weights stay below 2^15, and a row's first scores set its reference
        if (__any_sync(kFull, m - row_max > kLift)) {
          const float top = fmaxf(row_max, __fadd_ru(m, -kTileLift));
          const float f = top == -INFINITY ? 1.f : exp2_approx(row_max - top);
          row_max = top;
          row_sum *= f;
          large = __any_sync(kFull, fabsf(row_max) > 0x1p20f && row_max > -INFINITY);
          if (i > 0) {
            ok = wait_added();
            if (!ok) break;
#pragma unroll 1
            for (int j = 0; j < kD / 2; j += 16) {
              uint32_t o[16];
              const uint32_t at = lanes + Sh::kColO + half * (kD / 2) + j;
              tmem_ld(at, o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tmem_st16(at, o);
            }
          }
        }
        const float shift = row_max == -INFINITY ? 0.f : -row_max;
        unsigned long long sum2 = 0;
        if (is_new || large) {
          // Scores are rounded before the maximum is taken off them, like the maximum itself:
          // half a unit of it is 2^-4 at 2^20, but 2^8 at 2^33.  For all tiles, that takes the
          // chunk of 512 tokens from 353 to 366 us.  New rows' weights go into two bf16 parts,
          // as one would be off by as much as the result's own rounding where a token sees few
          // rows: the low ones take S's upper half (attend_block of perf/operators.py 18.1 us
          // with one part, 18.6 with two; a prompt of 8192 tokens over itself 1857, 1968).
#pragma unroll
          for (int j0 = 0; j0 < kHalf; j0 += 16) {
            uint32_t low[8];
#pragma unroll
            for (int j = j0; j < j0 + 16; j += 2) {
              const float lo = exp2_approx(__fadd_rn(__fmul_rn(__uint_as_float(s[j]), c), shift));
              const float hi = exp2_approx(__fadd_rn(__fmul_rn(__uint_as_float(s[j + 1]), c), shift));
              sum2 = f2_add(sum2, f2_pack(lo, hi));
              const uint32_t split = split_bf16(lo, hi, low[(j - j0) / 2]);
              s[j / 2] = is_new ? split : pack_f16(lo, hi);
            }
            if (is_new) tmem_st8(s_col + kKeys / 2 + half * (kHalf / 2) + j0 / 2, low);
          }
        } else {
          const unsigned long long c2 = f2_pack(c, c), shift2 = f2_pack(shift, shift);
#pragma unroll
          for (int j = 0; j < kHalf; j += 2) {
            float lo, hi;
            f2_unpack(f2_fma(f2_pack(__uint_as_float(s[j]), __uint_as_float(s[j + 1])), c2, shift2),
                      lo, hi);
            lo = exp2_approx(lo);
            hi = exp2_approx(hi);
            sum2 = f2_add(sum2, f2_pack(lo, hi));
            s[j / 2] = pack_f16(lo, hi);
          }
        }
        if (!Sh::kAlias) ok = wait_added();
        if (!ok) break;
        const uint32_t p_col =
            (Sh::kAlias ? s_col : lanes + Sh::kColP) + half * (kHalf / 2);
        if (kHalf >= 64) {
          tmem_st16(p_col, s);
          tmem_st16(p_col + 16, s + 16);
        } else {
          tmem_st16(p_col, s);
        }
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(p_full + 8 * (i & 1));
        row_sum += f2_hsum(sum2);
      }
      if (warp_wait(o_done + 8 * ((count - 1) % 3), ((count - 1) / 3) & 1, a.status,
                    a.wait_limit, dead))
        tc_fence_after();
    }
  } else if (warp < kProductWarp) {
    // K's warps or V's: their slices of the tiles, as the buffers become free
    // one code for both: the roles share the instruction cache
    constexpr int kUnits = ((kKeys / 8 + kValueWarps - 1) / kValueWarps * 8 * M + 31) / 32;
    const int lane = threadIdx.x & 31, which = warp - kSoftWarps;
    const int part = which >= kKeyWarps;  // 0: K, 1: V
    const int bufs = part ? kValueBufs : kKeyBufs;
    const Slice<kKeys> slice(part ? which - kKeyWarps : which, part ? kValueWarps : kKeyWarps);
    const size_t at = (size_t)seq * a.seq_rows + (size_t)head * a.cap +
                      (size_t)cached0 * kKeys + slice.first;
    const uint8_t* codes = (part ? a.v : a.k) + at * (kD / 2);
    const uint8_t* scales = (part ? a.vs : a.ks) + at * (kD / 16);
    const uint16_t* fresh_rows = (part ? a.v_new : a.k_new) + (new_row + (size_t)t0 * kKeys) * kD;
    const uint32_t raw = base + Sh::kRing + part * Sh::kRawCodes + slice.first * (kD / 2);
    const uint32_t raw_scales = base + Sh::kRing + 2 * Sh::kRawCodes + part * Sh::kRawScales +
                                slice.first * (kD / 16);
    const uint32_t bar = raw_full + 8 * kRaw * which;
    const int cached = count - fresh, left = n - cached0 * kKeys - slice.first;
    // tokens of the slice in the CTA's cached tile ci
    auto there = [&](int ci) { return min(slice.count, max(0, left - ci * kKeys)); };
    auto fetch = [&](int ci) {
      const int keys = there(ci), slot = ci % kRaw;
      if (keys == 0) return;
      const uint32_t scale_bytes = (uint32_t)((keys + 7) & ~7) * (kD / 16);  // within the capacity
      mbar_expect_tx(bar + 8 * slot, keys * (kD / 2) + scale_bytes);
      bulk_g2s(raw + slot * Sh::kRawBytes, codes + (size_t)ci * kKeys * (kD / 2), keys * (kD / 2),
               bar + 8 * slot);
      bulk_g2s(raw_scales + slot * Sh::kRawBytes, scales + (size_t)ci * kKeys * (kD / 16),
               scale_bytes, bar + 8 * slot);
    };
    if (lane == 0)
      for (int ci = 0; ci < min(kRaw, cached); ++ci) fetch(ci);
    int fetched = min(kRaw, cached);
    if (part && count > 0) warp_arrive(full);  // of the tile before the first
    bool ok = true;
    for (int i = 0; i < count; ++i) {
      const uint32_t dst =
          base + (part ? kKeyBufs + i % kValueBufs : i % kKeyBufs) * Sh::kTileBytes;
      CodeSlice<M, kUnits> x;
      if (i >= fresh) {
        const int ci = i - fresh, slot = ci % kRaw, keys = there(ci);
        if (keys > 0)
          ok = warp_wait(bar + 8 * slot, (ci / kRaw) & 1, a.status, a.wait_limit, dead);
        if (!ok) break;
        x.load(raw + slot * Sh::kRawBytes, raw_scales + slot * Sh::kRawBytes, keys, lane);
        __syncwarp();
        if (fetched < cached) {
          if (lane == 0) {
            fence_proxy_async_smem();
            fetch(fetched);
          }
          ++fetched;
        }
      }
      if (i >= bufs)
        ok = warp_wait((part ? o_done : s_done) + 8 * (i % bufs), (i / bufs + 1) & 1, a.status,
                       a.wait_limit, dead);
      if (!ok) break;
      if (i < fresh) {
        const uint16_t* src = fresh_rows + (size_t)i * kKeys * kD;
        // what is not finite in V is added at the end, to the rows that see it
        if (copy_rows<M>(src, keys_new - (t0 + i) * kKeys, dst, slice.first, slice.count, lane,
                         part != 0))
          *odd = 1;
      } else {
        x.unpack(dst, slice.first, slice.count, lane);
      }
      fence_proxy_async_smem();
      warp_arrive(full + 8 * ((i + part) & 3));
      if (!part && i == count - 1) warp_arrive(full + 8 * (count & 3));  // there is none
    }
    // nothing may be in flight when the ring's memory is used again
    if (!ok && lane == 0)
      for (int ci = max(0, fetched - kRaw); ci < fetched; ++ci)
        if (there(ci) > 0)
          mbar_wait(bar + 8 * (ci % kRaw), (ci / kRaw) & 1, a.status, kWaitLimit);
    __syncwarp();
  } else {
    if ((threadIdx.x & 31) == 0 && count > 0) {
      constexpr uint32_t kLead = kKeys * 128;
      bool ok = true;
      auto await = [&](uint32_t bar, uint32_t parity) {
        if (!tile_wait(bar, parity, a.status, a.wait_limit, dead)) ok = false;
      };
      // K of tile i and V of tile i - 1
      auto operands = [&](int i) { await(full + 8 * (i & 3), (i >> 2) & 1); };
      auto scores = [&](int i) {
        const uint32_t desc = i < fresh ? tc_desc(true, false, kKeys) : tc_desc(false, false, kKeys);
        const uint64_t kt = tc_smem(base + (i % kKeyBufs) * Sh::kTileBytes, kLead);
        const uint32_t s_col = tm + (i & 1) * kKeys;
#pragma unroll
        for (int k = 0; k < kD / 16; ++k)
          tc_mma(s_col, tm + Sh::kColQ + 8 * k, kt + (((k >> 2) * kLead + (k & 3) * 32) >> 4), desc,
                 k > 0);
        tc_commit(s_done + 8 * (i & 1));
      };
      auto values = [&](int i) {
        const uint32_t desc = i < fresh ? tc_desc(true, true, kD) : tc_desc(false, true, kD);
        const uint64_t vt = tc_smem(base + (kKeyBufs + i % kValueBufs) * Sh::kTileBytes, kLead);
        const uint32_t p_col = tm + (Sh::kAlias ? (i & 1) * kKeys : Sh::kColP);
        const uint32_t low_col = tm + (i & 1) * kKeys + kKeys / 2;
#pragma unroll
        for (int k = 0; k < kKeys / 16; ++k)
          tc_mma(tm + Sh::kColO, p_col + 8 * k, vt + ((2048 * k) >> 4), desc, i > 0 || k > 0);
        if (i < fresh) {
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k)
            tc_mma(tm + Sh::kColO, low_col + 8 * k, vt + ((2048 * k) >> 4), desc, true);
        }
        tc_commit(o_done + 8 * (i % 3));
      };
#pragma unroll 1
      for (int i = -1; i < count; ++i) {
        operands(i + 1);
        // S of tile i + 1 takes the place of the weights of tile i - 1, or of their low parts
        if (i > 0 && (Sh::kAlias || i - 1 < fresh)) await(o_done + 8 * ((i - 1) % 3), ((i - 1) / 3) & 1);
        if (i + 1 < count && (i + 1 == 0 || i + 1 == fresh)) await(q_full, i + 1 == 0 ? 0 : 1);
        tc_fence_after();
        if (ok && i + 1 < count) scores(i + 1);
        if (i < 0) continue;
        await(p_full + 8 * (i & 1), (i >> 1) & 1);
        if (!ok) break;
        tc_fence_after();
        values(i);
      }
      // every product that was issued is complete before the memory is used again
      tc_commit(drain);
      mbar_wait(drain, 0, a.status, kWaitLimit);
    }
    __syncwarp();
  }
  __syncthreads();

  const bool none = n == 0 && !a.k_new;  // no token to attend to
  float* stat = reinterpret_cast<float*>(smem + Sh::kStats);  // [max, sum, sum][row]
  if (warp < kSoftWarps) {
    if (half == 0) stat[lane_row] = row_max;
    stat[(1 + half) * kTileRows + lane_row] = row_sum;
  }
  __syncthreads();
  if (warp < kSoftWarps) {
    const bool valid = row < a.rows && !bad_len;
    const size_t at = (((size_t)seq * a.B + token) * a.heads + head) * a.group + row % a.group;
    row_sum = stat[kTileRows + lane_row] + stat[2 * kTileRows + lane_row];
    const float inv = none ? 0.f : 1.f / row_sum;
    if (a.cluster == 1 && valid && a.lse && half == 0)
      a.lse[at] = none ? -INFINITY : (row_max + kTileLift) / kLog2e + logf(row_sum * kTileUnlift);
#pragma unroll 1
    for (int j = half * (kD / 2); j < (half + 1) * (kD / 2); j += 16) {
      uint32_t o[16];
      if (count > 0) {
        tmem_ld(lanes + Sh::kColO + j, o);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = 0;
      }
      if (*odd) {  // the values that were left out
        for (int key = t0 * kKeys; key < min((t0 + fresh) * kKeys, token + 1); ++key)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint16_t x = a.v_new[(new_row + key) * kD + j + e];
            if ((x & 0x7f80u) == 0x7f80u)
              o[e] = __float_as_uint(__uint_as_float(o[e]) + __uint_as_float((uint32_t)x << 16));
          }
        __syncwarp();
      }
      if (a.cluster == 1) {
        if (valid)
#pragma unroll
          for (int e = 0; e < 16; e += 8) {
            uint32_t w[4];
#pragma unroll
            for (int f = 0; f < 4; ++f)
              w[f] = pack_bf16(__uint_as_float(o[e + 2 * f]) * inv,
                               __uint_as_float(o[e + 2 * f + 1]) * inv);
            st16(a.out + at * kD + j + e, make_uint4(w[0], w[1], w[2], w[3]));
          }
        __syncwarp();
      } else {  // [dim / 4][row][4]
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          st_shared16(base + (((j + e) / 4) * kTileRows + lane_row) * 16,
                      make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]));
      }
    }
    tc_fence_before();
  }
  if (a.cluster > 1)
    cluster_sync();
  else
    __syncthreads();
  if (warp == kProductWarp) {
    tc_fence_after();
    tmem_free(tm);
  }
  if (a.cluster == 1) return;
  // Each CTA writes its share of the rows (those that are there), from all CTAs' results in
  // rank order: first every CTA's factor for every row of the share, then the sums.
  const int rows = min(kTileRows, a.rows - row0);
  const int share = (rows + a.cluster - 1) / a.cluster;
  const int r0 = (int)rank * share, mine = bad_len ? 0 : max(0, min(share, rows - r0));
  const uint32_t stats = base + Sh::kStats;
  float* factor = reinterpret_cast<float*>(smem + Sh::kFactors);  // [cluster][share], maxima first
  float* sums = reinterpret_cast<float*>(smem + Sh::kSwap);       // the same
  for (int i = threadIdx.x; i < mine * a.cluster; i += kTileThreads) {
    const int q = i / mine, r = i % mine;
    factor[q * share + r] = ld_cluster_f32(mapa(stats + 4 * (r0 + r), q));
    sums[q * share + r] = ld_cluster_f32(mapa(stats + 4 * (kTileRows + r0 + r), q)) +
                          ld_cluster_f32(mapa(stats + 4 * (2 * kTileRows + r0 + r), q));
  }
  __syncthreads();
  if ((int)threadIdx.x < mine) {
    const int r = threadIdx.x, gr = row0 + r0 + r;
    float m = -INFINITY, l = 0.f;
    for (int q = 0; q < a.cluster; ++q) m = fmaxf(m, factor[q * share + r]);
    for (int q = 0; q < a.cluster; ++q) {
      const float mq = factor[q * share + r];
      // a CTA without tokens has sums of zero; one whose scores were all NaN has NaN sums
      const float f = mq == -INFINITY ? 1.f : exp2_approx(mq - m);
      l = fmaf(sums[q * share + r], f, l);
      factor[q * share + r] = f;
    }
    sums[r] = none ? 0.f : 1.f / l;  // the first CTA's, which this thread alone has read
    if (a.lse)
      a.lse[(((size_t)seq * a.B + gr / a.group) * a.heads + head) * a.group + gr % a.group] =
          none ? -INFINITY : (m + kTileLift) / kLog2e + logf(l * kTileUnlift);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < mine * (kD / 4); i += kTileThreads) {
    const int r = i % mine, dim4 = i / mine;  // neighbouring threads read neighbouring rows
    const uint32_t x_addr = base + (dim4 * kTileRows + r0 + r) * 16;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int q0 = 0; q0 < a.cluster; q0 += 4) {
      float4 x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q0 + q < a.cluster) x[q] = ld_cluster_f32x4(mapa(x_addr, q0 + q));
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q0 + q < a.cluster) {
          const float f = factor[(q0 + q) * share + r];
          acc.x = fmaf(x[q].x, f, acc.x);
          acc.y = fmaf(x[q].y, f, acc.y);
          acc.z = fmaf(x[q].z, f, acc.z);
          acc.w = fmaf(x[q].w, f, acc.w);
        }
    }
    const int gr = row0 + r0 + r;
    const size_t at =
        (((size_t)seq * a.B + gr / a.group) * a.heads + head) * a.group + gr % a.group;
    const float inv = sums[r];
    *reinterpret_cast<uint2*>(a.out + at * kD + 4 * dim4) =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  }
  cluster_sync();  // no CTA leaves while its results are read
}

}  // namespace vd
