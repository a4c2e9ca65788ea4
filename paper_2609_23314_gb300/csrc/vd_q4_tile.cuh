// vd_q4_tile.cuh -- attention over one layer of a 4-bit cache (vd_q4_attend in
// include/vd.h): the block kernel, for many query rows per KV head (blocks of block
// prompt processing, prompts).
//
// The formula is vd_q4_attend.cuh's.  128 query rows of a KV head are one CTA's tile (a
// row per thread of four warps and per lane of tensor memory), the tokens come in tiles
// of KT, and the two products run on tcgen05 with Q, the weights P and both results in
// tensor memory, so that shared memory carries K and V only:
//   S = Q K^T   (128 x KT, K's rows along the depth)
//   O += P V    (128 x head_dim, V's rows along the columns)
// Roles of the ten warps, which meet only at mbarriers:
//   0-3  a row each: maximum, weights, their sum; rescale O where the maximum has risen
//        by more than 2^8 (a smaller rise only makes the weights exceed 1);
//   4-7  cached codes to fp16 in the swizzled layout of the products (exact), or copies of
//        the new tokens' bf16 rows; two buffers each for K and V;
//   8    issues the products: S of tile i + 1 before O of tile i, so that the softmax of
//        one tile runs beside the products of its neighbours;
//   9    bulk copies of codes and scales into a ring.
// The new tokens' tiles come first, in bf16, then Q is rewritten in fp16 (rows scaled by
// powers of two, as in the streaming kernel) for the cached ones.  A cluster splits the
// tiles of a unit and joins the results through distributed shared memory.
//
// Bounds per tile of 128 tokens at head_dim 128: 2 x 2.1 M multiply-adds, 1024 cycles at
// 4096 a cycle; 128 exponentials per thread, 512 cycles; codes to fp16 about 350 issue
// slots per scheduler.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "vd_device.cuh"
#include "vd_q4.cuh"
#include "vd_q4_attend.cuh"
#include "vd_tcgen05.cuh"

namespace vd {

constexpr int kTileRows = 128;
constexpr int kTileThreads = 320;

template <int M>
struct TileShape {
  static constexpr int kD = 32 * M;
  static constexpr int kKeys = M <= 4 ? 128 : M <= 7 ? 64 : 32;  // tensor memory: see below
  static constexpr int kBlocks = (kD + 63) / 64;                 // 64-column blocks of a row
  static constexpr int kTileBytes = kBlocks * kKeys * 128;
  static constexpr int kCodeBytes = kKeys * 16 * M;
  static constexpr int kScaleBytes = kKeys * 2 * M;
  static constexpr int kRawBytes = 2 * (kCodeBytes + kScaleBytes);
  static constexpr int kRaw = M == 8 ? 4 : 3;  // stages of the ring
  static constexpr int kRing = 4 * kTileBytes;
  static constexpr int kUsed = kRing + kRaw * kRawBytes;
  static constexpr int kPartBytes = kTileRows * kD * 4;
  static constexpr int kStats = kUsed > kPartBytes ? kUsed : kPartBytes;
  static constexpr int kBars = kStats + 2 * kTileRows * 4;
  static constexpr int kNumBars = 2 * kRaw + 14;
  static constexpr int kMisc = kBars + kNumBars * 8;  // tensor memory address, flags
  // The base is rounded up to 1024.  Never two CTAs on an SM: the second would wait for
  // tensor memory, and the first, in one cluster with it, for the second.
  static constexpr int kNeed = kMisc + 16 + 1024;
  static constexpr int kTotal = kNeed > 120 * 1024 ? kNeed : 120 * 1024;
  // columns of tensor memory: two S, P (16-bit pairs), O, Q (16-bit pairs)
  static constexpr int kColP = 2 * kKeys;
  static constexpr int kColO = (kColP + kKeys / 2 + 31) / 32 * 32;
  static constexpr int kColQ = kColO + kD;
  static_assert(kColQ + kD / 2 <= 512, "tensor memory");
};

// Waits like mbar_wait, and gives up as well once another role has.
__device__ __forceinline__ bool tile_wait(uint32_t bar, uint32_t parity, unsigned* status,
                                          uint32_t limit, volatile int* dead) {
  for (uint32_t i = 0; i < limit; ++i) {
    uint32_t done;
    asm volatile(
        "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; "
        "selp.u32 %0, 1, 0, p; }"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    if (done) return true;
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

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

template <int M>
__global__ void __launch_bounds__(kTileThreads, 1) q4_tile_kernel(AttendArgs a) {
  using Sh = TileShape<M>;
  constexpr int kD = Sh::kD, kKeys = Sh::kKeys;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw_base = smem_addr(smem_raw);
  const uint32_t base = (raw_base + 1023u) & ~1023u;
  unsigned char* smem = smem_raw + (base - raw_base);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned rank = blockIdx.x % a.cluster;
  const unsigned item = blockIdx.x / a.cluster;
  const int tile = item % a.tiles;
  const unsigned unit = item / a.tiles;
  const int seq = unit / a.heads, head = unit % a.heads;

  const uint32_t bars = base + Sh::kBars;
  const uint32_t raw_full = bars, raw_empty = bars + 8 * Sh::kRaw;
  const uint32_t k_full = raw_empty + 8 * Sh::kRaw, k_empty = k_full + 16;
  const uint32_t v_full = k_empty + 16, v_empty = v_full + 16, s_full = v_empty + 16;
  const uint32_t p_full = s_full + 16, pv_done = p_full + 8, q_full = pv_done + 8;
  const uint32_t drain = q_full + 8;
  volatile int* dead = reinterpret_cast<volatile int*>(smem + Sh::kMisc + 4);
  volatile int* odd = dead + 1;  // a new row of V holds a value that is not finite
  if (threadIdx.x == 0) {
    for (int i = 0; i < Sh::kRaw; ++i) {
      mbar_init(raw_full + 8 * i, 1);
      mbar_init(raw_empty + 8 * i, 128);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(k_full + 8 * i, 128);
      mbar_init(k_empty + 8 * i, 1);
      mbar_init(v_full + 8 * i, 128);
      mbar_init(v_empty + 8 * i, 1);
      mbar_init(s_full + 8 * i, 1);
    }
    mbar_init(p_full, 128);
    mbar_init(pv_done, 1);
    mbar_init(q_full, 128);
    mbar_init(drain, 1);
    fence_mbar_init();
    *dead = 0;
    *odd = 0;
  }
  if (warp == 8) tmem_alloc(base + Sh::kMisc);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = *reinterpret_cast<volatile uint32_t*>(smem + Sh::kMisc);
  grid_dependency_wait();
  grid_launch_dependents();

  const int n = __ldcg(a.len + seq);
  const bool bad_len = n < 0 || n > a.cap;
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

  float row_max = -INFINITY, row_sum = 0.f;  // the softmax warps': in log2 units
  if (warp < 4) {
    const uint32_t lanes = tm + ((uint32_t)warp << 21);  // this warp's 32 lanes
    const int row = row0 + (int)threadIdx.x;
    const bool valid = row < a.rows;
    const int token = min(row, a.rows - 1) / a.group;
    const uint16_t* q = a.q + ((((size_t)seq * a.B + token) * a.heads + head) * a.group +
                               row % a.group) * kD;
    // Q: scaled so that the row's largest value lies in [1, 2), for bf16, or in [2^13, 2^14)
    uint32_t top = 0;
    if (count > 0 && valid)
#pragma unroll 4
      for (int i = 0; i < kD / 8; ++i) {
        const uint4 x = ld_cg16(q + 8 * i);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7fffu, (w[e] >> 16) & 0x7fffu));
      }
    const uint32_t ex = top ? min(253u, max(1u, top >> 7)) : 127u;
    const float up = __uint_as_float((254 - ex) << 23);
    const float unit = __uint_as_float(ex << 23) * (a.scale * kLog2e);
    auto write_q = [&](bool bf16) {
      const float f = bf16 ? 1.f : 0x1p13f;
#pragma unroll 1
      for (int i = 0; i < M; ++i) {
        uint32_t w[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (valid) x = ld_cg16(q + 32 * i + 8 * j);
          w[4 * j] = x.x, w[4 * j + 1] = x.y, w[4 * j + 2] = x.z, w[4 * j + 3] = x.w;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float lo = __uint_as_float(w[j] << 16) * up * f;
          const float hi = __uint_as_float(w[j] & 0xffff0000u) * up * f;
          w[j] = bf16 ? pack_bf16(lo, hi) : pack_f16(lo, hi);
        }
        __syncwarp();
        tmem_st16(lanes + Sh::kColQ + 16 * i, w);
      }
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(q_full);
    };
    __syncwarp();
    if (count > 0) write_q(fresh > 0);
    for (int i = 0; i < count; ++i) {
      const uint32_t s_col = lanes + (i & 1) * kKeys;
      if (!warp_wait(s_full + 8 * (i & 1), (i >> 1) & 1, a.status, kWaitLimit, dead))
        break;
      tc_fence_after();
      if (i == fresh - 1 && fresh < count) write_q(false);  // the last product of the bf16 form
      const bool is_new = i < fresh;
      // not 0, which would make a masked score a NaN
      const float c = fmaxf(is_new ? unit : unit * 0x1p-13f, 0x1p-126f);
      // tokens behind this row's last one do not count
      const int seen = is_new ? token - (t0 + i) * kKeys
                              : n - 1 - (cached0 + i - fresh) * kKeys;
      const bool edge = __any_sync(kFull, seen < kKeys - 1);
      // Half the columns at a time, the first half read once more for its weights: all of
      // them at once would not fit the registers
      constexpr int kPart = kKeys == 128 ? 64 : kKeys;
      uint32_t s[kPart];
      auto load = [&](int from) {
        tmem_ld(s_col + from, s);
        if (edge) {
#pragma unroll
          for (int j = 0; j < kPart; ++j)
            if (from + j > seen) s[j] = 0xff800000u;
        }
      };
      float m = -INFINITY;
#pragma unroll
      for (int from = 0; from < kKeys; from += kPart) {
        load(from);
#pragma unroll
        for (int j = 0; j < kPart; ++j) m = fmaxf(m, __uint_as_float(s[j]));
      }
      m *= c;
      bool waited = false;
      // the weights stay below 2^8, and a row's first scores set its maximum
      if (__any_sync(kFull, m > row_max + 8.f)) {
        const float up_to = fmaxf(row_max, m);
        const float f = up_to == -INFINITY ? 1.f : exp2_approx(row_max - up_to);
        row_max = up_to;
        row_sum *= f;
        if (i > 0) {
          waited = true;
          if (!warp_wait(pv_done, (i - 1) & 1, a.status, kWaitLimit, dead))
            break;
          tc_fence_after();
#pragma unroll 1
          for (int j = 0; j < kD; j += 32) {
            uint32_t o[32];
            tmem_ld(lanes + Sh::kColO + j, o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tmem_st32(lanes + Sh::kColO + j, o);
          }
        }
      }
      const float shift = row_max == -INFINITY ? 0.f : -row_max;
      const unsigned long long c2 = f2_pack(c, c), shift2 = f2_pack(shift, shift);
      unsigned long long sum2 = 0;
#pragma unroll
      for (int from = kKeys - kPart; from >= 0; from -= kPart) {
        if (from < kKeys - kPart) load(from);
#pragma unroll
        for (int j = 0; j < kPart; j += 2) {
          float lo, hi;
          f2_unpack(f2_fma(f2_pack(__uint_as_float(s[j]), __uint_as_float(s[j + 1])), c2, shift2),
                    lo, hi);
          lo = exp2_approx(lo);
          hi = exp2_approx(hi);
          sum2 = f2_add(sum2, f2_pack(lo, hi));
          s[j / 2] = is_new ? pack_bf16(lo, hi) : pack_f16(lo, hi);
        }
        if (from == kKeys - kPart && i > 0 && !waited) {
          waited = warp_wait(pv_done, (i - 1) & 1, a.status, kWaitLimit, dead);
          if (!waited) break;
          tc_fence_after();
        }
#pragma unroll
        for (int j = 0; j < kPart / 2; j += 16) tmem_st16(lanes + Sh::kColP + from / 2 + j, s + j);
      }
      if (i > 0 && !waited) break;
      row_sum += f2_hsum(sum2);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(p_full);
    }
    if (count > 0 && warp_wait(pv_done, (count - 1) & 1, a.status, kWaitLimit, dead))
      tc_fence_after();
  } else if (warp < 8) {
    const int t = threadIdx.x - 128;
    for (int i = 0; i < count; ++i) {
      const int b = i & 1;
      const uint32_t again = (i >> 1) + 1;  // parity of the release before: b's (i >> 1)-th
      const uint32_t kt = base + b * Sh::kTileBytes, vt = kt + 2 * Sh::kTileBytes;
      if (i < fresh) {  // copies of the new rows; what is behind the last one is zero
        const int key0 = (t0 + i) * kKeys;
        for (int part = 0; part < 2; ++part) {
          const uint16_t* src = (part ? a.v_new : a.k_new) + (new_row + key0) * kD;
          const uint32_t dst = part ? vt : kt;
          if (i > 1 && !warp_wait((part ? v_empty : k_empty) + 8 * b, again & 1, a.status,
                                  kWaitLimit, dead))
            break;
#pragma unroll 4
          for (int j = t; j < kKeys * (kD / 8); j += 128) {
            const int key = j / (kD / 8), chunk = j % (kD / 8);
            uint4 x = make_uint4(0, 0, 0, 0);
            if (key0 + key < keys_new) x = ld_cg16(src + (size_t)key * kD + 8 * chunk);
            if (part) {  // a value that is not finite is added at the end, to those that see it
              uint32_t w[4] = {x.x, x.y, x.z, x.w};
              bool found = false;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u, found = true;
                if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0xffffu, found = true;
              }
              if (found) *odd = 1;
              x = make_uint4(w[0], w[1], w[2], w[3]);
            }
            st_shared16(dst + (chunk >> 3) * (kKeys * 128) + key * 128 +
                            (((chunk & 7) ^ (key & 7)) << 4), x);
          }
          fence_proxy_async_smem();
          mbar_arrive((part ? v_full : k_full) + 8 * b);
        }
        if (*dead) break;
        continue;
      }
      const int ci = i - fresh, slot = ci % Sh::kRaw;
      const int left = n - (cached0 + ci) * kKeys;  // cached tokens of the tile
      const uint32_t raw = base + Sh::kRing + slot * Sh::kRawBytes;
      if (!warp_wait(raw_full + 8 * slot, (ci / Sh::kRaw) & 1, a.status, a.wait_limit, dead))
        break;
      bool gone = false;
      for (int part = 0; part < 2; ++part) {
        const uint32_t codes = raw + part * Sh::kCodeBytes;
        const uint32_t scales = raw + 2 * Sh::kCodeBytes + part * Sh::kScaleBytes;
        const uint32_t dst = part ? vt : kt;
        if (i > 1 && !warp_wait((part ? v_empty : k_empty) + 8 * b, again & 1, a.status,
                                kWaitLimit, dead)) {
          gone = true;
          break;
        }
#pragma unroll 4
        for (int j = t; j < kKeys * M; j += 128) {  // 32 values: 16 bytes of codes
          const int key = j / M, blk = j % M;
          uint4 x = ld_shared16(codes + j * 16);
          uint32_t sb = ld_shared_u16(scales + 2 * j);
          if (key >= left) x = make_uint4(0, 0, 0, 0), sb = 0;  // whatever lies there
          // the order of the four 16-byte stores, so that 8 neighbouring lanes meet 8
          // chunk positions
          const int turn = M == 4 ? (blk & 2) : M == 8 ? (blk >> 1) & 3 : 0;
          uint32_t w[4] = {x.x, x.y, x.z, x.w};
          if (M % 4 == 0) {
            if (turn & 1) {
              uint32_t u = w[0]; w[0] = w[1]; w[1] = u;
              u = w[2]; w[2] = w[3]; w[3] = u;
            }
            if (turn & 2) {
              uint32_t u = w[0]; w[0] = w[2]; w[2] = u;
              u = w[1]; w[1] = w[3]; w[3] = u;
            }
          }
          const uint32_t s_lo = (sb & 255u) * 0x00800080u, s_hi = (sb >> 8) * 0x00800080u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int at = e ^ turn;  // 8-value chunk of the 32
            const uint32_t sc = at < 2 ? s_lo : s_hi;
            uint32_t h[4];
            q4_unpack4(w[e], h);
            const int chunk = 4 * blk + at;
            st_shared16(dst + (chunk >> 3) * (kKeys * 128) + key * 128 +
                            (((chunk & 7) ^ (key & 7)) << 4),
                        make_uint4(h2_mul(h[0], sc), h2_mul(h[1], sc), h2_mul(h[2], sc),
                                   h2_mul(h[3], sc)));
          }
        }
        fence_proxy_async_smem();
        mbar_arrive((part ? v_full : k_full) + 8 * b);
      }
      if (gone) break;
      mbar_arrive(raw_empty + 8 * slot);
    }
  } else if (warp == 8) {
    if (lane == 0) {
      constexpr uint32_t kLead = kKeys * 128;
      auto values = [&](int i) {  // O += P V of tile i
        const bool bf16 = i < fresh;
        const uint32_t desc = bf16 ? tc_desc(true, true, kD) : tc_desc(false, true, kD);
        const uint32_t vt = base + (2 + (i & 1)) * Sh::kTileBytes;
        if (!tile_wait(p_full, i & 1, a.status, kWaitLimit, dead) ||
            !tile_wait(v_full + 8 * (i & 1), (i >> 1) & 1, a.status, kWaitLimit, dead))
          return false;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kKeys / 16; ++k)
          tc_mma(tm + Sh::kColO, tm + Sh::kColP + 8 * k, tc_smem(vt + 2048 * k, kLead), desc,
                 i > 0 || k > 0);
        tc_commit(v_empty + 8 * (i & 1));
        tc_commit(pv_done);
        return true;
      };
      bool ok = true;
      for (int i = 0; ok && i < count; ++i) {
        const bool bf16 = i < fresh;
        const uint32_t desc = bf16 ? tc_desc(true, false, kKeys) : tc_desc(false, false, kKeys);
        const uint32_t kt = base + (i & 1) * Sh::kTileBytes;
        if (i == 0) ok = tile_wait(q_full, 0, a.status, kWaitLimit, dead);
        if (i == fresh && i > 0) ok = tile_wait(q_full, 1, a.status, kWaitLimit, dead);
        ok = ok && tile_wait(k_full + 8 * (i & 1), (i >> 1) & 1, a.status, kWaitLimit, dead);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kD / 16; ++k)
          tc_mma(tm + (i & 1) * kKeys, tm + Sh::kColQ + 8 * k,
                 tc_smem(kt + (k >> 2) * kLead + (k & 3) * 32, kLead), desc, k > 0);
        tc_commit(k_empty + 8 * (i & 1));
        tc_commit(s_full + 8 * (i & 1));
        if (i > 0) ok = values(i - 1);
      }
      if (ok && count > 0) values(count - 1);
    }
    __syncwarp();
  } else {
    if (lane == 0) {
      const size_t unit_row = (size_t)seq * a.seq_rows + (size_t)head * a.cap;
      const int cached = count - fresh;
      int issued = 0;
      for (; issued < cached; ++issued) {
        const int slot = issued % Sh::kRaw;
        if (issued >= Sh::kRaw && !tile_wait(raw_empty + 8 * slot, (issued / Sh::kRaw + 1) & 1,
                                             a.status, kWaitLimit, dead))
          break;
        const size_t key0 = (size_t)(cached0 + issued) * kKeys;
        const int keys = min(kKeys, n - (int)key0);
        const uint32_t codes = (uint32_t)keys * (kD / 2);
        const uint32_t scales = (uint32_t)((keys + 7) & ~7) * (kD / 16);  // within the capacity
        const uint32_t dst = base + Sh::kRing + slot * Sh::kRawBytes, bar = raw_full + 8 * slot;
        fence_proxy_async_smem();
        mbar_expect_tx(bar, 2 * (codes + scales));
        bulk_g2s(dst, a.k + (unit_row + key0) * (kD / 2), codes, bar);
        bulk_g2s(dst + Sh::kCodeBytes, a.v + (unit_row + key0) * (kD / 2), codes, bar);
        bulk_g2s(dst + 2 * Sh::kCodeBytes, a.ks + (unit_row + key0) * (kD / 16), scales, bar);
        bulk_g2s(dst + 2 * Sh::kCodeBytes + Sh::kScaleBytes, a.vs + (unit_row + key0) * (kD / 16),
                 scales, bar);
      }
      // nothing may be in flight when the ring's memory is used again
      for (int i = max(0, issued - Sh::kRaw); i < issued; ++i)
        mbar_wait(raw_full + 8 * (i % Sh::kRaw), (i / Sh::kRaw) & 1, a.status, kWaitLimit);
    }
    __syncwarp();
  }
  // every product that was issued is complete before the memory is used again
  if (warp == 8 && lane == 0 && count > 0) {
    tc_commit(drain);
    mbar_wait(drain, 0, a.status, kWaitLimit);
  }
  __syncthreads();

  const bool none = n == 0 && !a.k_new;  // no token to attend to
  if (warp < 4) {
    const uint32_t lanes = tm + ((uint32_t)warp << 21);
    const int row = row0 + (int)threadIdx.x;
    const int token = min(row, a.rows - 1) / a.group;
    const bool valid = row < a.rows && !bad_len;
    const size_t at = (((size_t)seq * a.B + token) * a.heads + head) * a.group + row % a.group;
    const float inv = none ? 0.f : 1.f / row_sum;
    if (a.cluster == 1 && valid && a.lse)
      a.lse[at] = none ? -INFINITY : row_max / kLog2e + logf(row_sum);
    float* stat = reinterpret_cast<float*>(smem + Sh::kStats);
    stat[threadIdx.x] = row_max;
    stat[kTileRows + threadIdx.x] = row_sum;
#pragma unroll 1
    for (int j = 0; j < kD; j += 32) {
      uint32_t o[32];
      if (count > 0) {
        tmem_ld(lanes + Sh::kColO + j, o);
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0;
      }
      if (*odd) {  // the values that were left out
        for (int key = t0 * kKeys; key < min((t0 + fresh) * kKeys, token + 1); ++key)
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const uint16_t x = a.v_new[(new_row + key) * kD + j + e];
            if ((x & 0x7f80u) == 0x7f80u)
              o[e] = __float_as_uint(__uint_as_float(o[e]) + __uint_as_float((uint32_t)x << 16));
          }
      }
      if (a.cluster == 1) {
        if (valid)
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            uint32_t w[4];
#pragma unroll
            for (int f = 0; f < 4; ++f)
              w[f] = pack_bf16(__uint_as_float(o[e + 2 * f]) * inv,
                               __uint_as_float(o[e + 2 * f + 1]) * inv);
            st16(a.out + at * kD + j + e, make_uint4(w[0], w[1], w[2], w[3]));
          }
      } else {  // [dim / 4][row][4]
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          st_shared16(base + (((j + e) / 4) * kTileRows + threadIdx.x) * 16,
                      make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]));
      }
    }
    tc_fence_before();
  }
  if (a.cluster > 1)
    cluster_sync();
  else
    __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_free(tm);
  }
  if (a.cluster == 1) return;
  // each CTA writes its share of the rows, from all CTAs' results in rank order
  const int share = kTileRows / a.cluster;
  const uint32_t stats = base + Sh::kStats;
  for (int i = threadIdx.x; i < share * (kD / 4) && !bad_len; i += kTileThreads) {
    const int r = (int)rank * share + i % share, dim4 = i / share;
    const int row = row0 + r;
    if (row >= a.rows) continue;
    float m = -INFINITY;
    for (int q = 0; q < a.cluster; ++q) m = fmaxf(m, ld_cluster_f32(mapa(stats + 4 * r, q)));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
    for (int q = 0; q < a.cluster; ++q) {
      const float mq = ld_cluster_f32(mapa(stats + 4 * r, q));
      // a CTA without tokens has sums of zero; one whose scores were all NaN has NaN sums
      const float f = mq == -INFINITY ? 1.f : exp2_approx(mq - m);
      const uint32_t x = mapa(base + (dim4 * kTileRows + r) * 16, q);
      acc.x = fmaf(ld_cluster_f32(x), f, acc.x);
      acc.y = fmaf(ld_cluster_f32(x + 4), f, acc.y);
      acc.z = fmaf(ld_cluster_f32(x + 8), f, acc.z);
      acc.w = fmaf(ld_cluster_f32(x + 12), f, acc.w);
      l = fmaf(ld_cluster_f32(mapa(stats + 4 * (kTileRows + r), q)), f, l);
    }
    const size_t at =
        (((size_t)seq * a.B + row / a.group) * a.heads + head) * a.group + row % a.group;
    const float inv = none ? 0.f : 1.f / l;
    *reinterpret_cast<uint2*>(a.out + at * kD + 4 * dim4) =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    if (dim4 == 0 && a.lse) a.lse[at] = none ? -INFINITY : m / kLog2e + logf(l);
  }
  cluster_sync();  // no CTA leaves while its results are read
}

}  // namespace vd
