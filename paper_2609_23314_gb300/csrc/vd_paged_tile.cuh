// vd_paged_tile.cuh -- attention over one layer of a paged cache (vd_paged_attend in
// include/vd.h): the block kernel, for many query rows per KV head (blocks of block prompt
// processing, prompts).
//
// The formula is vd_paged_stream.cuh's; roles, barriers and tensor memory are those of the block
// kernel over a 4-bit cache (vd_q4_tile.cuh): 128 query rows of a KV head are one CTA's, the slots
// come in tiles, and both products run on tcgen05 with Q, the weights P and both results in
// tensor memory, so that shared memory carries K and V only.
//   0-7   softmax, a row per pair of threads;
//   8-11  K's tiles, a slice of the slots each: single asynchronous copies of bf16 rows into the
//         swizzled layout of the products, one tile ahead; e4m3 ones by way of registers to
//         fp16 (exact);
//   12-14 V's tiles, the same;
//   15    one thread issues the products.
// A cluster splits the tiles of a unit and joins the results through distributed shared memory.
//
// 128 new tokens over 2048, 8 KV heads of 4 query heads, 21 us: start and queries 4, 5 tiles of 2.2,
// the join.  A tile of 128 slots takes the softmax 2000 cycles, most of it the exponentials, and the
// products 2300, of which the weights' lower parts are 800; its 2.2 us are about 4500, the sum of the
// two, although the roles are there to overlap.  What keeps them apart has not been measured: copies
// that run one tile ahead only, with 5 tiles a CTA, or the chain from scores to weights to product.  8 sequences of 4000 slots, 16 rows 39 us (3.4 TB/s).
// Copies by lanes with a fixed chunk of every row: 26 us without.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "vd_attend.cuh"
#include "vd_device.cuh"
#include "vd_paged.cuh"
#include "vd_paged_attend.cuh"
#include "vd_paged_stream.cuh"
#include "vd_q4_tile.cuh"
#include "vd_tcgen05.cuh"

namespace vd {

// A CTA's part of a unit's slots, in tiles.
template <int kKeys>
struct BlockPlace {
  int rows_all, row0;  // query rows of the KV head, the tile's first one
  int keys, all_see;   // slots that the tile's last and first row see
  int t0, count;       // this CTA's tiles of them
  __device__ __forceinline__ BlockPlace(const PagedAttendArgs& a, int tile, int rank, int2 size)
      : rows_all(size.y * a.group), row0(tile * kTileRows) {
    const int last = (min(rows_all, row0 + kTileRows) - 1) / a.group;
    keys = row0 >= rows_all ? 0 : size.x + (a.causal ? last + 1 : 0);
    all_see = size.x + (a.causal ? row0 / a.group + 1 : 0);
    const int tiles = (keys + kKeys - 1) / kKeys;
    t0 = (int)((uint32_t)(tiles * rank) / a.cluster);  // below 2^24 tiles, 17 ranks
    count = (int)((uint32_t)(tiles * (rank + 1)) / a.cluster) - t0;
  }
};

template <int M, bool E4M3>
__global__ void __launch_bounds__(kTileThreads, 1)
    paged_tile_kernel(const __grid_constant__ PagedAttendArgs a) {
  using Sh = TileShape<M>;
  constexpr int kD = Sh::kD, kKeys = Sh::kKeys;
  constexpr int kKeyBufs = Sh::kKeyBufs, kValueBufs = Sh::kValueBufs;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw_base = smem_addr(smem_raw);
  const uint32_t base = (raw_base + 1023u) & ~1023u;
  unsigned char* smem = smem_raw + (base - raw_base);
  const int warp = threadIdx.x >> 5;
  const int item = blockIdx.x / a.cluster, rank = blockIdx.x - item * a.cluster;
  const int unit = item / a.tiles, tile = item - unit * a.tiles;
  const int seq = unit / a.heads, head = unit - seq * a.heads;

  // Barriers as in vd_q4_tile.cuh: full[i % 4]: K of tile i and V of the tile before it;
  // s_done[i % 2]: the tile's scores; o_done[i % 3]: it is added to O; p_full[i % 2]: its weights;
  // swap: a pair of softmax warps has exchanged its rows' maxima; Q written; all products complete
  const uint32_t full = base + Sh::kBars, s_done = full + 32, o_done = s_done + 16;
  const uint32_t p_full = o_done + 24, swap = p_full + 16, q_full = swap + 32;
  const uint32_t drain = q_full + 8;
  volatile int* dead = reinterpret_cast<volatile int*>(smem + Sh::kMisc + 4);
  volatile int* odd = dead + 1;  // a value of V that some rows do not see is not finite
  if (threadIdx.x == 0) {
    for (int i = 0; i < 4; ++i) mbar_init(full + 8 * i, kKeyWarps + kValueWarps);
    for (int i = 0; i < 3; ++i) mbar_init(o_done + 8 * i, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_done + 8 * i, 1);
      mbar_init(p_full + 8 * i, kSoftWarps);
    }
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

  // Queries and the table, which a wait for the length need not delay, into L2
  {
    const int r = tile * kTileRows + (threadIdx.x & 127);
    if (threadIdx.x < 256 && r < a.B * a.group) {
      const int tok = r / a.group;
      const char* q = reinterpret_cast<const char*>(
          a.q + ((((size_t)seq * a.B + tok) * a.heads + head) * a.group + r - tok * a.group) * a.d);
      prefetch_l2(q + (threadIdx.x >= 128 ? a.d : 0));
    }
    const int line = threadIdx.x - 256;  // of 32 entries
    if (line >= 0 && 32 * line < a.pages.max_pages)
      prefetch_l2(a.pages.table + (size_t)seq * a.pages.max_pages + 32 * line);
  }
  // kept where the loops need no registers for it
  volatile int* kept = reinterpret_cast<volatile int*>(smem + Sh::kFactors);
  const int2 size = seq_size(a, seq, rank == 0 && tile == 0 && head == 0 && threadIdx.x == 0);
  if (threadIdx.x == 0) {
    kept[0] = size.x;
    kept[1] = size.y;
  }
  const BlockPlace<kKeys> at_first(a, tile, rank, size);
  const int keys = at_first.keys, all_see = at_first.all_see, t0 = at_first.t0,
            count = at_first.count;

  const int half = (warp >> 2) & 1, lane_row = threadIdx.x & 127;  // of the softmax threads
  const uint32_t lanes = tm + ((uint32_t)(warp & 3) << 21);        // their warp's 32 lanes
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
      if (!warp_wait(swap + 8 * (warp & 3), turn & 1, a.pages.status, a.wait_limit, dead))
        return false;
      m = fmaxf(m, at[(half ^ 1) * kTileRows]);
      return true;
    };
    if (count > 0) {
      const int row = at_first.row0 + lane_row, rows_all = at_first.rows_all;
      const int token = min(row, rows_all - 1) / a.group;
      const int sees = size.x + (a.causal ? token + 1 : 0);
      const uint32_t q_col = lanes + Sh::kColQ + half * 8 * M;
      // Q, each row times its power of two (scale_of)
      float factor;
      bool ok;
      {
        const uint16_t* q =
            a.q + ((((size_t)seq * a.B + token) * a.heads + head) * a.group + row % a.group) * a.d;
        uint32_t w[8 * M];
#pragma unroll
        for (int i = 0; i < 2 * M; ++i) {
          const int d0 = half * 16 * M + 8 * i;
          uint4 x = make_uint4(0, 0, 0, 0);
          if (row < rows_all && d0 < a.d) x = ld_cg16(q + d0);
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
        const float ks = E4M3 && a.pages.k_scale ? __ldcg(a.pages.k_scale + head) : 1.f;
        factor = score_factor(qs.down, a.scale * ks);
        if (E4M3) factor = cached_factor(factor);
#pragma unroll
        for (int i = 0; i < 8 * M; ++i) {
          asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(w[i]) : "r"(qs.up));
          if (E4M3)
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
#pragma unroll 1
      for (int i = 0; ok && i < count; ++i) {
        const uint32_t s_col = lanes + (i & 1) * kKeys;
        ok = warp_wait(s_done + 8 * (i & 1), (i >> 1) & 1, a.pages.status, a.wait_limit, dead);
        if (!ok) break;
        tc_fence_after();
        uint32_t s[kHalf];
        tmem_ld(s_col + half * kHalf, s);
        const int seen = sees - (t0 + i) * kKeys - half * kHalf;  // of the half's slots
        if (__any_sync(kFull, seen < kHalf)) {
#pragma unroll
          for (int j = 0; j < kHalf; ++j)
            if (j >= seen) s[j] = 0xff800000u;
        }
        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < kHalf; j += 2)
          m4[(j >> 1) & 3] =
              max3(m4[(j >> 1) & 3], __uint_as_float(s[j]), __uint_as_float(s[j + 1]));
        float m = __fmul_rn(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), factor);
        // where weights lie over S: both halves have read their scores before either writes some
        if (Sh::kAlias || !E4M3) tc_fence_before();
        ok = exchange(m, i + 1);
        if (!ok) break;
        if (Sh::kAlias || !E4M3) tc_fence_after();
        bool added = i == 0;  // the tile before is in O, and P is free
        auto wait_added = [&] {
          if (!added)
            added = warp_wait(o_done + 8 * ((i - 1) % 3), ((i - 1) / 3) & 1, a.pages.status,
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
          if (i > 0) {
            ok = wait_added();
            if (!ok) break;
            constexpr int kStep = M == 4 ? 16 : 8;
#pragma unroll 1
            for (int j = 0; j < kD / 2; j += kStep) {
              uint32_t o[kStep];
              const uint32_t at = lanes + Sh::kColO + half * (kD / 2) + j;
              tmem_ld(at, o);
#pragma unroll
              for (int e = 0; e < kStep; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              if (kStep == 16)
                tmem_st16(at, o);
              else
                tmem_st8(at, o);
            }
          }
        }
        // Scores are rounded before the maximum is taken off them, like the maximum itself.  bf16
        // weights go in two parts, as one would be off by as much as the result's own rounding
        // where a token sees few slots: the low ones take S's upper half.
        const float shift = row_max == -INFINITY ? 0.f : -row_max;
        auto p_col = [&] { return (Sh::kAlias ? s_col : lanes + Sh::kColP) + half * (kHalf / 2); };
        // Weights are written as they come where registers are short: then P has to be free before
        constexpr bool kEarly = !E4M3 && M <= 3;
        if (kEarly) {
          ok = wait_added();
          if (!ok) break;
        }
        unsigned long long sum2 = 0;
#pragma unroll
        for (int j0 = 0; j0 < kHalf; j0 += 16) {
          uint32_t low[8];
#pragma unroll
          for (int j = j0; j < j0 + 16; j += 2) {
            float lo, hi;
            f2_unpack(f2_add(f2_mul(f2_pack(__uint_as_float(s[j]), __uint_as_float(s[j + 1])),
                                    f2_pack(factor, factor)),
                             f2_pack(shift, shift)),
                      lo, hi);
            lo = exp2_approx(lo);
            hi = exp2_approx(hi);
            sum2 = f2_add(sum2, f2_pack(lo, hi));
            s[j / 2] = E4M3 ? pack_f16(lo, hi) : split_weights(lo, hi, low[(j - j0) / 2]);
          }
          if (!E4M3) tmem_st8(s_col + kKeys / 2 + half * (kHalf / 2) + j0 / 2, low);
          if (kEarly) tmem_st8(p_col() + j0 / 2, s + j0 / 2);
        }
        if (!Sh::kAlias && !kEarly) ok = wait_added();
        if (!ok) break;
        if (!kEarly) {
          tmem_st16(p_col(), s);
          if (kHalf >= 64) tmem_st16(p_col() + 16, s + 16);
        }
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(p_full + 8 * (i & 1));
        row_sum += f2_hsum(sum2);
      }
      if (warp_wait(o_done + 8 * ((count - 1) % 3), ((count - 1) / 3) & 1, a.pages.status,
                    a.wait_limit, dead))
        tc_fence_after();
    }
  } else if (warp < kProductWarp) {
    // K's warps or V's: their slices of the tiles, as the buffers become free
    const int lane = threadIdx.x & 31, which = warp - kSoftWarps;
    const int part = which >= kKeyWarps;  // 0: K, 1: V
    const int bufs = part ? kValueBufs : kKeyBufs;
    const Slice<kKeys> slice(part ? which - kKeyWarps : which, part ? kValueWarps : kKeyWarps);
    const char* pool = (part ? a.pages.v : a.pages.k) + head * a.pages.head_stride;
    const int32_t* table = a.pages.table + (size_t)seq * a.pages.max_pages;
    constexpr uint32_t kNoRow = 0xffffffffu;
    // Rows of a tile's slots, in 16 bytes: of slot `lane` of the slice, and of slot 32 + lane
    struct Rows {
      int page[2];
      uint32_t in[2];  // of the page
    };
    auto lookup = [&](int i, Rows& r) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int key = 32 * u + lane, slot = (t0 + i) * kKeys + slice.first + key;
        const int place = a.pages.place_of(slot);
        r.page[u] = -2;
        r.in[u] = (uint32_t)(slot - place * a.pages.page_size) * a.slot16;
        if (i < count && key < slice.count && slot < keys) r.page[u] = __ldcg(table + place);
      }
    };
    auto row_of = [&](const Rows& r, int u) {
      if (r.page[u] == -2) return kNoRow;
      if ((unsigned)r.page[u] >= (unsigned)a.pages.n_page) {
        record_status(a.pages.status, kStDevicePage);
        return kNoRow;
      }
      return (uint32_t)r.page[u] * a.page16 + r.in[u];
    };
    // whether values of tile i have to be looked at: some rows do not see all of it
    auto hides = [&](int i) { return part && (t0 + i + 1) * kKeys > all_see; };
    auto done = [&](int i) {
      fence_proxy_async_smem();
      warp_arrive(full + 8 * ((i + part) & 3));
      if (!part && i == count - 1) warp_arrive(full + 8 * (count & 3));  // there is none
    };
    auto buffer = [&](int i) {
      return base + (part ? kKeyBufs + i % kValueBufs : i % kKeyBufs) * Sh::kTileBytes;
    };
    auto await_buffer = [&](int i) {
      return i < bufs || warp_wait((part ? o_done : s_done) + 8 * (i % bufs), (i / bufs + 1) & 1,
                                   a.pages.status, a.wait_limit, dead);
    };
    if (part && count > 0) warp_arrive(full);  // of the tile before the first
    Rows next;
    lookup(0, next);
    if (!E4M3) {
      const int chunks = a.d / 8;  // real ones
      auto land = [&](int i) {
        if (hides(i)) {  // what is not finite is added at the end, to the rows that see it
#pragma unroll 1
          for (int j = lane; j < slice.count * (kD / 8); j += 32) {
            const uint32_t at = tile_at<M>(buffer(i), slice.first + j / (kD / 8), j % (kD / 8));
            const uint4 x = ld_shared16(at);
            uint32_t w[4] = {x.x, x.y, x.z, x.w};
            bool found = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u, found = true;
              if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0xffffu, found = true;
            }
            if (found) {
              st_shared16(at, make_uint4(w[0], w[1], w[2], w[3]));
              *odd = 1;
            }
          }
        }
        done(i);
      };
      bool ok = true;
      int i = 0;
      for (; i < count; ++i) {
        const Rows now = next;
        lookup(i + 1, next);
        ok = await_buffer(i);
        if (!ok) break;
        constexpr int kRowChunks = kD / 8;
        const uint32_t dst = buffer(i);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (32 * u >= slice.count) break;
          const uint32_t mine = row_of(now, u);
          const int here = min(32, slice.count - 32 * u);  // slots, a multiple of 8
          constexpr bool kFixed = 32 % kRowChunks == 0;    // a lane has the same chunk of every row
          if (kFixed && chunks == kRowChunks &&
              __all_sync(kFull, mine != kNoRow || lane >= here)) {
            constexpr int kStep = 32 / kRowChunks, kBatch = 8 / kStep;  // rows, and copies of 8 rows
            const int chunk = lane % kRowChunks, key = lane / kRowChunks;
            const char* from = pool + chunk * 16;
            uint32_t to = tile_at<M>(dst, slice.first + 32 * u + key, chunk);
#pragma unroll 1
            for (int k0 = 0; k0 < here; k0 += 8, to += 8 * 128) {
              uint32_t row[kBatch];
#pragma unroll
              for (int j = 0; j < kBatch; ++j) row[j] = __shfl_sync(kFull, mine, k0 + kStep * j + key);
#pragma unroll
              for (int j = 0; j < kBatch; ++j)
                cp_async16((to ^ (kStep * j << 4)) + kStep * j * 128, from + (size_t)row[j] * 16);
            }
          } else {
#pragma unroll 1
            for (int j = lane; j < here * kRowChunks; j += 32) {
              const int key = j / kRowChunks, chunk = j % kRowChunks;
              const uint32_t row = __shfl_sync(kFull, mine, key);
              const bool real = row != kNoRow && chunk < chunks;
              cp_async16_or_zero(tile_at<M>(dst, slice.first + 32 * u + key, chunk),
                                 pool + (size_t)(real ? row + chunk : 0u) * 16, real);
            }
          }
        }
        cp_async_commit();
        if (i > 0) {
          cp_async_wait<1>();
          __syncwarp();  // a lane looks at what others copied
          land(i - 1);
        }
      }
      cp_async_wait<0>();
      __syncwarp();
      if (ok && count > 0) land(count - 1);
    } else {
      // 16 bytes of a row become two chunks of fp16
      constexpr int kUnits = ((kKeys / 8 + kValueWarps - 1) / kValueWarps * 8 * 2 * M + 31) / 32;
      const int chunks = a.d / 16;
      uint4 x[kUnits];
      auto load = [&](const Rows& r) {
        const uint32_t first = row_of(r, 0), second = row_of(r, 1);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          const int j = lane + 32 * u, key = j / (2 * M), chunk = j % (2 * M);
          const uint32_t r0 = __shfl_sync(kFull, first, key & 31),
                         r1 = __shfl_sync(kFull, second, key & 31), row = key < 32 ? r0 : r1;
          x[u] = make_uint4(0, 0, 0, 0);
          if (key < slice.count && row != kNoRow && chunk < chunks)
            x[u] = ld_cg16(pool + (size_t)(row + chunk) * 16);
        }
      };
      if (count > 0) {
        const Rows now = next;
        lookup(1, next);
        load(now);
      }
      for (int i = 0; i < count; ++i) {
        if (!await_buffer(i)) break;
        const uint32_t dst = buffer(i);
        const bool look = hides(i);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          const int j = lane + 32 * u, key = j / (2 * M), chunk = j % (2 * M);
          if (key >= slice.count) break;
          uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
          if (look) {
            bool found = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t nan = __vcmpeq4(w[e] & 0x7f7f7f7fu, 0x7f7f7f7fu);
              w[e] &= ~nan;
              found |= nan != 0;
            }
            if (found) *odd = 1;
          }
#pragma unroll
          for (int e = 0; e < 2; ++e)
            st_shared16(tile_at<M>(dst, slice.first + key, 2 * chunk + e),
                        make_uint4(e4m3_to_h2(w[2 * e], false), e4m3_to_h2(w[2 * e], true),
                                   e4m3_to_h2(w[2 * e + 1], false), e4m3_to_h2(w[2 * e + 1], true)));
        }
        done(i);
        if (i + 1 < count) {
          const Rows now = next;
          lookup(i + 2, next);
          load(now);
        }
      }
    }
    __syncwarp();
  } else {
    if ((threadIdx.x & 31) == 0 && count > 0) {
      constexpr uint32_t kLead = kKeys * 128;
      constexpr uint32_t kScoreDesc = tc_desc(!E4M3, false, kKeys), kValueDesc = tc_desc(!E4M3, true, kD);
      bool ok = true;
      auto await = [&](uint32_t bar, uint32_t parity) {
        if (!tile_wait(bar, parity, a.pages.status, a.wait_limit, dead)) ok = false;
      };
      auto scores = [&](int i) {
        const uint64_t kt = tc_smem(base + (i % kKeyBufs) * Sh::kTileBytes, kLead);
        const uint32_t s_col = tm + (i & 1) * kKeys;
#pragma unroll
        for (int k = 0; k < kD / 16; ++k)
          tc_mma(s_col, tm + Sh::kColQ + 8 * k, kt + (((k >> 2) * kLead + (k & 3) * 32) >> 4),
                 kScoreDesc, k > 0);
        tc_commit(s_done + 8 * (i & 1));
      };
      auto values = [&](int i) {
        const uint64_t vt = tc_smem(base + (kKeyBufs + i % kValueBufs) * Sh::kTileBytes, kLead);
        const uint32_t p_col = tm + (Sh::kAlias ? (i & 1) * kKeys : Sh::kColP);
        const uint32_t low_col = tm + (i & 1) * kKeys + kKeys / 2;
#pragma unroll
        for (int k = 0; k < kKeys / 16; ++k)
          tc_mma(tm + Sh::kColO, p_col + 8 * k, vt + ((2048 * k) >> 4), kValueDesc, i > 0 || k > 0);
        if (!E4M3) {
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k)
            tc_mma(tm + Sh::kColO, low_col + 8 * k, vt + ((2048 * k) >> 4), kValueDesc, true);
        }
        tc_commit(o_done + 8 * (i % 3));
      };
      await(q_full, 0);
#pragma unroll 1
      for (int i = -1; i < count; ++i) {
        await(full + 8 * ((i + 1) & 3), ((i + 1) >> 2) & 1);  // K of tile i + 1, V of tile i
        // S of tile i + 1 takes the place of the weights of tile i - 1, or of their low parts
        if (i > 0 && (Sh::kAlias || !E4M3)) await(o_done + 8 * ((i - 1) % 3), ((i - 1) / 3) & 1);
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
      mbar_wait(drain, 0, a.pages.status, kWaitLimit);
    }
    __syncwarp();
  }
  __syncthreads();

  const int2 size2 = make_int2(kept[0], kept[1]);
  const BlockPlace<kKeys> place(a, tile, rank, size2);
  const int rows_all = place.rows_all, row0 = place.row0, row = row0 + lane_row;
  const int token = min(row, max(rows_all, 1) - 1) / a.group;
  float* stat = reinterpret_cast<float*>(smem + Sh::kStats);  // [max, sum, sum][row]
  if (warp < kSoftWarps) {
    if (half == 0) stat[lane_row] = row_max;
    stat[(1 + half) * kTileRows + lane_row] = row_sum;
  }
  __syncthreads();
  const float vs = E4M3 && a.pages.v_scale ? __ldcg(a.pages.v_scale + head) : 1.f;
  // A row without a weight above 0 has a sum of 0
  auto inverse = [&](float sum) { return sum == 0.f ? 0.f : vs / sum; };
  auto log_sum = [&](float m, float sum) {
    return sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
  };
  if (warp < kSoftWarps) {
    const bool valid = row < rows_all;
    const size_t at = (((size_t)seq * a.B + token) * a.heads + head) * a.group + row % a.group;
    row_sum = stat[kTileRows + lane_row] + stat[2 * kTileRows + lane_row];
    const float inv = inverse(row_sum);
    if (a.cluster == 1 && valid && a.lse && half == 0) a.lse[at] = log_sum(row_max, row_sum);
#pragma unroll 1
    for (int j = half * (kD / 2); j < (half + 1) * (kD / 2); j += 16) {
      uint32_t o[16];
      if (place.count > 0) {
        tmem_ld(lanes + Sh::kColO + j, o);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = 0;
      }
      if (*odd && j < a.d) {  // the values that were left out, of tiles that some rows do not see
        const int sees = size2.x + (a.causal ? token + 1 : 0);
        const int k0 = max(place.t0, place.all_see / kKeys) * kKeys;
        for (int key = k0; key < min((place.t0 + place.count) * kKeys, sees); ++key) {
          const int page =
              __ldcg(a.pages.table + (size_t)seq * a.pages.max_pages + a.pages.place_of(key));
          if ((unsigned)page >= (unsigned)a.pages.n_page) continue;
          const char* v = a.pages.v + head * a.pages.head_stride + a.pages.row(page, key) +
                          j * (E4M3 ? 1 : 2);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if (j + e >= a.d) break;
            if (E4M3) {
              const uint8_t x = __ldcg(reinterpret_cast<const uint8_t*>(v) + e);
              if ((x & 0x7fu) == 0x7fu) o[e] = 0x7fffffffu;
            } else {
              const uint16_t x = __ldcg(reinterpret_cast<const uint16_t*>(v) + e);
              if ((x & 0x7f80u) == 0x7f80u)
                o[e] = __float_as_uint(__uint_as_float(o[e]) + __uint_as_float((uint32_t)x << 16));
            }
          }
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
            if (j + e < a.d) st16(a.out + at * a.d + j + e, make_uint4(w[0], w[1], w[2], w[3]));
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
  const int rows = max(0, min(kTileRows, rows_all - row0));
  const int share = (rows + a.cluster - 1) / a.cluster;
  const int r0 = rank * share, mine = max(0, min(share, rows - r0));
  const uint32_t stats = base + Sh::kStats;
  // [cluster][share], at most 128 + 15, maxima first, and the same of sums (kSwap follows kFactors)
  float* factor = reinterpret_cast<float*>(smem + Sh::kFactors);
  float* sums = reinterpret_cast<float*>(smem + Sh::kSwap) + 16;
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
      // a CTA without slots has sums of zero; one whose scores were all NaN has NaN sums
      const float f = mq == -INFINITY ? 1.f : exp2_approx(mq - m);
      l = fmaf(sums[q * share + r], f, l);
      factor[q * share + r] = f;
    }
    sums[r] = inverse(l);  // the first CTA's, which this thread alone has read
    if (a.lse)
      a.lse[(((size_t)seq * a.B + gr / a.group) * a.heads + head) * a.group + gr % a.group] =
          log_sum(m, l);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < mine * (a.d / 4); i += kTileThreads) {
    const int dim4 = i / mine, r = i - dim4 * mine;  // neighbouring threads read neighbouring rows
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
    *reinterpret_cast<uint2*>(a.out + at * a.d + 4 * dim4) =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  }
  // no CTA leaves while its results are read
  cluster_arrive_relaxed();
  cluster_wait();
}

template <int M, bool E4M3>
constexpr PagedKernel paged_tile() {
  return {paged_tile_kernel<M, E4M3>, TileShape<M>::kTotal, kTileRows, kTileThreads,
          TileShape<M>::kKeys};
}

}  // namespace vd
