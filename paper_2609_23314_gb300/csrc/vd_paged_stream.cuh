// vd_paged_stream.cuh -- attention over one layer of a paged cache (vd_paged_attend in
// include/vd.h): the streaming kernel, for few query rows per KV head.
//
//   s_ij = scale * q_i . k_j,  o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i)
//
// in one pass over the slots with a running maximum and sum.  A CTA takes its piece of the line
// (vd_paged_attend.cuh), a share of a unit at a time, in stages of 16 or 32 slots that go around a
// ring in shared memory.  Four warps copy: each looks up the pages of its stages, four of them
// ahead, and issues single asynchronous copies of 16 bytes, so that pages may be of any size and
// stride; one of the four also finds the shares.  The other warps compute, a stage each in turn
// with a running state of its own, meet in shared memory at the end of a share, and wait for
// nothing but their stages there: a warp that is done goes on to the next share.
//
// Per 16 slots a warp computes  S^T = K Q^T  and  O^T += V^T P^T  with slots and head dims on the
// 16-row side of m16n8k16, so that 8 query rows fill a tile.  bf16 pages are multiplied as
// they are, weights in two bf16 parts (1.06 * 2^-16 of a weight); e4m3 ones go to fp16 (exact), Q too
// with each row scaled by a power of two (QueryScale), weights are rounded to fp16.  Sums are
// fp32.
//
// Long batches are bound by DRAM: 512 KV heads around 4096 slots 131 us (6.2 TB/s, 92 % of the copy
// peak), 16 heads of 131000 slots 166 (95 %); in e4m3, where a slot's arithmetic takes 300 cycles of an
// SM for the 350 of its bytes, 77 to 86 from one machine to another (4.8 to 5.3 TB/s).  Small calls by a chain of latencies (length, page,
// slots, meeting, join): 8 heads of 4096 slots 11.7 us.  Copies in the computing warps took 40 % of
// their time (93 us for 84), boxes of tensor maps 119.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "vd_attend.cuh"
#include "vd_device.cuh"
#include "vd_paged.cuh"
#include "vd_paged_attend.cuh"

namespace vd {

// 16 bytes to shared memory, or zeros.
__device__ __forceinline__ void cp_async16_or_zero(uint32_t smem, const void* p, bool real) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(p),
               "r"(real ? 16 : 0)
               : "memory");
}

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

// c += a b, 16 x 8 x 16; not volatile, so that products and loads are free to overlap.
template <bool BF16>
__device__ __forceinline__ void product16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                          uint32_t b1) {
  if (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

__device__ __forceinline__ void prefetch_l2(const void* p) {
  asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}

// Arrives on the barrier once this thread's copies so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ bool bar_done(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; "
      "selp.u32 %0, 1, 0, p; }"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}

// Waits for a phase; gives up after `limit` polls, and once another warp has.  By a whole warp, whose
// lanes get the same answer: what follows a wait are products, shuffles and barriers of all of them, and
// a lane that has seen the phase end beside one that has run out of polls would wait there for ever.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* dead,
                                         const PagedAttendArgs& a) {
  bool done = bar_done(bar, parity);
  if (__all_sync(kFull, done)) return true;
#pragma unroll 1
  for (uint32_t i = 0; i < a.wait_limit; ++i) {
    if (!done) done = bar_done(bar, parity);
    if (__all_sync(kFull, done)) return true;
    if (__any_sync(kFull, *dead)) break;
  }
  *dead = 1;
  record_status(a.pages.status, kStTimeout);
  return false;
}

constexpr int kShares = 4;     // shares in shared memory: the copies run ahead

template <int NB>
struct StreamMem {
  uint64_t full[NB], empty[NB];      // the ring's places
  uint64_t share_full[kShares], share_free[kShares];
  uint64_t parts_full, parts_free;   // partial rows
  Share share[kShares];
  WalkMem walk;
  int dead;  // a wait has run out
};

template <int M, int NT, bool E4M3>
struct StreamShape {
  static constexpr int kD = 32 * M;  // head_dim, rounded up
  static constexpr int kRows = 8 * NT;
  static constexpr int kRowBytes = kD * (E4M3 ? 1 : 2);
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kGroups = (E4M3 && M <= 4) || M <= 2 ? 2 : 1;  // of 16 slots, in a stage
  static constexpr int kKeys = 16 * kGroups;
  static constexpr int kTileBytes = kKeys * kRowBytes;  // of K or V
  static constexpr int kStageBytes = 2 * kTileBytes;
  // Warps that compute and that copy: 12, of 168 registers each, or 8 where the sums take more
  static constexpr bool kWide = M > 4 || M * NT > 6;
  static constexpr int kWarpsUsed = !kWide ? 8 : M == 4 ? 6 : 4;
  static constexpr int kProducers = kWide && M == 4 ? 2 : 4;
  static constexpr int kStreamThreads = 32 * (kWarpsUsed + kProducers);
  static constexpr int kMost = 192 * 1024 / kStageBytes;
  static constexpr int kPlaces = (kMost > 32 ? 32 : kMost) / kWarpsUsed * kWarpsUsed;  // of the ring
  static constexpr int kRing = kPlaces * kStageBytes;
  static constexpr int kPart = kD + 4;  // floats of a partial row
  static constexpr int kParts = kRing;  // [warp][8 rows]
  static constexpr int kStats = kParts + kWarpsUsed * 8 * kPart * 4;  // [warp][8 rows] max, sum
  static constexpr int kMem = kStats + kWarpsUsed * 8 * 8;
  static constexpr int kTotal = kMem + (int)sizeof(StreamMem<kPlaces>);
  static_assert(kTotal <= 232448, "shared memory");
  static_assert(2 * kTotal > 228 * 1024, "one CTA on an SM, as the workspace has it");
  static_assert(kPlaces % kProducers == 0, "a place has one producer and one consumer");
};

// Chunk c (16 bytes) of a row lies at c ^ turn(row), so that the same chunk of 8 rows falls on
// different banks.
template <int kChunks>
struct Swizzle {
  static constexpr int kMask = kChunks % 8 == 0 ? 7 : kChunks % 4 == 0 ? 3 : 1;
  static __device__ __forceinline__ int turn(int row) {
    return (kMask == 7 ? row : kMask == 3 ? row >> 1 : row >> 2) & kMask;
  }
  // From the address of chunk 0 or 1 of a row to the chunk `even` further.
  static __device__ __forceinline__ uint32_t step(uint32_t addr, int even) {
    return (addr ^ ((even & kMask) << 4)) + ((even & ~kMask) << 4);
  }
};

// The running maximum less this is the point that weights are relative to: fp16 weights far below the
// largest keep their bits.  The point moves with every rise of the maximum that one of the warp's rows
// sees (there is no slack before it does).
template <bool E4M3>
constexpr float kPagedLift = E4M3 ? 15.f : 8.f;

// Whether one of a word's values is not finite.
template <bool E4M3>
__device__ __forceinline__ bool not_finite(uint32_t w) {
  if (E4M3) return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

// Two weights in bf16, and in `low` what that leaves of them: together within 1.06 * 2^-16 of a weight
// (half a step of the lower part, and 2^-20).
// The upper part is rounded towards zero and the lower one is of 2^-20 of the weight more, so that
// both are above 0 where the weight is (but for weights below 2^-113): an infinite value stays one.
__device__ __forceinline__ uint32_t split_weights(float x, float y, uint32_t& low) {
  uint32_t minus;
  asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(minus) : "f"(-y), "f"(-x));
  low = pack_bf16(fmaf(x, 1.f + 0x1p-20f, __uint_as_float(minus << 16)),
                  fmaf(y, 1.f + 0x1p-20f, __uint_as_float(minus & 0xffff0000u)));
  return minus ^ 0x80008000u;
}

template <int M, int NT, bool E4M3>
__global__ void __launch_bounds__((StreamShape<M, NT, E4M3>::kStreamThreads), 1)
    paged_stream_kernel(const __grid_constant__ PagedAttendArgs a) {
  using Sh = StreamShape<M, NT, E4M3>;
  using Sw = Swizzle<Sh::kChunks>;
  constexpr int kW = Sh::kWarpsUsed, kN = Sh::kPlaces, kG = Sh::kGroups;
  constexpr int kProducers = Sh::kProducers;
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t base = smem_addr(smem);
  auto& mem = *reinterpret_cast<StreamMem<kN>*>(smem + Sh::kMem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunks = a.d * (E4M3 ? 1 : 2) / 16;  // of a row in the pages
  if (threadIdx.x < kN) {
    mbar_init(smem_addr(&mem.full[threadIdx.x]), 32);
    mbar_init(smem_addr(&mem.empty[threadIdx.x]), 1);
  } else if (threadIdx.x < kN + kShares) {
    mbar_init(smem_addr(&mem.share_full[threadIdx.x - kN]), 1);
    mbar_init(smem_addr(&mem.share_free[threadIdx.x - kN]), kW + kProducers - 1);
  } else if (threadIdx.x == kN + kShares) {
    mbar_init(smem_addr(&mem.parts_full), kW);
    mbar_init(smem_addr(&mem.parts_free), kW);
    mem.dead = 0;
    mem.share[0].seq = -1;
  }
  fence_mbar_init();
  // what copies do not write: the chunks behind head_dim
  if (chunks < Sh::kChunks)
    for (int i = threadIdx.x; i < Sh::kRing / 16; i += Sh::kStreamThreads)
      st_shared16(base + 16 * i, make_uint4(0, 0, 0, 0));
  grid_dependency_wait();
  grid_launch_dependents();
  if (a.cluster > 1) {
    // queries and the table, which a wait for the length need not delay, into L2
    const int unit = blockIdx.x / a.cluster, head = unit / a.tiles, seq = head / a.heads;
    const int line = threadIdx.x - 32, row = (unit - head * a.tiles) * Sh::kRows + (lane & (Sh::kRows - 1));
    if (warp == 0 && row < a.B * a.group) {
      const int tok = row / a.group;
      const uint16_t* q = a.q + ((((size_t)seq * a.B + tok) * a.heads + head - seq * a.heads) * a.group +
                                 row - tok * a.group) * a.d;
      prefetch_l2(q + (lane >= Sh::kRows ? a.d / 2 : 0));
    } else if (line >= 0 && 32 * line < a.pages.max_pages) {
      prefetch_l2(a.pages.table + (size_t)seq * a.pages.max_pages + 32 * line);
    }
  }
  long long all = 0;
  if (a.cluster == 1 && a.n_seq > kFewSeqs) all = Walk::survey(a, mem.walk);
  __syncthreads();
  bool ok = true;

  if (warp >= kW) {
    // ------------------------------------------------------------------ copies
    const int p = warp - kW;
    Walk walk;
    if (p == 0 && a.cluster == 1) {
      walk = Walk(a, mem.walk, all);
      if (lane == 0) a.split[blockIdx.x] = make_int4(-1, 0, 0, 0);
    }
    int next = p;         // this warp's next stage, from the share's first one
    int place = p;        // of the ring
    uint32_t round = 0;   // how often the ring has gone around
    constexpr bool kFixed = 32 % Sh::kChunks == 0;  // a lane has the same chunk of every row
    for (int k = 0; ok; ++k) {
      Share& s = mem.share[k % kShares];
      const uint32_t turn = (uint32_t)(k / kShares);
      if (p == 0) {
        if (turn > 0) ok = bar_wait(smem_addr(&mem.share_free[k % kShares]), (turn - 1) & 1, &mem.dead, a);
        if (lane == 0) {
          const bool more = a.cluster > 1 ? k == 0 && cluster_share(a, s) : walk.next(a, mem.walk, s);
          if (!more) s.seq = -1;
          else if (s.slot >= 0 && s.s0 == 0) a.split[blockIdx.x] = walk.split_of(a, s);
          bar_arrive(smem_addr(&mem.share_full[k % kShares]));
        }
        __syncwarp();
      }
      ok = ok && bar_wait(smem_addr(&mem.share_full[k % kShares]), turn & 1, &mem.dead, a);
      if (!ok || s.seq < 0) break;
      const int s0 = s.s0, count = s.s1 - s.s0, total = seen_slots(a, s);
      const int32_t* table = a.pages.table + (size_t)s.seq * a.pages.max_pages;
      const long long in = s.head * a.pages.head_stride + (kFixed ? lane % Sh::kChunks * 16 : 0);
      const char *k_head = a.pages.k + in, *v_head = a.pages.v + in;
      if (p == 1 && lane < 2 * Sh::kRows) {  // its queries, which the other warps will want, into L2
        const long long row = out_row(a, s, lane & (Sh::kRows - 1));
        if (row >= 0) prefetch_l2(a.q + row * a.d + (lane < Sh::kRows ? 0 : a.d / 2));
      }
      if (p > 0) {
        __syncwarp();
        if (lane == 0) bar_arrive(smem_addr(&mem.share_free[k % kShares]));
      }
      // Pages of the lane's slots: kNone behind the last slot
      constexpr int kAhead = 4, kNone = -2;
      auto lookup = [&](int i) {
        const int slot = (s0 + i) * Sh::kKeys + (lane & (Sh::kKeys - 1));
        return i < count && slot < total ? __ldcg(table + a.pages.place_of(slot)) : kNone;
      };
      int page[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) page[u] = lookup(next + u * kProducers);
      while (ok && next < count) {
        int later[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) later[u] = lookup(next + (kAhead + u) * kProducers);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          if (next >= count || !ok) break;
          if (round > 0) {
            ok = bar_wait(smem_addr(&mem.empty[place]), (round - 1) & 1, &mem.dead, a);
            if (!ok) break;
          }
          bool real = page[u] != kNone;
          if (real && (unsigned)page[u] >= (unsigned)a.pages.n_page) {
            record_status(a.pages.status, kStDevicePage);
            real = false;
          }
          // where the lane's row lies, in 16 bytes
          const int slot = (s0 + next) * Sh::kKeys + (lane & (Sh::kKeys - 1));
          const uint32_t mine = (uint32_t)page[u] * a.page16 +
                                (uint32_t)(slot - a.pages.place_of(slot) * a.pages.page_size) * a.slot16;
          const uint32_t dst = base + place * Sh::kStageBytes;
          if (chunks == Sh::kChunks && __all_sync(kFull, real)) {
            constexpr int kCopies = Sh::kKeys * Sh::kChunks / 32;  // of K, and of V
            uint32_t row[kCopies];
#pragma unroll
            for (int i = 0; i < kCopies; ++i)
              row[i] = __shfl_sync(kFull, mine, (32 * i + lane) / Sh::kChunks);
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
              const int t = (32 * i + lane) / Sh::kChunks, ch = (32 * i + lane) % Sh::kChunks;
              const uint32_t to = dst + t * Sh::kRowBytes + ((ch ^ Sw::turn(t)) << 4);
              const size_t from = (size_t)(row[i] + (kFixed ? 0 : ch)) * 16;
              cp_async16(to, k_head + from);
              cp_async16(to + Sh::kTileBytes, v_head + from);
            }
          } else {
            // whole rows: a warp takes 32 / chunks of them at a time
            const int rows = 32 / chunks, t0 = lane / chunks, ch = lane - t0 * chunks;
            const int skip = kFixed ? ch - lane % Sh::kChunks : ch;
            const unsigned reals = __ballot_sync(kFull, real);
            for (int t = t0; t - t0 < Sh::kKeys; t += rows) {
              const uint32_t row = __shfl_sync(kFull, mine, t & (Sh::kKeys - 1));
              if (t0 < rows && t < Sh::kKeys) {
                const bool there = reals >> t & 1;
                const uint32_t to = dst + t * Sh::kRowBytes + ((ch ^ Sw::turn(t)) << 4);
                const long long from = there ? ((long long)row + skip) * 16 : 0;
                cp_async16_or_zero(to, k_head + from, there);
                cp_async16_or_zero(to + Sh::kTileBytes, v_head + from, there);
              }
            }
          }
          cp_async_arrive(smem_addr(&mem.full[place]));
          next += kProducers;
          place += kProducers;
          if (place >= kN) {
            place -= kN;
            ++round;
          }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) page[u] = later[u];
      }
      next -= count;
    }
    cp_async_commit();
    cp_async_wait<0>();
  } else {
    // ------------------------------------------------------------------ products
    float* parts = reinterpret_cast<float*>(smem + Sh::kParts);
    float2* stats = reinterpret_cast<float2*>(smem + Sh::kStats);
    const int r = lane >> 2, c = lane & 3;
    // Q: lane (r, c) holds row r of each n-tile
    uint32_t qf[NT][2 * M][2];
    auto load_queries = [&](const Share& s) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const long long row = out_row(a, s, 8 * t + r);
        const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q + (row < 0 ? 0 : row) * a.d);
#pragma unroll
        for (int j = 0; j < 2 * M; ++j) {
          // e4m3: chunk j's dims 4 c .. 4 c + 3; bf16: chunks 2 j and 2 j + 1, dims 2 c, 2 c + 1
          const int d0 = 16 * j + (E4M3 ? 4 : 2) * c, d1 = E4M3 ? d0 + 2 : d0 + 8;
          qf[t][j][0] = row >= 0 && d0 < a.d ? __ldcg(src + d0 / 2) : 0u;
          qf[t][j][1] = row >= 0 && d1 < a.d ? __ldcg(src + d1 / 2) : 0u;
        }
      }
    };
    auto share_known = [&](int k) {
      ok = ok && bar_wait(smem_addr(&mem.share_full[k % kShares]), k / kShares & 1, &mem.dead, a);
      return ok && mem.share[k % kShares].seq >= 0;
    };
  // Where a lane's row of the four 8 x 8 blocks of a matrix load lies in a tile: blocks of K are
  // slots 0-7, 8-15 of a chunk, then of the next one; of V in bf16, chunks go first
  const int slots8 = lane & 7, b3 = (lane >> 3) & 1, b4 = lane >> 4;
  const int k_slot = slots8 + 8 * b3, v_slot = slots8 + 8 * (E4M3 ? b3 : b4);
  const uint32_t k_lane = k_slot * Sh::kRowBytes + ((b4 ^ Sw::turn(k_slot)) << 4);
  const uint32_t v_lane = v_slot * Sh::kRowBytes + (((E4M3 ? b4 : b3) ^ Sw::turn(v_slot)) << 4);
  int next = warp;     // this warp's next stage, from the share's first one
  int place = warp;    // of the ring
  uint32_t phase = 0;  // of its barriers
  uint32_t met = 0;    // times that the warps have met
  bool more = share_known(0);
  if (more) load_queries(mem.share[0]);
  for (int k = 0; more; ++k) {
    const Share& s = mem.share[k % kShares];
    const int s0 = s.s0, count = s.s1 - s.s0, len = s.len;
    int sees[NT][2];  // slots that columns 2 c and 2 c + 1 see
    float qs[NT][2];  // what their scores are multiplied by for log2 units
    // some token does not see a slot that others see (what lies behind them all reads as zero)
    const bool unseen = a.causal && (s.tile * Sh::kRows) / a.group + 1 < s.add;
    const int all_see = a.causal ? len + (s.tile * Sh::kRows) / a.group + 1 : len;
    const float ks = E4M3 && a.pages.k_scale ? __ldcg(a.pages.k_scale + s.head) : 1.f;
    const float vs = E4M3 && a.pages.v_scale ? __ldcg(a.pages.v_scale + s.head) : 1.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        sees[t][e] = a.causal
                         ? len + (s.tile * Sh::kRows + 8 * t + 2 * c + e) / a.group + 1
                         : len;
      if (!E4M3) {
        qs[t][0] = qs[t][1] = a.scale * kLog2e;
      } else {
        uint32_t top = 0;  // largest magnitude of the row, as bits
#pragma unroll
        for (int j = 0; j < 2 * M; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t x = qf[t][j][e];
            top = max(top, max(x & 0x7fffu, (x >> 16) & 0x7fffu));
          }
        top = max(top, __shfl_xor_sync(kFull, top, 1));
        top = max(top, __shfl_xor_sync(kFull, top, 2));
        const QueryScale f = scale_of(top);
#pragma unroll
        for (int j = 0; j < 2 * M; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t x = qf[t][j][e];
            asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(x) : "r"(f.up));
            qf[t][j][e] = pack_f16(__uint_as_float(x << 16) * kTo16,
                                   __uint_as_float(x & 0xffff0000u) * kTo16);
          }
        const float factor = score_factor(f.down, a.scale * ks) * kFrom16;
        qs[t][0] = __shfl_sync(kFull, factor, 8 * c);
        qs[t][1] = __shfl_sync(kFull, factor, 8 * c + 4);
      }
    }
    float o[NT][2 * M][4];
    float mx[NT][2], sum[NT][2];  // references and sums of columns 2 c and 2 c + 1
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      mx[t][0] = mx[t][1] = -INFINITY;
      sum[t][0] = sum[t][1] = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * M; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][i][e] = 0.f;
    }

    const bool idle = next >= count;
    for (; next < count; next += kW) {
      ok = ok && bar_wait(smem_addr(&mem.full[place]), phase, &mem.dead, a);
      if (!ok) break;
      const uint32_t tile_k = base + place * Sh::kStageBytes, tile_v = tile_k + Sh::kTileBytes;
      const int key0 = (s0 + next) * Sh::kKeys;
      // Matrix loads go kBatch at a time ahead of their products; a query tile alone has two chains
      // of sums, so that products wait less for one another
      constexpr int kLoads = E4M3 ? M : 2 * M, kBatch = kLoads % 4 == 0 ? 4 : kLoads % 3 == 0 ? 3 : 2;
      constexpr int kChains = NT == 1 ? 2 : 1;
      float x[kG][NT][4], xs[kChains][kG][NT][4] = {};
#pragma unroll
      for (int g = 0; g < kG; ++g)
#pragma unroll
        for (int j0 = 0; j0 < kLoads; j0 += kBatch) {
          uint32_t w[kBatch][4];
#pragma unroll
          for (int j = 0; j < kBatch; ++j)
            ldmatrix4(Sw::step(tile_k + k_lane, 2 * (j0 + j)) + 16 * g * Sh::kRowBytes, w[j]);
#pragma unroll
          for (int j = 0; j < kBatch; ++j) {
            if (E4M3) {  // two chunks of 16 dims
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t f[4] = {
                    e4m3_to_h2(w[j][2 * h], false), e4m3_to_h2(w[j][2 * h + 1], false),
                    e4m3_to_h2(w[j][2 * h], true), e4m3_to_h2(w[j][2 * h + 1], true)};
#pragma unroll
                for (int t = 0; t < NT; ++t)
                  product16<false>(xs[h % kChains][g][t], f, qf[t][2 * (j0 + j) + h][0],
                                   qf[t][2 * (j0 + j) + h][1]);
              }
            } else {
#pragma unroll
              for (int t = 0; t < NT; ++t)
                product16<true>(xs[j % kChains][g][t], w[j], qf[t][j0 + j][0], qf[t][j0 + j][1]);
            }
          }
        }
#pragma unroll
      for (int g = 0; g < kG; ++g)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[g][t][e] = kChains == 1 ? xs[0][g][t][e] : xs[0][g][t][e] + xs[kChains - 1][g][t][e];
      // Scores, rounded before the maximum is taken off them (a difference of the unrounded
      // product would be off by half a unit of the maximum), into the running state
      const bool hides = key0 + Sh::kKeys > all_see;
      bool above = false;
      float top[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float m = -INFINITY;
#pragma unroll
          for (int g = 0; g < kG; ++g)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float& y = x[g][t][e + 2 * h];
              y = __fmul_rn(y, qs[t][e]);
              if (hides && key0 + 16 * g + 8 * h + r >= sees[t][e]) y = -INFINITY;
              m = fmaxf(m, y);
            }
          top[t][e] = __fadd_ru(m, -kPagedLift<E4M3>);
          above |= top[t][e] > mx[t][e];
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
      uint32_t ph[kG][NT][2], pl[kG][NT][2];  // weights of slots 2 c, 2 c + 1 (and + 8) for row r
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float m = mx[t][e] == -INFINITY ? 0.f : mx[t][e];
#pragma unroll
          for (int g = 0; g < kG; ++g) {
            x[g][t][e] = exp2_approx(__fadd_rn(x[g][t][e], -m));
            x[g][t][e + 2] = exp2_approx(__fadd_rn(x[g][t][e + 2], -m));
            sum[t][e] += x[g][t][e] + x[g][t][e + 2];
          }
        }
#pragma unroll
        for (int g = 0; g < kG; ++g)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (E4M3) {
              ph[g][t][h] = transposed(pack_f16(x[g][t][2 * h], x[g][t][2 * h + 1]));
            } else {
              uint32_t low;
              ph[g][t][h] = transposed(split_weights(x[g][t][2 * h], x[g][t][2 * h + 1], low));
              pl[g][t][h] = transposed(low);
            }
          }
      }
      // Calls use(i, f) with V's dims 16 i .. 16 i + 15 of a group of slots.  Rows of f: dims in
      // order (bf16), or dims 2 r for row r and 2 r + 1 for row r + 8
      auto values = [&](int g, auto&& use) {
#pragma unroll
        for (int j0 = 0; j0 < kLoads; j0 += kBatch) {
          uint32_t w[kBatch][4];
#pragma unroll
          for (int j = 0; j < kBatch; ++j)
            ldmatrix4_trans(Sw::step(tile_v + v_lane, 2 * (j0 + j)) + 16 * g * Sh::kRowBytes, w[j]);
#pragma unroll
          for (int j = 0; j < kBatch; ++j) {
            if (E4M3) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                // a word: dims 2 r, 2 r + 1 of slot 2 c, then of slot 2 c + 1
                const uint32_t lo = __byte_perm(w[j][2 * h], 0, 0x3120),
                               hi = __byte_perm(w[j][2 * h + 1], 0, 0x3120);
                const uint32_t f[4] = {e4m3_to_h2(lo, false), e4m3_to_h2(lo, true),
                                       e4m3_to_h2(hi, false), e4m3_to_h2(hi, true)};
                use(2 * (j0 + j) + h, f);
              }
            } else {
              use(j0 + j, w[j]);
            }
          }
        }
      };
      auto product = [&](float (&y)[4], const uint32_t (&f)[4], int g, int t) {
        product16<!E4M3>(y, f, ph[g][t][0], ph[g][t][1]);
        if (!E4M3) product16<true>(y, f, pl[g][t][0], pl[g][t][1]);
      };
      // A value that is not finite must not reach the tokens that do not see its slot, whose
      // weight for it is 0: then the slots go one by one, to those that do.
      bool odd = false;
      if (hides && unseen) {
        for (int i = lane; i < Sh::kTileBytes / 16; i += 32) {
          const uint4 w = ld_shared16(tile_v + 16 * i);
          odd |= not_finite<E4M3>(w.x) || not_finite<E4M3>(w.y) || not_finite<E4M3>(w.z) ||
                 not_finite<E4M3>(w.w);
        }
        odd = __any_sync(kFull, odd);
      }
      if (!odd) {
#pragma unroll
        for (int g = 0; g < kG; ++g)
          values(g, [&](int i, const uint32_t (&f)[4]) {
#pragma unroll
            for (int t = 0; t < NT; ++t) product(o[t][i], f, g, t);
          });
      } else {
#pragma unroll
        for (int g = 0; g < kG; ++g) {
#pragma unroll 1
          for (int slot = 0; slot < 16; ++slot) {
            const uint32_t keep = (slot & 7) >> 1 != c ? 0u : slot & 1 ? 0xffff0000u : 0xffffu;
            const uint32_t first = slot < 8 ? keep : 0u, second = slot < 8 ? 0u : keep;
            values(g, [&](int i, const uint32_t (&f)[4]) {
              const uint32_t one[4] = {f[0] & first, f[1] & first, f[2] & second, f[3] & second};
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                float y[4] = {0.f, 0.f, 0.f, 0.f};
                product(y, one, g, t);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (key0 + 16 * g + slot < sees[t][e & 1]) o[t][i][e] += y[e];
              }
            });
          }
        }
      }
      __syncwarp();
      if (lane == 0) bar_arrive(smem_addr(&mem.empty[place]));
      place += kW;
      if (place >= kN) {
        place -= kN;
        phase ^= 1;
      }
    }
    next -= count;
    if (!ok) break;
    // the next share's queries come while the warps meet
    more = share_known(k + 1);
    if (more) load_queries(mem.share[(k + 1) % kShares]);

    const bool whole = s.slot == kWhole;
    float* joint = reinterpret_cast<float*>(smem);  // of a cluster: [row][kD], [row] max, sum
    float2* joint_stats = reinterpret_cast<float2*>(joint + Sh::kRows * Sh::kD);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) sum[t][e] += __shfl_xor_sync(kFull, sum[t][e], off);
        // all scores NaN: so is the result
        if (sum[t][e] != sum[t][e] && mx[t][e] == -INFINITY) mx[t][e] = 0.f;
      }
      // where the rows of the last meeting have been read
      if (met > 0) ok = ok && bar_wait(smem_addr(&mem.parts_free), (met - 1) & 1, &mem.dead, a);
      float* mine = parts + warp * 8 * Sh::kPart;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float* row = mine + (2 * c + e) * Sh::kPart;
        if (!idle)
#pragma unroll
        for (int i = 0; i < 2 * M; ++i) {
          if (E4M3) {
            *reinterpret_cast<float2*>(row + 16 * i + 2 * r) = make_float2(o[t][i][e], o[t][i][e + 2]);
          } else {
            row[16 * i + r] = o[t][i][e];
            row[16 * i + 8 + r] = o[t][i][e + 2];
          }
        }
        if (r == 0) stats[warp * 8 + 2 * c + e] = make_float2(mx[t][e], sum[t][e]);
      }
      // Row q of the tile from all warps' parts, in their order
      auto combine = [&](int q, long long row) {
        float2 st[kW];
        float top = -INFINITY, total = 0.f, f[kW];
#pragma unroll
        for (int w = 0; w < kW; ++w) st[w] = stats[w * 8 + q];
#pragma unroll
        for (int w = 0; w < kW; ++w) top = fmaxf(top, st[w].x);
#pragma unroll
        for (int w = 0; w < kW; ++w) {
          // a warp that has seen nothing may have left nothing
          f[w] = st[w].x == -INFINITY ? 0.f : exp2_approx(st[w].x - top);
          total += st[w].x == -INFINITY ? 0.f : f[w] * st[w].y;
        }
        const float scale = whole ? (top == -INFINITY ? 0.f : vs / total) : vs;
        const size_t part = (size_t)s.slot * Sh::kRows + 8 * t + q;
        for (int d = 4 * lane; d < a.d; d += 128) {
          float4 z[kW], y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int w = 0; w < kW; ++w)
            z[w] = *reinterpret_cast<const float4*>(parts + (w * 8 + q) * Sh::kPart + d);
#pragma unroll
          for (int w = 0; w < kW; ++w) {
            const bool none = st[w].x == -INFINITY;
            y.x += none ? 0.f : f[w] * z[w].x;
            y.y += none ? 0.f : f[w] * z[w].y;
            y.z += none ? 0.f : f[w] * z[w].z;
            y.w += none ? 0.f : f[w] * z[w].w;
          }
          y = make_float4(y.x * scale, y.y * scale, y.z * scale, y.w * scale);
          if (whole)
            *reinterpret_cast<uint2*>(a.out + row * a.d + d) =
                make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
          else
            *reinterpret_cast<float4*>(s.slot == kOfCluster ? joint + (8 * t + q) * Sh::kD + d
                                                            : a.parts + part * a.d + d) = y;
        }
        if (lane == 0) {
          if (!whole)
            *(s.slot == kOfCluster ? joint_stats + 8 * t + q : a.stats + part) =
                make_float2(top, total);
          else if (a.lse)
            a.lse[row] = (top + log2f(total)) * kLn2;
        }
      };
      __syncwarp();
      if (lane == 0) bar_arrive(smem_addr(&mem.parts_full));
#pragma unroll 1
      for (int q = warp; q < 8; q += kW) {
        const long long row = out_row(a, s, 8 * t + q);
        if (row < 0) continue;
        ok = ok && bar_wait(smem_addr(&mem.parts_full), met & 1, &mem.dead, a);
        combine(q, row);
      }
      __syncwarp();
      if (lane == 0) bar_arrive(smem_addr(&mem.parts_free));
      ++met;
    }
    __syncwarp();
    if (lane == 0) bar_arrive(smem_addr(&mem.share_free[k % kShares]));
  }
  }
  // A cluster's CTAs join their parts; all of its threads come here
  if (a.cluster > 1) {
    Share& s = mem.share[0];
    cluster_sync();
    if (s.seq >= 0 && warp < kW) {
      float* joint = reinterpret_cast<float*>(smem);
      float2* joint_stats = reinterpret_cast<float2*>(joint + Sh::kRows * Sh::kD);
      for (int q = blockIdx.x % a.cluster + a.cluster * warp; q < Sh::kRows; q += a.cluster * kW) {
        const long long row = out_row(a, s, q);
        if (row < 0) continue;
        float2 mine = make_float2(-INFINITY, 0.f);
        if (lane < a.cluster) {
          const uint64_t w = ld_cluster_u64(mapa(smem_addr(joint_stats + q), lane));
          mine = make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
        }
        float top = mine.x;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, off));
        const float f = mine.x == -INFINITY ? 0.f : exp2_approx(mine.x - top);
        float total = mine.x == -INFINITY ? 0.f : f * mine.y;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) total += __shfl_xor_sync(kFull, total, off);
        const float inverse = top == -INFINITY ? 0.f : 1.f / total;
        const unsigned seen = __ballot_sync(kFull, mine.x != -INFINITY);
        for (int d0 = 0; d0 < a.d; d0 += 128) {
          const int d = d0 + 4 * lane;
          float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int k0 = 0; k0 < a.cluster; k0 += 8) {
            float4 z[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (d < a.d && (seen >> (k0 + k) & 1))
                z[k] = ld_cluster_f32x4(mapa(smem_addr(joint + q * Sh::kD + d), k0 + k));
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float g = __shfl_sync(kFull, f, k0 + k);
              if (d < a.d && (seen >> (k0 + k) & 1)) {
                y.x += g * z[k].x;
                y.y += g * z[k].y;
                y.z += g * z[k].z;
                y.w += g * z[k].w;
              }
            }
          }
          if (d < a.d)
            *reinterpret_cast<uint2*>(a.out + row * a.d + d) =
                make_uint2(pack_bf16(y.x * inverse, y.y * inverse),
                           pack_bf16(y.z * inverse, y.w * inverse));
        }
        if (lane == 0 && a.lse) a.lse[row] = (top + log2f(total)) * kLn2;
      }
    }
    // no CTA leaves while its results are read
    cluster_arrive_relaxed();
    cluster_wait();
  }
  write_empty(a);
}

struct PagedKernel {
  void (*kern)(PagedAttendArgs);
  int smem, rows, threads, stage_keys;
};

template <int M, int NT, bool E4M3>
constexpr PagedKernel paged_stream() {
  using Sh = StreamShape<M, NT, E4M3>;
  return {paged_stream_kernel<M, NT, E4M3>, Sh::kTotal, Sh::kRows, Sh::kStreamThreads,
          Sh::kKeys};
}

// [(head_dim + 31) / 32 - 1][kind]: the streaming kernel with tiles of 8 and of 16 rows (bf16 pages,
// where their sums fit the registers; else the first again), the block kernel
constexpr int kKinds = 3;
extern const PagedKernel kPagedBf16[8][kKinds], kPagedE4m3[8][kKinds];

}  // namespace vd
