// vd_paged_attend.cuh -- attention over one layer of a paged cache (vd_paged_attend in
// include/vd.h): how the work is divided and its parts are joined.
//
// A unit is a sequence's KV head and a tile of `rows` query rows; it takes ceil(slots /
// slots of a stage) stages.  The units' stages, sequence after sequence, make one line that is cut
// into equal pieces, one for each CTA, whatever the lengths are: the lengths are on the device,
// and a cut by them needs no plan on the host and leaves no CTA idle beside a long sequence.
// A CTA that holds all stages of a unit writes its output.  Of the others it writes a part (sums
// relative to a reference, the reference, the sum of weights), and paged_join_kernel puts
// the parts of a unit together, in order: the same bits every time.
//
// Where the units are so few that several CTAs can take each, a cluster takes a unit instead and
// joins its CTAs' parts through distributed shared memory: one launch, and no look at the other
// sequences.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "vd_attend.cuh"
#include "vd_device.cuh"
#include "vd_paged.cuh"

namespace vd {

struct PagedAttendArgs {
  Pages pages;
  const uint16_t* q;
  uint16_t* out;
  float* lse;            // nullable
  const int32_t* n_new;  // nullable
  int4* split;           // workspace: of each CTA the unit that it begins and does not end: the row
                         // of out of its KV head's first one, the tile's first row and the
                         // number of its rows, the last CTA with a part; or -1
  float2* stats;         // ... [2 CTAs][rows] references and sums of weights,
  float* parts;          // ... [2 CTAs][rows][d] sums
  int n_seq, heads, group, B, d;
  int rows;              // of a tile, a power of two
  int tiles;             // of B tokens
  int cluster;           // CTAs that share a unit, a power of two, or 1: pieces of the line
  int row_shift, stage_shift, cluster_shift;  // log2 of rows, of a stage's slots, of cluster
  int causal;
  float scale;
};

constexpr float kLn2 = 0.69314718055994531f;

// What a sequence has to do.
struct SeqWork {
  int len, add, total, tiles;  // slots, new tokens, slots that the last of them sees
  int stages;                  // of a unit
  __device__ __forceinline__ long long all(int heads) const {
    return (long long)stages * tiles * heads;
  }
};

__device__ __forceinline__ SeqWork seq_work(const PagedAttendArgs& a, int len, int add) {
  SeqWork w = {len, add, 0, 0, 0};
  w.total = add == 0 ? 0 : len + (a.causal ? add : 0);
  w.tiles = (add * a.group + a.rows - 1) >> a.row_shift;
  w.stages = (w.total + (1 << a.stage_shift) - 1) >> a.stage_shift;
  return w;
}

// Length and new tokens of a sequence, none of which where they are out of range.
__device__ __forceinline__ int2 seq_size(const PagedAttendArgs& a, int seq, bool report) {
  const int len = __ldcg(a.pages.len + seq), add = a.n_new ? __ldcg(a.n_new + seq) : a.B;
  if (add < 0 || add > a.B || len < 0 || len > a.pages.capacity() - (a.causal ? add : 0)) {
    if (report) record_status(a.pages.status, kStDeviceLen);
    return make_int2(0, 0);
  }
  return make_int2(len, add);
}

// Quotients, of which most fit 32 bits.
__device__ __forceinline__ long long divide(long long n, long long d) {
  return (unsigned long long)(n | d) >> 32 ? n / d : (long long)((uint32_t)n / (uint32_t)d);
}

// The line cut into `ctas` pieces: the first `more` have one stage more.
struct Cut {
  long long per;
  int ctas, more;
  __device__ __forceinline__ long long begin(int g) const {
    return per * g + (g < more ? g : more);
  }
  __device__ __forceinline__ int holder(long long at) const {
    const long long head = (per + 1) * more;
    return at < head ? (int)divide(at, per + 1) : more + (int)divide(at - head, per);
  }
};

// A CTA's share of a unit: stages [s0, s1).
constexpr int kWhole = -1, kOfCluster = -2;

struct Share {
  int seq, head, tile, s0, s1;
  int len, add, total;  // of the sequence, as in SeqWork
  int slot;  // of the part; kWhole: the whole unit, kOfCluster: a part of the cluster's unit
};

constexpr int kChunk = 64;  // sequences that are looked at together

struct WalkMem {
  Cut cut;
  long long end[kChunk];  // where each ends on the line
  int2 size[kChunk];
  long long sum[32];
};

// Walks over a CTA's piece of the line.  All threads of the CTA construct it together; then each
// warp may go its own way.
struct Walk {
  long long at, end;  // line positions: the next stage, the piece's end
  int chunk, seq, head, tile, stage;
  SeqWork w;          // of seq

  __device__ Walk() : at(0), end(0) {}
  // Pieces of `least` stages at least.
  __device__ Walk(const PagedAttendArgs& a, WalkMem& m, int least)
      : at(0), end(0), chunk(0), seq(0), head(0), tile(0), stage(0), w() {
    load(a, m, 0, blockIdx.x == 0);
    long long all = m.end[kChunk - 1];
    if (a.n_seq > kChunk) {
      long long mine = 0;
      for (int s = kChunk + threadIdx.x; s < a.n_seq; s += blockDim.x) {
        const int2 n = seq_size(a, s, blockIdx.x == 0);
        mine += seq_work(a, n.x, n.y).all(a.heads);
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) mine += __shfl_xor_sync(kFull, mine, off);
      if ((threadIdx.x & 31) == 0) m.sum[threadIdx.x >> 5] = mine;
      __syncthreads();
      for (int i = 0; i < (int)blockDim.x / 32; ++i) all += m.sum[i];
    }
    Cut cut;
    const long long most = divide(all, least);
    cut.ctas = most >= (long long)gridDim.x ? (int)gridDim.x : most > 1 ? (int)most : 1;
    cut.per = divide(all, cut.ctas);
    cut.more = (int)(all - cut.per * cut.ctas);
    if (threadIdx.x == 0) m.cut = cut;
    if ((int)blockIdx.x >= cut.ctas) return;
    at = cut.begin(blockIdx.x);
    end = cut.begin(blockIdx.x + 1);
    if (at >= end) return;
    // the first sequence and the place in it
    long long begin = 0, stop;
    while ((stop = m.end[kChunk - 1]) <= at) {
      begin = stop;
      chunk += kChunk;
      load(a, m, stop, false);
    }
    const int lane = threadIdx.x & 31;
    int done = 0;
#pragma unroll
    for (int i = 0; i < kChunk; i += 32)
      done += __popc(__ballot_sync(kFull, m.end[i + lane] <= at));
    if (done > 0) begin = m.end[done - 1];
    seq = chunk + done;
    w = seq_work(a, m.size[done].x, m.size[done].y);
    const int unit = (int)divide(at - begin, w.stages);
    stage = (int)(at - begin - (long long)unit * w.stages);
    head = unit / w.tiles;
    tile = unit - head * w.tiles;
  }
  // The ends of the chunk's sequences, the first of which begins at `begin`; by the first warp.
  __device__ void load(const PagedAttendArgs& a, WalkMem& m, long long begin, bool report) {
    __syncthreads();  // the last chunk's readers
    if (threadIdx.x < 32) {
      static_assert(kChunk == 64, "two sequences a lane");
      const int i = 2 * threadIdx.x, s = chunk + i;
      const int2 none = make_int2(0, 0), n0 = s < a.n_seq ? seq_size(a, s, report) : none,
                 n1 = s + 1 < a.n_seq ? seq_size(a, s + 1, report) : none;
      const long long x0 = seq_work(a, n0.x, n0.y).all(a.heads),
                      x1 = seq_work(a, n1.x, n1.y).all(a.heads);
      long long x = x0 + x1;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const long long y = __shfl_up_sync(kFull, x, off);
        if ((int)threadIdx.x >= off) x += y;
      }
      m.end[i] = begin + x - x1;
      m.end[i + 1] = begin + x;
      m.size[i] = n0;
      m.size[i + 1] = n1;
    }
    __syncthreads();
  }
  // The next share, if there is one.
  __device__ bool next(const PagedAttendArgs& a, const WalkMem& m, Share& s) {
    if (at >= end) return false;
    s.seq = seq;
    s.head = head;
    s.tile = tile;
    s.len = w.len;
    s.add = w.add;
    s.total = w.total;
    const int n = end - at < w.stages - stage ? (int)(end - at) : w.stages - stage;
    s.s0 = stage;
    s.s1 = stage += n;
    at += n;
    // a CTA's first share may begin inside a unit, its last one may end there
    s.slot = n == w.stages ? kWhole : 2 * (int)blockIdx.x + (s.s0 == 0 ? 1 : 0);
    if (stage == w.stages) {
      stage = 0;
      if (++tile == w.tiles) {
        tile = 0;
        if (++head == a.heads) {
          head = 0;
          if (at < end) do {
              ++seq;
              const int2 n = seq - chunk < kChunk ? m.size[seq - chunk] : seq_size(a, seq, false);
              w = seq_work(a, n.x, n.y);
            } while (w.all(a.heads) == 0);
        }
      }
    }
    return true;
  }
};

// The share of a CTA of a cluster, with no stage where there are fewer than CTAs; false: the unit
// has nothing to do.
__device__ __forceinline__ bool cluster_share(const PagedAttendArgs& a, Share& s) {
  const int rank = blockIdx.x & (a.cluster - 1), unit = blockIdx.x >> a.cluster_shift;
  const int head = unit / a.tiles;
  s.tile = unit - head * a.tiles;
  s.seq = head / a.heads;
  s.head = head - s.seq * a.heads;
  const int2 n = seq_size(a, s.seq, rank == 0 && s.tile == 0 && s.head == 0);
  const SeqWork w = seq_work(a, n.x, n.y);
  s.len = w.len;
  s.add = w.add;
  s.total = w.total;
  s.s0 = (int)((uint32_t)(w.stages * rank) >> a.cluster_shift);  // below 2^26 stages, 17 ranks
  s.s1 = (int)((uint32_t)(w.stages * (rank + 1)) >> a.cluster_shift);
  s.slot = kOfCluster;
  return s.tile < w.tiles && w.total > 0;
}

// What the join has to know of such a unit; `at`: the line's position behind the share.
__device__ __forceinline__ int4 split_of(const PagedAttendArgs& a, const Cut& cut, const Share& s,
                                         long long at) {
  const int row0 = s.tile * a.rows;
  const int left = seq_work(a, s.len, s.add).stages - s.s1;
  return make_int4((s.seq * a.B * a.heads + s.head) * a.group, row0,
                   min(a.rows, s.add * a.group - row0), cut.holder(at + left - 1));
}

// Where a tile's row lies: out and q at row * d, lse at row.  -1: no such row.
__device__ __forceinline__ long long out_row(const PagedAttendArgs& a, const Share& s, int row) {
  const int at = s.tile * a.rows + row, tok = at / a.group;
  if (tok >= s.add) return -1;
  return (((long long)s.seq * a.B + tok) * a.heads + s.head) * a.group + (at - tok * a.group);
}

// Outputs of tokens that see no slot: zeros and -infinity.
__device__ __forceinline__ void write_empty(const PagedAttendArgs& a) {
  for (int s = blockIdx.x; s < a.n_seq; s += gridDim.x) {
    const int2 n = seq_size(a, s, false);
    const SeqWork w = seq_work(a, n.x, n.y);
    if (w.add == 0 || w.total > 0) continue;
    const long long row0 = (long long)s * a.B * a.heads * a.group;
    const long long rows = (long long)w.add * a.heads * a.group;
    const int chunks = a.d / 8;
    for (long long i = threadIdx.x; i < rows * chunks; i += blockDim.x)
      st16(a.out + row0 * a.d + i * 8, make_uint4(0, 0, 0, 0));
    if (a.lse)
      for (long long i = threadIdx.x; i < rows; i += blockDim.x) a.lse[row0 + i] = -INFINITY;
  }
}

}  // namespace vd
