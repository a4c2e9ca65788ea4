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
  int cluster;           // CTAs that share a unit, at most 16, or 1: pieces of the line
  int row_shift, stage_shift;  // log2 of rows, of a stage's slots
  int causal;
  float scale;
  uint32_t page16, slot16;  // strides of the pages in 16 bytes (where a layer's rows lie fits 32 bits)
  uint32_t wait_limit;
};

constexpr float kLn2 = 0.69314718055994531f;

// What a sequence has to do.
struct SeqWork {
  int total, tiles;  // slots that its last token sees, tiles of its tokens
  int stages;        // of a unit
};

// What a unit costs beside its stages, in stages of a CTA: its queries, the meeting of the warps.
constexpr int kUnitCost = 16;

__device__ __forceinline__ SeqWork seq_work(const PagedAttendArgs& a, int2 size) {
  SeqWork w;
  w.total = size.y == 0 ? 0 : size.x + (a.causal ? size.y : 0);
  w.tiles = (size.y * a.group + a.rows - 1) >> a.row_shift;
  w.stages = (w.total + (1 << a.stage_shift) - 1) >> a.stage_shift;
  return w;
}

// The sequence's length on the line.
__device__ __forceinline__ long long line_length(const PagedAttendArgs& a, int2 size) {
  const SeqWork w = seq_work(a, size);
  return w.stages == 0 ? 0 : (long long)(w.stages + kUnitCost) * w.tiles * a.heads;
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

// The line cut into `ctas` pieces: the first `more` are longer by one.
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
  int seq, head, tile, s0, s1;  // seq -1: no more
  int len, add;                 // of the sequence
  int slot;  // of the part; kWhole: the whole unit, kOfCluster: a part of the cluster's unit
};

constexpr int kFewSeqs = 128;  // so many a warp takes in at once

// Sequences that a warp looks at together, one a lane.
struct WalkMem {
  int first;
  long long end[32];  // where each ends on the line
  int2 size[32];
  // many sequences: of each warp of the CTA, and what they found
  long long sum[16];
  int found_seq;
  long long found_at;
};

// Walks over a CTA's piece of the line.  One warp constructs it, all of it; its first lane goes on.
struct Walk {
  Cut cut;
  long long at, end;  // line positions: the next one, the piece's end
  int seq, head, tile, in;  // in: the next position in the unit
  int2 size;                // of seq

  // Where there are more than kFewSeqs sequences, all threads of the CTA come here first: the length
  // of the line, and a sequence near the piece's first one.
  static __device__ long long survey(const PagedAttendArgs& a, WalkMem& m) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int per = (a.n_seq + blockDim.x - 1) / blockDim.x, s0 = threadIdx.x * per,
              s1 = min(a.n_seq, s0 + per);
    long long mine = 0;
    for (int s = s0; s < s1; ++s) mine += line_length(a, seq_size(a, s, blockIdx.x == 0));
    const long long upto = warp_scan_i64(mine);
    if (lane == 31) m.sum[warp] = upto;
    __syncthreads();
    long long before = upto - mine, all = 0;
    for (int w = 0; w < warps; ++w) {
      if (w < warp) before += m.sum[w];
      all += m.sum[w];
    }
    const Cut cut = cut_of(all);
    const long long at = cut.begin(blockIdx.x);
    if ((int)blockIdx.x < cut.ctas && before <= at && at < before + mine) {
      m.found_seq = s0;
      m.found_at = before;
    }
    __syncthreads();
    return all;
  }
  // Pieces long enough that each has a stage wherever it begins.
  static __device__ __forceinline__ Cut cut_of(long long all) {
    Cut cut;
    const long long most = all / (2 * kUnitCost);
    cut.ctas = most >= (long long)gridDim.x ? (int)gridDim.x : most > 1 ? (int)most : 1;
    cut.per = divide(all, cut.ctas);
    cut.more = (int)(all - cut.per * cut.ctas);
    return cut;
  }

  __device__ Walk() : at(0), end(0) {}
  __device__ Walk(const PagedAttendArgs& a, WalkMem& m, long long all)
      : cut(), at(0), end(0), seq(0), head(0), tile(0), in(0), size() {
    int first = 0;
    long long begin = 0;
    if (a.n_seq <= kFewSeqs) {
      // all sequences, the lane's one of each 32, and where they end on the line
      const int lane = threadIdx.x & 31;
      int2 n[kFewSeqs / 32];
      long long end_of[kFewSeqs / 32], before[kFewSeqs / 32];
#pragma unroll
      for (int i = 0; i < kFewSeqs / 32; ++i) {
        const int s = 32 * i + lane;
        n[i] = s < a.n_seq ? seq_size(a, s, blockIdx.x == 0) : make_int2(0, 0);
      }
      all = 0;
#pragma unroll
      for (int i = 0; i < kFewSeqs / 32; ++i) {
        before[i] = all;
        end_of[i] = 0;
        if (32 * i < a.n_seq) {
          end_of[i] = all + warp_scan_i64(line_length(a, n[i]));
          all = __shfl_sync(kFull, end_of[i], 31);
        }
      }
      cut = cut_of(all);
      at = (int)blockIdx.x < cut.ctas ? cut.begin(blockIdx.x) : all;
#pragma unroll
      for (int i = 0; i < kFewSeqs / 32; ++i)
        if (32 * i < a.n_seq && at >= before[i]) {  // the last that holds
          first = 32 * i;
          begin = before[i];
          m.end[lane] = end_of[i];
          m.size[lane] = n[i];
        }
      m.first = first;
      __syncwarp();
    } else {
      cut = cut_of(all);
      at = (int)blockIdx.x < cut.ctas ? cut.begin(blockIdx.x) : all;
    }
    end = (int)blockIdx.x < cut.ctas ? cut.begin(blockIdx.x + 1) : at;
    if (at >= end) return;
    if (a.n_seq > kFewSeqs) {
      first = m.found_seq;
      begin = m.found_at;
      load(a, m, first, begin, false);
      while (m.end[31] <= at) {
        begin = m.end[31];
        first += 32;
        load(a, m, first, begin, false);
      }
    }
    const int done = __popc(__ballot_sync(kFull, m.end[threadIdx.x & 31] <= at));
    if (done > 0) begin = m.end[done - 1];
    seq = first + done;
    size = m.size[done];
    const SeqWork w = seq_work(a, size);
    const int unit = (int)divide(at - begin, w.stages + kUnitCost);
    in = (int)(at - begin - (long long)unit * (w.stages + kUnitCost));
    head = unit / w.tiles;
    tile = unit - head * w.tiles;
  }
  // The warp's next 32 sequences, the first of which begins at `begin`.
  static __device__ void load(const PagedAttendArgs& a, WalkMem& m, int first, long long begin,
                              bool report) {
    const int lane = threadIdx.x & 31, s = first + lane;
    const int2 n = s < a.n_seq ? seq_size(a, s, report) : make_int2(0, 0);
    const long long x = warp_scan_i64(line_length(a, n));
    __syncwarp();
    m.first = first;
    m.end[lane] = begin + x;
    m.size[lane] = n;
    __syncwarp();
  }
  // The next share, if there is one; by one thread.
  __device__ bool next(const PagedAttendArgs& a, const WalkMem& m, Share& s) {
    while (at < end) {
      SeqWork w = seq_work(a, size);
      const int length = w.stages + kUnitCost;
      const int n = end - at < length - in ? (int)(end - at) : length - in;
      s.seq = seq;
      s.head = head;
      s.tile = tile;
      s.len = size.x;
      s.add = size.y;
      s.s0 = max(0, in - kUnitCost);
      s.s1 = max(0, in + n - kUnitCost);
      // a CTA's first share may begin inside a unit, its last one may end there
      s.slot = s.s1 - s.s0 == w.stages ? kWhole : 2 * (int)blockIdx.x + (s.s0 == 0 ? 1 : 0);
      in += n;
      at += n;
      if (in == length) {
        in = 0;
        if (++tile == w.tiles) {
          tile = 0;
          if (++head == a.heads) {
            head = 0;
            if (at < end) do {
                ++seq;
                size = seq - m.first < 32 ? m.size[seq - m.first] : seq_size(a, seq, false);
                w = seq_work(a, size);
              } while (w.stages == 0);
          }
        }
      }
      if (s.s1 > s.s0) return true;
    }
    return false;
  }
  // What the join has to know of a unit that the last share began and did not end.
  __device__ int4 split_of(const PagedAttendArgs& a, const Share& s) const {
    const int row0 = s.tile * a.rows;
    const int left = seq_work(a, make_int2(s.len, s.add)).stages - s.s1;
    return make_int4((s.seq * a.B * a.heads + s.head) * a.group, row0,
                     min(a.rows, s.add * a.group - row0), cut.holder(at + left - 1));
  }
};

// The slots that the sequence's last token sees.
__device__ __forceinline__ int seen_slots(const PagedAttendArgs& a, const Share& s) {
  return s.len + (a.causal ? s.add : 0);
}

// The share of a CTA of a cluster, with no stage where there are fewer than CTAs; false: the unit
// has nothing to do.
__device__ __forceinline__ bool cluster_share(const PagedAttendArgs& a, Share& s) {
  const int unit = blockIdx.x / a.cluster, rank = blockIdx.x - unit * a.cluster;
  const int head = unit / a.tiles;
  s.tile = unit - head * a.tiles;
  s.seq = head / a.heads;
  s.head = head - s.seq * a.heads;
  const int2 n = seq_size(a, s.seq, rank == 0 && s.tile == 0 && s.head == 0);
  const SeqWork w = seq_work(a, n);
  s.len = n.x;
  s.add = n.y;
  s.s0 = (int)((uint32_t)(w.stages * rank) / a.cluster);  // below 2^26 stages, 17 ranks
  s.s1 = (int)((uint32_t)(w.stages * (rank + 1)) / a.cluster);
  s.slot = kOfCluster;
  return s.tile < w.tiles && w.total > 0;
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
    if (n.y == 0 || seq_work(a, n).total > 0) continue;
    const long long row0 = (long long)s * a.B * a.heads * a.group;
    const long long rows = (long long)n.y * a.heads * a.group;
    const int chunks = a.d / 8;
    for (long long i = threadIdx.x; i < rows * chunks; i += blockDim.x)
      st16(a.out + row0 * a.d + i * 8, make_uint4(0, 0, 0, 0));
    if (a.lse)
      for (long long i = threadIdx.x; i < rows; i += blockDim.x) a.lse[row0 + i] = -INFINITY;
  }
}

}  // namespace vd
