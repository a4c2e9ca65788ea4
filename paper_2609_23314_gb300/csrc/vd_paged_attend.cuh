// vd_paged_attend.cuh -- attention over one layer of a paged cache (vd_paged_attend in
// include/vd.h): how the work is divided and its parts are joined.
//
// A unit is a sequence's KV head and a tile of `rows` query rows; it takes ceil(slots /
// kStageKeys) stages.  The units' stages, sequence after sequence, make one line that is cut
// into equal pieces, one for each CTA, whatever the lengths are: the lengths are on the device,
// and a cut by them needs no plan on the host and leaves no CTA idle beside a long sequence.
// A CTA that holds all stages of a unit writes its output.  Of the others it writes a part (sums
// relative to a reference, the reference, the sum of weights), and paged_join_kernel puts
// the parts of a unit together, in order: the same bits every time.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "vd_attend.cuh"
#include "vd_device.cuh"
#include "vd_paged.cuh"

namespace vd {

constexpr int kStageKeys = 16;

struct PagedAttendArgs {
  Pages pages;
  const uint16_t* q;
  uint16_t* out;
  float* lse;            // nullable
  const int32_t* n_new;  // nullable
  int4* split;           // workspace: of each CTA (see split_of), ...
  float2* stats;         // ... [2 CTAs][rows] references and sums of weights,
  float* parts;          // ... [2 CTAs][rows][d] sums
  int n_seq, heads, group, B, d;
  int rows;              // of a tile
  int causal;
  float scale;
};

constexpr float kLn2 = 0.69314718055994531f;

// What a sequence has to do.
struct SeqWork {
  int len, add, total, tiles;  // slots, new tokens, slots that the last of them sees
  int stages;
  long long work;              // stages of all its units
};

__device__ __forceinline__ SeqWork seq_work(const PagedAttendArgs& a, int len, int add) {
  SeqWork w = {len, add, 0, 0, 0, 0};
  w.total = add == 0 ? 0 : len + (a.causal ? add : 0);
  w.tiles = (add * a.group + a.rows - 1) / a.rows;
  w.stages = (w.total + kStageKeys - 1) / kStageKeys;
  w.work = (long long)w.stages * w.tiles * a.heads;
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

// The line cut into `ctas` pieces: the first `more` have one stage more.
struct Cut {
  long long per;
  int ctas, more;
  __device__ __forceinline__ long long begin(int g) const {
    return per * g + (g < more ? g : more);
  }
  __device__ __forceinline__ int holder(long long at) const {
    const long long head = (per + 1) * more;
    return at < head ? (int)(at / (per + 1)) : more + (int)((at - head) / per);
  }
};

// A CTA's share of a unit: stages [s0, s1) of `stages`.
struct Share {
  int seq, head, tile, s0, s1;
  SeqWork w;
  bool whole;
  int slot;  // of the part
  int last;  // the last CTA that has a part of the unit, where this share begins it
};

constexpr int kChunk = 64;  // sequences that a walk looks at together

struct WalkMem {
  long long end[kChunk];  // where each ends on the line
  int2 size[kChunk];
  long long sum[32];
};

// Walks over a CTA's piece of the line.  All threads of the CTA make the same calls.
struct Walk {
  const PagedAttendArgs& a;
  WalkMem& m;
  Cut cut;
  long long at, end, seq_begin;  // line positions: the next stage, the piece's end, seq's first
  int seq, chunk;                // chunk: the first of the sequences in m

  // Pieces of `least` stages at least.
  __device__ Walk(const PagedAttendArgs& args, WalkMem& mem, int least)
      : a(args), m(mem), at(0), end(0), seq_begin(0), seq(0), chunk(0) {
    load(0, blockIdx.x == 0);
    long long all = m.end[kChunk - 1];
    if (a.n_seq > kChunk) {
      long long mine = 0;
      for (int s = kChunk + threadIdx.x; s < a.n_seq; s += blockDim.x) {
        const int2 n = seq_size(a, s, blockIdx.x == 0);
        mine += seq_work(a, n.x, n.y).work;
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) mine += __shfl_xor_sync(kFull, mine, off);
      if ((threadIdx.x & 31) == 0) m.sum[threadIdx.x >> 5] = mine;
      __syncthreads();
      for (int w = 0; w < (int)blockDim.x / 32; ++w) all += m.sum[w];
    }
    const long long most = all / least;
    cut.ctas = most >= (long long)gridDim.x ? (int)gridDim.x : most > 1 ? (int)most : 1;
    cut.per = all / cut.ctas;
    cut.more = (int)(all - cut.per * cut.ctas);
    if ((int)blockIdx.x >= cut.ctas) return;
    at = cut.begin(blockIdx.x);
    end = cut.begin(blockIdx.x + 1);
  }
  // The ends of the chunk's sequences, the first of which begins at `begin`; by the first warp.
  __device__ void load(long long begin, bool report) {
    __syncthreads();  // the last chunk's readers
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x;
#pragma unroll
      for (int i = 0; i < kChunk; i += 32) {
        const int s = chunk + i + lane;
        const int2 n = s < a.n_seq ? seq_size(a, s, report) : make_int2(0, 0);
        long long x = seq_work(a, n.x, n.y).work;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const long long y = __shfl_up_sync(kFull, x, off);
          if (lane >= off) x += y;
        }
        m.end[i + lane] = begin + x;
        m.size[i + lane] = n;
        begin += __shfl_sync(kFull, x, 31);
      }
    }
    __syncthreads();
  }
  // The next share, if there is one.
  __device__ bool next(Share& s) {
    if (at >= end) return false;
    long long stop;
    while ((stop = m.end[seq - chunk]) <= at) {  // a sequence that is done, or empty
      seq_begin = stop;
      ++seq;
      if (seq == chunk + kChunk) {
        chunk = seq;
        load(stop, false);
      }
    }
    s.seq = seq;
    s.w = seq_work(a, m.size[seq - chunk].x, m.size[seq - chunk].y);
    const long long in = at - seq_begin;
    const int unit = (int)(in / s.w.stages);
    s.s0 = (int)(in - (long long)unit * s.w.stages);
    s.head = unit / s.w.tiles;
    s.tile = unit - s.head * s.w.tiles;
    const long long left = end - at;
    s.s1 = s.w.stages - s.s0 <= left ? s.w.stages : s.s0 + (int)left;
    s.whole = s.s0 == 0 && s.s1 == s.w.stages;
    // a CTA's first share may begin inside a unit, its last one may end there
    s.slot = 2 * blockIdx.x + (s.s0 == 0 ? 1 : 0);
    at += s.s1 - s.s0;
    s.last = s.whole || s.s0 > 0 ? 0 : cut.holder(at + (s.w.stages - s.s1) - 1);
    return true;
  }
};

// Where a tile's row lies: out and q at row * d, lse at row.  -1: no such row.
__device__ __forceinline__ long long out_row(const PagedAttendArgs& a, const Share& s, int row) {
  const int at = s.tile * a.rows + row, tok = at / a.group;
  if (tok >= s.w.add) return -1;
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
