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

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

// What a sequence has to do.
struct SeqWork {
  int len, add, total, tiles;  // slots, new tokens, slots that the last of them sees
  int stages;
  long long work;              // stages of all its units
};

__device__ __forceinline__ SeqWork seq_work(const PagedAttendArgs& a, int seq, bool report) {
  SeqWork w;
  w.len = __ldcg(a.pages.len + seq);
  w.add = a.n_new ? __ldcg(a.n_new + seq) : a.B;
  if (w.add < 0 || w.add > a.B || w.len < 0 || w.len > a.pages.capacity() - (a.causal ? w.add : 0)) {
    if (report) record_status(a.pages.status, kStDeviceLen);
    w.len = w.add = 0;
  }
  w.total = w.add == 0 ? 0 : w.len + (a.causal ? w.add : 0);
  w.tiles = (w.add * a.group + a.rows - 1) / a.rows;
  w.stages = (w.total + kStageKeys - 1) / kStageKeys;
  w.work = (long long)w.stages * w.tiles * a.heads;
  return w;
}

__device__ __forceinline__ long long block_sum_i64(long long v, long long* sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(kFull, v, off);
  if (lane == 0) sh[warp] = v;
  __syncthreads();
  long long t = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) t += sh[w];
  __syncthreads();
  return t;
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
};

// Walks over a CTA's piece of the line.  All threads of the CTA make the same calls.
struct Walk {
  const PagedAttendArgs& a;
  long long* sh;  // kWarps + 1 + kThreads entries
  Cut cut;
  long long at, end, seq_begin;  // line positions: the next stage, the piece's end, seq's first
  int seq, chunk;                // chunk: first sequence of those whose ends are in sh

  __device__ Walk(const PagedAttendArgs& args, long long* shared, int least)
      : a(args), sh(shared), at(0), end(0), seq_begin(0), seq(0), chunk(0) {
    long long mine = 0;
    for (int s = threadIdx.x; s < a.n_seq; s += kThreads)
      mine += seq_work(a, s, blockIdx.x == 0).work;
    const long long all = block_sum_i64(mine, sh);
    const long long most = all / least;
    cut.ctas = most >= (long long)gridDim.x ? (int)gridDim.x : most > 1 ? (int)most : 1;
    cut.per = all / cut.ctas;
    cut.more = (int)(all - cut.per * cut.ctas);
    if ((int)blockIdx.x >= cut.ctas) return;
    at = cut.begin(blockIdx.x);
    end = cut.begin(blockIdx.x + 1);
    load(0);
  }
  // sh[kWarps + 1 + i]: where sequence chunk + i ends on the line
  __device__ void load(long long begin) {
    const int s = chunk + threadIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long x = s < a.n_seq ? seq_work(a, s, false).work : 0;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const long long y = __shfl_up_sync(kFull, x, off);
      if (lane >= off) x += y;
    }
    __syncthreads();  // the last chunk's readers
    if (lane == 31) sh[warp] = x;
    __syncthreads();
    for (int w = 0; w < warp; ++w) begin += sh[w];
    sh[kWarps + 1 + threadIdx.x] = begin + x;
    __syncthreads();
  }
  // The next share, if there is one.
  __device__ bool next(Share& s) {
    if (at >= end) return false;
    long long stop;
    while ((stop = sh[kWarps + 1 + seq - chunk]) <= at) {  // a sequence that is done, or empty
      seq_begin = stop;
      ++seq;
      if (seq == chunk + kThreads) {
        chunk = seq;
        load(stop);
      }
    }
    s.seq = seq;
    s.w = seq_work(a, seq, false);
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
    return true;
  }
  // What the join has to know of a share that begins a unit and does not end it: the unit and
  // the last CTA that has a part of it.
  __device__ int4 split_of(const Share& s) const {
    const long long unit_end = at + (s.w.stages - s.s1);
    return make_int4(s.seq, s.head, s.tile, cut.holder(unit_end - 1));
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
    const SeqWork w = seq_work(a, s, false);
    if (w.add == 0 || w.total > 0) continue;
    const long long row0 = (long long)s * a.B * a.heads * a.group;
    const long long rows = (long long)w.add * a.heads * a.group;
    const int chunks = a.d / 8;
    for (long long i = threadIdx.x; i < rows * chunks; i += kThreads)
      st16(a.out + row0 * a.d + i * 8, make_uint4(0, 0, 0, 0));
    if (a.lse)
      for (long long i = threadIdx.x; i < rows; i += kThreads) a.lse[row0 + i] = -INFINITY;
  }
}

}  // namespace vd
