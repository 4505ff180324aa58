// prompt_device.hpp -- device-side building blocks of the prompt pass: packed
// sequences and their division into chunks.
#pragma once

#include "attn_device.hpp"
#include "prompt.hpp"

namespace sla {

__device__ __forceinline__ void store4(bf16 *p, const float (&x)[4]) {
  *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
}
__device__ __forceinline__ void store4(float *p, const float (&x)[4]) {
  *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
}

// Sequences longer than min_len (-1: all) there can be.
__host__ __device__ inline int64_t most_longer(const PackedRows &r, int min_len) {
  const int64_t most = min_len < 0 ? r.B : r.tokens / (min_len + 1);
  return most < r.B ? most : r.B;
}

// Chunks of C tokens of the sequences longer than min_len (-1: of all, an empty one
// having one empty chunk).  Chunk c of sequence b has the slot start[b] / C + rank + c,
// rank counting the longer sequences before b: ceil(len / C) <= end / C - start / C + 1,
// so no two share one, and no table of chunk counts has to be summed up first.  Some
// slots stay empty.  With a window of w chunks, those behind the first `done`, chunk
// done + c has the slot w rank + c.
template <int C>
__host__ __device__ inline int64_t chunk_slots(const PackedRows &r, int min_len, int window = 0) {
  return window ? most_longer(r, min_len) * window : (int64_t)r.tokens / C + most_longer(r, min_len);
}
template <int C>
__host__ __device__ inline int first_slot(int start, int rank, int window = 0) {
  return window ? rank * window : start / C + rank;
}

// Whether the starts are in order and inside the rows (wave-uniform).  Every wave
// looks at all of them, here and in find_chunk: the loads are independent, 64 sequences
// at a time.  In batches of thousands this is what takes the time: single tokens of 8
// heads of 64 x 64 61 us for 1024 sequences, 455 for 4096 and 5000 for 16384, whose
// bytes are 53, 214 and 855 us; the convolution of 2048 channels 34, 322 and 4600 us, whose
// bytes are 12, 46 and 184.
__device__ __forceinline__ bool starts_ok(const PackedRows &r, int lane) {
  bool bad = false;
  for (int i = lane; i < r.B; i += kWave) {
    const int a = r.start[i], e = r.start[i + 1];
    bad = bad || a < 0 || a > e || e > r.tokens;
  }
  return !wave_any(bad);
}

// How many sequences are longer than sequence b, or as long and before it, in a batch
// of up to 64 (wave-uniform).
__device__ __forceinline__ int place_by_length(const PackedRows &r, int b, int lane) {
  const int len = lane < r.B ? r.start[lane + 1] - r.start[lane] : -1;
  const int mine = __builtin_amdgcn_readlane(len, b);
  return __popcll(__ballot(len > mine || (len == mine && lane < b)));
}

struct Chunk {
  int b;      // sequence, -1: none
  int row;    // first row
  int rows;   // 1..C, 0: the one chunk of an empty sequence
  int left;   // the sequence's rows from `row` on
  bool first; // of the sequence (of its window)
  int rank;   // longer sequences before its own
  int longer; // longer sequences in all
};

// The chunk of slot `slot`, from the sequence whose first slot is the last not behind
// it: its rows [start, end), that slot `front`, its rank.
template <int C>
__host__ __device__ inline void chunk_at(Chunk &c, int slot, int b, int start, int end, int front, int rank, int window, int done) {
  const int at = slot - front;
  if (window && at >= window) return;
  const int64_t row = start + (int64_t)(done + at) * C;
  if (at > 0 && row >= end) return;
  c.b = b;
  c.rank = rank;
  c.row = (int)row;
  c.left = end - c.row;
  c.rows = c.left < C ? c.left : C;
  c.first = at == 0;
}

// The chunk of a slot (wave-uniform).  `ok` says whether the starts are in order.
template <int C>
__device__ __forceinline__ Chunk find_chunk(const PackedRows &r, int min_len, int slot, int lane, bool &ok, int window = 0,
                                            int done = 0) {
  bool bad = false;
  int longer = 0, rank = 0, b = -1, start = 0, end = 0, front = 0;
  for (int i = 0; i < r.B; i += kWave) {
    const bool live = i + lane < r.B;
    const int a = live ? r.start[i + lane] : 0, e = live ? r.start[i + lane + 1] : 0;
    bad = bad || (live && (a < 0 || a > e || e > r.tokens));
    const uint64_t mask = __ballot(live && (int64_t)e - a > min_len);
    const int before = longer + __popcll(mask & ((1ull << lane) - 1));
    const int mine = first_slot<C>(a, before, window);
    const uint64_t reached = __ballot(mine <= slot) & mask;
    if (reached) {
      const int l = 63 - __builtin_clzll(reached);
      b = i + l;
      start = __builtin_amdgcn_readlane(a, l);
      end = __builtin_amdgcn_readlane(e, l);
      front = __builtin_amdgcn_readlane(mine, l);
      rank = __builtin_amdgcn_readlane(before, l);
    }
    longer += __popcll(mask);
  }
  ok = !wave_any(bad);
  Chunk c = {-1, 0, 0, 0, false, 0, longer};
  if (ok && b >= 0) chunk_at<C>(c, slot, b, start, end, front, rank, window, done);
  return c;
}

}  // namespace sla
