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

// Whether the starts are in order and inside the rows (wave-uniform).  Every
// wave looks at all of them: the loads are independent, 64 sequences at a time.
__device__ __forceinline__ bool starts_ok(const PackedRows &r, int lane) {
  bool bad = false;
  for (int i = lane; i < r.B; i += kWave) {
    const int a = r.start[i], b = r.start[i + 1];
    bad = bad || a < 0 || a > b || b > r.tokens;
  }
  return !wave_any(bad);
}

// Chunks of C tokens.  Sequence b's chunk c has the slot start[b] / C + b + c:
// ceil(len / C) <= end / C - start / C + 1, so no two share one, and no table of
// chunk counts has to be summed up first.  Some slots stay empty.
template <int C>
__host__ __device__ inline int64_t chunk_slots(const PackedRows &r) {
  return (int64_t)r.tokens / C + r.B;
}

// The sequence to be begun as number `place`: the longest first, for batches of up
// to 64, so that no long one is begun when the others have ended; else in order.
// (Wave-uniform; starts need not be in order.)
__device__ __forceinline__ int by_length(const PackedRows &r, int place, int lane) {
  if (r.B > kWave) return place;
  const int len = lane < r.B ? r.start[lane + 1] - r.start[lane] : 0;
  int rank = lane < r.B ? 0 : -1;
  for (int i = 0; i < r.B; ++i) {
    const int other = __builtin_amdgcn_readlane(len, i);
    rank += lane < r.B && (other > len || (other == len && i < lane));
  }
  return __builtin_ctzll(__ballot(rank == place));
}

struct Chunk {
  int b;      // sequence, -1: none
  int row;    // first row
  int rows;   // 1..C, 0: the one chunk of an empty sequence
  bool first, last;
};

// The chunk of a slot, of starts that are in order (wave-uniform): b is the
// last sequence whose first slot is not behind it, counted as in starts_ok.
// `ok` says whether the starts are in order.
template <int C>
__device__ __forceinline__ Chunk find_chunk(const PackedRows &r, int slot, int lane, bool &ok) {
  bool bad = false;
  int before = 0, a = 0, e = 0;
  for (int i = lane; i - lane < r.B; i += kWave) {
    const bool live = i < r.B;
    a = live ? r.start[i] : 0;
    e = live ? r.start[i + 1] : 0;
    bad = bad || (live && (a < 0 || a > e || e > r.tokens));
    before += __popcll(__ballot(live && a / C + i <= slot));
  }
  ok = !wave_any(bad);
  Chunk c = {-1, 0, 0, false, false};
  if (!ok || before == 0) return c;
  // (the last 64 sequences' starts are at hand)
  const int b = before - 1, kept = b - (r.B - 1) / kWave * kWave;
  const int start = kept >= 0 ? __shfl(a, kept) : r.start[b], end = kept >= 0 ? __shfl(e, kept) : r.start[b + 1];
  const int at = slot - (start / C + b);
  if (at > 0 && (int64_t)at * C >= end - start) return c;
  c.b = __builtin_amdgcn_readfirstlane(b);
  c.row = __builtin_amdgcn_readfirstlane(start + at * C);
  c.rows = __builtin_amdgcn_readfirstlane(min(C, end - c.row));
  c.first = at == 0;
  c.last = c.row + c.rows == end;
  return c;
}

}  // namespace sla
