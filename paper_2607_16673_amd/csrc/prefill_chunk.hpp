// prefill_chunk.hpp -- what the two kernels of the chunked recurrence share: the
// order of a chunk's tokens in matrix operands, those operands' types, and the
// workspace in which the first leaves them for the second.
//
// Every matrix instruction here is v_mfma_f32_16x16x32_bf16 or eight
// v_mfma_f32_16x16x4_f32 in a row.  Of an operand, lane l = 16 g + r holds row (or
// column) r and the 8 inner indices 32 ks + 8 g + e, e = 0..7, 8 neighbouring
// values; of a result, lane l holds column r of the rows 4 g + i, i = 0..3.  So
// that a result can be the next product's operand in the lane where it is, the
// 16-row tile 2 ks + h of 64 tokens (or of d_k) has as its row 4 g + i the index
//     32 ks + 8 g + 4 h + i:
// a pair of tiles then gives each lane its 8 neighbouring indices.
#pragma once

#include "prompt_device.hpp"

namespace sla {

constexpr int kChunk = 64;  // tokens of a chunk: four row tiles, one to a wave

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

// index of row `r` of tile `t`
__host__ __device__ constexpr int tile_row(int t, int r) { return 32 * (t / 2) + 8 * (r / 4) + 4 * (t % 2) + r % 4; }

// An operand: N bf16 planes, 8 bits of the values each, or fp32 values (as they lie in
// memory; see `planes`).
template <bool F32, int N>
struct Frag {
  using Piece = bf16x8;
  Piece p[N];
};
template <int N>
struct Frag<true, N> {
  using Piece = f32x4;
  Piece p[2];
};
// 16-byte pieces of a lane
template <bool F32, int N>
constexpr int kPiecesOf = F32 ? 2 : N;

// two values to one word, in one instruction
__device__ __forceinline__ uint32_t round_pair(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

// The bf16 planes of 4 values: each the rest of the ones before it, rounded to
// nearest, so that a rest is half a step at most and of either sign.  Three planes are
// the value itself, down to bf16's last bit of 2^-133: it has 24 bits, and a rest's
// sign is one.  (The first plane of 3.3961e38
// or more is infinite.  Holding it below cost 2 to 7% of the second kernel's time.)
template <int N>
__device__ __forceinline__ void split4(const float (&x)[4], uint2 (&p)[N]) {
  float r[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
  for (int n = 0; n < N; ++n) {
    p[n] = make_uint2(round_pair(r[0], r[1]), round_pair(r[2], r[3]));
    if (n + 1 < N) {
      r[0] -= __uint_as_float(p[n].x << 16);
      r[1] -= __uint_as_float(p[n].x & 0xffff0000u);
      r[2] -= __uint_as_float(p[n].y << 16);
      r[3] -= __uint_as_float(p[n].y & 0xffff0000u);
    }
  }
}

// An operand of the second kernel as bf16 planes.  Six products of those of fp32 values
// take 96 cycles where eight fp32 instructions take 256.  Planes of 1 <= |x| < 2 are
// 1, 2^-8 and 2^-17 at most, so the three products left out are 2 2^-25 + 2^-34 of a
// product's size at most, as a rounding of it would be.
template <int N>
__device__ __forceinline__ const Frag<false, N> &planes(const Frag<false, N> &f) { return f; }
template <int N>
__device__ __forceinline__ Frag<false, 3> planes(const Frag<true, N> &f) {
  const float lo[4] = {f.p[0][0], f.p[0][1], f.p[0][2], f.p[0][3]}, hi[4] = {f.p[1][0], f.p[1][1], f.p[1][2], f.p[1][3]};
  uint2 a[3], b[3];
  split4(lo, a);
  split4(hi, b);
  Frag<false, 3> s;
#pragma unroll
  for (int n = 0; n < 3; ++n) s.p[n] = __builtin_bit_cast(bf16x8, make_uint4(a[n].x, a[n].y, b[n].x, b[n].y));
  return s;
}

// A sum of products a b of NA and NB planes, those past the max(NA, NB) largest sizes
// left out.  It is held in S parts, by the products' size: a matrix instruction waits
// for the one before it on the same registers.
template <int S>
struct Sum {
  f32x4 s[S];
  __device__ __forceinline__ Sum() {
#pragma unroll
    for (int i = 0; i < S; ++i) s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  template <int NA, int NB, int N, int M>
  __device__ __forceinline__ void add(const Frag<false, N> &a, const Frag<false, M> &b) {
    constexpr int kMost = (NA > NB ? NA : NB) - 1;
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (i + j <= kMost) {
          f32x4 &c = s[i + j < S ? i + j : S - 1];
          c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[j], c, 0, 0, 0);
        }
  }
  template <int NA, int NB, int N, int M>
  __device__ __forceinline__ void add(const Frag<true, N> &a, const Frag<true, M> &b) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      s[e % S] = __builtin_amdgcn_mfma_f32_16x16x4f32(a.p[e / 4][e % 4], b.p[e / 4][e % 4], s[e % S], 0, 0, 0);
  }
  __device__ __forceinline__ f32x4 total() const {
    f32x4 t = s[S - 1];
#pragma unroll
    for (int i = S - 2; i >= 0; --i) t += s[i];
    return t;
  }
};

// Planes of an fp32 value.  Outputs that are rounded to bf16 take all three as well:
// with two of them they would differ in the last bit from those of fp32 products.
constexpr int kPlanes = 3;

// Row tile t of the lower triangular 64 x 64 matrices has the inner 32s ks <= t / 2.
__host__ __device__ constexpr int first_frag(int t) { return t < 2 ? t : 2 * t - 2; }
constexpr int kTriFrags = 6;

// What the first kernel leaves, operand by operand, 16 bytes a lane:
//   for every (slot, head): X beta, [6][pieces][64 lanes], the decayed Q K^T, fp32
//   [6][2][64 lanes] (planes would be a third more bytes, and each is cut once a
//   workgroup), and the decays G and D_63, fp32 [2][64];
//   for every (slot, key head): K^T [d_k / 16][2][pieces][64 lanes], and K and Q
//   [4][d_k / 32][pieces][64 lanes].  Keys and queries lie one token a row, often a
//   power of two apart, so that a head's rows all fall to one channel of the L2; the
//   workgroups of a head that read them chunk by chunk would wait there for one
//   another (one sequence of 32768 tokens, 16 heads, with planes that were cut: the second
//   kernel 998 us, 830 with them laid out, the first 30 longer).
//   behind them which sequences the second walks, the longest first in batches of up to
//   64, so that no long one is begun when the others have ended;
//   and in front of them, where every pass of a call finds them, the number of these
//   (-1: bad starts) and the tokens of the longest sequence.
struct Walk {
  int32_t b, start, len, slot;
};

template <bool F32, int DK>
struct ChunkSpace {
  static constexpr size_t kFront = 128;  // a line, so that the operands begin with one
  static constexpr size_t kPiece = 64 * 16;
  static constexpr size_t kSolve = kTriFrags * kPiecesOf<F32, kPlanes> * kPiece;
  static constexpr size_t kMix = kTriFrags * kPiecesOf<true, kPlanes> * kPiece;
  static constexpr size_t kDecay = kSolve + kMix, kRest = kDecay + kChunk * 4;
  static constexpr size_t kHead = kRest + kChunk * 4;
  static constexpr size_t kRows = 4 * (DK / 32) * kPiecesOf<F32, 1> * kPiece;  // of K, of Q, and of K^T
  static constexpr size_t kKeys = 3 * kRows;
  static size_t of_slot(int H, int Hk) { return H * kHead + Hk * kKeys; }

  unsigned char *base;
  size_t slots, walks;
  int H, Hk;

  __host__ __device__ size_t operands() const { return slots * (H * kHead + Hk * kKeys); }
  __host__ __device__ size_t walk_at(size_t i) const { return kFront + operands() + i * sizeof(Walk); }
  __host__ __device__ size_t bytes() const { return walk_at(walks); }
  __device__ int32_t *walk_count() const { return reinterpret_cast<int32_t *>(base); }
  __device__ int32_t *longest() const { return walk_count() + 1; }
  __device__ Walk *walk(int i) const { return reinterpret_cast<Walk *>(base + walk_at(i)); }
  __host__ __device__ unsigned char *head(size_t slot, int h) const { return base + kFront + (slot * H + h) * kHead; }
  __host__ __device__ unsigned char *keys(size_t slot, int kh) const {
    return base + kFront + slots * H * kHead + (slot * Hk + kh) * kKeys;
  }
};

template <bool F32, int DK>
__host__ __device__ inline ChunkSpace<F32, DK> chunk_space(const PrefillArgs &a) {
  return {static_cast<unsigned char *>(a.workspace), (size_t)chunk_slots<kChunk>(a.rows, a.serial_len, a.window),
          (size_t)most_longer(a.rows, a.serial_len), a.H, a.Hk};
}

// Each returns hipSuccess or the launch error (specialised in prefill_chunk.hip's units).
template <bool F32, int DK>
hipError_t launch_chunks(const PrefillArgs &a, hipStream_t s);

}  // namespace sla
