// prefill_chunk.hip -- the recurrence over packed sequences in chunks of 64
// tokens on the matrix cores (specialised by SLA_CHUNK_DK and SLA_CHUNK_F32).
//
// With D_ij the product of the gates j + 1 .. i and G_i of those up to i (from
// the chunk's start), H the state in front of it, Q, K, V its rows:
//     X = (I + L)^-1,  L_ij = beta_i D_ij k_i . k_j  (j < i)
//     U = X beta (V - G o (K H))          (no delta rule: U = V)
//     out = G o (Q H) + (D o Q K^T, lower) U
//     H' = G_63 H + K^T (D_63 o U)
// X beta and D o Q K^T do not depend on the state.  A first kernel makes them for
// all chunks at once; a second walks each sequence's chunks in order.  Gates are
// only multiplied: no logarithm, no quotient, so tiny ones do no harm.
//
// A sequence's NaN or infinity reaches all outputs of its chunk of 64 tokens, those
// of earlier tokens in it included, and no other sequence.
#include <type_traits>

#include "prefill_chunk.hpp"

namespace sla {
namespace {

constexpr int kThreads = 256;
constexpr int kPitch = 68;  // of a 64 x 64 fp32 matrix in LDS

// workgroup barrier for LDS: loads from memory stay in flight across it
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ------------------------------------------------------------ first kernel
// One workgroup = one chunk and one head.  Wave w owns the matrices' rows 16 w ..
// Rows past the sequence's end count as zero keys with gate 1 and strength 0.
// The inverse goes by blocks of 16: the diagonal ones by substitution on the vector
// ALUs, the others from them by fp32 matrix instructions, so that no power of L, which
// may be large where X is not, is ever formed.
//
// 537 chunks of 32 heads (16 key heads) of 128 take 281 us: 0.6 GB read and 0.96 GB
// written, 5.6 TB/s, the rate of a large copy, over a chain of steps in each workgroup
// that would take 214 us by itself (vector ALUs busy 43%, matrix cores 12%).  It took 429
// us before the matrices had the keys' place in LDS, 360 with loads that waited for one
// another behind their bounds checks (rows are clamped instead).  Registers hold three
// workgroups to a CU.  Heads of one key head on one XCD read half as much, and took 297.
template <bool F32, int DK>
struct MatricesLds {
  using T = typename std::conditional<F32, float, bf16>::type;
  static constexpr int kKeyPitch = DK + 16 / (int)sizeof(T);
  union {
    T k[kChunk * kKeyPitch];
    float x[kChunk * kPitch];  // L, then X, when the keys have been used
  };
  float d[4][16][16];        // D inside the diagonal blocks
  float upto[kChunk];        // product of a block's gates up to i
  float behind[kChunk];      // product of a block's gates behind j
  float total[4];            // of a block's gates
  float decay[kChunk];       // G
  float rest[kChunk];        // D_63
  float beta[kChunk];
};

// row r's 4 inner indices 4 g + e of a 16 x 16 block
__device__ __forceinline__ f32x4 block_a(const float *m, int bi, int bj, int g, int r) {
  return *reinterpret_cast<const f32x4 *>(m + (16 * bi + r) * kPitch + 16 * bj + 4 * g);
}
__device__ __forceinline__ f32x4 block_b(const float *m, int bi, int bj, int g, int r) {
  f32x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = m[(16 * bi + 4 * g + e) * kPitch + 16 * bj + r];
  return x;
}
__device__ __forceinline__ void block_store(float *m, int bi, int bj, int g, int r, f32x4 x) {
#pragma unroll
  for (int e = 0; e < 4; ++e) m[(16 * bi + 4 * g + e) * kPitch + 16 * bj + r] = x[e];
}
// c + a b of 16 x 16 blocks, inner index 4 g + e
__device__ __forceinline__ f32x4 block_mma(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// 8 neighbouring values as an operand of N planes, 16 bytes a lane and piece
template <bool F32, int N>
__device__ __forceinline__ void store_frag(unsigned char *at, int lane, const float (&x)[8]) {
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<f32x4 *>(at + (i * kWave + lane) * 16) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
  } else {
    const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    uint2 a[N], b[N];
    split4(lo, a);
    split4(hi, b);
#pragma unroll
    for (int n = 0; n < N; ++n)
      *reinterpret_cast<uint4 *>(at + (n * kWave + lane) * 16) = make_uint4(a[n].x, a[n].y, b[n].x, b[n].y);
  }
}

template <bool F32, int DK, bool DELTA>
__global__ __launch_bounds__(kThreads) void matrices_kernel(PrefillArgs a) {
  using L = MatricesLds<F32, DK>;
  using T = typename L::T;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  L &s = *reinterpret_cast<L *>(lds);
  const ChunkSpace<F32, DK> space = chunk_space<F32, DK>(a);
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int g = lane / 16, r = lane % 16;
  const unsigned wg = workgroup();
  const unsigned slot = wg / (unsigned)a.H;
  const int h = (int)(wg % (unsigned)a.H), group = a.H / a.Hk, kh = h / group;
  if (slot >= space.slots) return;
  if (a.done > 0 && slot > 0 && *space.longest() <= a.done * kChunk) return;  // a pass that no sequence reaches
  bool ok;
  const Chunk c = find_chunk<kChunk>(a.rows, a.serial_len, (int)slot, lane, ok, a.window, a.done);
  if (h == 0) {
    if (!ok && a.status)
      for (int64_t i = (int64_t)slot * kThreads + threadIdx.x; i < a.rows.B; i += (int64_t)space.slots * kThreads)
        a.status[i] = SLA_ERR_LENGTH;
    if (slot == 0 && threadIdx.x == 0) *space.walk_count() = ok ? c.longer : -1;
    if (slot == 0 && wave == 0 && a.window && a.done == 0) {  // for the passes behind this one
      int longest = 0;
      for (int i = lane; ok && i < a.rows.B; i += kWave) longest = max(longest, a.rows.start[i + 1] - a.rows.start[i]);
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) longest = max(longest, __shfl_xor(longest, o));
      if (lane == 0) *space.longest() = longest;
    }
    if (c.b >= 0 && c.first && wave == 0) {
      const int place = a.rows.B <= kWave ? place_by_length(a.rows, c.b, lane) : c.rank;
      if (lane == 0) {
        *space.walk(place) = Walk{c.b, c.row, a.window ? min(c.left, a.window * kChunk) : c.left, (int)slot};
        if (a.status) a.status[c.b] = SLA_OK;
      }
    }
  }
  if (c.b < 0 || c.rows == 0) return;

  // keys to LDS, queries to registers, gates
  const size_t gate = (size_t)(c.row + min(lane, c.rows - 1)) * a.H + h;
  const float alpha = a.alpha ? a.alpha[gate] : 1.f, beta = DELTA ? a.beta[gate] : 1.f;
  // (rows past the end repeat the last one until they are zeroed, so that no load waits for a branch)
  constexpr int kLanes = DK / 8, kLoads = kChunk * kLanes / kThreads, kWords = sizeof(T) / 2;
  const T *k = static_cast<const T *>(a.k) + (int64_t)c.row * a.k_stride + (size_t)kh * DK;
  u32x4 staged[kLoads][kWords];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int t = (threadIdx.x + i * kThreads) / kLanes, e = threadIdx.x % kLanes * 8;
#pragma unroll
    for (int j = 0; j < kWords; ++j)
      staged[i][j] = reinterpret_cast<const u32x4 *>(k + (int64_t)min(t, c.rows - 1) * a.k_stride + e)[j];
  }
  Frag<F32, 1> q[DK / 32];
  {
    const int t = 16 * wave + r;
    const T *row = static_cast<const T *>(a.q) + (int64_t)(c.row + min(t, c.rows - 1)) * a.q_stride + (size_t)kh * DK + 8 * g;
#pragma unroll
    for (int ks = 0; ks < DK / 32; ++ks)
#pragma unroll
      for (int j = 0; j < kPiecesOf<F32, 1>; ++j) {
        u32x4 x = reinterpret_cast<const u32x4 *>(row + 32 * ks)[j];
        if (t >= c.rows) x = u32x4{0, 0, 0, 0};
        reinterpret_cast<u32x4 *>(&q[ks])[j] = x;
      }
  }
  if (wave == 1) s.beta[lane] = lane < c.rows ? beta : 0.f;
  if (wave == 0) {
    // lane 16 b + j: column j of D's diagonal block b, and the products along the block
    const float al = lane < c.rows ? alpha : 1.f;
    float col = 0.f, run = 1.f, upto = 1.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float ai = __shfl(al, (lane & 48) + i);
      col = i == r ? 1.f : col * ai;
      run *= ai;
      if (i == r) upto = run;
      s.d[g][i][r] = i >= r ? col : 0.f;
    }
    const float t0 = __shfl(upto, 15), t1 = __shfl(upto, 31), t2 = __shfl(upto, 47), t3 = __shfl(upto, 63);
    const float front = g == 0 ? 1.f : g == 1 ? t0 : g == 2 ? t0 * t1 : t0 * t1 * t2;
    const float back = g == 3 ? 1.f : g == 2 ? t3 : g == 1 ? t2 * t3 : t1 * t2 * t3;
    s.upto[lane] = upto;
    s.behind[lane] = col;
    if (r == 15) s.total[g] = upto;
    s.decay[lane] = front * upto;
    s.rest[lane] = col * back;
  }
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int t = (threadIdx.x + i * kThreads) / kLanes, e = threadIdx.x % kLanes * 8;
#pragma unroll
    for (int j = 0; j < kWords; ++j)
      reinterpret_cast<u32x4 *>(s.k + t * L::kKeyPitch + e)[j] = t < c.rows ? staged[i][j] : u32x4{0, 0, 0, 0};
  }
  lds_barrier();

  unsigned char *const head = space.head(slot, h);
  auto key_frag = [&](int row, int ks) {
    Frag<F32, 1> f;
#pragma unroll
    for (int j = 0; j < kPiecesOf<F32, 1>; ++j)
      f.p[j] = reinterpret_cast<const typename Frag<F32, 1>::Piece *>(s.k + row * L::kKeyPitch + 32 * ks + 8 * g)[j];
    return f;
  };
  // Q K^T, decayed: the query tile `wave`, transposed, so that the lane has its
  // operand: query 16 wave + r, keys 32 ks + 8 g + e
  {
    const int query = 16 * wave + r;
    const float upto = s.upto[query];
    float p[2][8];  // row tiles 0 and 1 have no second inner 32; it is made all the same, without a branch
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int block = 2 * ks + g / 2;  // of the lane's keys
      float mid = upto;                  // ... times the blocks between
      mid *= wave - block > 1 ? s.total[block + 1 & 3] : 1.f;
      mid *= wave - block > 2 ? s.total[block + 2 & 3] : 1.f;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        Sum<2> sum;
#pragma unroll
        for (int i = 0; i < DK / 32; ++i) {
          if constexpr (F32) {
            sum.template add<1, 1>(key_frag(tile_row(2 * ks + t, r), i), q[i]);
          } else {
            sum.s[i % 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key_frag(tile_row(2 * ks + t, r), i).p[0], q[i].p[0], sum.s[i % 2], 0, 0, 0);
          }
        }
        const f32x4 qk = sum.total();
        const int key = 32 * ks + 8 * g + 4 * t;
        const f32x4 behind = *reinterpret_cast<const f32x4 *>(s.behind + key);
        const f32x4 same = *reinterpret_cast<const f32x4 *>(&s.d[wave][r][key % 16]);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[ks][4 * t + i] = key + i > query ? 0.f : qk[i] * (block == wave ? same[i] : mid * behind[i]);
      }
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      if (ks <= wave / 2)
        store_frag<true, kPlanes>(head + space.kSolve + (size_t)(first_frag(wave) + ks) * kPiecesOf<true, kPlanes> * space.kPiece, lane, p[ks]);
  }
  if (threadIdx.x < kChunk) {
    reinterpret_cast<float *>(head + space.kDecay)[threadIdx.x] = s.decay[threadIdx.x];
    reinterpret_cast<float *>(head + space.kRest)[threadIdx.x] = s.rest[threadIdx.x];
  }

  if (h % group == 0) {
    unsigned char *keys = space.keys(slot, kh);
#pragma unroll
    for (int ks = 0; ks < DK / 32; ++ks)
#pragma unroll
      for (int j = 0; j < kPiecesOf<F32, 1>; ++j) {
        const size_t at = (((size_t)wave * (DK / 32) + ks) * kPiecesOf<F32, 1> + j) * space.kPiece + lane * 16;
        *reinterpret_cast<u32x4 *>(keys + space.kRows + at) =
            reinterpret_cast<const u32x4 *>(s.k + tile_row(wave, r) * L::kKeyPitch + 32 * ks + 8 * g)[j];
        *reinterpret_cast<u32x4 *>(keys + 2 * space.kRows + at) = reinterpret_cast<const u32x4 *>(&q[ks])[j];
      }
    for (int f = wave; f < DK / 16 * 2; f += kThreads / kWave) {
      const T *from = s.k + (32 * (f % 2) + 8 * g) * L::kKeyPitch + tile_row(f / 2, r);
      unsigned char *to = keys + (size_t)f * kPiecesOf<F32, 1> * space.kPiece;
      if constexpr (F32) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from[e * L::kKeyPitch];
        store_frag<true, 1>(to, lane, x);
      } else {
        uint32_t x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from[e * L::kKeyPitch].bits;
        *reinterpret_cast<uint4 *>(to + lane * 16) =
            make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
      }
    }
  }

  if constexpr (DELTA) {
    // L: the 12 tiles up to the ones right of the diagonal, which the operands reach
    // (those are zeros); three to a wave
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x4 low[3];
    int ti[3], tj[3];
#pragma unroll
    for (int n = 0; n < 3; ++n) {
      const int tile = 3 * wave + n;  // (0, 0) (0, 1) (1, 0) (1, 1) (2, 0) .. (2, 3) (3, 0) .. (3, 3)
      ti[n] = tile < 4 ? tile / 2 : tile / 4 + 1;
      tj[n] = tile < 4 ? tile % 2 : tile % 4;
      Sum<1> sum;
#pragma unroll
      for (int ks = 0; ks < DK / 32; ++ks) sum.template add<1, 1>(key_frag(16 * ti[n] + r, ks), key_frag(16 * tj[n] + r, ks));
      const f32x4 kk = sum.total();
      float behind = s.behind[16 * tj[n] + r];
      behind *= ti[n] - tj[n] > 1 ? s.total[tj[n] + 1 & 3] : 1.f;
      behind *= ti[n] - tj[n] > 2 ? s.total[tj[n] + 2 & 3] : 1.f;
      const int row = 16 * ti[n] + 4 * g, col = 16 * tj[n] + r;
      const f32x4 beta = *reinterpret_cast<const f32x4 *>(s.beta + row), upto = *reinterpret_cast<const f32x4 *>(s.upto + row);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float d = ti[n] == tj[n] ? s.d[ti[n]][4 * g + i][r] : upto[i] * behind;
        low[n][i] = row + i <= col ? 0.f : beta[i] * d * kk[i];
      }
    }
    lds_barrier();  // every wave is done with the keys
#pragma unroll
    for (int n = 0; n < 3; ++n) block_store(s.x, ti[n], tj[n], g, r, low[n]);
    lds_barrier();
    {  // diagonal blocks: column r by forward substitution, in every 16 lanes alike
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = i == r ? 1.f : 0.f;
#pragma unroll
      for (int p = 0; p < 4; ++p) {  // four columns of L: what is known of x goes to all rows below at once
        f32x4 l[16];
#pragma unroll
        for (int i = 4 * p + 1; i < 16; ++i)
          l[i] = *reinterpret_cast<const f32x4 *>(s.x + (16 * wave + i) * kPitch + 16 * wave + 4 * p);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 4 * p + 1; i < 16; ++i)
            if (i > 4 * p + j) x[i] = __builtin_fmaf(-l[i][j], x[4 * p + j], x[i]);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i / 4 == g) s.x[(16 * wave + i) * kPitch + 16 * wave + r] = x[i];
    }
    lds_barrier();
    if (wave < 2) {  // X10 = -X11 L10 X00, X32 likewise
      const int b = 2 * wave;
      const f32x4 y = block_mma(block_a(s.x, b + 1, b, g, r), block_b(s.x, b, b, g, r), zero);
      block_store(s.x, b + 1, b, g, r, -block_mma(block_a(s.x, b + 1, b + 1, g, r), y, zero));
    }
    lds_barrier();
    f32x4 y2 = zero, y3 = zero;  // rows 2, 3 of L X, column `wave`
    if (wave < 2) {
      for (int m = wave; m < 2; ++m) {
        const f32x4 x = block_b(s.x, m, wave, g, r);
        y2 = block_mma(block_a(s.x, 2, m, g, r), x, y2);
        y3 = block_mma(block_a(s.x, 3, m, g, r), x, y3);
      }
    }
    lds_barrier();
    if (wave < 2) {
      block_store(s.x, 2, wave, g, r, -block_mma(block_a(s.x, 2, 2, g, r), y2, zero));
      block_store(s.x, 3, wave, g, r,
                  -block_mma(block_a(s.x, 3, 3, g, r), y3, block_mma(block_a(s.x, 3, 2, g, r), y2, zero)));
    }
    lds_barrier();
    // out: row tile `wave` as the second kernel's operand
    for (int ks = 0; ks <= wave / 2; ++ks) {
      const int at = 32 * ks + 8 * g;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s.x[tile_row(wave, r) * kPitch + at + e] * s.beta[at + e];
      store_frag<F32, kPlanes>(head + (size_t)(first_frag(wave) + ks) * kPiecesOf<F32, kPlanes> * space.kPiece, lane, x);
    }
  }
}

// ----------------------------------------------------------- second kernel
// One workgroup = one (sequence, head) and 16 NT columns of its state, which stay
// in the accumulators of four waves from the first chunk to the last: wave w has
// the row tiles w, w + 4, .. of d_k and the token tile w.  These waves do what the
// next state waits for: K H, R, the corrected values, the update.  Four others, one
// on the same SIMD as each, make the outputs from the same operands in LDS, in the
// time the first ones wait for one another: three barriers a chunk.  What comes
// from memory is asked for as soon as the chunk before has used its registers.
//
// The chain of chunks bounds one long sequence: 512 chunks, 16 heads of 128, 842 us or
// 3950 cycles a chunk: three products from LDS, their planes made and put back, the
// barriers, and waits for loads (with planes that were cut, 815 us in all: 870 without
// `touch` below, 617 with every chunk's lines the same, 532 with no loads).  Many
// sequences are bound by LDS, vector ALUs and matrix cores in turn (59, 51 and 47%
// busy): 32 sequences of up to 2048 tokens, 32 heads, 537 chunks in 605 us with two
// workgroups to a CU (a tenth less with two planes for the outputs; four column tiles to
// a workgroup and one were a tenth and half as much again slower).  fp32 activations are
// bound by the vector ALUs, busy 64%, which cut operands into planes (152 chunks of 12
// heads of 64 x 80 in 61 us; 80 with fp32 matrix instructions).
//
// Columns: lane r of column tile n has the column 32 (n / 2) + 8 (r / 4) + 4 (n % 2)
// + r % 4 of the slab, so that an output tile, made transposed, gives each lane 8
// neighbouring columns of a token.
template <bool F32, int DK, int NT>
struct StateLds {
  static constexpr size_t kFrag = (size_t)kPlanes * kWave * 16;
  static constexpr int kStateFrags = DK / 32 * NT, kRowFrags = 2 * NT;
  // H, V - G o (K H), D_63 o U, U
  static constexpr size_t kBytes = (kStateFrags + 3 * kRowFrags) * kFrag;
};

// half `half` (4 of 8 values) of a lane's operand
template <int N>
__device__ __forceinline__ void put_half(unsigned char *frag, int half, int lane, f32x4 x) {
  const float v[4] = {x[0], x[1], x[2], x[3]};
  uint2 p[N];
  split4(v, p);
#pragma unroll
  for (int n = 0; n < N; ++n) *reinterpret_cast<uint2 *>(frag + (n * kWave + lane) * 16 + 8 * half) = p[n];
}

template <int N>
__device__ __forceinline__ Frag<false, N> get_frag(const unsigned char *frag, int lane) {
  Frag<false, N> f;
#pragma unroll
  for (int n = 0; n < N; ++n) f.p[n] = *reinterpret_cast<const bf16x8 *>(frag + (n * kWave + lane) * 16);
  return f;
}

template <typename P>
__device__ __forceinline__ P load_piece(rsrc_t r, uint32_t voff, uint32_t soff) {
  return __builtin_bit_cast(P, __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, kPolicyDefault));
}

// The order of a phase: reads of operands from LDS run `AHEAD` operands in front of
// the `FRAGS` ones' products, R reads and M matrix instructions each, and LOADS loads
// from memory go in between, evenly: issued in a row, they would hold up the wave.
template <int AHEAD, int R, int M, int FRAGS, int LOADS = 0, int F = 0>
__device__ __forceinline__ void pace() {
  constexpr int kFirst = AHEAD < FRAGS ? AHEAD : FRAGS, kLoads = LOADS * (F + 1) / FRAGS - LOADS * F / FRAGS;
  if constexpr (F == 0) __builtin_amdgcn_sched_group_barrier(0x100, R * kFirst, 0);
  if constexpr (kLoads > 0) __builtin_amdgcn_sched_group_barrier(0x020, kLoads, 0);
  __builtin_amdgcn_sched_group_barrier(0x008, M, 0);
  if constexpr (F + kFirst < FRAGS) __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  if constexpr (F + 1 < FRAGS) pace<AHEAD, R, M, FRAGS, LOADS, F + 1>();
}

// matrix instructions of one product of N planes with an activation
template <bool F32, int N>
constexpr int kMfma = F32 ? 6 : N;

constexpr int kStateThreads = 512;
// of the state kernel: two workgroups to a CU where their registers hold the operands
template <bool F32, int DK, int NT>
constexpr int kWavesPerSimd = NT > 1 && DK <= (F32 ? 64 : 128) ? 4 : 2;
constexpr uint32_t kNowhere = 0x40000000u;  // an offset past any chunk's rows: reads give 0

// What a chunk reads of a tensor, as a descriptor that moves on by a constant from
// chunk to chunk.  Past the sequence's last row and last chunk it reads zeros,
// without a branch and without memory.
struct ChunkRows {
  const unsigned char *at;
  int64_t step;
  uint32_t whole, part;
  int last;
  __device__ __forceinline__ rsrc_t next(int c) {
    const rsrc_t r = make_rsrc(at, c < last ? whole : c == last ? part : 0u);
    at += step;
    return r;
  }
};

template <bool F32, int DK, int NT, bool DELTA>
__global__ __launch_bounds__(kStateThreads) __attribute__((amdgpu_waves_per_eu(kWavesPerSimd<F32, DK, NT>, kWavesPerSimd<F32, DK, NT>))) void state_kernel(PrefillArgs a, int slabs) {
  using T = typename std::conditional<F32, float, bf16>::type;
  using L = StateLds<F32, DK, NT>;
  using Piece = typename Frag<F32, 1>::Piece;
  constexpr int kKs = DK / 32, kTiles = DK / 64, w = sizeof(T);
  constexpr int kKeyPieces = kPiecesOf<F32, 1>, kSolvePieces = kPiecesOf<F32, kPlanes>, kMixPieces = kPiecesOf<true, kPlanes>;
  constexpr int kActs = F32 ? 3 : 1;  // planes of an activation
  constexpr int kParts = NT == 1 ? 3 : 1, kOutParts = NT == 1 ? 2 : 1;
  constexpr bool kTouch = kWavesPerSimd<F32, DK, NT> == 2;
  constexpr bool kTwoSets = NT == 1 && DK <= (F32 ? 64 : 128);
  constexpr int kAhead = NT == 1 ? 8 : 2;  // of the state's operands read in front of their products
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  unsigned char *const lds_h = lds, *const lds_r = lds + L::kStateFrags * L::kFrag, *const lds_u = lds_r + L::kRowFrags * L::kFrag,
                *const lds_o = lds_u + L::kRowFrags * L::kFrag;
  const ChunkSpace<F32, DK> space = chunk_space<F32, DK>(a);
  const int lane = threadIdx.x % kWave, role = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wave = role % 4;
  const int g = lane / 16, r = lane % 16;
  const int half = wave % 2;  // of the token tile `wave` in its pair

  // the slabs of a head, and neighbouring heads, one behind another on one XCD
  const unsigned wg = workgroup(), at = wg / kXcdCount;
  const unsigned place = at / (unsigned)slabs * kXcdCount + wg % kXcdCount;
  const int slab = (int)(at % (unsigned)slabs);
  if (place >= (unsigned)space.walks * (unsigned)a.H) return;
  const int number = (int)(place / (unsigned)a.H), h = (int)(place % (unsigned)a.H), kh = h / (a.H / a.Hk);
  if (number >= __builtin_amdgcn_readfirstlane(*space.walk_count())) return;
  const Walk walk = *space.walk(number);
  const int b = __builtin_amdgcn_readfirstlane(walk.b), start = __builtin_amdgcn_readfirstlane(walk.start),
            len = __builtin_amdgcn_readfirstlane(walk.len);
  const size_t unit = (size_t)b * a.H + h;
  const int chunks = (len + kChunk - 1) / kChunk, last = chunks - 1, tail = len - last * kChunk;
  const size_t slot0 = (size_t)__builtin_amdgcn_readfirstlane(walk.slot);
  auto rows_of = [&](const void *p, int64_t stride, size_t first, int width) {
    return ChunkRows{reinterpret_cast<const unsigned char *>(static_cast<const T *>(p) + start * stride + first),
                     kChunk * stride * w, (uint32_t)((kChunk - 1) * (int)stride + width) * w,
                     (uint32_t)((tail - 1) * (int)stride + width) * w, last};
  };
  ChunkRows head_rows = {space.head(slot0, h), (int64_t)(a.H * space.kHead), (uint32_t)space.kHead, (uint32_t)space.kHead, last};
  ChunkRows key_rows = {space.keys(slot0, kh), (int64_t)(a.Hk * space.kKeys), (uint32_t)space.kKeys, (uint32_t)space.kKeys, last};
  constexpr int kHeadLines = ChunkSpace<F32, DK>::kHead / 128, kLines = kHeadLines + ChunkSpace<F32, DK>::kKeys / 128;
  const int t0 = first_frag(wave);
  constexpr uint32_t kDecay = ChunkSpace<F32, DK>::kDecay, kRest = ChunkSpace<F32, DK>::kRest;
  constexpr uint32_t kPiece = ChunkSpace<F32, DK>::kPiece, kRows = ChunkSpace<F32, DK>::kRows;

  if (role < 4) {
    int col[NT];  // this lane's columns as an operand's row
#pragma unroll
    for (int n = 0; n < NT; ++n) col[n] = slab * 16 * NT + (NT == 1 ? r : 32 * (n / 2) + 8 * (r / 4) + 4 * (n % 2) + r % 4);
    // the state's row i of tile m is at h_off + (64 m + i) rows (columns past its own, and no state, read as zeros)
    uint32_t h_off[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) h_off[n] = col[n] < a.dv ? (uint32_t)(tile_row(wave, 4 * g) * a.dv + col[n]) * 4 : kNowhere;
    const size_t state_at = unit * DK * a.dv;
    const rsrc_t state_in = make_rsrc(a.state ? a.state + state_at : nullptr, a.state ? (uint32_t)DK * a.dv * 4 : 0u);
    f32x4 H[kTiles][NT];
#pragma unroll
    for (int m = 0; m < kTiles; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          H[m][n][i] = buf_load_f32<kPolicyDefault>(state_in, h_off[n], (uint32_t)((64 * m + i) * a.dv) * 4);

    ChunkRows v_rows = rows_of(a.v, a.v_stride, (size_t)h * a.dv, a.dv);
    uint32_t v_off[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
      v_off[n] = col[n] < a.dv ? (uint32_t)(tile_row(wave, 4 * g) * (int)a.v_stride + col[n]) * w : kNowhere;
    struct Operands {
      Frag<F32, 1> kf[kKs], key[kTiles][2];
      Frag<F32, kPlanes> ts[2];
      uint32_t vr[NT][4];
      f32x4 gr, gu;  // decays of the rows 4 g + i, and behind them
      float gc;      // of the whole chunk
    };
    auto load_k = [&](Operands &x, rsrc_t rs) {
#pragma unroll
      for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
        for (int j = 0; j < kKeyPieces; ++j)
          x.kf[ks].p[j] = load_piece<Piece>(rs, lane * 16 + j * kPiece, kRows + (wave * kKs + ks) * kKeyPieces * kPiece);
    };
    auto load_v = [&](Operands &x, int c, rsrc_t head) {
      const rsrc_t rs = v_rows.next(c);
      if (DELTA) x.gr = load_piece<f32x4>(head, tile_row(wave, 4 * g) * 4, kDecay);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t row = (uint32_t)(i * (int)a.v_stride * w);
          x.vr[n][i] = F32 ? __builtin_amdgcn_raw_buffer_load_b32(rs, v_off[n], row, kPolicyDefault)
                         : (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(rs, v_off[n], row, kPolicyDefault);
        }
    };
    auto load_decay = [&](Operands &x, rsrc_t rs) {
      x.gu = load_piece<f32x4>(rs, tile_row(wave, 4 * g) * 4, kRest);
      x.gc = buf_load_f32<kPolicyDefault>(rs, (kChunk - 1) * 4, kDecay);
    };
    auto load_matrix = [&](Operands &x, rsrc_t head) {  // row tiles 0 and 1 have no second inner 32
      const rsrc_t more = wave < 2 ? make_rsrc(head_rows.at, 0u) : head;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int j = 0; j < kSolvePieces; ++j)
          x.ts[ks].p[j] = load_piece<Piece>(ks ? more : head, lane * 16 + j * kPiece, (t0 + ks) * kSolvePieces * kPiece);
    };
    auto load_keys = [&](Operands &x, rsrc_t rs) {
#pragma unroll
      for (int m = 0; m < kTiles; ++m)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int j = 0; j < kKeyPieces; ++j)
            x.key[m][ks].p[j] = load_piece<Piece>(rs, lane * 16 + j * kPiece, ((wave + 4 * m) * 2 + ks) * kKeyPieces * kPiece);
    };
    auto put_state = [&](int m) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
        put_half<kPlanes>(lds_h + (size_t)((wave + 4 * m) / 2 * NT + n) * L::kFrag, half, lane, H[m][n]);
    };

    // One chunk, from the operands `x`; the next one's go to `y`.  Where registers
    // allow two sets, the loads lie between the products, a whole chunk ahead;
    // else they follow the last use of their registers.
    constexpr int kKeyLoads = 2 * kTiles * kKeyPieces, kRowLoads = kKs * kKeyPieces + 4 * NT + 1, kSolveLoads = 2 * kSolvePieces + 2;
    auto step = [&](int c, Operands &x, Operands &y) {
      lds_barrier();
      const rsrc_t head = head_rows.next(c + 1), keys = key_rows.next(c + 1);
      f32x4 u[NT];  // V - G o (K H), then U
      if constexpr (DELTA) {
        Sum<kParts> sum[NT];
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            sum[n].template add<kActs, kPlanes>(planes(x.kf[ks]), get_frag<kPlanes>(lds_h + (size_t)(ks * NT + n) * L::kFrag, lane));
        if (kTwoSets) {
          load_k(y, keys);
          load_v(y, c + 1, head);
        }
        pace<kAhead, kPlanes, kMfma<F32, 3>, kKs * NT, kTwoSets ? kRowLoads : 0>();
        __builtin_amdgcn_sched_barrier(0);
        if (!kTwoSets) load_k(y, keys);
#pragma unroll
        for (int n = 0; n < NT; ++n) u[n] = sum[n].total();
      } else if (kTwoSets) {
        load_v(y, c + 1, head);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = __uint_as_float(F32 ? x.vr[n][i] : x.vr[n][i] << 16);
          u[n][i] = DELTA ? __builtin_fmaf(-x.gr[i], u[n][i], v) : v;
        }
        if (DELTA) put_half<kPlanes>(lds_r + (size_t)(wave / 2 * NT + n) * L::kFrag, half, lane, u[n]);
      }
      if (!kTwoSets) load_v(y, c + 1, head);
      if constexpr (DELTA) {
        lds_barrier();
        Sum<kParts> sum[NT];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            sum[n].template add<kPlanes, kPlanes>(planes(x.ts[ks]), get_frag<kPlanes>(lds_r + (size_t)(ks * NT + n) * L::kFrag, lane));
        if (kTwoSets) {
          load_matrix(y, head);
          load_decay(y, head);
        }
        pace<2, kPlanes, 6, 2 * NT, kTwoSets ? kSolveLoads : 0>();
        __builtin_amdgcn_sched_barrier(0);
        if (!kTwoSets) load_matrix(y, head);
#pragma unroll
        for (int n = 0; n < NT; ++n) u[n] = sum[n].total();
      } else if (kTwoSets) {
        load_decay(y, head);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        put_half<kPlanes>(lds_u + (size_t)(wave / 2 * NT + n) * L::kFrag, half, lane, x.gu * u[n]);
        put_half<kPlanes>(lds_o + (size_t)(wave / 2 * NT + n) * L::kFrag, half, lane, u[n]);
      }
      const float whole = x.gc;
      if (!kTwoSets) load_decay(y, head);
      lds_barrier();
      Sum<kParts> next[kTiles][NT];
#pragma unroll
      for (int m = 0; m < kTiles; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) next[m][n].s[0] = H[m][n] * whole;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const Frag<false, kPlanes> uf = get_frag<kPlanes>(lds_u + (size_t)(ks * NT + n) * L::kFrag, lane);
#pragma unroll
          for (int m = 0; m < kTiles; ++m) next[m][n].template add<kActs, kPlanes>(planes(x.key[m][ks]), uf);
        }
      if (kTwoSets) load_keys(y, keys);
      pace<2, kPlanes, kTiles * kMfma<F32, 3>, 2 * NT, kTwoSets ? kKeyLoads : 0>();
      __builtin_amdgcn_sched_barrier(0);
      if (!kTwoSets) load_keys(y, keys);
#pragma unroll
      for (int m = 0; m < kTiles; ++m) {
#pragma unroll
        for (int n = 0; n < NT; ++n) H[m][n] = next[m][n].total();
        put_state(m);
      }
    };

    __builtin_amdgcn_s_setprio(2);
    Operands even;
    {
      const rsrc_t head = head_rows.next(0), keys = key_rows.next(0);
      if (chunks > 0) {
        if (DELTA) load_k(even, keys);
        load_v(even, 0, head);
        if (DELTA) load_matrix(even, head);
        load_decay(even, head);
        load_keys(even, keys);
      }
    }
#pragma unroll
    for (int m = 0; m < kTiles; ++m) put_state(m);
    if constexpr (kTwoSets) {
      Operands odd;
      int c = 0;
      for (; c + 1 < chunks; c += 2) {  // (with no branch between the two, which would wait for all loads)
        step(c, even, odd);
        step(c + 1, odd, even);
      }
      if (c < chunks) step(c, even, odd);
    } else {
      for (int c = 0; c < chunks; ++c) step(c, even, even);
    }
    const rsrc_t state_out = make_rsrc(a.state_out + state_at, (uint32_t)DK * a.dv * 4);
#pragma unroll
    for (int m = 0; m < kTiles; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          buf_store_f32<kPolicyDefault>(H[m][n][i], state_out, h_off[n], (uint32_t)((64 * m + i) * a.dv) * 4);
  } else {
    // lane: token 16 wave + r, columns 4 g + i of each tile
    const int token = 16 * wave + r;
    T *out = static_cast<T *>(a.out) + ((size_t)(start + token) * a.H + h) * a.dv + slab * 16 * NT + (NT == 1 ? 4 : 8) * g;
    const size_t out_step = (size_t)kChunk * a.H * a.dv;
    Frag<F32, 1> qf[kKs];
    Frag<true, kPlanes> to[2];
    float gq;  // decay of the token
    auto load_q = [&](int c) {
      const rsrc_t rs = key_rows.next(c);
#pragma unroll
      for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
        for (int j = 0; j < kKeyPieces; ++j)
          qf[ks].p[j] = load_piece<Piece>(rs, lane * 16 + j * kPiece, 2 * kRows + (wave * kKs + ks) * kKeyPieces * kPiece);
    };
    auto load_matrix = [&](int c) {
      const rsrc_t rs = head_rows.next(c), more = wave < 2 ? make_rsrc(head_rows.at, 0u) : rs;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int j = 0; j < kMixPieces; ++j)
          to[ks].p[j] = load_piece<f32x4>(ks ? more : rs, lane * 16 + j * kPiece,
                                          ChunkSpace<F32, DK>::kSolve + (t0 + ks) * kMixPieces * kPiece);
      gq = buf_load_f32<kPolicyDefault>(rs, token * 4, kDecay);
    };
    // Where one workgroup has a CU, nothing else runs while its loads take their time.
    // The lines that the head's workgroups will read two chunks on are brought to the
    // L2 by one load a wave, whose bytes nothing looks at: a part of the operands by
    // each workgroup, and its own values.  (Every wave loads every time, past the end
    // the last line again: a load that may not be there makes others wait for all.)
    const int line = min((wave * kWave + lane) * slabs + slab, kLines - 1);
    const bool of_head = line < kHeadLines;
    const unsigned char *const lines = of_head ? space.head(slot0, h) + (size_t)line * 128
                                               : space.keys(slot0, kh) + (size_t)(line - kHeadLines) * 128;
    const size_t line_step = of_head ? a.H * space.kHead : a.Hk * space.kKeys;
    const T *const values = static_cast<const T *>(a.v) + start * a.v_stride + (size_t)h * a.dv + min(slab * 16 * NT, a.dv - 16);
    uint32_t seen[2] = {};
    auto touch = [&](int c) {
      if (!kTouch) return;
      asm volatile("" ::"v"(seen[0]), "v"(seen[1]));  // the last ones' use: a chunk later they are there
      seen[0] = *reinterpret_cast<const uint32_t *>(lines + min(c, last) * line_step);
      seen[1] = *reinterpret_cast<const uint32_t *>(values + (int64_t)min(c * kChunk + 16 * wave + r, len - 1) * a.v_stride);
    };
    if (chunks > 0) {
      load_q(0);
      load_matrix(0);
      touch(1);
    }
    for (int c = 0; c < chunks; ++c) {
      lds_barrier();
      Sum<kOutParts> sum[NT];
#pragma unroll
      for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          sum[n].template add<kPlanes, kActs>(get_frag<kPlanes>(lds_h + (size_t)(ks * NT + n) * L::kFrag, lane), planes(qf[ks]));
      pace<kAhead, kPlanes, kMfma<F32, 3>, kKs * NT>();
      __builtin_amdgcn_sched_barrier(0);
      if (DELTA) lds_barrier();
      load_q(c + 1);
      const Frag<false, kPlanes> mix[2] = {planes(to[0]), planes(to[1])};  // while the others make the corrected values
      const float since = gq;
      __builtin_amdgcn_sched_barrier(0);
      load_matrix(c + 1);
      lds_barrier();
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < kOutParts; ++i) sum[n].s[i] *= since;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          sum[n].template add<kPlanes, kPlanes>(get_frag<kPlanes>(lds_o + (size_t)(ks * NT + n) * L::kFrag, lane), mix[ks]);
      f32x4 o[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) o[n] = sum[n].total();
      touch(c + 2);
      if (token < len - c * kChunk) {
        if constexpr (NT == 1) {
          const float x[4] = {o[0][0], o[0][1], o[0][2], o[0][3]};
          store4(out, x);
        } else {
#pragma unroll
          for (int n = 0; n < NT; n += 2) {
            const float x[8] = {o[n][0], o[n][1], o[n][2], o[n][3], o[n + 1][0], o[n + 1][1], o[n + 1][2], o[n + 1][3]};
            if (slab * 16 * NT + 16 * n + 8 * g < a.dv) store8(out + 16 * n, x);
          }
        }
      }
      out += out_step;
    }
    asm volatile("" ::"v"(seen[0]), "v"(seen[1]));
  }
}

// lets a kernel have more than 64 KiB of LDS
template <typename K>
hipError_t allow_lds(K kernel, size_t bytes) {
  if (bytes <= (64u << 10)) return hipSuccess;
  return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <bool F32, int DK, int NT, bool DELTA>
hipError_t launch_states(const PrefillArgs &a, hipStream_t s) {
  using L = StateLds<F32, DK, NT>;
  const auto second = state_kernel<F32, DK, NT, DELTA>;
  const hipError_t e = allow_lds(second, L::kBytes);
  if (e != hipSuccess) return e;
  const int slabs = (a.dv + 16 * NT - 1) / (16 * NT);
  const uint64_t units = ((uint64_t)most_longer(a.rows, a.serial_len) * a.H + kXcdCount - 1) / kXcdCount * kXcdCount;
  hipLaunchKernelGGL(second, grid_of(units * slabs), dim3(kStateThreads), L::kBytes, s, a, slabs);
  return hipGetLastError();
}

template <bool F32, int DK, bool DELTA>
hipError_t launch_family(const PrefillArgs &a, hipStream_t s) {
  using M = MatricesLds<F32, DK>;
  const auto first = matrices_kernel<F32, DK, DELTA>;
  hipError_t e = allow_lds(first, sizeof(M));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(first, grid_of((uint64_t)chunk_slots<kChunk>(a.rows, a.serial_len, a.window) * a.H), dim3(kThreads), sizeof(M), s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  // 16 columns of a state to a workgroup where 32 leave half of the CUs without one
  const int64_t wide = most_longer(a.rows, a.serial_len) * a.H * ((a.dv + 31) / 32);
  return wide <= device_cus() / 2 ? launch_states<F32, DK, 1, DELTA>(a, s) : launch_states<F32, DK, 2, DELTA>(a, s);
}

}  // namespace

template <bool F32, int DK>
hipError_t launch_chunks(const PrefillArgs &a, hipStream_t s) {
  return a.family == SLA_FAMILY_DECAY ? launch_family<F32, DK, false>(a, s) : launch_family<F32, DK, true>(a, s);
}

template hipError_t launch_chunks<SLA_CHUNK_F32, SLA_CHUNK_DK>(const PrefillArgs &a, hipStream_t s);

}  // namespace sla
