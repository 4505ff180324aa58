// attn_verify.hip -- attention of a draft's nodes over the paged cache:
//     o_j = sum_i p_ji v_i,  p_j = softmax_i(scale q_j . k_i),
// i over the committed rows and the nodes of j's root path.
//
// A kv head's queries are the rows r = node * G + g (G query heads to a kv
// head): all of them read the same keys.  A workgroup takes 16 to 256 rows of
// one kv head and a part of the keys, walks that in tiles of 16 KB of keys and
// 16 KB of values that it stages in LDS, and keeps the running maximum and sum of
// every row's softmax, so that the keys and values are read once (once for each
// block of rows, back to back on one XCD, whose L2 they then come from).  A
// sequence whose keys are divided over workgroups leaves unnormalised outputs and
// statistics in the workspace, and a second kernel joins them.
//
// What bounds it: for one token or few rows the cache's bytes, 256 sequences of
// up to 16384 keys 372 us, 5.8 TB/s.  For many rows no one unit: the waves of a
// SIMD wait for one another between products, exponentials and fragment reads.
// 64-node trees over up to 8192 keys with heads of 256 take 424 us, 830 TFLOP/s,
// the matrix cores busy 44% of the time and the LDS 27%; a 32-node tree over
// 131072 keys 54.8 us, 37% and 23%.  For short work it is the chain of loads that a
// workgroup starts with (length, page, rows) and the second launch, one token over
// 1000 keys 9.1 us.  (States in turn, the card warm.)
//
// On the matrix cores the scores are formed transposed, S^T = K Q^T: a lane
// of v_mfma_f32_16x16x32_bf16 then holds four consecutive keys of one query,
// which is what the B operand of O^T = V^T P^T takes, so the weights go from
// one product to the next within the lane, and a row's statistics are one
// value per lane.  V^T comes out of the row-major tile by ds_read_b64_tr_b16.
// fp32 activations use v_mfma_f32_16x16x4_f32 in the same arrangement, with
// exact products.
#include <algorithm>

#include "attn_device.hpp"

namespace sla {
namespace {

constexpr int kThreads = 256;       // of the join kernel
constexpr int kQueries = 16;        // queries of one matrix tile
// Equal parts (see Split): tiles of a workgroup from which they pay, the fewest
// workgroups for a kv head and block of queries that still fill the chip, and the
// tiles whose time a sequence's start takes (32 sequences of up to 3001 keys and
// 40-node trees in fp32: 148 us if it counted for none, 142 us).
constexpr int kLongWork = 40, kFewWorkers = 8, kStart = 2;
constexpr float kSlack = 8.f;       // how far, in powers of two, a score may pass its softmax's reference
constexpr float kNoScore = -3e38f;  // the reference before the first visible key

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(4))) int32_t const_int;  // read by scalar loads

// A tile of keys and values in LDS, 16 KB each, so that two of them and two
// workgroups fit a CU.  A wave fills it 1 KB at a time, 16 bytes a lane.  Piece
// c of row r lies at piece c ^ swizzle(r) of its row, so that a wave's fragment
// reads spread over the banks: 16 rows of one piece for K; for V four rows of
// two (bf16) or four (fp32) neighbouring ones.
template <typename T, int D>
struct Tile {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kRow = D * (int)sizeof(T);  // bytes of a row
  static constexpr int kBytes = 16384;
  static constexpr int kKeys = kBytes / kRow;
  static constexpr int kCols = kRow / 16;        // pieces of a row
  static constexpr int kLoads = kBytes / 1024;   // loads of a wave that fill the tile
  static constexpr int kLoadRows = 1024 / kRow;  // rows of one of them, 1..8
  static_assert(kLoadRows >= 1 && kLoadRows <= 8, "a load stays in one page");
  __host__ __device__ static constexpr int swizzle_k(int r) { return kRow >= 256 ? r % 16 : r / 2 % 8; }
  __host__ __device__ static constexpr int swizzle_v(int r) {
    return !kBf16 ? r & 12 : kRow >= 256 ? r * 2 % 16 : r & 6;
  }
};

// How a launch's keys are divided.  Either every sequence has as many ranges of
// whole tiles as its length asks for, one to a workgroup, so that the ranges of a
// batch are about equally long: the tiles of all sequences over `share`, at
// least, is a range's most, and `parts` bounds how many there are.  Or (workers >
// 0) the tiles of all sequences, one behind the other, are cut into `workers`
// equal parts, and a workgroup may end one sequence and begin the next: no
// workgroup has more to do than another, but a sequence's start costs some of
// them a second time what it costs to begin.  share and workers 0: a workgroup a
// sequence, and no workspace.
//
// The workspace has room for the parts of divided sequences alone, `slots` of
// them; a sequence that one workgroup has to itself goes straight to the output.
//   Ranges, fine: one each.
//   Ranges, by `share`: a divided sequence of t tiles in ranges of m < t has fewer
//   than 2 t / m of them, and all tiles over m are at most `share`: 2 share.
//   Equal parts: a worker may go on with one sequence that another began, the slot
//   of its number, and begin one that another goes on with, a slot behind those by
//   the sequence's number or, if there are fewer of them, by the worker's.
struct Split {
  int share, parts;
  bool fine;  // as many ranges as `parts` allows, rather than as few as `share` asks for
  int workers;
  int slots;
  __host__ __device__ bool divided() const { return share > 0 || workers > 0; }
  // the first part of sequence b, whose first range or worker is `first`
  __host__ __device__ int first_slot(int first, int b, int B) const {
    return workers == 0 ? first : workers + (B <= workers ? b : first);
  }
};

// A query fragment: the B operand of S^T = K Q^T for 16 queries.
template <typename T, int D>
struct Frag;
template <int D>
struct Frag<bf16, D> {
  bf16x8 x[D / 32];
};
template <int D>
struct Frag<float, D> {
  f32x4 x[D / 16];
};

// x without its infinite and NaN elements; `found` is set if there were any.
__device__ __forceinline__ u32x4 finite_part(u32x4 x, bool &found, bf16) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (x[i] & 0x7f80u) == 0x7f80u, hi = (x[i] & 0x7f800000u) == 0x7f800000u;
    found |= lo || hi;
    x[i] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
  }
  return x;
}
__device__ __forceinline__ u32x4 finite_part(u32x4 x, bool &found, float) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool bad = (x[i] & 0x7f800000u) == 0x7f800000u;
    found |= bad;
    if (bad) x[i] = 0;
  }
  return x;
}

// four consecutive activations
__device__ __forceinline__ f32x4 load4(const bf16 *p) {
  const uint2 x = *reinterpret_cast<const uint2 *>(p);
  return f32x4{__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
               __uint_as_float(x.y & 0xffff0000u)};
}
__device__ __forceinline__ f32x4 load4(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }

// The workspace of a split launch: unnormalised outputs [Hkv][slots][R][D],
// their reference and sum [Hkv][slots][R], each sequence's first part (the number
// of its range or worker) and how many it has [B], each part's error [slots].
__host__ __device__ inline size_t split_rows(const AttnVerifyArgs &a, const Split &s, int R) {
  return (size_t)a.cache.Hkv * s.slots * R;
}
__device__ __forceinline__ float2 *split_stats(const AttnVerifyArgs &a, const Split &s, int R) {
  return reinterpret_cast<float2 *>(static_cast<float *>(a.workspace) + split_rows(a, s, R) * a.cache.D);
}
__device__ __forceinline__ int2 *split_parts(const AttnVerifyArgs &a, const Split &s, int R) {
  return reinterpret_cast<int2 *>(split_stats(a, s, R) + split_rows(a, s, R));
}
__device__ __forceinline__ int32_t *split_errors(const AttnVerifyArgs &a, const Split &s, int R) {
  return reinterpret_cast<int32_t *>(split_parts(a, s, R) + a.B);
}

// Sum over the lanes up to this one, by rows of 16, then across them.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast 31 into rows 2 and 3
  return x;
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), kWave - 1); }

__device__ __forceinline__ uint64_t uniform64(uint64_t x) {
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)x) |
         (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}

// x / d; in 32 bits for all but the largest batches
__device__ __forceinline__ uint64_t quotient(uint64_t x, uint32_t d) {
  return x >> 32 ? x / d : (uint32_t)x / d;
}

// A sequence's tiles of keys (one, if its length is bad, to tell of that).
template <int KEYS>
__device__ __forceinline__ int tiles_of(const AttnVerifyArgs &a, int len) {
  return length_ok(a.rows, a.cache.page_shift, len, a.n) && len <= a.max_len ? (len + a.n + KEYS - 1) / KEYS : 1;
}

struct Range {
  int b, part, parts, first;  // the sequence, which of its ranges, how many, the slot of the first
};

// The range number `item` of a launch: false if there are fewer.  All threads
// of a workgroup call it.  The longest range is the smallest of kTries lengths,
// from the tiles over `parts` to the tiles over `share`, that makes no more
// than `parts` of them; the last always does, for a sequence's last range is
// the only one that may be shorter.
template <int KEYS, int WAVES>
__device__ __forceinline__ bool pick_range(const AttnVerifyArgs &a, const Split &s, int item, Range &r) {
  constexpr int kTries = 4;
  __shared__ uint32_t sum_s[2][WAVES];
  __shared__ int count_s[kTries][WAVES], scan_s[2][WAVES];
  __shared__ Range found_s;
  auto tiles_of = [&](int b) { return sla::tiles_of<KEYS>(a, a.rows.len[b]); };
  auto over = [](int tiles, int most) { return (tiles + most - 1) / most; };
  if (s.share == 0) {
    r = Range{item, 0, 1, item};
    return item < a.B;
  }
  if (a.B == 1) {
    const int tiles = tiles_of(0);
    r = Range{0, item, over(tiles, over(tiles, s.parts)), 0};
    return item < r.parts;
  }
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int own = (a.B + WAVES * kWave - 1) / (WAVES * kWave);  // sequences of a thread
  const int b0 = min(tid * own, a.B), b1 = min(b0 + own, a.B);
  // (a batch's tiles pass 32 bits: summed by halves of 16)
  uint32_t low = 0, high = 0;
  for (int b = b0; b < b1; ++b) {
    const int t = tiles_of(b);
    low += t & 0xffff;
    high += t >> 16;
  }
  low = wave_sum(low);
  high = wave_sum(high);
  if (lane == 0) {
    sum_s[0][wave] = low;
    sum_s[1][wave] = high;
  }
  __syncthreads();
  unsigned long long sum = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) sum += sum_s[0][w] + ((unsigned long long)sum_s[1][w] << 16);
  int most[kTries], count[kTries] = {};
  // (2^30 tiles are more than a sequence has: with them each has one range)
  const int hi = (int)min((sum + s.share - 1) / s.share, 1ull << 30);
  const int lo = s.fine ? (int)((sum + s.parts - 1) / s.parts) : hi;
#pragma unroll
  for (int i = 0; i < kTries; ++i) most[i] = max(lo + (int)((long long)(hi - lo) * i / (kTries - 1)), 1);
  int divided = 0;  // ranges of this thread's divided sequences, by `share`
  for (int b = b0; b < b1; ++b) {
    const int t = tiles_of(b);
#pragma unroll
    for (int i = 0; i < kTries; ++i) count[i] += over(t, most[i]);
    if (!s.fine && t > hi) divided += over(t, hi);
  }
#pragma unroll
  for (int i = 0; i < kTries; ++i) {
    const int total = wave_sum(count[i]);
    if (lane == 0) count_s[i][wave] = total;
  }
  __syncthreads();
  int longest = most[kTries - 1], mine = count[kTries - 1], all = 0;
  bool chosen = false;
#pragma unroll
  for (int i = 0; i < kTries; ++i) {
    int c = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) c += count_s[i][w];
    if (!chosen && (c <= s.parts || i == kTries - 1)) {
      chosen = true;
      longest = most[i];
      mine = count[i];
      all = c;
    }
  }
  if (item >= all) return false;
  // ranges of this thread's sequences and of those in front of them; and slots
  int before = wave_scan(mine), slot = wave_scan(divided);
  if (lane == kWave - 1) {
    scan_s[0][wave] = before;
    scan_s[1][wave] = slot;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w)
    if (w < wave) {
      before += scan_s[0][w];
      slot += scan_s[1][w];
    }
  int first = before - mine;
  slot -= divided;
  if (item >= first && item < before)
    for (int b = b0; b < b1; ++b) {
      const int parts = over(tiles_of(b), longest);
      if (item < first + parts) {
        found_s = Range{b, item - first, parts, s.fine ? first : slot};
        break;
      }
      first += parts;
      if (parts > 1) slot += parts;
    }
  __syncthreads();
  r = found_s;
  return true;
}

// The batch's tiles one behind the other, each sequence's start counted as kStart
// more.  All threads of a workgroup call these; every thread counts some
// neighbouring sequences.
template <int KEYS, int WAVES>
struct Tiles {
  int b0, b1;             // this thread's sequences
  uint64_t before, mine;  // tiles in front of them, and theirs

  // returns the tiles of all sequences
  __device__ __forceinline__ uint64_t count(const AttnVerifyArgs &a) {
    __shared__ uint32_t sum_s[2][WAVES];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int own = (a.B + WAVES * kWave - 1) / (WAVES * kWave);
    b0 = min(tid * own, a.B);
    b1 = min(b0 + own, a.B);
    // (a batch's tiles pass 32 bits: summed by halves of 16)
    uint32_t low = 0, high = 0;
    for (int b = b0; b < b1; ++b) {
      const int t = tiles_of<KEYS>(a, a.rows.len[b]) + kStart;
      low += t & 0xffff;
      high += t >> 16;
    }
    const uint32_t low_to = wave_scan(low), high_to = wave_scan(high);
    if (lane == kWave - 1) {
      sum_s[0][wave] = low_to;
      sum_s[1][wave] = high_to;
    }
    __syncthreads();
    mine = low + ((uint64_t)high << 16);
    before = low_to + ((uint64_t)high_to << 16) - mine;
    uint64_t all = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const uint64_t sum = sum_s[0][i] + ((uint64_t)sum_s[1][i] << 16);
      if (i < wave) before += sum;
      all += sum;
    }
    return uniform64(all);
  }

  // the sequence that holds a tile, its length, and the tiles in front of it
  __device__ __forceinline__ int find(const AttnVerifyArgs &a, uint64_t tile, uint64_t &front, int &len) const {
    __shared__ int found_b, found_len;
    __shared__ uint64_t found_front;
    if (before <= tile && tile < before + mine) {
      uint64_t at = before;
      for (int b = b0; b < b1; ++b) {
        const int l = a.rows.len[b], t = tiles_of<KEYS>(a, l) + kStart;
        if (tile < at + t) {
          found_b = b;
          found_len = l;
          found_front = at;
          break;
        }
        at += t;
      }
    }
    __syncthreads();
    front = uniform64(found_front);
    len = __builtin_amdgcn_readfirstlane(found_len);
    return __builtin_amdgcn_readfirstlane(found_b);
  }
};

// A lane's 32-bit offset from a wave-uniform base, kept apart from it: added up
// ahead of a loop, every such address would hold two registers through it.
__device__ __forceinline__ uint32_t own_offset(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// -x; and 0 times x: zeros, and NaN where x is infinite or NaN.  (Opaque, so that a
// branch around them stays one.)
__device__ __forceinline__ bf16x8 minus(bf16x8 x) {
  u32x4 y = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = own_offset(y[i]) ^ 0x80008000u;
  return __builtin_bit_cast(bf16x8, y);
}
__device__ __forceinline__ bf16x8 zero_times(bf16x8 x) {
  u32x4 y = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = own_offset(y[i]);
    y[i] = ((w & 0x7f80u) == 0x7f80u ? 0x7fc0u : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0x7fc00000u : 0u);
  }
  return __builtin_bit_cast(bf16x8, y);
}

// Where the piece at `offset` of a row lies for a lane whose swizzle is `lane`
// (below 256): a few exclusive-ors for a row, the rest in the reads' immediates.
__device__ __forceinline__ int place(int offset, int lane) { return (offset % 256 ^ lane) + offset / 256 * 256; }

// Order of a block of fragment reads and the products that take them: AHEAD
// fragments (READS reads each) first, then each fragment's PRODUCTS products
// followed by the reads of the one AHEAD behind it.
template <int AHEAD, int READS, int PRODUCTS, int FRAGS>
__device__ __forceinline__ void pace() {
  constexpr int kRead = 0x100, kMfma = 0x8;
  constexpr int kFirst = AHEAD < FRAGS ? AHEAD : FRAGS;
  __builtin_amdgcn_sched_group_barrier(kRead, kFirst * READS, 0);
#pragma unroll
  for (int f = 0; f < FRAGS; ++f) {
    __builtin_amdgcn_sched_group_barrier(kMfma, PRODUCTS, 0);
    if (f + kFirst < FRAGS) __builtin_amdgcn_sched_group_barrier(kRead, READS, 0);
  }
}

// WK waves share a query's keys (each takes its part of every tile), the
// workgroup's waves / WK groups of them take QT query tiles each.
template <typename T, int D, int QT, int WK, int WAVES, bool SPAN>
__global__ __launch_bounds__(WAVES * kWave, 2) void verify_kernel(AttnVerifyArgs a, Split split, int qtiles) {
  using L = Tile<T, D>;
  constexpr int kKeyTiles = L::kKeys / 16 / WK;  // of a wave
  // fragments read ahead of their products, as the registers allow
  constexpr int kAhead = QT * D >= 320 ? (L::kBf16 ? 4 : 2) : 8;
  static_assert(kKeyTiles >= 1 && (!L::kBf16 || kKeyTiles % 2 == 0), "whole matrix tiles");
  __shared__ __attribute__((aligned(1024))) char stage[2][2 * L::kBytes];
  __shared__ uint64_t anc_s[kWave];
  __shared__ int bad_value;
  __shared__ bool bad_page_s[WAVES];

  const int n = a.n, Hkv = a.cache.Hkv, G = a.Hq / Hkv, R = n * G;
  // the query tiles of one key range, which read the same keys, are numbered
  // back to back on one XCD
  const unsigned turn = workgroup() / kXcdCount;
  unsigned u = turn / qtiles * kXcdCount + blockIdx.x % kXcdCount;
  const int qt0 = turn % qtiles * (WAVES / WK * QT * kQueries);
  const int kv = u % Hkv, item = u / Hkv;
  const bool reports = kv == 0 && qt0 == 0;  // this workgroup tells of its parts and their errors
  const int shift = a.cache.page_shift;
  const const_int *const lens = (const const_int *)(uintptr_t)a.rows.len;
  // sequence b's tiles from..to of `tiles`; its first part is number `first`, this
  // one's slot `slot` if the sequence is divided
  auto attend = [&](const int b, const int len, const int tiles, const int from, const int to, const int first,
                    const int slot, auto parts_of) __attribute__((always_inline)) {
    // (opaque where registers are short: what is formed from it is formed again
    // for the next sequence, or next to its use, and not kept)
    const int tid = SPAN || QT * D >= 512 ? own_offset(threadIdx.x) : threadIdx.x, lane = tid % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int g = lane / 16, col = lane % 16;
    const bool whole = from == 0 && to == tiles;  // no other workgroup has keys of these rows
    int32_t *const err = !whole ? split_errors(a, split, R) + slot : a.status ? a.status + b : nullptr;
    if (reports && split.divided() && from == 0 && tid == 0) split_parts(a, split, R)[b] = make_int2(first, parts_of());
    if (!length_ok(a.rows, shift, len, n) || len > a.max_len) {
      if (reports && err && tid == 0) *err = SLA_ERR_LENGTH;
      return;
    }
    const int total = len + n, k_begin = from * L::kKeys, k_end = min(to * L::kKeys, total);
    bool bad_page = false, bad_topology = false;

    // A tile goes through registers: its rows are read while the tile before is
    // worked on and written to LDS after that.  (Loads that go to LDS by
    // themselves were slower, 64-node trees with heads of 256 608 us against 482:
    // the first fragment read behind one waits for all of them.)  A wave's load i
    // brings rows `first`.. of the 16 that share a page.  The page comes from the
    // table by a scalar load, for it is the same in all lanes; a row past the last
    // one lies in whatever page the table names there (page 0 if it names none),
    // and is masked.
    constexpr int kOwnLoads = L::kLoads / WAVES;
    const const_int *const table = (const const_int *)(uintptr_t)(a.rows.table + (size_t)b * a.rows.max_pages);
    // Keys and values travel together, 32 KB of a workgroup's reads at a time,
    // but where the registers hold one of them only: there the values are read
    // when the keys have been written.
    constexpr bool kTogether = QT * D < (L::kBf16 ? 512 : 320);
    u32x4 rows[kTogether ? 2 : 1][kOwnLoads];
    constexpr int kV = kTogether ? 1 : 0;  // the values' rows
    auto read_rows = [&](int k0, bool keys, bool values) __attribute__((always_inline)) {
      const uint32_t own = own_offset(lane * 16);
#pragma unroll
      for (int i = 0; i < kOwnLoads; ++i) {
        const int first = (wave + i * WAVES) * L::kLoadRows, k = k0 + first / 16 * 16;
        int pg = table[min(k >> shift, a.rows.max_pages - 1)];
        if ((unsigned)pg >= (unsigned)a.cache.n_pages) {
          bad_page |= k < k_end;
          pg = 0;
        }
        const uint64_t off = (page_row(a.cache, pg, kv) + ((k & ((1 << shift) - 1)) + first % 16)) * L::kRow;
        if (keys) rows[0][i] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.cache.k) + off + own);
        if (values) rows[kV][i] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.cache.v) + off + own);
      }
    };
    auto write_rows = [&](char *dst, bool keys, bool values) __attribute__((always_inline)) {
      const int own = kTogether ? lane : own_offset(lane);
#pragma unroll
      for (int i = 0; i < kOwnLoads; ++i) {
        const int r = (wave + i * WAVES) * L::kLoadRows + own / L::kCols, piece = own % L::kCols;
        if (keys) *reinterpret_cast<u32x4 *>(dst + r * L::kRow + (piece ^ L::swizzle_k(r)) * 16) = rows[0][i];
        if (values) *reinterpret_cast<u32x4 *>(dst + L::kBytes + r * L::kRow + (piece ^ L::swizzle_v(r)) * 16) = rows[kV][i];
      }
    };
    read_rows(k_begin, true, kTogether);
    if (!kTogether) {
      write_rows(stage[0], true, false);
      read_rows(k_begin, false, true);
    }

    // this wave's queries
    const int r0 = qt0 + wave / WK * (QT * kQueries), wk = wave % WK;
    const bool active = r0 < R;
    const float sign = a.scale > 0.f ? 1.f : a.scale < 0.f ? -1.f : 0.f;
    Frag<T, D> qf[QT];
    int node[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int r = min(r0 + t * kQueries + col, R - 1);
      node[t] = r / G;
      const T *q = static_cast<const T *>(a.q) + (((size_t)b * n + r / G) * a.Hq + (size_t)kv * G + r % G) * D;
      if constexpr (L::kBf16) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) qf[t].x[c] = *reinterpret_cast<const bf16x8 *>(q + 32 * c + 8 * g);
      } else {
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          const f32x4 x = *reinterpret_cast<const f32x4 *>(q + 16 * c + 4 * g);
          qf[t].x[c] = x * sign;
        }
      }
    }

    f32x4 o[QT][D / 16];
    float m[QT], l[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      m[t] = kNoScore;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Weights are powers of two; the scale's sign is in the queries, and so is a
    // scale of 0: times 0, masked scores would not stay -inf.
    const float scale = sign == 0.f ? 1.f : fabsf(a.scale) * 1.44269504088896341f;

    // fragment reads: this lane's row of a key tile, and the pieces' places in it
    const int k_row = (wk * kKeyTiles * 16 + col) * L::kRow;
    const int k_piece = (g ^ L::swizzle_k(col)) * 16;
    // V, bf16: row 4 g + col / 4 of a key tile, 8 bytes of the piece pair of 16
    // elements; the lane receives element col of rows 4 g..4 g + 3.  fp32: row
    // 4 g + i, element col.
    const int v_in = L::kBf16 ? 4 * g + col / 4 : 4 * g;
    const int v_row = L::kBytes + (wk * kKeyTiles * 16 + v_in) * L::kRow;
    const int v_piece = L::kBf16 ? ((col % 4 / 2) ^ L::swizzle_v(v_in)) * 16 + col % 2 * 8
                                 : ((col / 4) ^ L::swizzle_v(v_in)) * 16 + col % 4 * 4;

    if (tid == 0) bad_value = 0;  // (the first tile's barrier follows)
    // attends to the staged tile `cur`
    auto step = [&](int k0, char *cur, char *next) {
      const bool edge = k0 + L::kKeys > len;  // the tile reaches into the draft
      if (edge) {
        if (wave == 0 && (k0 == k_begin || k0 <= len)) {  // the range's first such tile
          const int p = lane < n ? a.parent[(size_t)b * n + lane] : -1;
          bad_topology = !parents_ok(p, n, lane, a.chain);
          anc_s[lane] = bad_topology ? 0 : node_ancestors(p, lane);
        }
        // a weight of 0 does not remove an infinity or a NaN from a product: a
        // draft row's are left out here and given to the queries that see the
        // row at the end (a committed row's reach every query in any case)
        for (int c = tid; c < L::kBytes / 16; c += WAVES * kWave) {
          const int k = k0 + c / L::kCols;
          if (k < len) continue;
          u32x4 *const piece = reinterpret_cast<u32x4 *>(cur + L::kBytes) + c;
          bool found = false;
          const u32x4 x = finite_part(*piece, found, T{});
          if (found) {
            *piece = x;
            if (k < total) bad_value = 1;
          }
        }
        __syncthreads();
      }
      f32x4 s[QT][kKeyTiles];
      if (active) {
        const int k_own = own_offset(k_piece);
        // scores, transposed: keys 4 g + i of key tile kt, query col
#pragma unroll
        for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
          for (int t = 0; t < QT; ++t) s[t][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (L::kBf16) {
          constexpr int kChunks = D / 32, kFrags = kKeyTiles * kChunks;
          bf16x8 kf[kFrags];
#pragma unroll
          for (int f = 0; f < kFrags; ++f)
            kf[f] = *reinterpret_cast<const bf16x8 *>(cur + k_row + f / kChunks * 16 * L::kRow + place(f % kChunks * 64, k_own));
#pragma unroll
          for (int f = 0; f < kFrags; ++f)
#pragma unroll
            for (int t = 0; t < QT; ++t)
              s[t][f / kChunks] =
                  __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[f], qf[t].x[f % kChunks], s[t][f / kChunks], 0, 0, 0);
          pace<kAhead, 1, QT, kFrags>();
        } else {
          constexpr int kChunks = D / 16, kFrags = kKeyTiles * kChunks;
          f32x4 kf[kFrags];
#pragma unroll
          for (int f = 0; f < kFrags; ++f)
            kf[f] = *reinterpret_cast<const f32x4 *>(cur + k_row + f / kChunks * 16 * L::kRow + place(f % kChunks * 64, k_own));
#pragma unroll
          for (int f = 0; f < kFrags; ++f)
#pragma unroll
            for (int t = 0; t < QT; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                s[t][f / kChunks] =
                    __builtin_amdgcn_mfma_f32_16x16x4f32(kf[f][i], qf[t].x[f % kChunks][i], s[t][f / kChunks], 0, 0, 0);
          pace<(kAhead < 4 ? kAhead : 4), 1, QT * 4, kFrags>();
        }
        __builtin_amdgcn_sched_barrier(0);
        if (edge) {
#pragma unroll
          for (int kt = 0; kt < kKeyTiles; ++kt) {
            // bit i: the query sees key 4 g + i, draft node rel + i.  Bits of nodes
            // past the draft are clear in every mask.
            const int rel = k0 + (wk * kKeyTiles + kt) * 16 + 4 * g - len;
#pragma unroll
            for (int t = 0; t < QT; ++t) {
              const int up = -rel & 63;
              const uint64_t anc = anc_s[node[t]];
              uint64_t see = rel >= 0 ? anc >> (rel & 63) : anc << up | ((1ull << up) - 1);
              see = rel >= 64 ? 0 : rel <= -4 ? ~0ull : see;
#pragma unroll
              for (int i = 0; i < 4; ++i) s[t][kt][i] = (uint32_t)see >> i & 1 ? s[t][kt][i] : -INFINITY;
            }
          }
        }
      }
      if (!kTogether && k0 + L::kKeys < k_end) {
        write_rows(next, true, false);
        read_rows(k0 + L::kKeys, false, true);
      }
      if (active) {
        // softmax against a reference that only moves when a score exceeds it by
        // more than 2^kSlack: weights stay below 2^kSlack, where fp32 sums and bf16
        // weights are as precise as below 1, and most tiles neither reduce a
        // maximum over the lanes nor rescale the output (64-node trees with heads
        // of 256 1419 us with a maximum for every tile, 918 without)
        float top[QT];
        bool passed = false;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          top[t] = -INFINITY;
#pragma unroll
          for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[t] = fmaxf(top[t], s[t][kt][i]);
          top[t] *= scale;
          passed |= top[t] - m[t] > kSlack;
        }
        if (wave_any(passed)) {
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            top[t] = fmaxf(top[t], __shfl_xor(top[t], 16));
            top[t] = fmaxf(top[t], __shfl_xor(top[t], 32));
            top[t] = fmaxf(top[t], m[t]);
            const float shrink = __builtin_amdgcn_exp2f(m[t] - top[t]);
            m[t] = top[t];
            l[t] *= shrink;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[t][d] *= shrink;
          }
        }
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              s[t][kt][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][kt][i], scale, -m[t]));
              l[t] += s[t][kt][i];
            }
      }
      if (active) {
        const int v_own = own_offset(v_piece);
        // O^T += V^T P^T, for bf16 with the weights rounded to bf16 for the matrix
        // cores: each is off by up to 2^-8 of itself, as the output's rounding is
        if constexpr (L::kBf16) {
          constexpr int kSteps = D / 16, kFrags = kKeyTiles / 2 * kSteps;
          bf16x8 pf[QT][kKeyTiles / 2], vf[kFrags];
#pragma unroll
          for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int kp = 0; kp < kKeyTiles / 2; ++kp)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                pf[t][kp][i] = static_cast<__bf16>(s[t][2 * kp][i]);
                pf[t][kp][4 + i] = static_cast<__bf16>(s[t][2 * kp + 1][i]);
              }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int f = 0; f < kFrags; ++f) {
            char *piece = cur + v_row + f / kSteps * 32 * L::kRow + place(f % kSteps * 32, v_own);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)piece);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(piece + 16 * L::kRow));
            vf[f] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          }
#pragma unroll
          for (int f = 0; f < kFrags; ++f)
#pragma unroll
            for (int t = 0; t < QT; ++t)
              o[t][f % kSteps] =
                  __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[f], pf[t][f / kSteps], o[t][f % kSteps], 0, 0, 0);
          pace<kAhead, 2, QT, kFrags>();
        } else {
#pragma unroll
          for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float vf = *reinterpret_cast<const float *>(cur + v_row + (kt * 16 + i) * L::kRow + place(d * 64, v_own));
#pragma unroll
                for (int t = 0; t < QT; ++t)
                  o[t][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf, s[t][kt][i], o[t][d], 0, 0, 0);
              }
        }
      }
    };

    write_rows(stage[0], kTogether, true);
    if (k_begin + L::kKeys < k_end) read_rows(k_begin + L::kKeys, true, kTogether);
    // Two workgroups share a CU.  With one ahead of the other at the issue ports
    // their phases part: while one forms products the other takes exponentials
    // (64 sequences of 16-node trees, heads of 128, 50.7 -> 48.7 us).  Workgroups
    // numbered 256 apart usually meet.  Ten other loads of four-wave forms, fp32 and
    // single tokens among them, are within 2% with and without it, but the same
    // trees with heads of 64: 36.4 us with, 35.2 without.
    if (WAVES == 4 && (blockIdx.x >> 8) & 1) __builtin_amdgcn_s_setprio(2);
    if constexpr (L::kBf16) {
      // (here, where nothing waits for them yet: as they are read, one token takes 9.23 us, not 9.00)
      if (!(sign > 0.f)) {
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (auto &x : qf[t].x) x = sign < 0.f ? minus(x) : zero_times(x);
      }
    }
    int buf = 0;
    for (int k0 = k_begin; k0 < k_end; k0 += L::kKeys, buf ^= 1) {
      __syncthreads();  // the tile is whole, and the other buffer free
      step(k0, stage[buf], stage[buf ^ 1]);
      if (k0 + L::kKeys < k_end) write_rows(stage[buf ^ 1], kTogether, true);
      if (k0 + 2 * L::kKeys < k_end) read_rows(k0 + 2 * L::kKeys, true, kTogether);
    }

    if (reports && err) {
      if (lane == 0) bad_page_s[wave] = bad_page;
      __syncthreads();
      if (tid == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) bad_page |= bad_page_s[w];
        *err = bad_topology ? SLA_ERR_TOPOLOGY : bad_page ? SLA_ERR_PAGE : SLA_OK;
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      l[t] += __shfl_xor(l[t], 16);
      l[t] += __shfl_xor(l[t], 32);
    }
    if constexpr (WK > 1) {
      // the waves of a query join theirs, half of them handing over to the rest
      // in each round, one query tile at a time
      float *const box = reinterpret_cast<float *>(stage[0]);
      constexpr int kBox = (D / 16 * 4 + 2) * kWave;  // floats of a wave
      static_assert(WAVES / 2 * kBox * 4 <= (int)sizeof(stage), "the first round's hand-over fits");
#pragma unroll
      for (int half = WK / 2; half >= 1; half /= 2) {
        float *const x = box + (wave / WK * (WK / 2) + wk % half) * kBox + lane;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          __syncthreads();
          if (wk >= half && wk < 2 * half) {
            x[0] = m[t];
            x[kWave] = l[t];
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
              for (int i = 0; i < 4; ++i) x[(2 + d * 4 + i) * kWave] = o[t][d][i];
          }
          __syncthreads();
          if (wk < half) {
            const float top = fmaxf(m[t], x[0]);
            const float w0 = __builtin_amdgcn_exp2f(m[t] - top), w1 = __builtin_amdgcn_exp2f(x[0] - top);
            m[t] = top;
            l[t] = w0 * l[t] + w1 * x[kWave];
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[t][d][i] = w0 * o[t][d][i] + w1 * x[(2 + d * 4 + i) * kWave];
          }
        }
      }
      if (wk > 0) return;
    }
    if (!active) return;

    if (bad_value) {  // written before the last tile's barrier
      for (int k = max(k_begin, len); k < k_end; ++k) {
        const int pg = table[k >> shift];
        const T *row = static_cast<const T *>(a.cache.v) +
                       (page_row(a.cache, (unsigned)pg < (unsigned)a.cache.n_pages ? pg : 0, kv) + (k & ((1 << shift) - 1))) * D;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          const f32x4 v = load4(row + d * 16 + 4 * g);
#pragma unroll
          for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!(fabsf(v[e]) < INFINITY) && (anc_s[node[t]] >> (k - len)) & 1ull) o[t][d][e] += v[e];
        }
      }
    }

    float *const ws = static_cast<float *>(a.workspace);
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int r = r0 + t * kQueries + col;
      if (r >= R) continue;
      if (whole) {
        const float inv = 1.f / l[t];
        T *out = static_cast<T *>(a.out) + (((size_t)b * n + r / G) * a.Hq + (size_t)kv * G + r % G) * D + 4 * g;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          const f32x4 x = o[t][d] * inv;
          if constexpr (L::kBf16)
            *reinterpret_cast<uint2 *>(out + d * 16) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
          else
            *reinterpret_cast<f32x4 *>(out + d * 16) = x;
        }
      } else {
        const size_t row = ((size_t)kv * split.slots + slot) * R + r;
        float *out = ws + row * D + 4 * g;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4 *>(out + d * 16) = o[t][d];
        if (g == 0) split_stats(a, split, R)[row] = make_float2(m[t], l[t]);
      }
    }
  };

  if constexpr (!SPAN) {
    Range range;
    if (!pick_range<L::kKeys, WAVES>(a, split, item, range)) return;
    const int b = __builtin_amdgcn_readfirstlane(range.b), parts = __builtin_amdgcn_readfirstlane(range.parts);
    const int part = __builtin_amdgcn_readfirstlane(range.part), len = lens[b], tiles = tiles_of<L::kKeys>(a, len);
    const int first = __builtin_amdgcn_readfirstlane(range.first);
    attend(b, len, tiles, (int)((int64_t)tiles * part / parts), (int)((int64_t)tiles * (part + 1) / parts), first,
           first + part, [&] { return parts; });
  } else {
    // This worker's part [begin, end) of the tiles of all sequences: the first
    // `more` workers have one more than `each`.
    Tiles<L::kKeys, WAVES> count;
    const uint64_t all = count.count(a);
    const uint32_t workers = all < (uint64_t)split.workers ? (uint32_t)all : split.workers;
    if ((uint32_t)item >= workers) return;
    const uint64_t each = uniform64(quotient(all, workers));
    const uint32_t more = (uint32_t)(all - each * workers);
    uint64_t begin = each * item + min((uint32_t)item, more);
    const uint64_t end = begin + each + ((uint32_t)item < more);
    uint64_t before;
    int len, b = count.find(a, begin, before, len);
    for (;;) {
      const int tiles = tiles_of<L::kKeys>(a, len);
      before += kStart;
      const int from = begin > before ? (int)(begin - before) : 0;
      const int to = end < before + tiles ? (int)(end - before) : tiles;  // not above 0 if the part ends in the start's share
      const int next = lens[min(b + 1, a.B - 1)];
      if (from < to)
        attend(b, len, tiles, from, to, item, from > 0 ? item : split.first_slot(item, b, a.B), [&] {
          // up to the worker that has the sequence's last tile
          const uint64_t last = before + tiles - 1, longer = (each + 1) * more;
          return 1 - item + (int)(last < longer ? quotient(last, (uint32_t)each + 1)
                                                : more + quotient(last - longer, (uint32_t)each));
        });
      before += tiles;
      if (before >= end) return;
      begin = before;
      len = next;
      ++b;
      __syncthreads();  // the waves have left the sequence's last tile
    }
  }
}

// Joins the parts of a row, sum_s w_s x_s / sum_s w_s l_s with w_s = 2^(m_s - max m).
// GROUPS groups of D / 4 lanes, four elements a lane, take every GROUPS-th part,
// kBatch of them read at a time, and meet in LDS.  One pass, bounded by the parts'
// bytes (from the L2 for the most part) or, for few rows, by its launch and two
// dependent loads: 3.8 us of the 9.1 us of one token over 1000 keys.
template <typename T, int D, int GROUPS>
__global__ __launch_bounds__(kThreads) void join_kernel(AttnVerifyArgs a, Split split) {
  constexpr int kLanes = D / 4, kSlots = kThreads / kLanes, kBatch = 4;
  __shared__ f32x4 part_x[GROUPS > 1 ? kSlots : 1][kLanes];
  __shared__ float2 part_ml[GROUPS > 1 ? kSlots : 1];
  const int n = a.n, Hkv = a.cache.Hkv, G = a.Hq / Hkv, R = n * G;
  const size_t rows = (size_t)a.B * Hkv * R;
  const int slot = threadIdx.x / kLanes, grp = slot % GROUPS, e = threadIdx.x % kLanes * 4;
  const size_t i = (size_t)workgroup() * (kSlots / GROUPS) + slot / GROUPS;
  const int r = i % R, kv = i / R % Hkv, b = min((int)(i / R / Hkv), a.B - 1);
  const int2 own = split_parts(a, split, R)[b];
  const bool live = i < rows && own.y > 1;  // else written whole
  const int parts = live ? own.y : 0, slot0 = split.first_slot(own.x, b, a.B);
  auto slot_of = [&](int s) { return s > 0 ? own.x + s : slot0; };
  const size_t row0 = (size_t)kv * split.slots * R + r;
  const float *const ws = static_cast<const float *>(a.workspace) + row0 * D + e;
  const float2 *const ml = split_stats(a, split, R) + row0;
  float ref = kNoScore, l = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = grp; s0 < parts; s0 += kBatch * GROUPS) {
    float2 st[kBatch];
    f32x4 y[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const size_t s = slot_of(min(s0 + k * GROUPS, parts - 1));
      st[k] = ml[s * R];
      y[k] = *reinterpret_cast<const f32x4 *>(ws + s * R * D);
    }
    float top = ref;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) top = fmaxf(top, st[k].x);
    const float shrink = __builtin_amdgcn_exp2f(ref - top);
    ref = top;
    l *= shrink;
    x *= shrink;
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (s0 + k * GROUPS < parts) {
        const float w = __builtin_amdgcn_exp2f(st[k].x - ref);
        l = __builtin_fmaf(w, st[k].y, l);
        x += w * y[k];
      }
  }
  if constexpr (GROUPS > 1) {
    part_x[slot][e / 4] = x;
    if (e == 0) part_ml[slot] = make_float2(ref, l);
    __syncthreads();
    if (grp > 0) return;
    float top = ref;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) top = fmaxf(top, part_ml[slot + k].x);
    const float w0 = __builtin_amdgcn_exp2f(ref - top);
    l *= w0;
    x *= w0;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) {
      const float w = __builtin_amdgcn_exp2f(part_ml[slot + k].x - top);
      l = __builtin_fmaf(w, part_ml[slot + k].y, l);
      x += w * part_x[slot + k][e / 4];
    }
  }
  if (a.status && live && kv == 0 && r == 0) {
    // the sequence's first row tells of it: its kLanes lanes alone, for a wave
    // holds the first rows of several sequences where these have few
    const uint64_t lanes = (~0ull >> (kWave - kLanes)) << (threadIdx.x % kWave / kLanes * kLanes);
    bool topology = false, page = false, length = false;
    for (int s = e / 4; s < own.y; s += kLanes) {
      const int err = split_errors(a, split, R)[slot_of(s)];
      topology |= err == SLA_ERR_TOPOLOGY;
      length |= err == SLA_ERR_LENGTH;
      page |= err == SLA_ERR_PAGE;
    }
    topology = __ballot(topology) & lanes;
    length = __ballot(length) & lanes;
    page = __ballot(page) & lanes;
    if (e == 0) a.status[b] = topology ? SLA_ERR_TOPOLOGY : length ? SLA_ERR_LENGTH : page ? SLA_ERR_PAGE : SLA_OK;
  }
  if (!live) return;
  x *= 1.f / l;
  T *out = static_cast<T *>(a.out) + (((size_t)b * n + r / G) * a.Hq + (size_t)kv * G + r % G) * D + e;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2 *>(out) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  else
    *reinterpret_cast<f32x4 *>(out) = x;
}

// How a workgroup is laid out for the rows of a kv head: `qt` query tiles a
// wave, `wk` waves that share a query's keys, `waves` in all.
struct Form {
  int qt, wk, waves;
  int tiles() const { return waves / wk * qt; }
  int rows() const { return tiles() * kQueries; }
};

// fp32: every wave holds all of a workgroup's queries and takes its share of each
// tile's keys, as far as the registers hold the queries next to a tile in
// flight: up to this many query tiles.  A fragment is read from LDS by one wave
// only, and the products, which bound it, are spread evenly whatever the number
// of rows: 90 rows as two workgroups of three query tiles 95 us, as five and one
// 152 us (40 sequences of up to 3001 keys, heads of 64).  A tile of heads of 256
// has one key tile: nothing to share.
template <int D>
constexpr int key_split_tiles() {
  return D == 64 ? 5 : D == 128 ? 2 : 0;
}

// bf16: a wave has all keys of its own query tiles (shared keys, as in fp32,
// were no faster for one query tile and slower for three, 41 us against 37 for
// 64 sequences of 512 to 4096 keys and 48 rows: joining the waves cost more than
// idle ones).  Two query tiles a wave halve the fragments that it reads, from 65
// rows on; with heads of 256 the registers are short for it, and eight waves of
// one are better up to 128 rows, 98 us against 118.  Four waves up to 128 rows:
// eight would be half idle, 49 us against 44 for 96 rows and 52 against 48 for 128.
template <typename T, int D>
Form form_of(int R) {
  const int tiles = (R + kQueries - 1) / kQueries;
  if constexpr (sizeof(T) == 2) {
    if (tiles <= 4) return Form{1, 1, 4};
    if (D == 256 && tiles <= 8) return Form{1, 1, 8};
    return Form{2, 1, tiles <= 8 ? 4 : 8};
  } else if constexpr (D == 256) {
    return Form{1, 1, 8};
  } else {
    constexpr int kSplit = std::min(Tile<T, D>::kKeys / 16, 4);
    constexpr int kGroups = 4 / kSplit, kTake = key_split_tiles<D>() * kGroups;  // groups of waves, query tiles of a workgroup
    const int blocks = (tiles + kTake - 1) / kTake;
    return Form{(tiles + blocks * kGroups - 1) / (blocks * kGroups), kSplit, 4};
  }
}

template <typename T, int D>
Split plan(const AttnVerifyArgs &a) {
  constexpr int kKeys = Tile<T, D>::kKeys;
  const int R = a.n * (a.Hq / a.cache.Hkv);
  const Form f = form_of<T, D>(R);
  const int64_t tiles = ((int64_t)a.max_len + a.n + kKeys - 1) / kKeys;  // of the longest sequence there may be
  if (tiles == 1) return Split{0, a.B, false, 0, 0};
  // workgroups that run at once, and the ranges that makes of the batch's keys
  const int64_t slots = (int64_t)device_cus() * (8 / f.waves);
  const int64_t want = std::max<int64_t>(1, slots / ((int64_t)a.cache.Hkv * ((R + f.rows() - 1) / f.rows())));
  // Long work goes in equal parts: 256 sequences of up to 16384 keys and one
  // token 392 -> 375 us, 64 of up to 8192 and 64-node trees 498 -> 451 us; the
  // start of a second sequence costs short work more than it saves, 64 of up to
  // 4096 and 16-node trees 49 -> 52 us.
  if (a.B > 1 && want >= kFewWorkers && a.B * tiles >= kLongWork * want)
    return Split{0, (int)(want + a.B - 1), false, (int)want, (int)(want + std::min<int64_t>(want, a.B))};
  for (int64_t ranges = want; ranges <= 2 * want; ranges += want)
    if (ranges > a.B) {
      const int parts = (int)std::min<int64_t>(ranges, a.B * tiles);
      return Split{(int)(ranges - a.B), parts, true, 0, parts};
    }
  // more sequences than that: only one much longer than a workgroup's even share is divided
  const int64_t share = (want + 1) / 2;
  return Split{(int)share, (int)std::min<int64_t>(share + 1 + a.B, a.B * tiles), false, 0, (int)(2 * share)};
}

template <typename T, int D, int QT, int WK, int WAVES>
hipError_t launch_form(const AttnVerifyArgs &a, const Form &f, const Split &split, hipStream_t s) {
  const int R = a.n * (a.Hq / a.cache.Hkv), qtiles = (R + f.rows() - 1) / f.rows();
  const uint64_t items = (uint64_t)(split.workers ? split.workers : split.parts) * a.cache.Hkv;
  const uint64_t blocks = (items + kXcdCount - 1) / kXcdCount * kXcdCount * qtiles;
  auto *const kernel = split.workers ? verify_kernel<T, D, QT, WK, WAVES, true> : verify_kernel<T, D, QT, WK, WAVES, false>;
  hipLaunchKernelGGL(kernel, grid_of(blocks), dim3(WAVES * kWave), 0, s, a, split, qtiles);
  return hipGetLastError();
}

template <typename T, int D, int GROUPS>
hipError_t launch_join(const AttnVerifyArgs &a, const Split &split, hipStream_t s) {
  constexpr int kRows = kThreads / (D / 4) / GROUPS;  // of a workgroup
  const uint64_t rows = (uint64_t)a.B * a.n * a.Hq;
  hipLaunchKernelGGL((join_kernel<T, D, GROUPS>), grid_of((rows + kRows - 1) / kRows), dim3(kThreads), 0, s, a, split);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_d(const AttnVerifyArgs &a, hipStream_t s) {
  const Form f = form_of<T, D>(a.n * (a.Hq / a.cache.Hkv));
  const Split split = plan<T, D>(a);
  hipError_t e = hipErrorInvalidConfiguration;
  if constexpr (sizeof(T) == 2) {
    if (f.qt == 1 && f.waves == 4) e = launch_form<T, D, 1, 1, 4>(a, f, split, s);
    if constexpr (D == 256) {
      if (f.qt == 1 && f.waves == 8) e = launch_form<T, D, 1, 1, 8>(a, f, split, s);
    } else {
      if (f.qt == 2 && f.waves == 4) e = launch_form<T, D, 2, 1, 4>(a, f, split, s);
    }
    if (f.qt == 2 && f.waves == 8) e = launch_form<T, D, 2, 1, 8>(a, f, split, s);
  } else if constexpr (D == 256) {
    e = launch_form<T, D, 1, 1, 8>(a, f, split, s);
  } else {
    constexpr int kSplit = std::min(Tile<T, D>::kKeys / 16, 4), kMost = key_split_tiles<D>();
    if (f.qt == 1) e = launch_form<T, D, 1, kSplit, 4>(a, f, split, s);
    if (f.qt == 2) e = launch_form<T, D, 2, kSplit, 4>(a, f, split, s);
    if constexpr (kMost >= 3) {
      if (f.qt == 3) e = launch_form<T, D, 3, kSplit, 4>(a, f, split, s);
      if (f.qt == 4) e = launch_form<T, D, 4, kSplit, 4>(a, f, split, s);
      if (f.qt == 5) e = launch_form<T, D, 5, kSplit, 4>(a, f, split, s);
    }
  }
  if (e != hipSuccess || !split.divided()) return e;
  // a group for every four parts of a sequence of mean length, up to the whole workgroup
  if (split.parts <= 4 * (int64_t)a.B) return launch_join<T, D, 1>(a, split, s);
  if (split.parts <= 8 * (int64_t)a.B) return launch_join<T, D, 2>(a, split, s);
  return launch_join<T, D, kThreads / (D / 4)>(a, split, s);
}

template <typename T>
hipError_t launch_t(const AttnVerifyArgs &a, hipStream_t s) {
  switch (a.cache.D) {
    case 64: return launch_d<T, 64>(a, s);
    case 128: return launch_d<T, 128>(a, s);
    default: return launch_d<T, 256>(a, s);
  }
}

}  // namespace

size_t attn_workspace_bytes(const AttnVerifyArgs &a, int dtype) {
  const bool bf = dtype == SLA_DTYPE_BF16;
  const Split split = a.cache.D == 64    ? (bf ? plan<bf16, 64>(a) : plan<float, 64>(a))
                      : a.cache.D == 128 ? (bf ? plan<bf16, 128>(a) : plan<float, 128>(a))
                                         : (bf ? plan<bf16, 256>(a) : plan<float, 256>(a));
  if (!split.divided()) return 0;
  return split_rows(a, split, a.n * (a.Hq / a.cache.Hkv)) * (a.cache.D + 2) * sizeof(float) +
         (size_t)a.B * sizeof(int2) + (size_t)split.slots * sizeof(int32_t);
}

hipError_t launch_attn_verify(const AttnVerifyArgs &a, int dtype, hipStream_t s) {
  return dtype == SLA_DTYPE_BF16 ? launch_t<bf16>(a, s) : launch_t<float>(a, s);
}

}  // namespace sla
