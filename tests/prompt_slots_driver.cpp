// The index arithmetic of sla_prefill's chunked kernels, on the CPU (built and run by
// tests/test_prompt_slots.py).  prefill.hip's host code runs as it is, over a HIP runtime
// of stubs; instead of the chunked kernels' launches stands a walk through what their
// workgroups address, with the functions they use themselves (first_slot, chunk_at,
// chunk_space): every chunk of every sequence is made once, in its own slot, before the
// walk that reads it, and every byte that either kernel addresses, also in advance or past
// a sequence's end, lies in its buffer or behind its descriptor's.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <random>
#include <vector>

#include "prefill_chunk.hpp"

static long failures = 0, checks = 0, passes = 0, calls = 0, several = 0, narrow = 0;
#define CHECK(c)                                                                          \
  do {                                                                                    \
    ++checks;                                                                             \
    if (!(c) && ++failures < 20) fprintf(stderr, "check failed: %s (line %d)\n", #c, __LINE__); \
  } while (0)

// ------------------------------------------------------- a runtime of stubs
static long serial_launches = 0;
extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3, dim3, size_t, hipStream_t) { return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *, dim3 *, size_t *, hipStream_t *) { return hipSuccess; }
hipError_t hipLaunchKernel(const void *, dim3, dim3, void **, size_t, hipStream_t) { return ++serial_launches, hipSuccess; }
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipGetDevice(int *d) { return *d = 0, hipSuccess; }
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }
}

namespace sla {

static std::vector<int32_t> starts;
static std::vector<int> chunks_done;  // of each sequence, by the passes so far
static size_t given;                  // bytes of workspace

static int longer_than(const PackedRows &r, int min_len) {
  int n = 0;
  for (int b = 0; b < r.B; ++b) n += (int64_t)r.start[b + 1] - r.start[b] > min_len;
  return n;
}

// find_chunk without lanes
static Chunk chunk_of(const PackedRows &r, int min_len, int slot, int window, int done) {
  Chunk c = {-1, 0, 0, 0, false, 0, 0};
  int at = -1, front = 0, rank = 0, longer = 0;
  for (int b = 0; b < r.B; ++b) {
    if ((int64_t)r.start[b + 1] - r.start[b] <= min_len) continue;
    const int mine = first_slot<kChunk>(r.start[b], longer, window);
    if (mine <= slot) at = b, front = mine, rank = longer;
    ++longer;
  }
  if (at >= 0) chunk_at<kChunk>(c, slot, at, r.start[at], r.start[at + 1], front, rank, window, done);
  return c;
}

// state_kernel's reads and writes of one (sequence, head) and slab
template <bool F32, int DK, int NT>
static void walk_through(const PrefillArgs &a, const ChunkSpace<F32, DK> &space, const Walk &walk, int h, int slab, int slabs) {
  constexpr int w = F32 ? 4 : 2;
  const size_t bytes = space.bytes();
  const int chunks = (walk.len + kChunk - 1) / kChunk, last = chunks - 1, tail = walk.len - last * kChunk;
  const int kh = h / (a.H / a.Hk);
  const auto begin = [&](const unsigned char *p) { return (size_t)(p - space.base); };
  // operands: the descriptor of each chunk covers a slot's, the ones behind the last are empty
  for (int c : {0, chunks / 2, last}) {
    if (c < 0) continue;
    CHECK(begin(space.head(walk.slot, h)) + (size_t)c * a.H * space.kHead == begin(space.head(walk.slot + c, h)));
    CHECK(begin(space.keys(walk.slot, kh)) + (size_t)c * a.Hk * space.kKeys == begin(space.keys(walk.slot + c, kh)));
    CHECK((size_t)walk.slot + c < space.slots && begin(space.head(walk.slot + c, h)) + space.kHead <= space.kFront + space.slots * a.H * space.kHead);
    CHECK(begin(space.keys(walk.slot + c, kh)) + space.kKeys <= space.walk_at(0) && space.walk_at(0) <= bytes);
  }
  // lines brought to the L2 in advance
  using Space = ChunkSpace<F32, DK>;
  constexpr int head_lines = Space::kHead / 128, lines = head_lines + Space::kKeys / 128;
  for (int id : {0, 1, 100, 255}) {
    if (chunks == 0) break;
    const int line = std::min(id * slabs + slab, lines - 1);
    const bool of_head = line < head_lines;
    const size_t at = of_head ? begin(space.head(walk.slot, h)) + (size_t)line * 128
                              : begin(space.keys(walk.slot, kh)) + (size_t)(line - head_lines) * 128;
    CHECK(at + (size_t)last * (of_head ? a.H * space.kHead : a.Hk * space.kKeys) + 128 <= space.walk_at(0) && at % 128 == 0);
  }
  // values: rows and columns inside the tensor, or behind the descriptor
  constexpr uint32_t nowhere = 0x40000000u;
  for (int c = 0; c < chunks; c += std::max(1, chunks / 3)) {
    const int rows = c < last ? kChunk : tail;
    const uint64_t records = (uint64_t)((rows - 1) * a.v_stride + a.dv) * w;
    CHECK(records < nowhere && walk.start + c * kChunk + rows <= starts[walk.b + 1]);
    const uint64_t end = ((uint64_t)(walk.start + c * kChunk) * a.v_stride + (uint64_t)h * a.dv) * w + records;
    CHECK(end <= ((uint64_t)(a.rows.tokens - 1) * a.v_stride + (uint64_t)a.H * a.dv) * w);
    for (int t = 0; t < 4; ++t)
      for (int g = 0; g < 4; ++g)
        for (int i = 0; i < 4; ++i)
          for (int r = 0; r < 16; ++r)
            for (int n = 0; n < NT; ++n) {
              const int col = slab * 16 * NT + (NT == 1 ? r : 32 * (n / 2) + 8 * (r / 4) + 4 * (n % 2) + r % 4);
              const uint64_t off = col < a.dv ? (uint64_t)(tile_row(t, 4 * g) * a.v_stride + col) * w : nowhere;
              const uint64_t reach = off + (uint64_t)(i * a.v_stride * w);
              CHECK(reach < 1ull << 32);
              const int row = tile_row(t, 4 * g) + i;
              CHECK((reach < records) == (col < a.dv && row < rows));
              const uint64_t state = (col < a.dv ? (uint64_t)(tile_row(t, 4 * g) * a.dv + col) * 4 : nowhere) +
                                     (uint64_t)((DK - 64 + i) * a.dv) * 4;
              CHECK(col >= a.dv || state + 4 <= (uint64_t)DK * a.dv * 4);
            }
  }
  CHECK(std::min(slab * 16 * NT, a.dv - 16) >= 0);
}

template <bool F32, int DK>
hipError_t launch_chunks(const PrefillArgs &a, hipStream_t) {
  const auto space = chunk_space<F32, DK>(a);
  const PackedRows &r = a.rows;
  ++passes;
  CHECK(space.bytes() <= given && space.slots > 0 && space.slots < 1ull << 31);
  CHECK(space.slots * (size_t)a.H < 1ull << 31 && a.window >= 0 && a.done >= 0 && (a.window > 0 || a.done == 0));
  const int longer = longer_than(r, a.serial_len);
  CHECK((size_t)longer <= space.walks);
  std::vector<char> taken(space.slots, 0);
  std::vector<Walk> walks(longer, Walk{-1, 0, 0, 0});
  // the slots that have a chunk, and those around each window's ends
  int rank = 0;
  for (int b = 0; b < r.B; ++b) {
    const int len = r.start[b + 1] - r.start[b];
    if (len <= a.serial_len) continue;
    const int front = first_slot<kChunk>(r.start[b], rank, a.window);
    const int all = std::max(1, (len + kChunk - 1) / kChunk) - a.done, mine = a.window ? std::min(all, a.window) : all;
    CHECK(all >= 1 && chunks_done[b] == a.done && (size_t)front + mine <= space.slots);
    for (int c = 0; c < mine; ++c) {
      CHECK(!taken[front + c]);
      taken[front + c] = 1;
      if (c > 2 && c < mine - 2 && mine > 200) continue;
      const Chunk k = chunk_of(r, a.serial_len, front + c, a.window, a.done);
      CHECK(k.b == b && k.rank == rank && k.first == (c == 0) && k.row == r.start[b] + (a.done + c) * kChunk);
      CHECK(k.rows == std::min(kChunk, len - (a.done + c) * kChunk) && k.left == len - (a.done + c) * kChunk);
      if (c == 0) {
        int place = rank;
        if (r.B <= 64) {
          place = 0;
          for (int o = 0; o < r.B; ++o) {
            const int other = r.start[o + 1] - r.start[o];
            place += other > len || (other == len && o < b);
          }
        }
        CHECK(place < longer && walks[place].b < 0);
        walks[place] = Walk{b, k.row, a.window ? std::min(k.left, a.window * kChunk) : k.left, front + c};
        CHECK(space.walk_at(place + 1) <= space.bytes() && space.walk_at(0) == space.kFront + space.operands());
      }
    }
    if (mine < all || !a.window) {  // the slot behind the last is not this sequence's
      const size_t behind = (size_t)front + mine;
      if (behind < space.slots) CHECK(chunk_of(r, a.serial_len, (int)behind, a.window, a.done).b != b);
    }
    chunks_done[b] += mine;
    ++rank;
  }
  for (int i = 0; i < longer; ++i) {
    const Walk &k = walks[i];
    CHECK(k.b >= 0);
    const int chunks = (k.len + kChunk - 1) / kChunk;
    for (int c = 0; c < chunks; ++c) CHECK(taken[k.slot + c]);
    if (i % std::max(1, longer / 3)) continue;
    const int h = i % 2 ? a.H - 1 : 0;
    const int one = (a.dv + 15) / 16, two = (a.dv + 31) / 32;
    walk_through<F32, DK, 1>(a, space, k, h, 0, one);
    walk_through<F32, DK, 1>(a, space, k, h, one - 1, one);
    walk_through<F32, DK, 2>(a, space, k, h, 0, two);
    walk_through<F32, DK, 2>(a, space, k, h, two - 1, two);
  }
  return hipSuccess;
}
template hipError_t launch_chunks<false, 64>(const PrefillArgs &, hipStream_t);
template hipError_t launch_chunks<false, 128>(const PrefillArgs &, hipStream_t);
template hipError_t launch_chunks<false, 256>(const PrefillArgs &, hipStream_t);
template hipError_t launch_chunks<true, 64>(const PrefillArgs &, hipStream_t);
template hipError_t launch_chunks<true, 128>(const PrefillArgs &, hipStream_t);
template hipError_t launch_chunks<true, 256>(const PrefillArgs &, hipStream_t);

static std::mt19937_64 rng(3);
static int64_t upto(int64_t n) { return (int64_t)(rng() % (uint64_t)(n + 1)); }
template <typename T>
static T one_of(std::initializer_list<T> x) { return x.begin()[rng() % x.size()]; }

static void call(std::vector<int> lens, int before, int behind, int H, int Hk, int dk, int dv, int dtype, int family) {
  starts.assign(1, before);
  for (int n : lens) starts.push_back(starts.back() + n);
  PrefillArgs a;
  memset(&a, 0, sizeof(a));
  a.rows = PackedRows{starts.data(), (int)lens.size(), starts.back() + behind};
  a.H = H, a.Hk = Hk, a.dk = dk, a.dv = dv, a.family = family;
  const int64_t width = (int64_t)H * dv;
  a.v_stride = one_of<int64_t>({width, width + 64, 1 << 22});
  given = prefill_workspace_bytes(a, dtype);
  chunks_done.assign(lens.size(), 0);
  // addresses are told from a base that is never read
  a.workspace = reinterpret_cast<void *>((uintptr_t)1 << 40);
  float state_out;
  a.state_out = &state_out;
  const long serial = serial_launches, before_passes = passes;
  CHECK(launch_prefill(a, dtype, nullptr) == hipSuccess);
  ++calls;
  several += passes - before_passes > 1;
  narrow += passes - before_passes > 1 && H * lens.size() > 64;
  for (size_t b = 0; b < lens.size(); ++b) {
    const int all = std::max(1, (lens[b] + kChunk - 1) / kChunk);
    // all chunks, or none: a short sequence of a call with a token-by-token launch
    CHECK(chunks_done[b] == all || (chunks_done[b] == 0 && serial_launches > serial && lens[b] <= 24));
  }
}

}  // namespace sla

int main() {
  using namespace sla;
  for (int i = 0; i < 6000; ++i) {
    const int B = one_of({1, 2, 3, 7, 30, 63, 64, 65, 130, 400}), top = one_of({0, 1, 6, 7, 24, 25, 64, 65, 300, 3000});
    std::vector<int> lens;
    for (int b = 0; b < B; ++b) lens.push_back((int)upto(rng() % 5 ? top : top / 8));
    if (rng() % 3 == 0) lens[upto(B - 1)] = (int)upto(5000);
    const int Hk = one_of({1, 2, 3, 16, 64});
    call(lens, (int)(rng() % 2 ? 0 : upto(200)), (int)(rng() % 2 ? 0 : upto(200)), Hk * one_of({1, 2, 4}), Hk, one_of({64, 128, 256}),
         16 * one_of({1, 2, 3, 5, 8, 16, 64}), (int)upto(1), (int)upto(2));
  }
  // calls of several passes: long ones, alone and among short ones, many at once
  for (int i = 0; i < 60; ++i) {
    std::vector<int> lens;
    switch (i % 4) {
      case 0: lens = {(int)(200000 + upto(1 << 20))}; break;
      case 1: lens = {(int)upto(9), (int)(60000 + upto(400000)), 0, (int)upto(200000), 65}; break;
      case 2: lens.assign(64 + upto(100), (int)(1500 + upto(3000))); break;
      default:
        for (int b = 0; b < 300; ++b) lens.push_back((int)(rng() % 8 ? upto(30) : upto(8000)));
    }
    const int Hk = one_of({8, 16, 32});
    call(lens, (int)upto(3), (int)upto(3), Hk * one_of({1, 2}), Hk, one_of({64, 128, 256}), 16 * one_of({1, 2, 5, 8, 16}), (int)upto(1),
         (int)upto(2));
  }
  CHECK(several > 40 && narrow > 10 && serial_launches > 500);
  printf("%ld calls, %ld of several passes, %ld passes, %ld checks\n", calls, several, passes, checks);
  if (!failures) printf("prompt slot checks passed\n");
  return failures != 0;
}
