// conv_prefill.hip -- the short causal convolution along packed sequences,
// behind their conv states, and the states behind their last tokens.
//
// One wave = kStrip tokens of one sequence and 512 channels, 8 per lane.  A lane
// reads its strip's rows and the K - 1 rows in front of it (of the sequence, or
// of its state) at once and forms every window from registers: each row is read
// from memory once, and K - 1 of kStrip once more from a cache.  The bound is HBM,
// rows in, rows out: 16900 rows of 6144 bf16 channels 82 us, 5.1 TB/s, the rate of
// a large copy.  Longer strips, which read weights and the rows in front less often,
// were slower: 16 tokens 90 us, 32 tokens 98.  So were loads each behind its own
// bounds check (121 us), for which a wave waits one by one.
//
// The state's only readers are the windows of a sequence's first K - 1 tokens, all
// in its first wave, which therefore also writes the next state: from x, or the
// old state, if the sequence is shorter than K - 1.
#include "prompt_device.hpp"

namespace sla {
namespace {

constexpr int kThreads = 256;
constexpr int kChannels = kWave * 8;  // of a wave
constexpr int kStrip = 8;             // tokens of a wave
constexpr int kTokens = kStrip * kThreads / kWave;
static_assert(kStrip >= SLA_CONV_MAX_KERNEL - 1, "the first strip alone reads the state");

// 8 channels of a row as they lie in memory
template <typename T>
struct Packed {
  uint4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Packed<T> load_packed(const T *p) {
  Packed<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = reinterpret_cast<const uint4 *>(p)[i];
  return r;
}
__device__ __forceinline__ void widen(const Packed<bf16> &r, float (&f)[8]) {
  const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __uint_as_float(w[e] << 16);
    f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen(const Packed<float> &r, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f[4 * i] = __uint_as_float(r.w[i].x);
    f[4 * i + 1] = __uint_as_float(r.w[i].y);
    f[4 * i + 2] = __uint_as_float(r.w[i].z);
    f[4 * i + 3] = __uint_as_float(r.w[i].w);
  }
}

template <typename T, int K>
__global__ __launch_bounds__(kThreads) void conv_prefill_kernel(ConvPrefillArgs a, int chunks) {
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned wg = workgroup();
  const int slot = (int)(wg / (unsigned)chunks), chunk = (int)(wg % (unsigned)chunks);
  if (slot >= chunk_slots<kTokens>(a.rows, -1)) return;
  bool ok;
  const Chunk c = find_chunk<kTokens>(a.rows, -1, slot, lane, ok);
  if (a.status && chunk == 0 && threadIdx.x == 0) {
    if (!ok && slot < a.rows.B) a.status[slot] = SLA_ERR_LENGTH;
    if (ok && c.b >= 0 && c.first) a.status[c.b] = SLA_OK;
  }
  if (c.b < 0) return;
  const int d = chunk * kChannels + lane * 8;
  const int from = wave * kStrip, n = min(kStrip, c.rows - from);
  if (d >= a.D || (n <= 0 && !(c.first && wave == 0))) return;
  const T *x = static_cast<const T *>(a.x) + (int64_t)c.row * a.x_stride + d;
  // rows past the strip's end repeat its last one, so that no load waits for a branch
  const T *const strip = x + (int64_t)from * a.x_stride;
  Packed<T> rows[kStrip];
  if (n > 0)
#pragma unroll
    for (int i = 0; i < kStrip; ++i) rows[i] = load_packed(strip + (int64_t)min(i, n - 1) * a.x_stride);

  float z[kStrip + K - 1][8];  // z[K - 1 + i]: the strip's token i
  if (!c.first || wave > 0) {
    Packed<T> before[K - 1 > 0 ? K - 1 : 1];
#pragma unroll
    for (int i = 0; i < K - 1; ++i) before[i] = load_packed(strip + (i - (K - 1)) * a.x_stride);
#pragma unroll
    for (int i = 0; i < K - 1; ++i) widen(before[i], z[i]);
  } else {
#pragma unroll
    for (int i = 0; i < K - 1; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) z[i][e] = 0.f;
    if (a.state)
#pragma unroll
      for (int i = 0; i < K - 1; ++i) load_f32(a.state + ((size_t)c.b * (K - 1) + i) * a.D + d, z[i]);
  }

  if (K > 1 && c.first && wave == 0) {
    const int len = a.rows.start[c.b + 1] - c.row;
    float state[K - 1 > 0 ? K - 1 : 1][8];
#pragma unroll
    for (int i = 0; i < K - 1; ++i) {
      const int t = len - (K - 1) + i;  // the token of the next state's row i, below 0 the old state's row K - 1 + t
      if (t >= 0) {
        load_f32(x + (int64_t)t * a.x_stride, state[i]);
      } else {
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
          if (j == K - 1 + t)
#pragma unroll
            for (int e = 0; e < 8; ++e) state[i][e] = z[j][e];
      }
    }
#pragma unroll
    for (int i = 0; i < K - 1; ++i) store8(a.state_out + ((size_t)c.b * (K - 1) + i) * a.D + d, state[i]);
  }
  if (n <= 0) return;

  float w[8][K], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int i = 0; i < K; ++i) w[e][i] = a.weight[(size_t)(d + e) * K + i];
    bias[e] = a.bias ? a.bias[d + e] : 0.f;
  }
  T *y = static_cast<T *>(a.y) + (int64_t)(c.row + from) * a.D + d;
#pragma unroll
  for (int i = 0; i < kStrip; ++i) widen(rows[i], z[K - 1 + i]);
#pragma unroll
  for (int i = 0; i < kStrip; ++i) {
    if (i >= n) continue;
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float s = bias[e];
#pragma unroll
      for (int j = K - 1; j >= 0; --j) s = __builtin_fmaf(w[e][j], z[i + j][e], s);  // newest first, as conv.hip
      o[e] = a.silu ? silu(s) : s;
    }
    store8(y + (int64_t)i * a.D, o);
  }
}

template <typename T, int K>
hipError_t launch_k(const ConvPrefillArgs &a, hipStream_t s) {
  const int chunks = (a.D + kChannels - 1) / kChannels;
  hipLaunchKernelGGL((conv_prefill_kernel<T, K>), grid_of((uint64_t)chunk_slots<kTokens>(a.rows, -1) * chunks), dim3(kThreads), 0, s,
                     a, chunks);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const ConvPrefillArgs &a, hipStream_t s) {
  switch (a.K) {
    case 1: return launch_k<T, 1>(a, s);
    case 2: return launch_k<T, 2>(a, s);
    case 3: return launch_k<T, 3>(a, s);
    default: return launch_k<T, 4>(a, s);
  }
}

}  // namespace

hipError_t launch_conv_prefill(const ConvPrefillArgs &a, int dtype, hipStream_t s) {
  return dtype == SLA_DTYPE_BF16 ? launch_t<bf16>(a, s) : launch_t<float>(a, s);
}

}  // namespace sla
