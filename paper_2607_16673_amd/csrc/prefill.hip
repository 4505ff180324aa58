// prefill.hip -- the recurrence over packed sequences: which of them go token by
// token and which in chunks (prefill_chunk.hip), and the kernel of the former.
//
// One workgroup = one (sequence, head) and 64 columns of its state, which stay in
// registers from the first token to the last: wave w holds the rows w dk / 4 ..,
// a lane 4 columns of every fourth of them.  With a = S_{t-1} k and b = S_{t-1} q
// reduced at once, a token needs one exchange between the waves:
//     u = beta (v - alpha a),  o = alpha b + u (k . q),  S = alpha S + u k^T.
// Queries, keys and gates of 16 tokens are staged in LDS at a time.  One read and
// one write of the state bound it for sequences of a token (256 of 16 heads of 128 x
// 256: 212 us, 5.1 TB/s, the rate of a large copy), the chain of exchanges (1.2 us a
// token where the chip is not full) for longer ones.
#include <algorithm>
#include <type_traits>

#include "prefill_chunk.hpp"

namespace sla {
namespace {

constexpr int kThreads = 256;
constexpr int kCols = 64;   // columns of a workgroup
constexpr int kStage = 16;  // tokens staged at a time

__device__ __forceinline__ void load4(const float *p, float (&x)[4]) { load_f32(p, x); }
__device__ __forceinline__ void load4(const bf16 *p, float (&x)[4]) {
  const uint2 w = *reinterpret_cast<const uint2 *>(p);
  x[0] = __uint_as_float(w.x << 16);
  x[1] = __uint_as_float(w.x & 0xffff0000u);
  x[2] = __uint_as_float(w.y << 16);
  x[3] = __uint_as_float(w.y & 0xffff0000u);
}

template <typename T, int DK, bool DELTA>
__global__ __launch_bounds__(kThreads) void serial_kernel(PrefillArgs a, int slabs) {
  constexpr int kRows = DK / 16;  // of a lane
  __shared__ float sk[kStage][DK], sq[kStage][DK];
  __shared__ float salpha[kStage], sbeta[kStage];
  __shared__ float red[2][4][9][16];  // [parity][wave][a 0-3, b 0-3, k.q][columns of 4]
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int g = lane / 16, cl = lane % 16;
  const unsigned wg = workgroup();
  const unsigned unit = wg / (unsigned)slabs;
  const int slab = (int)(wg % (unsigned)slabs);
  if (unit >= (unsigned)a.rows.B * (unsigned)a.H) return;
  const int b = (int)(unit / (unsigned)a.H), h = (int)(unit % (unsigned)a.H);
  const int start = a.rows.start[b], len = a.rows.start[b + 1] - start;
  const bool ok = starts_ok(a.rows, lane);
  if (ok && len > a.serial_len) return;
  if (a.status && h == 0 && slab == 0 && threadIdx.x == 0) a.status[b] = ok ? SLA_OK : SLA_ERR_LENGTH;
  if (!ok) return;
  const int col = slab * kCols + cl * 4;
  const bool live = col < a.dv;
  const int kh = h / (a.H / a.Hk);

  // lane's row i: wave DK / 4 + 4 i + g
  float S[kRows][4];
  const size_t base = ((size_t)unit * DK + wave * (DK / 4) + g) * a.dv + col;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
#pragma unroll
    for (int e = 0; e < 4; ++e) S[i][e] = 0.f;
    if (a.state && live) load4(a.state + base + (size_t)(4 * i) * a.dv, S[i]);
  }
  const T *q = static_cast<const T *>(a.q) + (int64_t)start * a.q_stride + (size_t)kh * DK;
  const T *k = static_cast<const T *>(a.k) + (int64_t)start * a.k_stride + (size_t)kh * DK;
  const T *v = static_cast<const T *>(a.v) + (int64_t)start * a.v_stride + (size_t)h * a.dv + col;
  T *out = static_cast<T *>(a.out) + ((size_t)start * a.H + h) * a.dv + col;
  const size_t gate = (size_t)start * a.H + h;

  for (int t0 = 0; t0 < len; t0 += kStage) {
    const int n = min(kStage, len - t0);
    __syncthreads();  // the last stage has been read
    for (int i = threadIdx.x; i < n * (DK / 8); i += kThreads) {
      const int t = i / (DK / 8), e = i % (DK / 8) * 8;
      float x[8];
      load_f32(k + (int64_t)(t0 + t) * a.k_stride + e, x);
      store8(&sk[t][e], x);
      load_f32(q + (int64_t)(t0 + t) * a.q_stride + e, x);
      store8(&sq[t][e], x);
    }
    if (threadIdx.x < n) {
      salpha[threadIdx.x] = a.alpha ? a.alpha[gate + (size_t)(t0 + threadIdx.x) * a.H] : 1.f;
      sbeta[threadIdx.x] = DELTA ? a.beta[gate + (size_t)(t0 + threadIdx.x) * a.H] : 1.f;
    }
    __syncthreads();
    for (int t = 0; t < n; ++t) {
      float x[9] = {};  // S k, S q of 4 columns, k . q
      float kr[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int r = wave * (DK / 4) + 4 * i + g;
        kr[i] = sk[t][r];
        const float qr = sq[t][r];
        x[8] = __builtin_fmaf(kr[i], qr, x[8]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (DELTA) x[e] = __builtin_fmaf(S[i][e], kr[i], x[e]);
          x[4 + e] = __builtin_fmaf(S[i][e], qr, x[4 + e]);
        }
      }
#pragma unroll
      for (int e = DELTA ? 0 : 4; e < 9; ++e) {
        x[e] += __shfl_xor(x[e], 16);
        x[e] += __shfl_xor(x[e], 32);
        if (g == 0) red[t & 1][wave][e][cl] = x[e];
      }
      float val[4] = {};
      if (live) load4(v + (int64_t)(t0 + t) * a.v_stride, val);
      __syncthreads();
      float s[9] = {};
#pragma unroll
      for (int e = DELTA ? 0 : 4; e < 9; ++e)
#pragma unroll
        for (int w = 0; w < 4; ++w) s[e] += red[t & 1][w][e][cl];
      const float alpha = salpha[t], beta = sbeta[t];
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float u = DELTA ? beta * (val[e] - alpha * s[e]) : val[e];
        o[e] = __builtin_fmaf(u, s[8], alpha * s[4 + e]);
#pragma unroll
        for (int i = 0; i < kRows; ++i) S[i][e] = apply_factor(S[i][e], alpha, kr[i], u);
      }
      if (live && threadIdx.x < 16) store4(out + (size_t)(t0 + t) * a.H * a.dv, o);
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i)
    if (live) store4(a.state_out + base + (size_t)(4 * i) * a.dv, S[i]);
}

template <typename T, int DK>
hipError_t launch_serial(const PrefillArgs &a, hipStream_t s) {
  const int slabs = (a.dv + kCols - 1) / kCols;
  const dim3 grid = grid_of((uint64_t)a.rows.B * a.H * slabs);
  if (a.family == SLA_FAMILY_DECAY)
    hipLaunchKernelGGL((serial_kernel<T, DK, false>), grid, dim3(kThreads), 0, s, a, slabs);
  else
    hipLaunchKernelGGL((serial_kernel<T, DK, true>), grid, dim3(kThreads), 0, s, a, slabs);
  return hipGetLastError();
}

// Which sequences go token by token: a chunk takes the chunked kernels about as long
// whether it is full or not.  16 heads of 128, microseconds token by token and in
// chunks: one sequence of 6 tokens 11.9 and 13.7, of 8 tokens 14.7 and 13.7; 8
// sequences of 6 tokens 18.1 and 21.6; 256 sequences, whose states fill the chip, of 4
// tokens 126 and 452, of 24 tokens 388 and 464.  Lengths are on the device: each kernel
// passes over the others' sequences, and a launch that may find none of its own costs
// 3 us.  So where all tokens together are few enough for one sequence, one launch does;
// where an average sequence is long (few workgroups: longer than the limit; many: 64
// tokens) all go in chunks, and short ones among them cost little beside the others.
constexpr int kFewSerial = 6, kManySerial = 24, kManyAverage = 64;
// workgroups of a sequence, and the batches whose workgroups fill the chip
int64_t workgroups_of(const PrefillArgs &a) { return (int64_t)a.H * ((a.dv + kCols - 1) / kCols); }
int64_t filling_batch() { return 4 * device_cus(); }

PrefillArgs divided(PrefillArgs a) {
  const bool fills = a.rows.B * workgroups_of(a) >= filling_batch();
  a.serial_len = fills ? kManySerial : kFewSerial;
  if (a.rows.tokens > (fills ? kManyAverage : kFewSerial) * (int64_t)a.rows.B) a.serial_len = -1;
  return a;
}

// Sequences in chunks that a call of up to so many tokens and sequences can have: the
// most of the three divisions of its work, so that a workspace for the largest call
// serves all smaller ones, whichever way they go.
int64_t most_chunked(const PrefillArgs &a) {
  const int64_t T = a.rows.tokens, B = a.rows.B;
  const int64_t few = (filling_batch() - 1) / workgroups_of(a);  // the largest batch that does not fill the chip
  const int64_t all_of_few = T > 0 ? (T - 1) / kFewSerial : 0;   // ... all of it in chunks, or those past the limit
  const int64_t many = T / (kManySerial + 1);                    // as many as are all in chunks (T > 64 B), or more
  return std::min(B, std::max(many, std::min(few, all_of_few)));
}
bool all_serial(const PrefillArgs &a) { return a.rows.tokens <= a.serial_len; }

// Slots of the workspace.  All chunks of a call at once take 0.9 to 3.5 KB a token and
// head, so past kMostBytes, or eight times the states where that is more, a call goes in passes:
// each takes some chunks of every sequence that has any left, from the states that the
// pass before has written to state_out.
constexpr int64_t kMostBytes = 2ll << 30;
int64_t workspace_slots(const PrefillArgs &a, size_t of_slot) {
  const int64_t walks = most_chunked(a), all = a.rows.tokens / kChunk + walks;
  const int64_t states = (int64_t)a.rows.B * a.H * a.dk * a.dv * 4;
  return std::min(all, std::max(walks, std::max(kMostBytes, 8 * states) / (int64_t)of_slot));
}

// The chunks in one pass, or in several.  The lengths are on the device: the host goes by
// how many sequences can have more than the chunks that are done, so passes grow as
// fewer can, and there are 1 + ln(B) times as many as evenly long sequences fill; the
// others look at the longest sequence and end.
template <bool F32, int DK>
hipError_t launch_passes(PrefillArgs a, hipStream_t s) {
  const int64_t slots = workspace_slots(a, ChunkSpace<F32, DK>::of_slot(a.H, a.Hk));
  if (chunk_slots<kChunk>(a.rows, a.serial_len) <= slots) return launch_chunks<F32, DK>(a, s);
  const int64_t most = (a.rows.tokens + kChunk - 1) / kChunk;  // chunks of a sequence
  for (int64_t left = most; left > 0; left -= a.window) {
    a.done = (int32_t)(most - left);
    if (a.done > 0) {
      a.serial_len = a.done * kChunk;
      a.state = a.state_out;
    }
    const int64_t longer = most_longer(a.rows, a.serial_len);
    a.window = (int32_t)std::min(left, slots / longer);
    const hipError_t e = launch_chunks<F32, DK>(a, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <bool F32, int DK>
hipError_t launch_dk(const PrefillArgs &a, hipStream_t s) {
  using T = typename std::conditional<F32, float, bf16>::type;
  if (a.serial_len >= 0) {
    const hipError_t e = launch_serial<T, DK>(a, s);
    if (e != hipSuccess || all_serial(a)) return e;
  }
  return launch_passes<F32, DK>(a, s);
}

template <bool F32>
hipError_t launch_t(const PrefillArgs &a, hipStream_t s) {
  switch (a.dk) {
    case 64: return launch_dk<F32, 64>(a, s);
    case 128: return launch_dk<F32, 128>(a, s);
    default: return launch_dk<F32, 256>(a, s);
  }
}

template <bool F32, int DK>
size_t bytes_dk(const PrefillArgs &a) {
  using Space = ChunkSpace<F32, DK>;
  return Space{nullptr, (size_t)workspace_slots(a, Space::of_slot(a.H, a.Hk)), (size_t)most_chunked(a), a.H, a.Hk}.bytes();
}
template <bool F32>
size_t bytes_t(const PrefillArgs &a) {
  switch (a.dk) {
    case 64: return bytes_dk<F32, 64>(a);
    case 128: return bytes_dk<F32, 128>(a);
    default: return bytes_dk<F32, 256>(a);
  }
}

}  // namespace

size_t prefill_workspace_bytes(const PrefillArgs &a, int dtype) {
  if (most_chunked(a) == 0) return 0;  // fewer tokens than any sequence in chunks has
  return dtype == SLA_DTYPE_BF16 ? bytes_t<false>(a) : bytes_t<true>(a);
}

hipError_t launch_prefill(const PrefillArgs &a, int dtype, hipStream_t s) {
  return dtype == SLA_DTYPE_BF16 ? launch_t<false>(divided(a), s) : launch_t<true>(divided(a), s);
}

}  // namespace sla
