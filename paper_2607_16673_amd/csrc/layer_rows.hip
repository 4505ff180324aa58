// layer_rows.hip -- the row-by-row steps around a recurrent layer's core: the
// recurrence's inputs (L2 norms of queries and keys, gates) in front of it, and
// the gated norm of its output behind it.
//
// One pass each: every element is read once and written once, so memory bounds
// them for many rows (32768 rows of 32 gates, 16 heads of 128 bf16: inputs 98 us, 5.6
// TB/s; of 32 heads: norm 142 us, 5.7 TB/s; a large copy reaches 5.1) and the launch for
// few (1024 rows: 4.4 and 5.1 us).  A head is the work of neighbouring lanes, 8
// elements (16 bytes of bf16) each; its sum of squares is a butterfly over those lanes.
#include "attn_device.hpp"
#include "prompt.hpp"

namespace sla {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f));
}

// log(1 + exp(x)), without overflow and with the tail of a small exp(x)
__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.f) + log1pf(expf(-fabsf(x))); }

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void inputs_kernel(InputsArgs a, unsigned head_blocks) {
  constexpr int kLanes = D / 8;
  constexpr int kHeads = kThreads / kLanes;  // heads of one workgroup
  const unsigned wg = workgroup();
  if (wg >= head_blocks) {  // gates: a thread each
    const int64_t i = (int64_t)(wg - head_blocks) * kThreads + threadIdx.x;
    if (i >= (int64_t)a.rows * a.H) return;
    const int64_t row = i / a.H;
    const int h = (int)(i - row * a.H);
    if (a.alpha) {
      const float x = to_f32(static_cast<const T *>(a.a)[row * a.a_stride + h]) + (a.dt_bias ? a.dt_bias[h] : 0.f);
      a.alpha[i] = expf(-expf(a.a_log[h]) * softplus(x));
    }
    if (a.beta) a.beta[i] = sigmoid(to_f32(static_cast<const T *>(a.b)[row * a.b_stride + h]));
    return;
  }
  const int64_t item = (int64_t)wg * kHeads + threadIdx.x / kLanes;
  if (item >= (int64_t)a.rows * 2 * a.Hk) return;  // whole heads: the shuffles stay among live lanes
  const int64_t row = item / (2 * a.Hk);
  int h = (int)(item - row * 2 * a.Hk);
  const bool query = h < a.Hk;
  if (!query) h -= a.Hk;
  const int e = threadIdx.x % kLanes * 8;
  const T *src = query ? static_cast<const T *>(a.q) + row * a.q_stride : static_cast<const T *>(a.k) + row * a.k_stride;
  float x[8];
  load_f32(src + (size_t)h * D + e, x);
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) ss += __shfl_xor(ss, o);
  const float r = (query ? a.q_scale : 1.f) / sqrtf(ss + a.eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= r;
  T *dst = static_cast<T *>(query ? a.q_out : a.k_out) + ((size_t)row * a.Hk + h) * a.repeat * D + e;
  for (int i = 0; i < a.repeat; ++i) store8(dst + (size_t)i * D, x);
}

template <typename T, int D>
hipError_t launch_inputs_d(const InputsArgs &a, hipStream_t s) {
  const uint64_t per = kThreads / (D / 8);
  const uint64_t heads = ((uint64_t)a.rows * 2 * a.Hk + per - 1) / per;
  const uint64_t gates = a.alpha || a.beta ? ((uint64_t)a.rows * a.H + kThreads - 1) / kThreads : 0;
  hipLaunchKernelGGL((inputs_kernel<T, D>), grid_of(heads + gates), dim3(kThreads), 0, s, a, (unsigned)heads);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_inputs_t(const InputsArgs &a, hipStream_t s) {
  switch (a.dk) {
    case 64: return launch_inputs_d<T, 64>(a, s);
    case 128: return launch_inputs_d<T, 128>(a, s);
    default: return launch_inputs_d<T, 256>(a, s);
  }
}

// L lanes to a head, P pieces of 8 elements to a lane: dv <= 8 L P.
template <typename X, typename T, int L, int P>
__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a) {
  constexpr int kHeads = kThreads / L;
  const int64_t item = (int64_t)workgroup() * kHeads + threadIdx.x / L;
  if (item >= (int64_t)a.rows * a.H) return;  // whole heads
  const int64_t row = item / a.H;
  const int h = (int)(item - row * a.H);
  const int lane = threadIdx.x % L;
  float x[P][8], z[P][8];
  float ss = 0.f;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int e = (p * L + lane) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[p][i] = z[p][i] = 0.f;
    if (e < a.dv) {
      load_f32(static_cast<const X *>(a.x) + item * a.dv + e, x[p]);
      if (a.gate != SLA_GATE_NONE) load_f32(static_cast<const T *>(a.z) + row * a.z_stride + (size_t)h * a.dv + e, z[p]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[p][i], x[p][i], ss);
  }
#pragma unroll
  for (int o = 1; o < L; o <<= 1) ss += __shfl_xor(ss, o);
  const float r = 1.f / sqrtf(ss / (float)a.dv + a.eps);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int e = (p * L + lane) * 8;
    if (e >= a.dv) continue;
    float w[8], y[8];
    if (a.weight) load_f32(a.weight + e, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i] = x[p][i] * r * (a.weight ? w[i] : 1.f);
      if (a.gate == SLA_GATE_SILU) y[i] *= silu(z[p][i]);
      else if (a.gate == SLA_GATE_SIGMOID) y[i] *= sigmoid(z[p][i]);
    }
    store8(static_cast<T *>(a.y) + item * a.dv + e, y);
  }
}

template <typename X, typename T, int L, int P>
hipError_t launch_norm_l(const NormArgs &a, hipStream_t s) {
  const uint64_t per = kThreads / L;
  hipLaunchKernelGGL((norm_kernel<X, T, L, P>), grid_of(((uint64_t)a.rows * a.H + per - 1) / per), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <typename X, typename T>
hipError_t launch_norm_t(const NormArgs &a, hipStream_t s) {
  if (a.dv <= 16) return launch_norm_l<X, T, 2, 1>(a, s);
  if (a.dv <= 32) return launch_norm_l<X, T, 4, 1>(a, s);
  if (a.dv <= 64) return launch_norm_l<X, T, 8, 1>(a, s);
  if (a.dv <= 128) return launch_norm_l<X, T, 16, 1>(a, s);
  if (a.dv <= 256) return launch_norm_l<X, T, 32, 1>(a, s);
  if (a.dv <= 512) return launch_norm_l<X, T, 64, 1>(a, s);
  return launch_norm_l<X, T, 64, 2>(a, s);
}

}  // namespace

hipError_t launch_recurrent_inputs(const InputsArgs &a, int dtype, hipStream_t s) {
  return dtype == SLA_DTYPE_BF16 ? launch_inputs_t<bf16>(a, s) : launch_inputs_t<float>(a, s);
}

hipError_t launch_gated_norm(const NormArgs &a, int x_dtype, int dtype, hipStream_t s) {
  if (x_dtype == SLA_DTYPE_BF16)
    return dtype == SLA_DTYPE_BF16 ? launch_norm_t<bf16, bf16>(a, s) : launch_norm_t<bf16, float>(a, s);
  return dtype == SLA_DTYPE_BF16 ? launch_norm_t<float, bf16>(a, s) : launch_norm_t<float, float>(a, s);
}

}  // namespace sla
