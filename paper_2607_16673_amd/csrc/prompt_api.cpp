// prompt_api.cpp -- host side of the prompt-pass calls of include/sla.h:
// argument validation, alias checks and kernel launches on the caller's stream.
// Nothing here allocates device memory or keeps state between calls.
#include <stdint.h>
#include <string.h>

#include <cmath>

#include "prompt.hpp"
#include "sla.h"

namespace {

constexpr int32_t kMaxRows = 1 << 30;
constexpr int64_t kMaxStride = 1 << 22;
constexpr size_t kMost = (size_t)1 << 56;  // bytes of a buffer past any memory

bool dtype_ok(int dtype) { return dtype == SLA_DTYPE_F32 || dtype == SLA_DTYPE_BF16; }
size_t act_bytes(int dtype) { return dtype == SLA_DTYPE_BF16 ? 2 : 4; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Span {
  const void *p;  // NULL: none
  size_t bytes;
};

// count x width x size bytes at p
Span span_of(const void *p, size_t count, size_t width, size_t size) {
  const unsigned __int128 bytes = (unsigned __int128)count * width * size;
  return Span{p, bytes < kMost ? (size_t)bytes : kMost};
}

// `rows` rows of `width` elements, `stride` apart
Span rows_of(const void *p, int32_t rows, int64_t width, int64_t stride, size_t size) {
  return Span{rows > 0 ? p : nullptr, rows > 0 ? ((size_t)(rows - 1) * (size_t)stride + (size_t)width) * size : 0};
}

bool overlaps(const Span &x, const Span &y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
  return x.p && y.p && x.bytes && y.bytes && a < b + y.bytes && b < a + x.bytes;
}

// Whether an output overlaps another one or a buffer the call reads.
template <int W, int N>
bool aliased(const Span (&writes)[W], const Span (&reads)[N]) {
  for (int i = 0; i < W; ++i) {
    for (int j = 0; j < i; ++j)
      if (overlaps(writes[i], writes[j])) return true;
    for (int j = 0; j < N; ++j)
      if (overlaps(writes[i], reads[j])) return true;
  }
  return false;
}

bool stride_ok(int64_t stride, size_t size) { return stride <= kMaxStride && stride * (int64_t)size % 16 == 0; }

int hip_status(hipError_t e) { return e == hipSuccess ? SLA_OK : SLA_ERR_HIP; }

bool rows_ok(int32_t rows) { return rows >= 0 && rows <= kMaxRows; }

int check_prefill(const sla_prefill_shape *s) {
  if (!s) return SLA_ERR_NULL;
  if (!rows_ok(s->tokens) || s->batch < 1 || s->batch > 65535) return SLA_ERR_SHAPE;
  if (s->heads < 1 || s->heads > (1 << 16) || s->k_heads < 1 || s->heads % s->k_heads) return SLA_ERR_SHAPE;
  if (s->d_k < 1 || s->d_v < 16 || s->d_v > 1024 || s->d_v % 16) return SLA_ERR_SHAPE;
  if (!dtype_ok(s->qkv_dtype)) return SLA_ERR_DTYPE;
  if (s->family < SLA_FAMILY_GDN || s->family > SLA_FAMILY_GLA) return SLA_ERR_SHAPE;
  if (s->family == SLA_FAMILY_GLA) return SLA_ERR_UNSUPPORTED;
  if (s->d_k != 64 && s->d_k != 128 && s->d_k != 256) return SLA_ERR_UNSUPPORTED;
  // the numbers of a launch's workgroups fit 32 bits, a row's elements a stride
  if (((int64_t)s->tokens / 64 + s->batch) * s->heads >= (1ll << 31)) return SLA_ERR_SHAPE;
  if ((int64_t)s->batch * s->heads * ((s->d_v + 15) / 16) >= (1ll << 31)) return SLA_ERR_SHAPE;
  if ((int64_t)s->heads * (s->d_v > s->d_k ? s->d_v : s->d_k) > kMaxStride) return SLA_ERR_SHAPE;
  return SLA_OK;
}

sla::PrefillArgs prefill_args(const sla_prefill_shape *s) {
  sla::PrefillArgs a;
  memset(&a, 0, sizeof(a));
  a.rows = sla::PackedRows{nullptr, s->batch, s->tokens};
  a.H = s->heads;
  a.Hk = s->k_heads;
  a.dk = s->d_k;
  a.dv = s->d_v;
  a.family = s->family;
  return a;
}

int check_conv(const sla_conv_prefill_shape *s) {
  if (!s) return SLA_ERR_NULL;
  if (!rows_ok(s->tokens) || s->batch < 1 || s->batch > 65535) return SLA_ERR_SHAPE;
  if (s->channels < 8 || s->channels % 8 || s->channels > (1 << 20)) return SLA_ERR_SHAPE;
  if (s->kernel_size < 1 || s->kernel_size > SLA_CONV_MAX_KERNEL) return SLA_ERR_SHAPE;
  if (!dtype_ok(s->x_dtype)) return SLA_ERR_DTYPE;
  if (s->activation != SLA_ACT_NONE && s->activation != SLA_ACT_SILU) return SLA_ERR_SHAPE;
  // the numbers of a launch's workgroups fit 32 bits
  if (((int64_t)s->tokens / 8 + s->batch) * ((s->channels + 511) / 512) >= (1ll << 31)) return SLA_ERR_SHAPE;
  return SLA_OK;
}

}  // namespace

extern "C" {

size_t sla_prefill_workspace_bytes(const sla_prefill_shape *shape) {
  if (check_prefill(shape) != SLA_OK) return 0;
  return sla::prefill_workspace_bytes(prefill_args(shape), shape->qkv_dtype);
}

int sla_prefill(const sla_prefill_shape *shape, const float *state, const void *q, int64_t q_stride, const void *k,
                int64_t k_stride, const void *v, int64_t v_stride, const float *alpha, const float *beta,
                const int32_t *seq_start, void *out, float *state_out, void *workspace, size_t workspace_bytes,
                int32_t *status, hipStream_t stream) {
  const int st = check_prefill(shape);
  if (st != SLA_OK) return st;
  const int32_t T = shape->tokens;
  const bool reads_alpha = shape->family != SLA_FAMILY_DELTANET, reads_beta = shape->family != SLA_FAMILY_DECAY;
  if (!seq_start || !state_out) return SLA_ERR_NULL;
  if (T > 0 && (!q || !k || !v || !out || (reads_alpha && !alpha) || (reads_beta && !beta))) return SLA_ERR_NULL;
  const int64_t kd = (int64_t)shape->k_heads * shape->d_k, vd = (int64_t)shape->heads * shape->d_v;
  if (q_stride < kd || k_stride < kd || v_stride < vd) return SLA_ERR_SHAPE;
  sla::PrefillArgs a = prefill_args(shape);
  const size_t need = sla::prefill_workspace_bytes(a, shape->qkv_dtype);
  if (need && !workspace) return SLA_ERR_NULL;
  if (need && workspace_bytes < need) return SLA_ERR_SHAPE;
  const size_t w = act_bytes(shape->qkv_dtype);
  const size_t states = (size_t)shape->batch * shape->heads * shape->d_k;
  const Span writes[] = {rows_of(out, T, vd, vd, w), span_of(state_out, states, shape->d_v, 4),
                         Span{need ? workspace : nullptr, need}, span_of(status, shape->batch, 1, 4)};
  const Span reads[] = {rows_of(q, T, kd, q_stride, w),
                        rows_of(k, T, kd, k_stride, w),
                        rows_of(v, T, vd, v_stride, w),
                        rows_of(reads_alpha ? alpha : nullptr, T, shape->heads, shape->heads, 4),
                        rows_of(reads_beta ? beta : nullptr, T, shape->heads, shape->heads, 4),
                        span_of(seq_start, (size_t)shape->batch + 1, 1, 4),
                        span_of(state != state_out ? state : nullptr, states, shape->d_v, 4)};
  if (aliased(writes, reads)) return SLA_ERR_ALIAS;
  if (!aligned16(state) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(state_out) ||
      !aligned16(workspace) || !stride_ok(q_stride, w) || !stride_ok(k_stride, w) || !stride_ok(v_stride, w))
    return SLA_ERR_UNSUPPORTED;
  a.rows.start = seq_start;
  a.state = state;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.alpha = reads_alpha ? alpha : nullptr;
  a.beta = reads_beta ? beta : nullptr;
  a.out = out;
  a.state_out = state_out;
  a.workspace = workspace;
  a.status = status;
  return hip_status(sla::launch_prefill(a, shape->qkv_dtype, stream));
}

int sla_conv_prefill(const sla_conv_prefill_shape *shape, const float *conv_state, const void *x, int64_t x_stride,
                     const float *weight, const float *bias, const int32_t *seq_start, void *y, float *conv_state_out,
                     int32_t *status, hipStream_t stream) {
  const int st = check_conv(shape);
  if (st != SLA_OK) return st;
  const int32_t T = shape->tokens, D = shape->channels, K = shape->kernel_size;
  if (!weight || !seq_start || (T > 0 && (!x || !y)) || (K > 1 && !conv_state_out)) return SLA_ERR_NULL;
  if (x_stride < D) return SLA_ERR_SHAPE;
  const size_t w = act_bytes(shape->x_dtype);
  const size_t rows = (size_t)shape->batch * (K - 1);
  if (K == 1) conv_state = conv_state_out = nullptr;
  const Span writes[] = {rows_of(y, T, D, D, w), span_of(conv_state_out, rows, D, 4), span_of(status, shape->batch, 1, 4)};
  const Span reads[] = {rows_of(x, T, D, x_stride, w), span_of(weight, D, K, 4), span_of(bias, D, 1, 4),
                        span_of(seq_start, (size_t)shape->batch + 1, 1, 4),
                        span_of(conv_state != conv_state_out ? conv_state : nullptr, rows, D, 4)};
  if (aliased(writes, reads)) return SLA_ERR_ALIAS;
  if (!aligned16(conv_state) || !aligned16(x) || !aligned16(weight) || !aligned16(bias) || !aligned16(y) ||
      !aligned16(conv_state_out) || !stride_ok(x_stride, w))
    return SLA_ERR_UNSUPPORTED;
  sla::ConvPrefillArgs a;
  memset(&a, 0, sizeof(a));
  a.rows = sla::PackedRows{seq_start, shape->batch, T};
  a.D = D;
  a.K = K;
  a.silu = shape->activation == SLA_ACT_SILU;
  a.state = conv_state;
  a.x = x;
  a.x_stride = x_stride;
  a.weight = weight;
  a.bias = bias;
  a.y = y;
  a.state_out = conv_state_out;
  a.status = status;
  return hip_status(sla::launch_conv_prefill(a, shape->x_dtype, stream));
}

int sla_recurrent_inputs(const sla_inputs_shape *s, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                         const void *a, int64_t a_stride, const void *b, int64_t b_stride, const float *a_log,
                         const float *dt_bias, void *q_out, void *k_out, float *alpha, float *beta, hipStream_t stream) {
  if (!s) return SLA_ERR_NULL;
  if (!rows_ok(s->rows) || s->heads < 1 || s->heads > (1 << 16) || s->k_heads < 1 || s->k_heads > (1 << 16) ||
      s->repeat < 1 || s->repeat > 64 || s->d_k < 1 || !std::isfinite(s->q_scale) || !(s->eps >= 0.f) ||
      !std::isfinite(s->eps))
    return SLA_ERR_SHAPE;
  if (!dtype_ok(s->dtype)) return SLA_ERR_DTYPE;
  if (s->d_k != 64 && s->d_k != 128 && s->d_k != 256) return SLA_ERR_UNSUPPORTED;
  const int64_t kd = (int64_t)s->k_heads * s->d_k;
  if (kd > kMaxStride) return SLA_ERR_SHAPE;
  // a launch's workgroups are numbered in 32 bits: 8 heads or 256 gates to one at least
  if (((int64_t)s->rows * 2 * s->k_heads) / 8 + ((int64_t)s->rows * s->heads) / 256 >= (1ll << 31)) return SLA_ERR_SHAPE;
  const int32_t N = s->rows;
  if (N > 0) {
    if (!q || !k || !q_out || !k_out) return SLA_ERR_NULL;
    if (alpha ? !a || !a_log : !!a) return SLA_ERR_NULL;
    if (beta ? !b : !!b) return SLA_ERR_NULL;
  }
  if (q_stride < kd || k_stride < kd || (alpha && a_stride < s->heads) || (beta && b_stride < s->heads))
    return SLA_ERR_SHAPE;
  const size_t w = act_bytes(s->dtype);
  const int64_t od = kd * s->repeat;
  const Span writes[] = {rows_of(q_out, N, od, od, w), rows_of(k_out, N, od, od, w),
                         rows_of(alpha, N, s->heads, s->heads, 4), rows_of(beta, N, s->heads, s->heads, 4)};
  const Span reads[] = {rows_of(q, N, kd, q_stride, w),
                        rows_of(k, N, kd, k_stride, w),
                        rows_of(alpha ? a : nullptr, N, s->heads, a_stride, w),
                        rows_of(beta ? b : nullptr, N, s->heads, b_stride, w),
                        span_of(alpha ? a_log : nullptr, s->heads, 1, 4),
                        span_of(alpha ? dt_bias : nullptr, s->heads, 1, 4)};
  if (aliased(writes, reads)) return SLA_ERR_ALIAS;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !stride_ok(q_stride, w) ||
      !stride_ok(k_stride, w) || (alpha && a_stride > kMaxStride) || (beta && b_stride > kMaxStride))
    return SLA_ERR_UNSUPPORTED;
  if (N == 0) return SLA_OK;
  sla::InputsArgs g;
  memset(&g, 0, sizeof(g));
  g.rows = N;
  g.H = s->heads;
  g.Hk = s->k_heads;
  g.repeat = s->repeat;
  g.dk = s->d_k;
  g.q_scale = s->q_scale;
  g.eps = s->eps;
  g.q = q;
  g.k = k;
  g.a = a;
  g.b = b;
  g.q_stride = q_stride;
  g.k_stride = k_stride;
  g.a_stride = a_stride;
  g.b_stride = b_stride;
  g.a_log = a_log;
  g.dt_bias = dt_bias;
  g.q_out = q_out;
  g.k_out = k_out;
  g.alpha = alpha;
  g.beta = beta;
  return hip_status(sla::launch_recurrent_inputs(g, s->dtype, stream));
}

int sla_gated_norm(const sla_norm_shape *s, const void *x, const void *z, int64_t z_stride, const float *weight, void *y,
                   hipStream_t stream) {
  if (!s) return SLA_ERR_NULL;
  if (!rows_ok(s->rows) || s->heads < 1 || s->heads > (1 << 16) || s->d_v < 16 || s->d_v > 1024 || s->d_v % 16 ||
      !(s->eps >= 0.f) || !std::isfinite(s->eps))
    return SLA_ERR_SHAPE;
  if (!dtype_ok(s->x_dtype) || !dtype_ok(s->dtype)) return SLA_ERR_DTYPE;
  if (s->gate < SLA_GATE_NONE || s->gate > SLA_GATE_SIGMOID) return SLA_ERR_SHAPE;
  const int64_t d = (int64_t)s->heads * s->d_v;
  // a launch's workgroups are numbered in 32 bits: 2 heads or more to one
  if (d > kMaxStride || (int64_t)s->rows * s->heads / 2 >= (1ll << 31)) return SLA_ERR_SHAPE;
  const int32_t N = s->rows;
  const bool gated = s->gate != SLA_GATE_NONE;
  if (N > 0 && (!x || !y || (gated && !z))) return SLA_ERR_NULL;
  if (gated && z_stride < d) return SLA_ERR_SHAPE;
  const size_t w = act_bytes(s->dtype), xw = act_bytes(s->x_dtype);
  // every head is read whole before it is written, so y may be x or z
  const bool over_x = y == x && xw == w, over_z = gated && y == z && z_stride == d;
  const Span writes[] = {rows_of(y, N, d, d, w)};
  const Span reads[] = {rows_of(over_x ? nullptr : x, N, d, d, xw), rows_of(gated && !over_z ? z : nullptr, N, d, z_stride, w),
                        span_of(weight, s->d_v, 1, 4)};
  if (aliased(writes, reads)) return SLA_ERR_ALIAS;
  if (!aligned16(x) || !aligned16(y) || !aligned16(weight) || (gated && (!aligned16(z) || !stride_ok(z_stride, w))))
    return SLA_ERR_UNSUPPORTED;
  if (N == 0) return SLA_OK;
  sla::NormArgs a;
  memset(&a, 0, sizeof(a));
  a.rows = N;
  a.H = s->heads;
  a.dv = s->d_v;
  a.gate = s->gate;
  a.eps = s->eps;
  a.x = x;
  a.z = z;
  a.z_stride = z_stride;
  a.weight = weight;
  a.y = y;
  return hip_status(sla::launch_gated_norm(a, s->x_dtype, s->dtype, stream));
}

}  // extern "C"
