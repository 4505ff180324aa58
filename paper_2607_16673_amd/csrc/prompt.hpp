// prompt.hpp -- launch interface between the host ABI (prompt_api.cpp) and the
// kernels of a recurrent layer's prompt pass: the recurrence and the
// convolution over packed sequences, and the row-by-row steps around them.
// Plain structs of device pointers and sizes; the host side has already
// validated what it can see.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace sla {

// Packed sequences: sequence b has the rows start[b] .. start[b + 1] - 1 of `tokens`.
struct PackedRows {
  const int32_t *start;  // [B + 1]
  int32_t B, tokens;
};

struct PrefillArgs {
  PackedRows rows;
  int32_t H, Hk, dk, dv;
  int32_t family;
  int32_t serial_len;    // sequences up to this length go token by token, longer ones in chunks (-1: all in chunks)
  int32_t window, done;  // a pass of the chunked kernels takes so many chunks of each sequence, behind so many (0: all)
  const float *state;    // [B][H][dk][dv] or null
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;  // elements from row to row
  const float *alpha, *beta;             // [T][H]
  void *out;             // [T][H][dv]
  float *state_out;
  void *workspace;
  int32_t *status;
};

struct ConvPrefillArgs {
  PackedRows rows;
  int32_t D, K;
  bool silu;
  const float *state;    // [B][K-1][D] or null
  const void *x;
  int64_t x_stride;
  const float *weight;   // [D][K]
  const float *bias;     // [D] or null
  void *y;               // [T][D]
  float *state_out;
  int32_t *status;
};

struct InputsArgs {
  int32_t rows, H, Hk, repeat, dk;
  float q_scale, eps;
  const void *q, *k, *a, *b;
  int64_t q_stride, k_stride, a_stride, b_stride;
  const float *a_log, *dt_bias;
  void *q_out, *k_out;
  float *alpha, *beta;
};

struct NormArgs {
  int32_t rows, H, dv;
  int32_t gate;
  float eps;
  const void *x, *z;
  int64_t z_stride;
  const float *weight;
  void *y;
};

// Each launcher returns hipSuccess or the launch error.  `dtype` is
// SLA_DTYPE_F32 or SLA_DTYPE_BF16.
hipError_t launch_prefill(const PrefillArgs &a, int dtype, hipStream_t s);
size_t prefill_workspace_bytes(const PrefillArgs &a, int dtype);
hipError_t launch_conv_prefill(const ConvPrefillArgs &a, int dtype, hipStream_t s);
hipError_t launch_recurrent_inputs(const InputsArgs &a, int dtype, hipStream_t s);
hipError_t launch_gated_norm(const NormArgs &a, int x_dtype, int dtype, hipStream_t s);

}  // namespace sla
