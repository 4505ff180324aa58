// The host side of the prompt-pass calls (prompt_api.cpp) for AddressSanitizer
// and UndefinedBehaviorSanitizer builds (built and run by
// tests/test_prompt_sanitizers.py; no GPU code is involved: the launchers are
// stubs that look at what they are given).  Random shapes, sizes at the ends of
// their types, and pointers at the ends of the address space go through the
// argument checks; a launcher may only ever see what the checks let pass.
#include <stdint.h>
#include <stdio.h>

#include <cmath>
#include <random>

#include "prompt.hpp"
#include "sla.h"

static long launched[4] = {}, refused = 0, failures = 0;
#define CHECK(c)                                                     \
  do {                                                               \
    if (!(c)) {                                                      \
      fprintf(stderr, "check failed: %s (line %d)\n", #c, __LINE__); \
      ++failures;                                                    \
    }                                                                \
  } while (0)

namespace sla {
static void seen(const PackedRows &r) { CHECK(r.start && r.B >= 1 && r.B <= 65535 && r.tokens >= 0 && r.tokens <= 1 << 30); }
size_t prefill_workspace_bytes(const PrefillArgs &a, int) { return a.rows.tokens <= 4ll * a.rows.B ? 0 : 1u << 20; }
hipError_t launch_prefill(const PrefillArgs &a, int, hipStream_t) {
  seen(a.rows);
  CHECK(a.H >= 1 && a.Hk >= 1 && a.H % a.Hk == 0 && a.dv >= 16 && a.dv <= 1024 && a.dv % 16 == 0);
  CHECK(a.dk == 64 || a.dk == 128 || a.dk == 256);
  CHECK(a.family >= 0 && a.family < SLA_FAMILY_GLA && a.state_out);
  CHECK(a.rows.tokens == 0 || (a.q && a.k && a.v && a.out && (a.family == SLA_FAMILY_DELTANET) == !a.alpha &&
                               (a.family == SLA_FAMILY_DECAY) == !a.beta));
  CHECK(a.q_stride >= (int64_t)a.Hk * a.dk && a.q_stride <= 1 << 22 && a.v_stride >= (int64_t)a.H * a.dv);
  CHECK(((int64_t)a.rows.tokens / 64 + a.rows.B) * a.H < 1ll << 31 && (int64_t)a.rows.B * a.H * (a.dv / 16) < 1ll << 31);
  ++launched[0];
  return hipSuccess;
}
hipError_t launch_conv_prefill(const ConvPrefillArgs &a, int, hipStream_t) {
  seen(a.rows);
  CHECK(a.D >= 8 && a.D % 8 == 0 && a.K >= 1 && a.K <= 4 && a.weight && (a.K == 1 ? !a.state && !a.state_out : !!a.state_out));
  CHECK((a.rows.tokens == 0 || (a.x && a.y)) && a.x_stride >= a.D && a.x_stride <= 1 << 22);
  CHECK(((int64_t)a.rows.tokens / 32 + a.rows.B) * ((a.D + 511) / 512) < 1ll << 31);
  ++launched[1];
  return hipSuccess;
}
hipError_t launch_recurrent_inputs(const InputsArgs &a, int, hipStream_t) {
  CHECK(a.rows > 0 && a.q && a.k && a.q_out && a.k_out && !a.alpha == !a.a && !a.beta == !a.b && (!a.alpha || a.a_log));
  CHECK(a.repeat >= 1 && a.repeat <= 64 && std::isfinite(a.q_scale) && a.eps >= 0 && a.q_stride >= (int64_t)a.Hk * a.dk);
  CHECK((int64_t)a.rows * 2 * a.Hk / 8 + (int64_t)a.rows * a.H / 256 < 1ll << 31);
  ++launched[2];
  return hipSuccess;
}
hipError_t launch_gated_norm(const NormArgs &a, int, int, hipStream_t) {
  CHECK(a.rows > 0 && a.x && a.y && (a.gate == SLA_GATE_NONE || (a.z && a.z_stride >= (int64_t)a.H * a.dv)));
  CHECK(a.dv >= 16 && a.dv <= 1024 && a.dv % 16 == 0 && (int64_t)a.rows * a.H / 2 < 1ll << 31);
  ++launched[3];
  return hipSuccess;
}
}  // namespace sla

static std::mt19937_64 rng(7);
static int32_t pick(std::initializer_list<int32_t> usual) {
  static const int32_t ends[] = {INT32_MIN, -1, 0, 1, 65535, 65536, 1 << 20, 1 << 30, INT32_MAX};
  if (rng() % 12 == 0) return ends[rng() % 9];
  return usual.begin()[rng() % usual.size()];
}
static void *place(size_t i) {
  switch (rng() % 40) {
    case 0: return nullptr;
    case 1: return reinterpret_cast<void *>(~(uintptr_t)15);
    case 2: return reinterpret_cast<void *>((uintptr_t)64);
    case 3: return reinterpret_cast<void *>(((uintptr_t)i << 44) + 4);
    case 4: return reinterpret_cast<void *>((uintptr_t)1 << 44);
    default: return reinterpret_cast<void *>((uintptr_t)i << 44);
  }
}
static int64_t stride(int64_t dense) {
  switch (rng() % 12) {
    case 0: return INT64_MIN;
    case 1: return INT64_MAX;
    case 2: return dense - 8;
    case 3: return dense + 64;
    default: return dense;
  }
}

int main() {
  for (int i = 0; i < 400000; ++i) {
    void *p[12];
    for (size_t j = 0; j < 12; ++j) p[j] = place(j + 1);
    auto f = [&](int j) { return static_cast<float *>(p[j]); };
    auto n = [&](int j) { return static_cast<int32_t *>(p[j]); };
    int code;
    if (i % 4 == 0) {
      const sla_prefill_shape s = {pick({0, 1, 100, 5000, 1 << 20}), pick({1, 3, 64, 4096}), pick({1, 4, 16, 64}), pick({1, 2, 4}),
                                   pick({64, 128, 256}), pick({16, 80, 128, 1024}), pick({0, 1}), pick({0, 1, 2, 3})};
      const size_t need = sla_prefill_workspace_bytes(&s);
      const int64_t kd = (int64_t)s.k_heads * s.d_k, vd = (int64_t)s.heads * s.d_v;
      code = sla_prefill(&s, f(0), p[1], stride(kd), p[2], stride(kd), p[3], stride(vd), f(4), f(5), n(6), p[7],
                         rng() % 3 ? f(8) : f(0), p[9], rng() % 8 ? need : need / 2, n(10), nullptr);
    } else if (i % 4 == 1) {
      const sla_conv_prefill_shape s = {pick({0, 1, 100, 5000, 1 << 20}), pick({1, 3, 64}), pick({8, 1000, 6144}), pick({1, 2, 3, 4}),
                                        pick({0, 1}), pick({0, 1})};
      code = sla_conv_prefill(&s, f(0), p[1], stride(s.channels), f(2), f(3), n(4), p[5], rng() % 3 ? f(6) : f(0), n(7), nullptr);
    } else if (i % 4 == 2) {
      const float odd[] = {0.f, 1e-6f, -1.f, INFINITY, NAN, 3e38f};
      const sla_inputs_shape s = {pick({0, 1, 1000, 1 << 20}), pick({1, 16}), pick({1, 8}), pick({1, 2, 64}), pick({64, 128, 256}),
                                  pick({0, 1}), odd[rng() % 6], odd[rng() % 6]};
      const int64_t kd = (int64_t)s.k_heads * s.d_k;
      const bool no_a = rng() % 4 == 0, no_b = rng() % 4 == 0;
      code = sla_recurrent_inputs(&s, p[0], stride(kd), p[1], stride(kd), no_a ? nullptr : p[2], stride(s.heads), no_b ? nullptr : p[3],
                                  stride(s.heads), f(4), f(5), p[6], p[7], no_a ? nullptr : f(8), no_b ? nullptr : f(9), nullptr);
    } else {
      const sla_norm_shape s = {pick({0, 1, 1000, 1 << 20}), pick({1, 16}), pick({16, 80, 1024}), pick({0, 1}), pick({0, 1}),
                                pick({0, 1, 2}), rng() % 5 ? 1e-6f : NAN};
      code = sla_gated_norm(&s, p[0], p[1], stride((int64_t)s.heads * s.d_v), f(2), rng() % 4 ? p[3] : p[0], nullptr);
    }
    CHECK(code <= 0 && code >= SLA_ERR_LENGTH);
    refused += code != SLA_OK;
  }
  for (long l : launched) CHECK(l > 1000);
  CHECK(refused > 1000);
  printf("%ld %ld %ld %ld launched, %ld refused\n", launched[0], launched[1], launched[2], launched[3], refused);
  if (!failures) printf("sanitized prompt checks passed\n");
  return failures != 0;
}
