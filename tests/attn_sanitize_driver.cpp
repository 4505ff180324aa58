// The host side of the attention calls (attn_api.cpp) for AddressSanitizer and
// UndefinedBehaviorSanitizer builds (built and run by
// tests/test_attn_sanitizers.py; no GPU code is involved: the launchers are
// stubs that look at what they are given).  Random shapes, sizes at the ends
// of their types, and pointers at the ends of the address space go through the
// argument checks; a launcher may only ever see what the checks let pass.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <random>

#include "attn.hpp"
#include "sla.h"

static long launched = 0, refused = 0, failures = 0;
#define CHECK(c)                                                     \
  do {                                                               \
    if (!(c)) {                                                      \
      fprintf(stderr, "check failed: %s (line %d)\n", #c, __LINE__); \
      ++failures;                                                    \
    }                                                                \
  } while (0)

namespace sla {
static void seen(const PagedCache &c) {
  CHECK(c.k && c.v && c.Hkv >= 1 && c.n_pages >= 1 && c.page_shift >= 4 && c.page_shift <= 8);
  CHECK(c.D == 64 || c.D == 128 || c.D == 256);
}
static void seen(const CacheRows &r, int shift, int B, int n) {
  CHECK(r.table && r.len && r.max_pages >= 1 && ((int64_t)r.max_pages << shift) <= (1ll << 30));
  CHECK(B >= 1 && B <= 65535 && n >= 1 && n <= 64);
}
hipError_t launch_attn_append(const AttnAppendArgs &a, int, hipStream_t) {
  seen(a.cache);
  seen(a.rows, a.cache.page_shift, a.B, a.n);
  CHECK(a.Hq % a.cache.Hkv == 0 && a.q_stride >= (int64_t)a.Hq * a.cache.D);
  CHECK(a.rope_dim % 16 == 0 && a.rope_dim >= 0 && a.rope_dim <= a.cache.D && (!a.rope_dim || (a.rope && a.rope_len > 0)));
  ++launched;
  return hipSuccess;
}
hipError_t launch_attn_verify(const AttnVerifyArgs &a, int, hipStream_t) {
  seen(a.cache);
  seen(a.rows, a.cache.page_shift, a.B, a.n);
  CHECK(a.max_len > 0 && a.max_len <= (int64_t)a.rows.max_pages << a.cache.page_shift);
  ++launched;
  return hipSuccess;
}
hipError_t launch_attn_commit(const AttnCommitArgs &a, int, hipStream_t) {
  seen(a.cache);
  seen(a.rows, a.cache.page_shift, a.B, a.n);
  CHECK(a.layers >= 1 && (int64_t)a.layers * a.cache.Hkv <= (1 << 20));
  ++launched;
  return hipSuccess;
}
hipError_t launch_page_copy(const PageCopyArgs &a, int, hipStream_t) {
  seen(a.cache);
  CHECK(a.copies >= 1 && a.layers >= 1 && a.src && a.dst);
  ++launched;
  return hipSuccess;
}
size_t attn_workspace_bytes(const AttnVerifyArgs &a, int) { return (size_t)a.B * 64; }
}  // namespace sla

int main() {
  std::mt19937_64 rng(7);
  auto pick = [&](std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); };
  auto size = [&](int64_t good) {
    return (int32_t)(rng() % 40 ? good : pick({0, -1, 1, INT32_MAX, INT32_MIN, 1 << 16, 1 << 26, 65}));
  };
  auto address = [&](int slot) {
    const uint64_t good = ((uint64_t)slot + 1) << 40;
    switch (rng() % 60) {
      case 0: return (void *)nullptr;
      case 1: return (void *)(uintptr_t)(good + 4);
      case 2: return (void *)(UINTPTR_MAX - 15);
      case 3: return (void *)(uintptr_t)(((uint64_t)slot) << 40);
      default: return (void *)(uintptr_t)good;
    }
  };
  for (int it = 0; it < 200000; ++it) {
    sla_attn_shape s;
    memset(&s, 0, sizeof(s));
    s.batch = size(1 + rng() % 300);
    s.kv_heads = size(1 + rng() % 9);
    s.q_heads = size((int64_t)(1 + rng() % 8) * (s.kv_heads > 0 && s.kv_heads < 1000 ? s.kv_heads : 1));
    s.head_dim = size(64 << rng() % 3);
    s.n_nodes = size(1 + rng() % 64);
    s.qkv_dtype = size(rng() % 2);
    s.topology = size(rng() % 2);
    s.page_size = size(16 << rng() % 5);
    s.n_pages = size(1 + rng() % 5000);
    s.max_pages = size(1 + rng() % 1000);
    s.max_len = size(rng() % 3000);
    sla_attn_transform t;
    memset(&t, 0, sizeof(t));
    t.q_norm = (const float *)address(20);
    t.k_norm = (const float *)address(21);
    t.eps = rng() % 20 ? 1e-6f : -1.f;
    t.rope = (const float *)address(22);
    t.rope_dim = size(16 * (rng() % 5));
    t.rope_len = size(1 + rng() % 100000);
    t.layout = size(rng() % 2);
    int32_t *st = (int32_t *)address(12);
    const int64_t qs = rng() % 30 ? 16384 : pick({0, -8, INT64_MAX, 3, 1ll << 40});
    int r;
    switch (it % 4) {
      case 0:
        r = sla_attn_append(&s, rng() % 3 ? &t : nullptr, address(0), qs, address(1), qs, address(2), qs,
                            (int32_t *)address(3), (int32_t *)address(4), (int32_t *)address(5), address(6), address(7),
                            address(8), st, nullptr);
        break;
      case 1:
        r = sla_attn_verify(&s, 0.1f, address(0), address(7), address(8), (int32_t *)address(3), (int32_t *)address(4),
                            (int32_t *)address(5), address(6), address(9), rng() % 10 ? 1 << 22 : rng() % 4096, st, nullptr);
        break;
      case 2:
        r = sla_attn_commit(&s, size(1 + rng() % 40), address(7), address(8), (int32_t *)address(3),
                            (int32_t *)address(10), (int32_t *)address(11), (int32_t *)address(4), (int32_t *)address(5),
                            (int32_t *)address(13), st, nullptr);
        break;
      default:
        r = sla_page_copy(&s, size(1 + rng() % 40), address(7), address(8), (int32_t *)address(3), (int32_t *)address(4),
                          (int32_t *)address(5), size(1 + rng() % 1000), st, nullptr);
    }
    if (r != SLA_OK) ++refused;
    sla_attn_workspace_bytes(&s);
  }
  CHECK(launched > 20000 && refused > 20000);
  printf("%ld launched, %ld refused\n", launched, refused);
  if (failures == 0) printf("sanitized attention checks passed\n");
  return failures != 0;
}
