// attn_device.hpp -- device-side building blocks of the attention kernels: a
// draft's ancestors and depths, its rows in the paged cache, and the
// activation types' 8-element pieces.
#pragma once

#include "attn.hpp"
#include "device.hpp"

namespace sla {

// A launch's work-items are counted in 32 bits in each dimension, so large ones
// go on in the second: workgroup `number` of up to 2^32.  The width is a multiple
// of the XCDs and of 256.
constexpr unsigned kGridWidth = 1u << 22;
__device__ __forceinline__ unsigned workgroup() { return blockIdx.y * kGridWidth + blockIdx.x; }
inline dim3 grid_of(uint64_t workgroups) {
  if (workgroups <= kGridWidth) return dim3((unsigned)workgroups);
  return dim3(kGridWidth, (unsigned)((workgroups + kGridWidth - 1) / kGridWidth));
}

// round to nearest even, two values to one word
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return (uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(lo)) |
         ((uint32_t)__builtin_bit_cast(uint16_t, static_cast<__bf16>(hi)) << 16);
}

__device__ __forceinline__ void store8(bf16 *p, const float (&x)[8]) {
  *reinterpret_cast<uint4 *>(p) =
      make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
  reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Whether lane j < n may have the parent p (wave-uniform).
__device__ __forceinline__ bool parents_ok(int p, int n, int lane, bool chain) {
  const bool live = lane < n;
  return !wave_any(live && (p < -1 || p >= lane || (chain && p != lane - 1)));
}

// depth(j) of lane j from its parent p, the parents being in topological
// order: every step doubles the distance a lane has looked up its path.
__device__ __forceinline__ int node_depth(int p) {
  int d = 1, a = p;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const int src = a >= 0 ? a : 0;
    const int da = __shfl(d, src), aa = __shfl(a, src);
    if (a >= 0) {
      d += da;
      a = aa;
    }
  }
  return d;
}

// Inclusive ancestor mask of lane j, by the same doubling.
__device__ __forceinline__ uint64_t node_ancestors(int p, int lane) {
  uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
  int a = p;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const int src = a >= 0 ? a : 0;
    const uint32_t l = __shfl(lo, src), h = __shfl(hi, src);
    const int aa = __shfl(a, src);
    if (a >= 0) {
      lo |= l;
      hi |= h;
      a = aa;
    }
  }
  return ((uint64_t)hi << 32) | lo;
}

// The first row of page `page` in head h of one layer, in rows of D elements.
__device__ __forceinline__ size_t page_row(const PagedCache &c, int page, int h) {
  return ((size_t)page * c.Hkv + h) << c.page_shift;
}

// Whether rows [0, len + n) fit the sequence's page-table row.
__device__ __forceinline__ bool length_ok(const CacheRows &r, int page_shift, int len, int n) {
  return len >= 0 && (int64_t)len + n <= (int64_t)r.max_pages << page_shift;
}

}  // namespace sla
