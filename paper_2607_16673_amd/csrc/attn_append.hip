// attn_append.hip -- the draft's rows of an attention layer: queries and keys
// normalised over the head and rotated by their node's position, queries to
// q_out, keys and values to the paged cache.
//
// One pass: every element is read once and written once, so memory bounds it
// for large drafts (256 sequences of 64 nodes of 16 + 2 + 2 fp32 heads of 256:
// 132 us, 5.1 TB/s, the rate of a large copy) and the launch with its chain of loads
// (length, page, rotation) for small ones (64 of
// 16 nodes of heads of 128 in bf16: 5.6 us).  Norms,
// angles and products are fp32, rounded once at the end.  A head is the work of
// D / 8 neighbouring lanes, 8 elements (16 bytes of bf16) each: the mean
// square is a butterfly over those lanes, and the partner of a rotated pair is
// in the same lane (interleaved pairs) or rope_dim / 16 lanes away (halves).
#include "attn_device.hpp"

namespace sla {
namespace {

constexpr int kThreads = 256;

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void append_kernel(AttnAppendArgs a) {
  constexpr int kLanes = D / 8;
  constexpr int kHeads = kThreads / kLanes;  // heads of one workgroup
  const int b = blockIdx.y;
  const int lane = threadIdx.x % kWave;
  const int n = a.n, Hkv = a.cache.Hkv;
  const int per_node = a.Hq + 2 * Hkv;

  // every wave looks at the whole draft: lane j at node j
  const int p = lane < n ? a.parent[(size_t)b * n + lane] : -1;
  const int len = a.rows.len[b];
  int err = SLA_OK, depth = 1, page = 0;
  if (!parents_ok(p, n, lane, a.chain)) {
    err = SLA_ERR_TOPOLOGY;
  } else if (!length_ok(a.rows, a.cache.page_shift, len, n)) {
    err = SLA_ERR_LENGTH;
  } else {
    depth = node_depth(p);
    if (lane < n) page = a.rows.table[(size_t)b * a.rows.max_pages + ((len + lane) >> a.cache.page_shift)];
    if (wave_any(a.rope_dim > 0 && lane < n && len + depth > a.rope_len)) err = SLA_ERR_LENGTH;
    else if (wave_any(page < 0 || page >= a.cache.n_pages)) err = SLA_ERR_PAGE;
  }
  if (a.status && blockIdx.x == 0 && threadIdx.x == 0) a.status[b] = err;
  if (err != SLA_OK) return;

  const int item = blockIdx.x * kHeads + threadIdx.x / kLanes;
  const int j = min(item / per_node, n - 1);
  const int pos = len + __shfl(depth, j) - 1;
  const int pg = __shfl(page, j);
  if (item >= n * per_node) return;
  int h = item % per_node;
  const int e = threadIdx.x % kLanes * 8;  // first element of this lane
  const size_t node = (size_t)b * n + j;
  const size_t row_in_page = (size_t)((len + j) & ((1 << a.cache.page_shift) - 1));

  if (h >= a.Hq + Hkv) {  // a value: its bits
    h -= a.Hq + Hkv;
    const T *src = static_cast<const T *>(a.v) + node * a.v_stride + (size_t)h * D + e;
    T *dst = static_cast<T *>(a.cache.v) + (page_row(a.cache, pg, h) + row_in_page) * D + e;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      reinterpret_cast<uint4 *>(dst)[i] = reinterpret_cast<const uint4 *>(src)[i];
    return;
  }
  const bool query = h < a.Hq;
  if (!query) h -= a.Hq;
  const T *src = query ? static_cast<const T *>(a.q) + node * a.q_stride + (size_t)h * D + e
                       : static_cast<const T *>(a.k) + node * a.k_stride + (size_t)h * D + e;
  T *dst = query ? static_cast<T *>(a.q_out) + (node * a.Hq + h) * D + e
                 : static_cast<T *>(a.cache.k) + (page_row(a.cache, pg, h) + row_in_page) * D + e;
  float x[8];
  load_f32(src, x);
  const float *norm = query ? a.q_norm : a.k_norm;
  if (norm) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) ss += __shfl_xor(ss, o);
    const float r = 1.f / sqrtf(ss * (1.f / D) + a.eps);
    float w[8];
    load_f32(norm + e, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
  }
  const int half = a.rope_dim / 2;
  if (half > 0) {
    const float *row = a.rope + (size_t)pos * a.rope_dim;
    const bool turned = e < a.rope_dim;
    if (a.interleaved) {
      if (turned) {
        float c[4], s[4];
        load_f32(row + e / 2, c);
        load_f32(row + half + e / 2, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = x[2 * i], v = x[2 * i + 1];
          x[2 * i] = u * c[i] - v * s[i];
          x[2 * i + 1] = v * c[i] + u * s[i];
        }
      }
    } else {
      const bool first = e < half;
      const int partner = lane + (turned ? (first ? half / 8 : -(half / 8)) : 0);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], partner);
      if (turned) {
        float c[8], s[8];
        load_f32(row + (first ? e : e - half), c);
        load_f32(row + half + (first ? e : e - half), s);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = first ? x[i] * c[i] - y[i] * s[i] : x[i] * c[i] + y[i] * s[i];
      }
    }
  }
  store8(dst, x);
}

template <typename T, int D>
hipError_t launch_d(const AttnAppendArgs &a, hipStream_t s) {
  const int heads = kThreads / (D / 8);
  const unsigned blocks = (unsigned)((a.n * (a.Hq + 2 * a.cache.Hkv) + heads - 1) / heads);
  hipLaunchKernelGGL((append_kernel<T, D>), dim3(blocks, (unsigned)a.B), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const AttnAppendArgs &a, hipStream_t s) {
  switch (a.cache.D) {
    case 64: return launch_d<T, 64>(a, s);
    case 128: return launch_d<T, 128>(a, s);
    default: return launch_d<T, 256>(a, s);
  }
}

}  // namespace

hipError_t launch_attn_append(const AttnAppendArgs &a, int dtype, hipStream_t s) {
  return dtype == SLA_DTYPE_BF16 ? launch_t<bf16>(a, s) : launch_t<float>(a, s);
}

}  // namespace sla
