// attn.hpp -- launch interface between the host ABI (attn_api.cpp) and the
// kernels of the attention layer over a paged cache: append, verify, commit
// and page copy.  Plain structs of device pointers and sizes; the host side
// has already validated what it can see.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace sla {

// One layer's cache, or `layers` layers of it for commit and copy.
struct PagedCache {
  void *k, *v;         // [layers][n_pages][Hkv][page][D]
  int32_t Hkv, D;
  int32_t page_shift;  // log2 of the rows of a page
  int32_t n_pages;
};

// Where a batch's rows lie in the cache.
struct CacheRows {
  const int32_t *table;  // [B][max_pages]
  const int32_t *len;    // [B]
  int32_t max_pages;
};

struct AttnAppendArgs {
  int32_t B, n, Hq;
  bool chain;
  PagedCache cache;
  CacheRows rows;
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;  // elements from node to node
  const float *q_norm, *k_norm;
  float eps;
  const float *rope;
  int32_t rope_dim, rope_len;
  bool interleaved;
  const int32_t *parent;
  void *q_out;
  int32_t *status;
};

struct AttnVerifyArgs {
  int32_t B, n, Hq;
  int32_t max_len;
  bool chain;
  PagedCache cache;
  CacheRows rows;
  float scale;
  const void *q;
  const int32_t *parent;
  void *out;
  void *workspace;
  int32_t *status;
};

struct AttnCommitArgs {
  int32_t B, n, layers;
  PagedCache cache;
  CacheRows rows;
  const int32_t *parent, *path, *accepted;
  int32_t *new_len;
  int32_t *status;
};

struct PageCopyArgs {
  int32_t copies, layers;
  PagedCache cache;
  const int32_t *src, *dst, *rows;
  int32_t *status;
};

// Each launcher returns hipSuccess or the launch error.  `dtype` is
// SLA_DTYPE_F32 or SLA_DTYPE_BF16.
hipError_t launch_attn_append(const AttnAppendArgs &a, int dtype, hipStream_t s);
hipError_t launch_attn_verify(const AttnVerifyArgs &a, int dtype, hipStream_t s);
hipError_t launch_attn_commit(const AttnCommitArgs &a, int dtype, hipStream_t s);
hipError_t launch_page_copy(const PageCopyArgs &a, int dtype, hipStream_t s);
// bytes of partial results the launch for this shape writes
size_t attn_workspace_bytes(const AttnVerifyArgs &a, int dtype);

}  // namespace sla
