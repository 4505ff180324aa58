// attn_api.cpp -- host side of the attention calls of include/sla.h: argument
// validation, alias checks and kernel launches on the caller's stream.
// Nothing here allocates device memory or keeps state between calls.
#include <stdint.h>
#include <string.h>

#include <cmath>

#include "attn.hpp"
#include "sla.h"

namespace {

size_t act_bytes(int dtype) { return dtype == SLA_DTYPE_BF16 ? 2 : 4; }

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Span {
  const void *p;  // NULL: none
  size_t bytes;
};

Span span_of(const void *p, size_t count, size_t size) { return Span{p, count * size}; }

bool overlaps(const Span &x, const Span &y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
  return x.p && y.p && a < b + y.bytes && b < a + x.bytes;
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

// A pool of `layers` layers; a size past any memory counts as 2^56 bytes.
Span pool_span(const sla_attn_shape *s, int32_t layers, const void *p) {
  const unsigned __int128 bytes = (unsigned __int128)layers * s->n_pages * s->kv_heads * s->page_size *
                                  (unsigned)s->head_dim * act_bytes(s->qkv_dtype);
  const unsigned __int128 most = (unsigned __int128)1 << 56;
  return Span{p, (size_t)(bytes < most ? bytes : most)};
}

int hip_status(hipError_t e) { return e == hipSuccess ? SLA_OK : SLA_ERR_HIP; }

int page_shift(int page) {
  int s = 0;
  while ((1 << s) < page) ++s;
  return s;
}

// the fields every call reads
int check_pool(const sla_attn_shape *s) {
  if (!s) return SLA_ERR_NULL;
  if (s->kv_heads < 1 || s->kv_heads > (1 << 16) || s->n_pages < 1 || s->head_dim < 1) return SLA_ERR_SHAPE;
  if (s->page_size < 16 || s->page_size > 256 || (s->page_size & (s->page_size - 1))) return SLA_ERR_SHAPE;
  if (s->qkv_dtype != SLA_DTYPE_F32 && s->qkv_dtype != SLA_DTYPE_BF16) return SLA_ERR_DTYPE;
  if (s->head_dim != 64 && s->head_dim != 128 && s->head_dim != 256) return SLA_ERR_UNSUPPORTED;
  return SLA_OK;
}

int check_rows(const sla_attn_shape *s) {
  const int st = check_pool(s);
  if (st != SLA_OK) return st;
  if (s->batch < 1 || s->batch > 65535 || s->n_nodes < 1 || s->n_nodes > SLA_MAX_NODES || s->max_pages < 1)
    return SLA_ERR_SHAPE;
  if ((int64_t)s->max_pages * s->page_size > (1ll << 30)) return SLA_ERR_SHAPE;
  return SLA_OK;
}

int check_shape(const sla_attn_shape *s) {
  const int st = check_rows(s);
  if (st != SLA_OK) return st;
  if (s->q_heads < 1 || s->q_heads % s->kv_heads || s->q_heads > (1 << 16) || s->max_len < 0) return SLA_ERR_SHAPE;
  if (s->topology != SLA_TOPO_TREE && s->topology != SLA_TOPO_CHAIN) return SLA_ERR_SHAPE;
  // the rows' numbers, and those of a launch's workgroups, which are not many more, fit 32 bits
  if ((int64_t)s->batch * s->n_nodes * s->q_heads >= (1ll << 31)) return SLA_ERR_SHAPE;
  return SLA_OK;
}

bool layers_ok(const sla_attn_shape *s, int32_t layers) {
  // a launch's first dimension stays far inside 2^32 work-items
  return layers >= 1 && layers <= (1 << 16) && (int64_t)layers * s->kv_heads <= (1 << 20);
}

sla::PagedCache cache_of(const sla_attn_shape *s, void *k, void *v) {
  return sla::PagedCache{k, v, s->kv_heads, s->head_dim, page_shift(s->page_size), s->n_pages};
}

sla::AttnVerifyArgs verify_args(const sla_attn_shape *s) {
  sla::AttnVerifyArgs a;
  memset(&a, 0, sizeof(a));
  const int64_t capacity = (int64_t)s->max_pages * s->page_size;
  a.B = s->batch;
  a.n = s->n_nodes;
  a.Hq = s->q_heads;
  a.max_len = s->max_len > 0 && s->max_len < capacity ? s->max_len : (int32_t)capacity;
  a.chain = s->topology == SLA_TOPO_CHAIN;
  a.cache = cache_of(s, nullptr, nullptr);
  a.rows.max_pages = s->max_pages;
  return a;
}

}  // namespace

extern "C" {

int sla_attn_append(const sla_attn_shape *shape, const sla_attn_transform *t, const void *q, int64_t q_stride,
                    const void *k, int64_t k_stride, const void *v, int64_t v_stride, const int32_t *parent_idx,
                    const int32_t *page_table, const int32_t *cache_len, void *q_out, void *k_cache, void *v_cache,
                    int32_t *status, hipStream_t stream) {
  const int st = check_shape(shape);
  if (st != SLA_OK) return st;
  if (!q || !k || !v || !parent_idx || !page_table || !cache_len || !q_out || !k_cache || !v_cache) return SLA_ERR_NULL;
  const int D = shape->head_dim;
  const size_t w = act_bytes(shape->qkv_dtype);
  const int64_t qd = (int64_t)shape->q_heads * D, kd = (int64_t)shape->kv_heads * D;
  if (q_stride < qd || k_stride < kd || v_stride < kd) return SLA_ERR_SHAPE;
  if (t) {
    if (t->rope_dim < 0 || t->rope_dim > D || t->rope_dim % 16 || !(t->eps >= 0.f)) return SLA_ERR_SHAPE;
    if (t->layout != SLA_ROPE_HALF && t->layout != SLA_ROPE_INTERLEAVED) return SLA_ERR_SHAPE;
    if (t->rope_dim > 0 && t->rope_len < 1) return SLA_ERR_SHAPE;
    if (t->rope_dim > 0 && !t->rope) return SLA_ERR_NULL;
  }
  const size_t rows = (size_t)shape->batch, nodes = rows * shape->n_nodes;
  const Span writes[] = {span_of(q_out, nodes * (size_t)qd, w), pool_span(shape, 1, k_cache),
                         pool_span(shape, 1, v_cache), span_of(status, rows, 4)};
  const Span reads[] = {span_of(q, (nodes - 1) * (size_t)q_stride + (size_t)qd, w),
                        span_of(k, (nodes - 1) * (size_t)k_stride + (size_t)kd, w),
                        span_of(v, (nodes - 1) * (size_t)v_stride + (size_t)kd, w),
                        span_of(parent_idx, nodes, 4),
                        span_of(page_table, rows * shape->max_pages, 4),
                        span_of(cache_len, rows, 4),
                        span_of(t ? t->q_norm : nullptr, D, 4),
                        span_of(t ? t->k_norm : nullptr, D, 4),
                        span_of(t && t->rope_dim ? t->rope : nullptr, t ? (size_t)t->rope_dim * t->rope_len : 0, 4)};
  if (aliased(writes, reads)) return SLA_ERR_ALIAS;
  const int64_t step = 16 / (int64_t)w;  // elements of 16 bytes
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_cache) ||
      !aligned16(v_cache) || q_stride % step || k_stride % step || v_stride % step)
    return SLA_ERR_UNSUPPORTED;
  if (t && ((t->q_norm && !aligned16(t->q_norm)) || (t->k_norm && !aligned16(t->k_norm)) ||
            (t->rope_dim && !aligned16(t->rope))))
    return SLA_ERR_UNSUPPORTED;
  sla::AttnAppendArgs a;
  memset(&a, 0, sizeof(a));
  a.B = shape->batch;
  a.n = shape->n_nodes;
  a.Hq = shape->q_heads;
  a.chain = shape->topology == SLA_TOPO_CHAIN;
  a.cache = cache_of(shape, k_cache, v_cache);
  a.rows = sla::CacheRows{page_table, cache_len, shape->max_pages};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  if (t) {
    a.q_norm = t->q_norm;
    a.k_norm = t->k_norm;
    a.eps = t->eps;
    a.rope = t->rope;
    a.rope_dim = t->rope_dim;
    a.rope_len = t->rope_len;
    a.interleaved = t->layout == SLA_ROPE_INTERLEAVED;
  }
  a.parent = parent_idx;
  a.q_out = q_out;
  a.status = status;
  return hip_status(sla::launch_attn_append(a, shape->qkv_dtype, stream));
}

size_t sla_attn_workspace_bytes(const sla_attn_shape *shape) {
  if (check_shape(shape) != SLA_OK) return 0;
  return sla::attn_workspace_bytes(verify_args(shape), shape->qkv_dtype);
}

int sla_attn_verify(const sla_attn_shape *shape, float scale, const void *q, const void *k_cache, const void *v_cache,
                    const int32_t *parent_idx, const int32_t *page_table, const int32_t *cache_len, void *out,
                    void *workspace, size_t workspace_bytes, int32_t *status, hipStream_t stream) {
  const int st = check_shape(shape);
  if (st != SLA_OK) return st;
  if (!q || !k_cache || !v_cache || !parent_idx || !page_table || !cache_len || !out) return SLA_ERR_NULL;
  if (!std::isfinite(scale)) return SLA_ERR_SHAPE;
  sla::AttnVerifyArgs a = verify_args(shape);
  const size_t need = sla::attn_workspace_bytes(a, shape->qkv_dtype);
  if (need && !workspace) return SLA_ERR_NULL;
  if (need && workspace_bytes < need) return SLA_ERR_SHAPE;
  const size_t rows = (size_t)shape->batch, nodes = rows * shape->n_nodes;
  const size_t values = nodes * shape->q_heads * shape->head_dim, w = act_bytes(shape->qkv_dtype);
  const Span writes[] = {span_of(out, values, w), span_of(need ? workspace : nullptr, need, 1), span_of(status, rows, 4)};
  const Span reads[] = {span_of(q, values, w), pool_span(shape, 1, k_cache), pool_span(shape, 1, v_cache),
                        span_of(parent_idx, nodes, 4), span_of(page_table, rows * shape->max_pages, 4),
                        span_of(cache_len, rows, 4)};
  if (aliased(writes, reads)) return SLA_ERR_ALIAS;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) || !aligned16(workspace))
    return SLA_ERR_UNSUPPORTED;
  a.cache.k = const_cast<void *>(k_cache);
  a.cache.v = const_cast<void *>(v_cache);
  a.rows = sla::CacheRows{page_table, cache_len, shape->max_pages};
  a.scale = scale;
  a.q = q;
  a.parent = parent_idx;
  a.out = out;
  a.workspace = workspace;
  a.status = status;
  return hip_status(sla::launch_attn_verify(a, shape->qkv_dtype, stream));
}

int sla_attn_commit(const sla_attn_shape *shape, int32_t layers, void *k_cache, void *v_cache,
                    const int32_t *parent_idx, const int32_t *path, const int32_t *len, const int32_t *page_table,
                    const int32_t *cache_len, int32_t *new_len, int32_t *status, hipStream_t stream) {
  const int st = check_rows(shape);
  if (st != SLA_OK) return st;
  if (!layers_ok(shape, layers)) return SLA_ERR_SHAPE;
  if (!k_cache || !v_cache || !parent_idx || !path || !len || !page_table || !cache_len) return SLA_ERR_NULL;
  const size_t rows = (size_t)shape->batch, nodes = rows * shape->n_nodes;
  const Span writes[] = {pool_span(shape, layers, k_cache), pool_span(shape, layers, v_cache), span_of(new_len, rows, 4),
                         span_of(status, rows, 4)};
  const Span reads[] = {span_of(parent_idx, nodes, 4), span_of(path, nodes, 4), span_of(len, rows, 4),
                        span_of(page_table, rows * shape->max_pages, 4), span_of(cache_len, rows, 4)};
  if (aliased(writes, reads)) return SLA_ERR_ALIAS;
  if (!aligned16(k_cache) || !aligned16(v_cache)) return SLA_ERR_UNSUPPORTED;
  sla::AttnCommitArgs a;
  memset(&a, 0, sizeof(a));
  a.B = shape->batch;
  a.n = shape->n_nodes;
  a.layers = layers;
  a.cache = cache_of(shape, k_cache, v_cache);
  a.rows = sla::CacheRows{page_table, cache_len, shape->max_pages};
  a.parent = parent_idx;
  a.path = path;
  a.accepted = len;
  a.new_len = new_len;
  a.status = status;
  return hip_status(sla::launch_attn_commit(a, shape->qkv_dtype, stream));
}

int sla_page_copy(const sla_attn_shape *shape, int32_t layers, void *k_cache, void *v_cache, const int32_t *src,
                  const int32_t *dst, const int32_t *rows, int32_t copies, int32_t *status, hipStream_t stream) {
  const int st = check_pool(shape);
  if (st != SLA_OK) return st;
  if (!layers_ok(shape, layers) || copies < 1 || copies > (1 << 24)) return SLA_ERR_SHAPE;
  if (!k_cache || !v_cache || !src || !dst) return SLA_ERR_NULL;
  const Span writes[] = {pool_span(shape, layers, k_cache), pool_span(shape, layers, v_cache), span_of(status, copies, 4)};
  const Span reads[] = {span_of(src, copies, 4), span_of(dst, copies, 4), span_of(rows, copies, 4)};
  if (aliased(writes, reads)) return SLA_ERR_ALIAS;
  if (!aligned16(k_cache) || !aligned16(v_cache)) return SLA_ERR_UNSUPPORTED;
  sla::PageCopyArgs a;
  memset(&a, 0, sizeof(a));
  a.copies = copies;
  a.layers = layers;
  a.cache = cache_of(shape, k_cache, v_cache);
  a.src = src;
  a.dst = dst;
  a.rows = rows;
  a.status = status;
  return hip_status(sla::launch_page_copy(a, shape->qkv_dtype, stream));
}

}  // extern "C"
