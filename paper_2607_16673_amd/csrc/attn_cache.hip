// attn_cache.hip -- moving rows of the paged cache: the accepted path's rows
// behind the committed tokens (commit), and whole or partly filled pages
// (copy).  Both move bits.  A commit is bound by its chain of loads (length, path,
// parents, page table, rows): 64 sequences of 16 nodes 4.4 us, 256 of 64 nodes in
// six layers of 4 heads of 256 11.8 us for 26 MB read and written, 2.2 TB/s.  A
// copy is bound by memory, 1.6 GB read and written 322 us, 5.0 TB/s, or by its
// launch, half a page 3.7 us.
#include "attn_device.hpp"

namespace sla {
namespace {

constexpr int kThreads = 256;

// Commit.  Row len + path[t] goes to row len + t; along a root path of a
// topologically ordered draft path[t] >= t and rises, so moving t upwards
// never overwrites a row that is still to be read.  A thread owns one 16-byte
// column of one head of one layer's keys or values and moves it for every t,
// so that order is its own program order and no two threads meet.  Groups of
// kGroup steps are read before they are written: the reads of a group overlap
// one another, and a later group's rows lie above the rows written.
constexpr int kGroup = 8;

template <int COLS>
__global__ __launch_bounds__(kThreads) void commit_kernel(AttnCommitArgs a) {
  const int b = blockIdx.y;
  const int lane = threadIdx.x % kWave;
  const int n = a.n;
  const int len = a.rows.len[b], m = a.accepted[b];
  const int32_t *parent = a.parent + (size_t)b * n, *path = a.path + (size_t)b * n;
  const int shift = a.cache.page_shift, mask = (1 << shift) - 1;

  // every wave looks at the whole path: lane t at step t.  A parent behind its
  // child (an array out of topological order) would break the rising order.
  int err = check_path(parent, n, path, m, lane);
  if (err == SLA_OK && wave_any(lane > 0 && lane < m && path[lane] <= path[lane - 1])) err = SLA_ERR_PATH;
  int from = 0, src = 0, dst = 0;
  if (err == SLA_OK && !length_ok(a.rows, shift, len, n)) err = SLA_ERR_LENGTH;
  if (err == SLA_OK) {
    if (lane < m) {
      const int32_t *table = a.rows.table + (size_t)b * a.rows.max_pages;
      from = path[lane];
      src = table[(len + from) >> shift];
      dst = table[(len + lane) >> shift];
    }
    if (wave_any(src < 0 || src >= a.cache.n_pages || dst < 0 || dst >= a.cache.n_pages)) err = SLA_ERR_PAGE;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (a.status) a.status[b] = err;
    if (a.new_len) a.new_len[b] = err == SLA_OK ? len + m : len;
  }
  if (err != SLA_OK) return;
  // the rows in front of the first one that moves are in place
  const uint64_t moved = __ballot(lane < m && from != lane);
  if (!moved) return;
  const int t0 = __builtin_ctzll(moved);

  const int Hkv = a.cache.Hkv;
  const unsigned item = blockIdx.x * (kThreads / COLS) + threadIdx.x / COLS;  // (layer, keys or values, head)
  const int h = item % Hkv, kv = item / Hkv % 2, layer = item / Hkv / 2;
  const bool live = layer < a.layers;  // a launch's last workgroup may have columns to spare
  uint4 *base = static_cast<uint4 *>(kv ? a.cache.v : a.cache.k) +
                (live ? (((size_t)layer * a.cache.n_pages * Hkv) << shift) * COLS : 0) + threadIdx.x % COLS;
  for (int t = t0; t < m; t += kGroup) {
    uint4 x[kGroup];
#pragma unroll
    for (int i = 0; i < kGroup; ++i)
      if (live && t + i < m) {
        const int page = __builtin_amdgcn_readlane(src, t + i), row = (len + __builtin_amdgcn_readlane(from, t + i)) & mask;
        x[i] = base[(page_row(a.cache, page, h) + row) * COLS];
      }
#pragma unroll
    for (int i = 0; i < kGroup; ++i)
      if (live && t + i < m) {
        const int page = __builtin_amdgcn_readlane(dst, t + i), row = (len + t + i) & mask;
        base[(page_row(a.cache, page, h) + row) * COLS] = x[i];
      }
  }
}

template <int COLS>
hipError_t launch_commit_c(const AttnCommitArgs &a, hipStream_t s) {
  const int per = kThreads / COLS;
  const unsigned blocks = (unsigned)((a.layers * 2 * a.cache.Hkv + per - 1) / per);
  hipLaunchKernelGGL(commit_kernel<COLS>, dim3(blocks, (unsigned)a.B), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

// Copy.  One workgroup: the rows of one page in one head of one layer's keys
// or values, which are contiguous; of more than one page if there are more copies
// than a launch is high.
constexpr int kGridHeight = 65535;

__global__ __launch_bounds__(kThreads) void page_copy_kernel(PageCopyArgs a, int cols) {
  const int Hkv = a.cache.Hkv, shift = a.cache.page_shift;
  const int piece = blockIdx.x;
  const int h = piece % Hkv, kv = piece / Hkv % 2, layer = piece / Hkv / 2;
  uint4 *base = static_cast<uint4 *>(kv ? a.cache.v : a.cache.k) + (((size_t)layer * a.cache.n_pages * Hkv) << shift) * cols;
  for (int i = blockIdx.y; i < a.copies; i += kGridHeight) {
    const int src = a.src[i], dst = a.dst[i], rows = a.rows ? a.rows[i] : 1 << shift;
    int err = SLA_OK;
    if (src < 0 || src >= a.cache.n_pages || dst < 0 || dst >= a.cache.n_pages) err = SLA_ERR_PAGE;
    else if (rows < 0 || rows > 1 << shift) err = SLA_ERR_LENGTH;
    if (a.status && piece == 0 && threadIdx.x == 0) a.status[i] = err;
    if (err != SLA_OK || src == dst) continue;
    const uint4 *from = base + page_row(a.cache, src, h) * cols;
    uint4 *to = base + page_row(a.cache, dst, h) * cols;
    const int total = rows * cols;
    for (int c = threadIdx.x; c < total; c += kThreads) to[c] = from[c];
  }
}

}  // namespace

hipError_t launch_attn_commit(const AttnCommitArgs &a, int dtype, hipStream_t s) {
  switch (a.cache.D * (dtype == SLA_DTYPE_BF16 ? 2 : 4) / 16) {
    case 8: return launch_commit_c<8>(a, s);
    case 16: return launch_commit_c<16>(a, s);
    case 32: return launch_commit_c<32>(a, s);
    default: return launch_commit_c<64>(a, s);
  }
}

hipError_t launch_page_copy(const PageCopyArgs &a, int dtype, hipStream_t s) {
  const int cols = a.cache.D * (dtype == SLA_DTYPE_BF16 ? 2 : 4) / 16;
  const dim3 grid((unsigned)(a.layers * 2 * a.cache.Hkv), (unsigned)(a.copies < kGridHeight ? a.copies : kGridHeight));
  hipLaunchKernelGGL(page_copy_kernel, grid, dim3(kThreads), 0, s, a, cols);
  return hipGetLastError();
}

}  // namespace sla
