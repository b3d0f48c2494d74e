// Pages of a paged cache: reference counts on the host, and the moves and table
// rewrites that a fork or a compaction needs on the device (contracts in
// include/moe_api.h).
#include <hip/hip_runtime.h>

#include <functional>
#include <new>
#include <queue>
#include <utility>
#include <vector>

#include "moe_device.h"

namespace moe {
namespace {

constexpr int kCopyThreads = 256;
constexpr int kCopyPieces = 4;                 // 16-byte pieces a thread has in flight
constexpr int kCopyBytes = kCopyThreads * kCopyPieces * 16;

// One workgroup copies kCopyBytes of one page of one layer: four 16-byte loads a thread,
// then the stores. Bound by HBM, a byte read and a byte written for each byte moved: 400
// pages of 74 KB in 8 layers, 472 MB, in 90 us (5.2 TB/s); 24 pages in 24 layers, 85 MB, in
// 15 us.
__global__ void __launch_bounds__(kCopyThreads)
    page_copy_kernel(char* __restrict__ pages, int64_t layer_bytes, int64_t page_bytes, int n_pages, int parts,
                     const int2* __restrict__ pairs, uint32_t* status) {
  const int2 p = pairs[blockIdx.x / parts];
  if ((unsigned)p.x >= (unsigned)n_pages || (unsigned)p.y >= (unsigned)n_pages) {
    if (threadIdx.x == 0 && status) atomicOr(status, MOE_STATUS_BAD_PAGE);
    return;
  }
  char* layer = pages + (int64_t)blockIdx.y * layer_bytes;
  const char* from = layer + p.x * page_bytes;
  char* to = layer + p.y * page_bytes;
  const int64_t at = (int64_t)(blockIdx.x % parts) * kCopyBytes + threadIdx.x * 16;
  U4 v[kCopyPieces];
#pragma unroll
  for (int k = 0; k < kCopyPieces; ++k)
    if (at + k * kCopyThreads * 16 < page_bytes) v[k] = ld16(from + at + k * kCopyThreads * 16);
#pragma unroll
  for (int k = 0; k < kCopyPieces; ++k)
    if (at + k * kCopyThreads * 16 < page_bytes) *reinterpret_cast<U4*>(to + at + k * kCopyThreads * 16) = v[k];
}

// One entry a thread; latency (2,000 entries: 3.9 us).
__global__ void __launch_bounds__(256)
    page_remap_kernel(const int32_t* table_in, int64_t n, const int32_t* __restrict__ remap, int n_pages,
                      int32_t* table_out, uint32_t* status) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  int32_t p = table_in[i];
  if (p >= n_pages) {
    if (status) atomicOr(status, MOE_STATUS_BAD_PAGE);
  } else if (p >= 0) {
    p = remap[p];
  }
  table_out[i] = p;
}

}  // namespace
}  // namespace moe

struct moe_page_pool {
  int n_pages = 0, page_tokens = 0;
  std::vector<int32_t> refs;
  // free page ids, the lowest first
  std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>> free_ids;
};

namespace {

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// every id a live page
bool live(const moe_page_pool* p, const int32_t* pages, int n) {
  for (int i = 0; i < n; ++i)
    if (pages[i] < 0 || pages[i] >= p->n_pages || p->refs[pages[i]] < 1) return false;
  return true;
}

void take(moe_page_pool* p, int n, int32_t* out) {
  for (int i = 0; i < n; ++i) {
    out[i] = p->free_ids.top();
    p->free_ids.pop();
    p->refs[out[i]] = 1;
  }
}

}  // namespace

extern "C" {

int moe_page_pool_create(int n_pages, int page_tokens, moe_page_pool** out) {
  if (!out || n_pages < 1 || n_pages > (1 << 24) || page_tokens < 1 || page_tokens > 4096) return MOE_EINVAL;
  try {
    moe_page_pool* p = new moe_page_pool;
    p->n_pages = n_pages;
    p->page_tokens = page_tokens;
    try {
      p->refs.assign(n_pages, 0);
      std::vector<int32_t> ids(n_pages);
      for (int i = 0; i < n_pages; ++i) ids[i] = i;
      p->free_ids = decltype(p->free_ids)(std::greater<int32_t>(), std::move(ids));
    } catch (...) {
      delete p;
      throw;
    }
    *out = p;
    return MOE_OK;
  } catch (const std::bad_alloc&) {
    return MOE_ENOMEM;
  }
}

int moe_page_pool_destroy(moe_page_pool* p) {
  if (!p) return MOE_EINVAL;
  delete p;
  return MOE_OK;
}

int moe_page_pool_available(const moe_page_pool* p) { return p ? (int)p->free_ids.size() : MOE_EINVAL; }

int moe_page_pool_refs(const moe_page_pool* p, int page) {
  if (!p || page < 0 || page >= p->n_pages) return MOE_EINVAL;
  return p->refs[page];
}

int moe_page_pool_alloc(moe_page_pool* p, int n, int32_t* pages) {
  if (!p || n < 0 || (n && !pages)) return MOE_EINVAL;
  if ((size_t)n > p->free_ids.size()) return MOE_ENOMEM;
  take(p, n, pages);
  return MOE_OK;
}

int moe_page_pool_fork(moe_page_pool* p, const int32_t* pages, int64_t n_tokens, int32_t* forked, int32_t* copy) {
  if (!p || n_tokens < 0 || n_tokens > (int64_t)p->n_pages * p->page_tokens) return MOE_EINVAL;
  const int n = (int)((n_tokens + p->page_tokens - 1) / p->page_tokens);
  if (n == 0) return 0;
  const bool partial = n_tokens % p->page_tokens != 0;
  if (!pages || !forked || (partial && !copy) || !live(p, pages, n)) return MOE_EINVAL;
  if (partial && p->free_ids.empty()) return MOE_ENOMEM;
  const int shared = partial ? n - 1 : n;
  for (int i = 0; i < shared; ++i) {
    ++p->refs[pages[i]];
    forked[i] = pages[i];
  }
  if (!partial) return 0;
  const int32_t from = pages[n - 1];
  take(p, 1, forked + n - 1);
  copy[0] = from;
  copy[1] = forked[n - 1];
  return 1;
}

int moe_page_pool_free(moe_page_pool* p, const int32_t* pages, int n) {
  if (!p || n < 0 || (n && !pages)) return MOE_EINVAL;
  // all or none: an id may stand several times, as often as it is referenced
  for (int i = 0; i < n; ++i) {
    const int32_t id = pages[i];
    if (id < 0 || id >= p->n_pages || p->refs[id] < 1) {
      for (int k = 0; k < i; ++k) ++p->refs[pages[k]];
      return MOE_EINVAL;
    }
    --p->refs[id];
  }
  for (int i = 0; i < n; ++i)
    if (p->refs[pages[i]] == 0) {
      p->free_ids.push(pages[i]);    // (room for every page is reserved: nothing is allocated)
      p->refs[pages[i]] = -1;        // (pushed: the id may stand again)
    }
  for (int i = 0; i < n; ++i)
    if (p->refs[pages[i]] < 0) p->refs[pages[i]] = 0;
  return MOE_OK;
}

int moe_page_pool_compact(moe_page_pool* p, int32_t* moves, int32_t* remap) {
  if (!p || !moves || !remap) return MOE_EINVAL;
  const int live_n = p->n_pages - (int)p->free_ids.size();
  std::vector<int32_t> ids;
  try {
    ids.reserve(p->n_pages);
  } catch (const std::bad_alloc&) {
    return MOE_ENOMEM;
  }
  for (int i = 0; i < p->n_pages; ++i) remap[i] = p->refs[i] > 0 ? i : -1;
  int n = 0, hole = 0;
  for (int i = live_n; i < p->n_pages; ++i) {
    ids.push_back(i);
    if (p->refs[i] == 0) continue;
    while (p->refs[hole] > 0) ++hole;  // (as many holes below live_n as live pages above)
    moves[2 * n] = i;
    moves[2 * n + 1] = hole;
    remap[i] = hole;
    p->refs[hole] = p->refs[i];
    p->refs[i] = 0;
    ++n;
  }
  p->free_ids = decltype(p->free_ids)(std::greater<int32_t>(), std::move(ids));
  return n;
}

int moe_page_copy(void* pages, int n_layers, int64_t layer_bytes, int64_t page_bytes, int n_pages,
                  const int32_t* pairs, int n, uint32_t* status, void* stream) {
  if (n_layers < 1 || n_layers > 65535 || n_pages < 1 || n < 0 || page_bytes < 16 || page_bytes % 16 ||
      page_bytes > (int64_t(1) << 32) || layer_bytes % 16 ||
      (n_layers > 1 && layer_bytes / n_pages < page_bytes))
    return MOE_EINVAL;
  if (n == 0) return MOE_OK;
  if (!pages || !pairs) return MOE_EINVAL;
  if (misaligned(pages, 16) || misaligned(pairs, 8) || misaligned(status, 4)) return MOE_EALIGN;
  const int parts = (int)((page_bytes + moe::kCopyBytes - 1) / moe::kCopyBytes);
  if ((int64_t)n * parts * moe::kCopyThreads > (int64_t)UINT32_MAX) return MOE_EINVAL;  // (a grid's threads)
  hipLaunchKernelGGL(moe::page_copy_kernel, dim3((unsigned)n * parts, n_layers), dim3(moe::kCopyThreads), 0,
                     static_cast<hipStream_t>(stream), static_cast<char*>(pages), layer_bytes, page_bytes, n_pages,
                     parts, reinterpret_cast<const int2*>(pairs), status);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_EHIP;
}

int moe_page_remap(const int32_t* table_in, int64_t n, const int32_t* remap, int n_pages, int32_t* table_out,
                   uint32_t* status, void* stream) {
  if (n < 0 || n > (int64_t(1) << 31) || n_pages < 1) return MOE_EINVAL;
  if (n == 0) return MOE_OK;
  if (!table_in || !remap || !table_out) return MOE_EINVAL;
  if (misaligned(table_in, 4) || misaligned(remap, 4) || misaligned(table_out, 4) || misaligned(status, 4))
    return MOE_EALIGN;
  hipLaunchKernelGGL(moe::page_remap_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), table_in, n, remap, n_pages, table_out, status);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_EHIP;
}

}  // extern "C"
