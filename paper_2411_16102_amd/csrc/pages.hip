// Copies of pages inside the pools of a cache.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <vector>

#include "../../include/blendstep_bits.h"
#include "common.hpp"
#include "context.hpp"
#include "pages.hpp"

using namespace bs;

namespace {

// A workgroup per page and pool.  pools [n_pools] addresses (two words each), then n pairs (src, dst), in pinned memory; 16-byte
// units of a page.  Bound by memory: 502 pages of 64 KB in 16 pools 196 to 210 us, 5.0 to 5.4 TB/s; 120 copies of 15 pages in 32 pools, whose sources
// the caches hold, 76 us; 4 pages in 32 pools 7 us.
__global__ __launch_bounds__(256) void copy_pages_kernel(const int32_t *list, int n_pools, int units) {
  const int pool = blockIdx.y;
  u32x4_t *base = *reinterpret_cast<u32x4_t *const *>(list + 2 * pool);
  const int32_t *pair = list + 2 * n_pools + 2 * blockIdx.x;
  const u32x4_t *src = base + (size_t)pair[0] * units;
  u32x4_t *dst = base + (size_t)pair[1] * units;
  for (int i = threadIdx.x; i < units; i += 256) dst[i] = src[i];
}

int check_pools(bs_ctx *c, void *const *pools, int32_t n_pools, int64_t n_pages) {
  if (ctx_view(c).device == BS_DEVICE_NONE) return ctx_fail(c, BS_EINVAL, "host-only context");
  if (n_pools < 0 || n_pools > 65535 || (n_pools > 0 && !pools)) return ctx_fail(c, BS_EINVAL, "n_pools=%d (0 to 65535, with their addresses)", n_pools);
  if (n_pages < 0 || n_pages > (int64_t)0x7fffffff) return ctx_fail(c, BS_EINVAL, "n_pages=%lld out of range", (long long)n_pages);
  for (int i = 0; i < n_pools; ++i)
    if (!pools[i] || (reinterpret_cast<uintptr_t>(pools[i]) & 15)) return ctx_fail(c, BS_EINVAL, "pool %d is NULL or not 16-byte aligned", i);
  return BS_OK;
}

// (the pairs have been checked)
int copy_pairs(bs_ctx *c, void *const *pools, int32_t n_pools, int64_t page_bytes, const int32_t *src, const int32_t *dst, int32_t n, hipStream_t stream) {
  if (n == 0 || n_pools == 0) return BS_OK;
  CTX_HIP_TRY(c, hipSetDevice(ctx_view(c).device));
  int32_t *list = nullptr;
  if (const int rc = ctx_stage(c, 2L * n_pools + 2L * n, stream, &list)) return rc;
  for (int i = 0; i < n_pools; ++i) std::memcpy(list + 2 * i, &pools[i], sizeof(void *));
  for (int i = 0; i < n; ++i) {
    list[2 * n_pools + 2 * i] = src[i];
    list[2 * n_pools + 2 * i + 1] = dst[i];
  }
  const int units = (int)(page_bytes / 16);
  hipLaunchKernelGGL(copy_pages_kernel, dim3(n, n_pools), dim3(256), 0, stream, list, n_pools, units);
  CTX_HIP_TRY(c, hipGetLastError());
  return BS_OK;
}

int copy_pages(bs_ctx *c, const char *what, void *const *pools, int32_t n_pools, int64_t n_pages, int64_t page_bytes, const int32_t *src, const int32_t *dst,
               int32_t n, void *stream) {
  if (const int rc = check_pools(c, pools, n_pools, n_pages)) return rc;
  if (n < 0 || (n > 0 && (!src || !dst))) return ctx_fail(c, BS_EINVAL, "%s: bad list of %d pairs", what, n);
  for (int i = 0; i < n; ++i)
    if (src[i] < 0 || src[i] >= n_pages || dst[i] < 0 || dst[i] >= n_pages)
      return ctx_fail(c, BS_EINVAL, "pair %d (%d, %d) outside the pool of %lld pages", i, src[i], dst[i], (long long)n_pages);
  std::vector<int32_t> to(dst, dst + n);
  std::sort(to.begin(), to.end());
  const auto twice = std::adjacent_find(to.begin(), to.end());
  if (twice != to.end()) return ctx_fail(c, BS_EINVAL, "page %d is copied to twice", *twice);
  for (int i = 0; i < n; ++i)
    if (std::binary_search(to.begin(), to.end(), src[i])) return ctx_fail(c, BS_EINVAL, "page %d is copied from and to", src[i]);
  return copy_pairs(c, pools, n_pools, page_bytes, src, dst, n, (hipStream_t)stream);
}

int compact(bs_ctx *c, const char *what, void *const *pools, int32_t n_pools, int64_t n_pages, int64_t page_bytes, const int32_t *tables, int64_t n,
            int32_t *tables_out, int32_t *n_live, void *stream) {
  if (const int rc = check_pools(c, pools, n_pools, n_pages)) return rc;
  if (n < 0 || !n_live || (n > 0 && (!tables || !tables_out))) return ctx_fail(c, BS_EINVAL, "%s: bad argument", what);
  std::vector<char> named((size_t)n_pages, 0);
  for (int64_t i = 0; i < n; ++i) {
    if (tables[i] == BS_PAGE_NONE) continue;
    if (tables[i] < 0 || tables[i] >= n_pages) return ctx_fail(c, BS_EINVAL, "tables[%lld]=%d outside the pool of %lld pages", (long long)i, tables[i], (long long)n_pages);
    named[tables[i]] = 1;
  }
  std::vector<int32_t> to, src, dst;
  const int32_t live = plan_compaction(named, to, src, dst);
  if (const int rc = copy_pairs(c, pools, n_pools, page_bytes, src.data(), dst.data(), (int32_t)src.size(), (hipStream_t)stream)) return rc;
  for (int64_t i = 0; i < n; ++i) tables_out[i] = tables[i] == BS_PAGE_NONE ? BS_PAGE_NONE : to[tables[i]];
  *n_live = live;
  return BS_OK;
}

}  // namespace

extern "C" {

int bs_kv_copy_pages(bs_ctx *c, void *const *pools, int32_t n_pools, int64_t n_pages, const int32_t *src, const int32_t *dst, int32_t n,
                     void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&] { return copy_pages(c, "bs_kv_copy_pages", pools, n_pools, n_pages, bs_kv_page_bytes(c), src, dst, n, stream); });
}

int bs_kv_compact(bs_ctx *c, void *const *pools, int32_t n_pools, int64_t n_pages, const int32_t *tables, int64_t n, int32_t *tables_out,
                  int32_t *n_live, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&] { return compact(c, "bs_kv_compact", pools, n_pools, n_pages, bs_kv_page_bytes(c), tables, n, tables_out, n_live, stream); });
}

int bs_kv4_copy_pages(bs_ctx *c, void *const *pools, int32_t n_pools, int64_t n_pages, int32_t group, const int32_t *src, const int32_t *dst,
                      int32_t n, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    const int64_t bytes = bs_kv4_page_bytes(c, group);
    if (bytes == 0) return ctx_fail(c, BS_EINVAL, "bs_kv4_copy_pages: groups of %d channels are not supported", group);
    return copy_pages(c, "bs_kv4_copy_pages", pools, n_pools, n_pages, bytes, src, dst, n, stream);
  });
}

int bs_kv4_compact(bs_ctx *c, void *const *pools, int32_t n_pools, int64_t n_pages, int32_t group, const int32_t *tables, int64_t n,
                   int32_t *tables_out, int32_t *n_live, void *stream) {
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    const int64_t bytes = bs_kv4_page_bytes(c, group);
    if (bytes == 0) return ctx_fail(c, BS_EINVAL, "bs_kv4_compact: groups of %d channels are not supported", group);
    return compact(c, "bs_kv4_compact", pools, n_pools, n_pages, bytes, tables, n, tables_out, n_live, stream);
  });
}

}  // extern "C"
