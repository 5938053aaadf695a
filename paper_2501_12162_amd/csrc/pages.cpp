// Host side of the entry points of the cache's pages: argument validation,
// which runs before any HIP call, and the launches.
#include "pages.h"

#include <hip/hip_runtime.h>

#include "adaserve.h"
#include "host_device.h"
#include "host_plan.h"

namespace {

using namespace adaserve;

constexpr int32_t kMaxStride = 1 << 24, kMaxPageTokens = 1 << 16;

// An array of the call: an input, or an output, which may be the input `same` itself.
struct Array {
  const char *name;
  const void *p;
  int64_t bytes;
  bool output;
  const void *same;
};

int32_t validate_arrays(const Array *a, int n) {
  for (int i = 0; i < n; ++i) {
    if (a[i].bytes > 0 && !a[i].p) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "%s is NULL", a[i].name);
    if (!aligned(a[i].p, 4)) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "%s is not aligned to its elements", a[i].name);
    for (int k = 0; k < i; ++k) {
      const char *x = (const char *)a[i].p, *y = (const char *)a[k].p;
      if (a[i].bytes == 0 || a[k].bytes == 0 || !(a[i].output || a[k].output)) continue;
      if (x >= y + a[k].bytes || y >= x + a[i].bytes) continue;
      if (x == y && (a[i].same == y || a[k].same == x)) continue;
      return fail(ADASERVE_ERR_INVALID_ARGUMENT, "%s overlaps %s", a[i].name, a[k].name);
    }
  }
  return ADASERVE_OK;
}

int32_t validate_pool(const char *what, int32_t rows, int32_t num_pages, int32_t stride) {
  if (rows < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "%s %d < 0", what, rows);
  if (num_pages < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_pages %d < 0", num_pages);
  if (stride < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "block_table_stride %d < 0", stride);
  if (rows > kPagesMaxRows) return fail(ADASERVE_ERR_UNSUPPORTED, "%s %d > %d", what, rows, kPagesMaxRows);
  if (num_pages > kPagesMaxPages) return fail(ADASERVE_ERR_UNSUPPORTED, "num_pages %d > %d", num_pages, kPagesMaxPages);
  if (stride > kMaxStride) return fail(ADASERVE_ERR_UNSUPPORTED, "block_table_stride %d > %d", stride, kMaxStride);
  return ADASERVE_OK;
}

int32_t validate_page_size(int32_t page_size) {
  if (page_size < 1) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "page_size %d < 1", page_size);
  if (page_size > kMaxPageTokens) return fail(ADASERVE_ERR_UNSUPPORTED, "page_size %d > %d", page_size, kMaxPageTokens);
  return ADASERVE_OK;
}

// The workspace's parts, after its checks; none of a call without rows and pages.
int32_t set_space(PagesArgs &a, int32_t rows, int32_t num_pages, void *workspace, size_t given) {
  const PagesSpace s = pages_space(rows, num_pages);
  if (s.bytes == 0) return ADASERVE_OK;
  if (!workspace || given < s.bytes)
    return fail(ADASERVE_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace ? given : (size_t)0, s.bytes);
  if (!aligned(workspace, 256)) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "workspace must be 256-byte aligned");
  char *ws = (char *)workspace;
  a.ws_want = (int32_t *)ws;
  a.ws_list = (int32_t *)(ws + s.list);
  a.ws_bits = (unsigned long long *)(ws + s.list);
  a.ws_runs = (int32_t *)(ws + s.runs);
  return ADASERVE_OK;
}

}  // namespace

extern "C" {

size_t adaserve_pages_workspace_bytes(int32_t num_rows, int32_t num_pages) {
  if (validate_pool("num_rows", num_rows, num_pages, 0) != ADASERVE_OK) return SIZE_MAX;
  return pages_space(num_rows, num_pages).bytes;
}

int32_t adaserve_update_pages(int32_t num_requests, const int32_t *context_len, const int32_t *need_len, int32_t window,
                              int32_t sinks, int32_t page_size, const int32_t *block_table, int32_t block_table_stride,
                              const int32_t *page_refs, int32_t num_pages, int32_t *new_block_table,
                              int32_t *new_page_refs, int32_t *capacity, void *workspace, size_t workspace_bytes,
                              void *stream) {
  int32_t st = validate_pool("num_requests", num_requests, num_pages, block_table_stride);
  if (st != ADASERVE_OK) return st;
  st = validate_page_size(page_size);
  if (st != ADASERVE_OK) return st;
  if (window < 0 || sinks < 0)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "window %d and sinks %d must not be negative", window, sinks);
  if ((need_len == nullptr) != (capacity == nullptr) && num_requests > 0)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "need_len and capacity go together");
  const int64_t lens = 4ll * num_requests, table = lens * block_table_stride, refs = 4ll * num_pages;
  PagesArgs a{};
  st = set_space(a, num_requests, num_pages, workspace, workspace_bytes);
  if (st != ADASERVE_OK) return st;
  const Array arrays[] = {{"context_len", context_len, lens, false, nullptr},
                          {"need_len", need_len, need_len ? lens : 0, false, nullptr},
                          {"block_table", block_table, table, false, nullptr},
                          {"page_refs", page_refs, refs, false, nullptr},
                          {"new_block_table", new_block_table, table, true, block_table},
                          {"new_page_refs", new_page_refs, refs, true, page_refs},
                          {"capacity", capacity, capacity ? lens : 0, true, nullptr},
                          {"workspace", workspace, (int64_t)pages_space(num_requests, num_pages).bytes, true, nullptr}};
  st = validate_arrays(arrays, sizeof(arrays) / sizeof(arrays[0]));
  if (st != ADASERVE_OK) return st;
  if (num_requests == 0 && num_pages == 0) return ADASERVE_OK;
  st = check_device();
  if (st != ADASERVE_OK) return st;
  a.rows = num_requests;
  a.context_len = context_len;
  a.need_len = need_len;
  a.window = window;
  a.sinks = sinks;
  a.page_size = page_size;
  a.table = block_table;
  a.stride = block_table_stride;
  a.refs = page_refs;
  a.pages = num_pages;
  a.new_table = new_block_table;
  a.new_refs = new_page_refs;
  a.capacity = capacity;
  return launch_status(launch_update_pages(a, (hipStream_t)stream), "page update launch");
}

int32_t adaserve_fork_pages(int32_t num_sources, int32_t num_requests, const int32_t *source, const int32_t *context_len,
                            int32_t page_size, const int32_t *block_table, int32_t block_table_stride,
                            const int32_t *page_refs, int32_t num_pages, int32_t *new_block_table,
                            int32_t *new_context_len, int32_t *new_page_refs, int32_t *copy_src, int32_t *copy_dst,
                            void *workspace, size_t workspace_bytes, void *stream) {
  int32_t st = validate_pool("num_requests", num_requests, num_pages, block_table_stride);
  if (st != ADASERVE_OK) return st;
  st = validate_pool("num_sources", num_sources, num_pages, block_table_stride);
  if (st != ADASERVE_OK) return st;
  st = validate_page_size(page_size);
  if (st != ADASERVE_OK) return st;
  const int32_t most = num_sources > num_requests ? num_sources : num_requests;
  const int64_t old = 4ll * num_sources, lens = 4ll * num_requests, refs = 4ll * num_pages;
  PagesArgs a{};
  st = set_space(a, most, num_pages, workspace, workspace_bytes);
  if (st != ADASERVE_OK) return st;
  const Array arrays[] = {{"source", source, lens, false, nullptr},
                          {"context_len", context_len, old, false, nullptr},
                          {"block_table", block_table, old * block_table_stride, false, nullptr},
                          {"page_refs", page_refs, refs, false, nullptr},
                          {"new_block_table", new_block_table, lens * block_table_stride, true, nullptr},
                          {"new_context_len", new_context_len, lens, true, nullptr},
                          {"new_page_refs", new_page_refs, refs, true, page_refs},
                          {"copy_src", copy_src, lens, true, nullptr},
                          {"copy_dst", copy_dst, lens, true, nullptr},
                          {"workspace", workspace, (int64_t)pages_space(most, num_pages).bytes, true, nullptr}};
  st = validate_arrays(arrays, sizeof(arrays) / sizeof(arrays[0]));
  if (st != ADASERVE_OK) return st;
  if (most == 0 && num_pages == 0) return ADASERVE_OK;
  st = check_device();
  if (st != ADASERVE_OK) return st;
  a.rows = num_requests;
  a.sources = num_sources;
  a.source = source;
  a.context_len = context_len;
  a.page_size = page_size;
  a.table = block_table;
  a.stride = block_table_stride;
  a.refs = page_refs;
  a.pages = num_pages;
  a.new_table = new_block_table;
  a.new_len = new_context_len;
  a.new_refs = new_page_refs;
  a.copy_src = copy_src;
  a.copy_dst = copy_dst;
  return launch_status(launch_fork_pages(a, (hipStream_t)stream), "page fork launch");
}

int32_t adaserve_compact_pages(int32_t num_requests, const int32_t *block_table, int32_t block_table_stride,
                               const int32_t *page_refs, int32_t num_pages, int32_t *new_block_table,
                               int32_t *new_page_refs, int32_t *new_place, int32_t *move_src, int32_t *move_dst,
                               int32_t *counts, void *workspace, size_t workspace_bytes, void *stream) {
  int32_t st = validate_pool("num_requests", num_requests, num_pages, block_table_stride);
  if (st != ADASERVE_OK) return st;
  const int64_t table = 4ll * num_requests * block_table_stride, refs = 4ll * num_pages;
  if (table / 4 + num_pages >= (int64_t)1 << 31)   // a thread each
    return fail(ADASERVE_ERR_UNSUPPORTED, "%lld entries of block tables exceed a launch", (long long)(table / 4));
  PagesArgs a{};
  st = set_space(a, num_requests, num_pages, workspace, workspace_bytes);
  if (st != ADASERVE_OK) return st;
  const Array arrays[] = {{"block_table", block_table, table, false, nullptr},
                          {"page_refs", page_refs, refs, false, nullptr},
                          {"new_block_table", new_block_table, table, true, block_table},
                          {"new_page_refs", new_page_refs, refs, true, page_refs},
                          {"new_place", new_place, refs, true, nullptr},
                          {"move_src", move_src, refs, true, nullptr},
                          {"move_dst", move_dst, refs, true, nullptr},
                          {"counts", counts, 8, true, nullptr},
                          {"workspace", workspace, (int64_t)pages_space(num_requests, num_pages).bytes, true, nullptr}};
  st = validate_arrays(arrays, sizeof(arrays) / sizeof(arrays[0]));
  if (st != ADASERVE_OK) return st;
  st = check_device();
  if (st != ADASERVE_OK) return st;
  a.rows = num_requests;
  a.table = block_table;
  a.stride = block_table_stride;
  a.refs = page_refs;
  a.pages = num_pages;
  a.new_table = new_block_table;
  a.new_refs = new_page_refs;
  a.new_place = new_place;
  a.copy_src = move_src;
  a.copy_dst = move_dst;
  a.counts = counts;
  return launch_status(launch_compact_pages(a, (hipStream_t)stream), "page compaction launch");
}

int32_t adaserve_copy_pages(int32_t num_copies, const int32_t *src, const int32_t *dst, const int32_t *count,
                            void *k_pages, void *v_pages, int32_t num_layers, int64_t layer_stride, int32_t num_pages,
                            int32_t num_kv_heads, int32_t page_size, int32_t head_dim, int32_t dtype, void *stream) {
  int32_t st = validate_pool("num_copies", 0, num_pages, 0);
  if (st != ADASERVE_OK) return st;
  if (num_copies < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_copies %d < 0", num_copies);
  if (num_layers < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_layers %d < 0", num_layers);
  if (num_copies > kPagesMaxPages || num_layers > kPagesMaxRows)
    return fail(ADASERVE_ERR_UNSUPPORTED, "num_copies %d > %d, or num_layers %d > %d", num_copies, kPagesMaxPages,
                num_layers, kPagesMaxRows);
  st = validate_page_size(page_size);
  if (st != ADASERVE_OK) return st;
  if (dtype != ADASERVE_F32 && dtype != ADASERVE_BF16)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "dtype %d is neither F32 nor BF16", dtype);
  const int64_t esz = dtype == ADASERVE_BF16 ? 2 : 4;
  if (num_kv_heads < 1 || head_dim < 1)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_kv_heads %d and head_dim %d must be positive", num_kv_heads, head_dim);
  if (num_kv_heads > 4096 || head_dim > 4096 || head_dim * esz % 16 != 0)
    return fail(ADASERVE_ERR_UNSUPPORTED, "num_kv_heads %d, head_dim %d: at most 4096 each, rows a multiple of 16 bytes",
                num_kv_heads, head_dim);
  const int64_t page_bytes = (int64_t)num_kv_heads * page_size * head_dim * esz;
  if (page_bytes > (int64_t)1 << 30)
    return fail(ADASERVE_ERR_UNSUPPORTED, "pages of %lld bytes exceed 2^30", (long long)page_bytes);
  if (num_layers > 1) {
    // (its range first: the products with the element's size are within 64 bits then)
    if (layer_stride > ((int64_t)1 << 48) / num_layers)
      return fail(ADASERVE_ERR_UNSUPPORTED, "%d layers %lld elements apart span more than 2^48 elements", num_layers,
                  (long long)layer_stride);
    if (layer_stride < page_bytes / esz * num_pages || layer_stride * esz % 16 != 0)
      return fail(ADASERVE_ERR_INVALID_ARGUMENT, "layer_stride %lld: less than a pool, or not a multiple of 16 bytes",
                  (long long)layer_stride);
  }
  if (num_copies == 0 || num_layers == 0 || num_pages == 0) return ADASERVE_OK;
  if (!src || !dst || !k_pages || !v_pages) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "a required device pointer is NULL");
  if (!aligned(src, 4) || !aligned(dst, 4) || !aligned(count, 4) || !aligned(k_pages, 16) || !aligned(v_pages, 16))
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "src, dst and count must be aligned to 4 bytes, k_pages and v_pages to 16");
  st = check_device();
  if (st != ADASERVE_OK) return st;
  CopyPagesArgs a{};
  a.copies = num_copies;
  a.src = src;
  a.dst = dst;
  a.count = count;
  a.pool[0] = (char *)k_pages;
  a.pool[1] = (char *)v_pages;
  a.layers = num_layers;
  a.layer_bytes = num_layers > 1 ? layer_stride * esz : 0;
  a.page_bytes = page_bytes;
  a.pages = num_pages;
  return launch_status(launch_copy_pages(a, (hipStream_t)stream), "page copy launch");
}

}  // extern "C"
