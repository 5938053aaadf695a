// Internal interface between the host entry points of the cache's pages
// (pages.cpp) and their kernels (pages.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace adaserve {

constexpr int kPagesThreads = 256;
constexpr int kPagesMaxRows = 1 << 16;
constexpr int kPagesMaxPages = 1 << 23;
constexpr int kPagesRun = 1024;          // pages that a wave counts at a time

struct PagesArgs {
  int32_t rows;                  // of the new table
  int32_t sources;               // of the old one (fork)
  const int32_t *source;         // [rows] (fork)
  const int32_t *context_len;    // [rows], of a fork [sources]
  const int32_t *need_len;       // [rows], or null
  int32_t window, sinks;
  int32_t page_size;
  const int32_t *table;          // [sources or rows, stride]
  int32_t stride;
  const int32_t *refs;           // [pages]
  int32_t pages;
  int32_t *new_table;            // [rows, stride]
  int32_t *new_refs;             // [pages]
  int32_t *capacity;             // [rows]
  int32_t *new_len;              // [rows]
  int32_t *copy_src, *copy_dst;  // [rows], of a compaction [pages]
  int32_t *new_place;            // [pages]
  int32_t *counts;               // [2]
  // workspace
  int32_t *ws_want;              // [rows] pages wanted
  int32_t *ws_list;              // [pages] ranks of moves (compaction)
  unsigned long long *ws_bits;   // [runs, kPagesRun / 64] free pages (in the same place)
  int32_t *ws_runs;              // [runs] free pages, or pages in use, per run
};

// Caches small enough for one workgroup (pages_small.hip), whose counts and rows'
// scalars lie in LDS.  One launch against three or four, us on the device (in a
// graph): update of 24 rows of 256 entries, 4096 pages 8.0 | 11.4 (in place 7.9 | 7.5),
// 12288 pages 11.0 | 11.4 (10.2 | 7.7), of 128 rows of 40 12.6 | 11.7; fork of 24 rows
// of 256, 4096 pages 10.3 | 10.4, 12288 12.6 | 10.7, of 128 of 128 18.4 | 10.5;
// compaction of 128 rows of 128, 4096 pages 8.1 | 10.3, of 256 11.0 | 10.4.  A call by
// itself takes its launches' time on the host: 8.5 | 16.6 us.  The limits are where the times in a
// graph meet, but for the entries of an update, which are those of forks: none beyond them were measured.
constexpr int kSmallPages = 8192;
constexpr int kSmallRows = 512;          // of either table
constexpr int kSmallUpdateRows = 64;
constexpr int kSmallCompactPages = 4096; // (places and holes lie there, too)
constexpr int kSmallEntries = 6144;
constexpr int kSmallCompactEntries = 24576;

struct CopyPagesArgs {
  int32_t copies;
  const int32_t *src, *dst;
  const int32_t *count;          // or null
  char *pool[2];                 // keys, values
  int32_t layers;
  int64_t layer_bytes, page_bytes;
  int32_t pages;
};

// Offsets of the workspace.
struct PagesSpace {
  size_t list, runs, bytes;
};
inline PagesSpace pages_space(int32_t rows, int32_t pages) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  PagesSpace s;
  const size_t runs = ((size_t)pages + kPagesRun - 1) / kPagesRun;
  s.list = up((size_t)rows * 4);
  s.runs = s.list + up(runs * kPagesRun * 4);
  s.bytes = s.runs + up(runs * 4);
  return s;
}

hipError_t launch_update_pages(const PagesArgs &a, hipStream_t stream);
hipError_t launch_fork_pages(const PagesArgs &a, hipStream_t stream);
hipError_t launch_compact_pages(const PagesArgs &a, hipStream_t stream);
hipError_t launch_update_small(const PagesArgs &a, hipStream_t stream);
hipError_t launch_fork_small(const PagesArgs &a, hipStream_t stream);
hipError_t launch_compact_small(const PagesArgs &a, hipStream_t stream);
hipError_t launch_copy_pages(const CopyPagesArgs &a, hipStream_t stream);

}  // namespace adaserve
