// The pages of the cache on gfx950: tables, reference counts and contents.
//
// References are changed by atomic additions, whose sum has no order; free pages
// are handed out by rank -- the i-th free page in order of numbers to the i-th
// place in order of rows and entries -- so every result is a function of the inputs.
//
// Bound by their launches, each of which waits for the one before.  On the device, us: a step of
// 250 rows of 2048 entries, 100003 pages: references copied 2.1, rows 5.0, free pages 3.0,
// pages taken 8.0; 8000 pages compacted: counted 4.6, ranked 6.2, tables 3.9.
#include "device_common.h"
#include "pages.h"

namespace adaserve {

namespace {

constexpr int kThreads = kPagesThreads;
constexpr int kRunWords = kPagesRun / 64;

__device__ __forceinline__ bool in_pool(const PagesArgs &a, int32_t p) { return p >= 0 && p < a.pages; }

// Sum over a workgroup of 4 waves, in every thread; `parts` is free again after the next barrier.
__device__ __forceinline__ int32_t group_sum(int32_t x, int32_t *parts) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = x;
  __syncthreads();
  return parts[0] + parts[1] + parts[2] + parts[3];
}

// Lane i's pages p0 + i, p0 + 64 + i, ... of a run; `none` past the last one.
__device__ __forceinline__ void load_run(const int32_t *refs, int32_t pages, int64_t p0, int32_t none, int32_t (&x)[kRunWords]) {
#pragma unroll
  for (int i = 0; i < kRunWords; ++i) x[i] = refs[min(p0 + i * 64 + (threadIdx.x & 63), (int64_t)pages - 1)];
#pragma unroll
  for (int i = 0; i < kRunWords; ++i) {
    asm volatile("" : "+v"(x[i]));   // (loaded by now: no load goes behind a ballot)
    if (p0 + i * 64 + (threadIdx.x & 63) >= pages) x[i] = none;
  }
}

__global__ __launch_bounds__(kThreads) void copy_refs_kernel(PagesArgs a) {
  const int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (p < a.pages) a.new_refs[p] = a.refs[p];
}

// The entries [first, last) of a row that are to have pages.
__device__ __forceinline__ void wanted_range(const PagesArgs &a, int64_t c, int64_t need, int32_t &first, int32_t &last) {
  const int64_t ps = a.page_size;
  first = (int32_t)min((c + ps - 1) / ps, (int64_t)a.stride);
  last = need > 0 ? (int32_t)min((need + ps - 1) / ps, (int64_t)a.stride) : 0;
  if (last < first) last = first;
}

// A workgroup per row: entries that nothing sees any more go, the others are
// written as they are; and how many pages the row wants.
__global__ __launch_bounds__(kThreads) void update_drop_kernel(PagesArgs a) {
  __shared__ int32_t parts[4];
  const int r = blockIdx.x;
  const int64_t c = a.context_len[r], ps = a.page_size;
  const int32_t *in = a.table + (int64_t)r * a.stride;
  int32_t *out = a.new_table + (int64_t)r * a.stride;
  // entries [from, to) go
  int64_t from = 0, to = a.stride;
  if (c >= 0) {
    from = ((int64_t)a.sinks + ps - 1) / ps;
    to = a.window > 0 && c + 1 > a.window ? (c + 1 - a.window) / ps : 0;
  }
  int32_t first = 0, last = 0;
  if (a.need_len && c >= 0) wanted_range(a, c, a.need_len[r], first, last);
  const bool same = a.new_table == a.table;
  int32_t want = 0;
  for (int32_t e = threadIdx.x; e < a.stride; e += kThreads) {
    int32_t p = in[e];
    const bool has = in_pool(a, p);
    if (e >= from && e < to) {
      if (has) atomicAdd(&a.new_refs[p], -1);
      out[e] = -1;   // (never one of [first, last): the window ends before them)
    } else {
      if (!same) out[e] = p;
      want += e >= first && e < last && !has;
    }
  }
  if (!a.need_len) return;
  want = group_sum(want, parts);
  if (threadIdx.x == 0) a.ws_want[r] = want;
}

// Which pages are free, a bit each, and how many per run of kPagesRun; a wave per
// run.  (All of a lane's loads before the first ballot: a ballot per load takes one
// round trip each, 8.7 us for 8000 pages.)
__global__ __launch_bounds__(kThreads) void free_pages_kernel(PagesArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t run = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t p0 = run * kPagesRun;
  if (p0 >= a.pages) return;
  int32_t x[kRunWords];
  load_run(a.new_refs, a.pages, p0, 1, x);
  unsigned long long mine = 0;
  int32_t n = 0;
#pragma unroll
  for (int i = 0; i < kRunWords; ++i) {
    const unsigned long long word = __ballot(x[i] <= 0);
    n += __popcll(word);
    if (lane == i) mine = word;
  }
  if (lane < kRunWords) a.ws_bits[run * kRunWords + lane] = mine;
  if (lane == 0) a.ws_runs[run] = n;
}

// The sums of the runs' free pages before each, in LDS; all of them.  For a
// workgroup of 4 waves.
__device__ __forceinline__ int32_t sum_runs(const PagesArgs &a, int32_t *before) {
  __shared__ int64_t parts[2][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t runs = (a.pages + kPagesRun - 1) / kPagesRun;
  int64_t sum = 0;
  int flip = 0;
  for (int32_t i0 = 0; i0 < runs; i0 += kThreads, flip ^= 1) {
    const int32_t i = i0 + tid, x = i < runs ? a.ws_runs[i] : 0;
    int64_t at = wave_inclusive_scan(x);
    if (lane == 63) parts[flip][wave] = at;
    __syncthreads();
    at += sum;
    for (int w = 0; w < 4; ++w) {
      if (w < wave) at += parts[flip][w];
      sum += parts[flip][w];
    }
    if (i < runs) before[i] = (int32_t)(at - x);
  }
  __syncthreads();
  return (int32_t)sum;
}

// The rank-th free page.
__device__ __forceinline__ int32_t free_page(const PagesArgs &a, const int32_t *before, int32_t rank) {
  int32_t lo = 0, hi = (a.pages + kPagesRun - 1) / kPagesRun;   // the last run with before[run] <= rank that has any
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) / 2;
    if (before[mid] <= rank) lo = mid;
    else hi = mid;
  }
  rank -= before[lo];
  unsigned long long words[kRunWords];
#pragma unroll
  for (int i = 0; i < kRunWords; ++i) words[i] = a.ws_bits[(int64_t)lo * kRunWords + i];
  unsigned long long word = 0;
  int32_t page = lo * kPagesRun;
  bool found = false;
#pragma unroll
  for (int i = 0; i < kRunWords; ++i) {
    const int32_t n = __popcll(words[i]);
    if (!found && rank < n) {
      found = true;
      word = words[i];
      page += i * 64;
    }
    if (!found) rank -= n;
  }
#pragma unroll
  for (int half = 32; half >= 1; half /= 2) {
    const int32_t n = __popcll(word & ((1ull << half) - 1));
    if (rank >= n) {
      rank -= n;
      word >>= half;
      page += half;
    }
  }
  return page;
}

// What rows [0, n) want, for a workgroup of 4 waves.
__device__ __forceinline__ int64_t wanted_before(const PagesArgs &a, int32_t n, int64_t *parts) {
  int64_t sum = 0;
  for (int32_t i = threadIdx.x; i < n; i += kThreads) sum += a.ws_want[i];
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = sum;
  __syncthreads();
  return parts[0] + parts[1] + parts[2] + parts[3];
}

// A workgroup per row: its entries without a page get the row's share of the free
// ones, in order; and how far the row reaches.
__global__ __launch_bounds__(kThreads) void update_assign_kernel(PagesArgs a) {
  extern __shared__ int32_t before[];
  __shared__ int32_t parts[2][4];
  __shared__ int64_t sums[4];
  __shared__ int32_t missing;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t c = a.context_len[r], need = a.need_len[r], ps = a.page_size;
  if (c < 0) {
    if (tid == 0) a.capacity[r] = 0;
    return;
  }
  int32_t first, last, got = 0;
  wanted_range(a, c, need, first, last);
  if (tid == 0) missing = a.stride;
  int32_t *row = a.new_table + (int64_t)r * a.stride;
  int64_t rank0 = 0;
  if (a.ws_want[r] > 0) {
    rank0 = wanted_before(a, r, sums);
    got = sum_runs(a, before);
  }
  __syncthreads();
  // (an entry that holds some of the c tokens is looked at, and left as it is)
  const int32_t begin = (int32_t)min(c / ps, (int64_t)a.stride);
  int flip = 0;
  for (int32_t e0 = begin; e0 < last; e0 += kThreads, flip ^= 1) {
    const int32_t e = e0 + tid;
    const bool without = e < last && !in_pool(a, row[e]);
    const unsigned long long wants = __ballot(without && e >= first);
    if (lane == 0) parts[flip][wave] = __popcll(wants);
    __syncthreads();
    int64_t rank = rank0 + __popcll(wants & ((1ull << lane) - 1));
    for (int w = 0; w < 4; ++w) {
      if (w < wave) rank += parts[flip][w];
      rank0 += parts[flip][w];
    }
    if (without) {
      if (e >= first && rank < got) {
        const int32_t p = free_page(a, before, (int32_t)rank);
        row[e] = p;
        a.new_refs[p] = 1;
      } else {
        atomicMin(&missing, e);
      }
    }
  }
  __syncthreads();
  if (tid == 0) {
    // the first position from c on without a page: in the entry that lacks one, or past the row
    const int64_t at = max(c, (int64_t)missing * ps);
    a.capacity[r] = (int32_t)(need > c && at < need ? at : need);
  }
}

// Workgroups 0 .. sources - 1: an old row's references, by how many take it.
// The others: the new rows.
__global__ __launch_bounds__(kThreads) void fork_rows_kernel(PagesArgs a) {
  __shared__ int32_t parts[4];
  const int tid = threadIdx.x;
  const int64_t ps = a.page_size;
  const bool old = (int32_t)blockIdx.x < a.sources;
  const int32_t r = old ? -1 : (int32_t)blockIdx.x - a.sources;
  const int32_t s = old ? (int32_t)blockIdx.x : a.source[r];
  // the new rows before r (of an old row: all) that take s
  const bool any = s >= 0 && s < a.sources;
  int32_t takers = 0;
  if (any)
    for (int32_t i = tid; i < (old ? a.rows : r); i += kThreads) takers += a.source[i] == s;
  takers = group_sum(takers, parts);
  const int64_t c = any ? min(max((int64_t)a.context_len[s], (int64_t)0), (int64_t)a.stride * ps) : 0;
  const int32_t whole = (int32_t)(c / ps);
  const int32_t *in = a.table + (int64_t)(any ? s : 0) * a.stride;
  if (old) {
    for (int32_t e = tid; e < a.stride; e += kThreads) {
      const int32_t p = in[e], more = e < whole ? takers - 1 : takers > 0 ? 0 : -1;
      if (in_pool(a, p) && more != 0) atomicAdd(&a.new_refs[p], more);
    }
    return;
  }
  int32_t *out = a.new_table + (int64_t)r * a.stride;
  const int32_t upto = !any ? 0 : takers == 0 ? a.stride : whole;   // entries that are the old row's
  for (int32_t e = tid; e < a.stride; e += kThreads) out[e] = e < upto ? in[e] : -1;
  if (tid == 0) {
    a.ws_want[r] = any && takers > 0 && c % ps != 0 && in_pool(a, in[whole]);
    a.new_len[r] = (int32_t)c;
    a.copy_src[r] = a.copy_dst[r] = -1;
  }
}

// The copies' pages, a thread per row.
__global__ __launch_bounds__(kThreads) void fork_assign_kernel(PagesArgs a) {
  extern __shared__ int32_t before[];
  __shared__ int32_t parts[4];
  __shared__ int64_t sums[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t r0 = blockIdx.x * kThreads, r = r0 + tid;
  const bool want = r < a.rows && a.ws_want[r] != 0;
  const unsigned long long wants = __ballot(want);
  if (lane == 0) parts[wave] = __popcll(wants);
  int64_t rank = wanted_before(a, r0, sums) + __popcll(wants & ((1ull << lane) - 1));
  for (int w = 0; w < wave; ++w) rank += parts[w];
  const int32_t got = sum_runs(a, before);
  if (!want) return;
  const int32_t whole = a.new_len[r] / a.page_size;
  if (rank < got) {
    const int32_t p = free_page(a, before, (int32_t)rank);
    a.copy_src[r] = a.table[(int64_t)a.source[r] * a.stride + whole];
    a.copy_dst[r] = p;
    a.new_table[(int64_t)r * a.stride + whole] = p;
    a.new_refs[p] = 1;
  } else {
    a.new_len[r] = whole * a.page_size;
  }
}

// Pages in use per run of kPagesRun, a wave each.
__global__ __launch_bounds__(kThreads) void compact_count_kernel(PagesArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t run = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t p0 = run * kPagesRun;
  if (p0 >= a.pages) return;
  int32_t x[kRunWords], n = 0;
  load_run(a.refs, a.pages, p0, 0, x);
#pragma unroll
  for (int i = 0; i < kRunWords; ++i) n += __popcll(__ballot(x[i] > 0));
  if (lane == 0) a.ws_runs[run] = n;
}

// Ranks: of the pages in use from U on, and of the free places below U.
// ws_list: a move's rank, -1 of a page that stays, -2 of one that is free.
__global__ __launch_bounds__(kThreads) void compact_rank_kernel(PagesArgs a) {
  __shared__ int32_t parts[3][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t runs = (a.pages + kPagesRun - 1) / kPagesRun;
  const int32_t run0 = blockIdx.x * 4, run = run0 + wave;
  int32_t x[kRunWords];
  if (run < runs) load_run(a.refs, a.pages, (int64_t)run * kPagesRun, 0, x);
  int32_t all = 0, before = 0;
  for (int32_t i = tid; i < runs; i += kThreads) {
    const int32_t n = a.ws_runs[i];
    all += n;
    if (i < run0) before += n;
  }
  const int32_t used = group_sum(all, parts[0]);
  before = group_sum(before, parts[1]);
  // pages in use below U: whole runs, and the one that U lies in
  int32_t front = 0;
  for (int32_t i = tid; i < used / kPagesRun; i += kThreads) front += a.ws_runs[i];
  for (int32_t p = used / kPagesRun * kPagesRun + tid; p < used; p += kThreads) front += a.refs[p] > 0;
  front = group_sum(front, parts[2]);
  const int32_t moves = used - front;
  if (blockIdx.x == 0 && tid == 0) {
    a.counts[0] = used;
    a.counts[1] = moves;
  }
  if (run >= runs) return;
  for (int32_t i = run0; i < run; ++i) before += a.ws_runs[i];
  const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < kRunWords; ++i) {
    const int32_t p = run * kPagesRun + i * 64 + lane;
    const bool is_used = x[i] > 0;
    const unsigned long long mask = __ballot(is_used);
    const int32_t rank = before + __popcll(mask & below);   // pages in use before p
    before += __popcll(mask);
    if (p >= a.pages) continue;
    int32_t what = is_used ? -1 : -2;
    if (is_used && p >= used) {
      what = rank - front;
      a.copy_src[what] = p;
    } else {
      a.new_place[p] = is_used ? p : -1;
      if (!is_used && p < used) a.copy_dst[p - rank] = p;
    }
    a.ws_list[p] = what;
    if (p >= moves) a.copy_src[p] = a.copy_dst[p] = -1;
  }
}

// What follows from the moves: places and references, and the tables' entries.
__global__ __launch_bounds__(kThreads) void compact_apply_kernel(PagesArgs a, int64_t page_blocks) {
  if ((int64_t)blockIdx.x < page_blocks) {
    const int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (p >= a.pages) return;
    const int32_t what = a.ws_list[p], used = a.counts[0];
    if (what >= 0) {
      const int32_t n = a.refs[p], to = a.copy_dst[what];
      a.new_place[p] = to;
      a.new_refs[to] = n;
      a.new_refs[p] = 0;
    } else if (p >= used) {
      a.new_refs[p] = 0;
    } else if (what == -1 && a.new_refs != a.refs) {
      a.new_refs[p] = a.refs[p];
    }
    return;
  }
  const int64_t i = ((int64_t)blockIdx.x - page_blocks) * kThreads + threadIdx.x;
  if (i >= (int64_t)a.rows * a.stride) return;
  int32_t p = a.table[i];
  if (in_pool(a, p)) {
    const int32_t what = a.ws_list[p];
    p = what >= 0 ? a.copy_dst[what] : what == -1 ? p : -1;
  }
  a.new_table[i] = p;
}

// A workgroup copies pieces of 16 KB, key pools and value pools of all layers.  128 MB of
// pages of 32 KB in 43 us, called again and again on one state.
constexpr int kPiece = 16384;
__global__ __launch_bounds__(kThreads) void copy_pages_kernel(CopyPagesArgs a, int32_t pieces) {
  constexpr int kVec = kPiece / 16 / kThreads;
  const int64_t copies = a.count ? min(max(*a.count, 0), a.copies) : a.copies;
  const int64_t per_copy = (int64_t)a.layers * 2 * pieces;
  for (int64_t item = blockIdx.x; item < copies * per_copy; item += gridDim.x) {
    const int64_t i = item / per_copy;
    int64_t rest = item - i * per_copy;
    const int32_t from = a.src[i], to = a.dst[i];
    if (from < 0 || from >= a.pages || to < 0 || to >= a.pages || from == to) continue;
    const int32_t piece = (int32_t)(rest % pieces);
    rest /= pieces;
    char *pool = a.pool[rest & 1] + (rest >> 1) * a.layer_bytes;
    const char *s = pool + from * a.page_bytes;
    char *d = pool + to * a.page_bytes;
    const int64_t at = (int64_t)piece * kPiece + threadIdx.x * 16;
    u32x4 x[kVec];
#pragma unroll
    for (int v = 0; v < kVec; ++v)
      if (at + v * kThreads * 16 < a.page_bytes) x[v] = *(const u32x4 *)(s + at + v * kThreads * 16);
#pragma unroll
    for (int v = 0; v < kVec; ++v)
      if (at + v * kThreads * 16 < a.page_bytes) *(u32x4 *)(d + at + v * kThreads * 16) = x[v];
  }
}

unsigned blocks_of(int64_t n, int64_t per) { return (unsigned)((n + per - 1) / per); }

hipError_t copy_refs(const PagesArgs &a, hipStream_t stream) {
  if (a.new_refs == a.refs || a.pages == 0) return hipSuccess;
  hipLaunchKernelGGL(copy_refs_kernel, dim3(blocks_of(a.pages, kThreads)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

// Whether one workgroup is sooner done than several launches.
bool small(const PagesArgs &a, int32_t rows, int64_t entries, int32_t pages) {
  const int32_t most = a.rows > a.sources ? a.rows : a.sources;
  return a.pages <= pages && most <= rows && (int64_t)most * a.stride <= entries;
}

hipError_t find_free(const PagesArgs &a, hipStream_t stream) {
  if (a.pages == 0) return hipSuccess;
  hipLaunchKernelGGL(free_pages_kernel, dim3(blocks_of(a.pages, 4 * kPagesRun)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

// LDS of the kernels that hand out free pages: at most 32 KB, of 2^23 pages.
unsigned run_bytes(const PagesArgs &a) { return blocks_of(a.pages, kPagesRun) * 4; }

}  // namespace

hipError_t launch_update_pages(const PagesArgs &a, hipStream_t stream) {
  if (small(a, kSmallUpdateRows, kSmallEntries, kSmallPages)) return launch_update_small(a, stream);
  hipError_t e = copy_refs(a, stream);
  if (e != hipSuccess || a.rows == 0) return e;
  hipLaunchKernelGGL(update_drop_kernel, dim3((unsigned)a.rows), dim3(kThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || !a.need_len) return e;
  e = find_free(a, stream);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(update_assign_kernel, dim3((unsigned)a.rows), dim3(kThreads), run_bytes(a), stream, a);
  return hipGetLastError();
}

hipError_t launch_fork_pages(const PagesArgs &a, hipStream_t stream) {
  if (small(a, kSmallRows, kSmallEntries, kSmallPages)) return launch_fork_small(a, stream);
  hipError_t e = copy_refs(a, stream);
  if (e != hipSuccess || a.rows + a.sources == 0) return e;
  hipLaunchKernelGGL(fork_rows_kernel, dim3((unsigned)(a.sources + a.rows)), dim3(kThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.rows == 0) return e;
  e = find_free(a, stream);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fork_assign_kernel, dim3(blocks_of(a.rows, kThreads)), dim3(kThreads), run_bytes(a), stream, a);
  return hipGetLastError();
}

hipError_t launch_compact_pages(const PagesArgs &a, hipStream_t stream) {
  if (small(a, kSmallRows, kSmallCompactEntries, kSmallCompactPages)) return launch_compact_small(a, stream);
  const unsigned runs = blocks_of(a.pages, 4 * kPagesRun);
  if (runs > 0) hipLaunchKernelGGL(compact_count_kernel, dim3(runs), dim3(kThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_rank_kernel, dim3(runs > 0 ? runs : 1), dim3(kThreads), 0, stream, a);   // (the counts of no page)
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t page_blocks = blocks_of(a.pages, kThreads);
  const int64_t grid = page_blocks + blocks_of((int64_t)a.rows * a.stride, kThreads);
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL(compact_apply_kernel, dim3((unsigned)grid), dim3(kThreads), 0, stream, a, page_blocks);
  return hipGetLastError();
}

hipError_t launch_copy_pages(const CopyPagesArgs &a, hipStream_t stream) {
  const int32_t pieces = (int32_t)((a.page_bytes + kPiece - 1) / kPiece);
  const int64_t items = (int64_t)a.copies * a.layers * 2 * pieces;
  if (items == 0) return hipSuccess;
  const unsigned grid = (unsigned)(items < 2048 ? items : 2048);
  hipLaunchKernelGGL(copy_pages_kernel, dim3(grid), dim3(kThreads), 0, stream, a, pieces);
  return hipGetLastError();
}

}  // namespace adaserve
