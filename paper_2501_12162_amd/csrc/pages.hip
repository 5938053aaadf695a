// The pages of the cache on gfx950: tables, reference counts and contents.
//
// References are changed by atomic additions, whose sum has no order; free pages
// are handed out by rank -- the i-th free page in order of numbers to the i-th
// place in order of rows and entries -- so every result is a function of the inputs.
#include "device_common.h"
#include "pages.h"

namespace adaserve {

namespace {

constexpr int kThreads = kPagesThreads;
constexpr int kTakeThreads = 1024;
constexpr int kTakeWaves = kTakeThreads / 64;

__device__ __forceinline__ bool in_pool(const PagesArgs &a, int32_t p) { return p >= 0 && p < a.pages; }

// Sum over a workgroup of 4 waves, in every thread; `parts` is free again after the next barrier.
__device__ __forceinline__ int32_t group_sum(int32_t x, int32_t *parts) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = x;
  __syncthreads();
  return parts[0] + parts[1] + parts[2] + parts[3];
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
      out[e] = -1;
      want += e >= first && e < last;
    } else {
      if (!same) out[e] = p;
      want += e >= first && e < last && !has;
    }
  }
  if (!a.need_len) return;
  want = group_sum(want, parts);
  if (threadIdx.x == 0) a.ws_want[r] = want;
}

// One workgroup: the sums of the rows' wants before each row, and the list of
// as many free pages as all want, or as there are; then `after`.
template <class After>
__device__ __forceinline__ void take_pages(const PagesArgs &a, After after) {
  __shared__ int64_t parts[2][kTakeWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const unsigned long long below = (1ull << lane) - 1;
  // exclusive sum over the workgroup, and the total (of 2^10 wants of up to 2^24)
  auto scan = [&](int64_t x, int64_t *p, int64_t &total) {
    int64_t upto = wave_inclusive_scan(x);
    if (lane == 63) p[wave] = upto;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kTakeWaves; ++w) {
      if (w < wave) upto += p[w];
      total += p[w];
    }
    return upto - x;
  };
  int32_t want = 0;   // (wants beyond the pages that there are need not be told apart)
  int flip = 0;
  for (int32_t r0 = 0; r0 < a.rows; r0 += kTakeThreads, flip ^= 1) {
    const int32_t r = r0 + tid;
    int64_t total;
    const int64_t x = r < a.rows ? min(a.ws_want[r], a.pages) : 0;
    const int64_t at = scan(x, parts[flip], total);
    if (r < a.rows) a.ws_want[r] = (int32_t)min(want + at, (int64_t)a.pages);
    want = (int32_t)min(want + total, (int64_t)a.pages);
  }
  int32_t got = 0;
  constexpr int kPer = kPagesRun / 64;
  for (int64_t base = 0; base < a.pages && got < want; base += kTakeWaves * kPagesRun, flip ^= 1) {
    const int64_t p0 = base + (int64_t)wave * kPagesRun + lane;
    unsigned long long free[kPer];
    int32_t n = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int64_t p = p0 + i * 64;
      free[i] = __ballot(p < a.pages && a.new_refs[min(p, (int64_t)a.pages - 1)] <= 0);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) n += __popcll(free[i]);
    if (lane == 0) parts[flip][wave] = n;
    __syncthreads();
    int32_t at = got, all = 0;
    for (int w = 0; w < kTakeWaves; ++w) {
      const int32_t x = (int32_t)parts[flip][w];
      if (w < wave) at += x;
      all += x;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int32_t rank = at + __popcll(free[i] & below);
      if (((free[i] >> lane) & 1) && rank < want) {
        a.ws_list[rank] = (int32_t)(p0 + i * 64);
        a.new_refs[p0 + i * 64] = 1;
      }
      at += __popcll(free[i]);
    }
    got = min(want, got + all);
  }
  if (tid == 0) a.ws_total[0] = got;
  __syncthreads();   // the list and the sums, for this workgroup's own reads
  after(got);
}

__global__ __launch_bounds__(kTakeThreads) void update_take_kernel(PagesArgs a) {
  take_pages(a, [](int32_t) {});
}

// A workgroup per row: its entries without a page get the row's share of the
// list, in order; and how far the row reaches.
__global__ __launch_bounds__(kThreads) void update_assign_kernel(PagesArgs a) {
  __shared__ int32_t parts[2][4];
  __shared__ int32_t missing;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t c = a.context_len[r], need = a.need_len[r], ps = a.page_size;
  if (c < 0) {
    if (tid == 0) a.capacity[r] = 0;
    return;
  }
  int32_t first, last;
  wanted_range(a, c, need, first, last);
  if (tid == 0) missing = a.stride;
  int32_t *row = a.new_table + (int64_t)r * a.stride;
  int32_t rank0 = a.ws_want[r];
  const int32_t got = a.ws_total[0];
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
    int32_t rank = rank0 + __popcll(wants & ((1ull << lane) - 1));
    for (int w = 0; w < 4; ++w) {
      if (w < wave) rank += parts[flip][w];
      rank0 += parts[flip][w];
    }
    if (without) {
      if (e >= first && rank < got) row[e] = a.ws_list[rank];
      else atomicMin(&missing, e);
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

// The copies' pages.  (After the launch before, ws_want tells who wants one; the
// sums that take_pages leaves there tell it by their steps.)
__global__ __launch_bounds__(kTakeThreads) void fork_take_kernel(PagesArgs a) {
  take_pages(a, [&](int32_t got) {
    for (int32_t r = threadIdx.x; r < a.rows; r += kTakeThreads) {
      const int32_t s = a.source[r];
      if (s < 0 || s >= a.sources) continue;
      const int64_t c = a.new_len[r];
      const int32_t whole = (int32_t)(c / a.page_size);
      if (c % a.page_size == 0) continue;
      int32_t *entry = a.new_table + (int64_t)r * a.stride + whole;
      const int32_t from = a.table[(int64_t)s * a.stride + whole], rank = a.ws_want[r];
      if (*entry == from || !in_pool(a, from)) continue;   // (its own, as the first that takes it)
      if (rank < got) {
        a.copy_src[r] = from;
        a.copy_dst[r] = *entry = a.ws_list[rank];
      } else {
        a.new_len[r] = whole * a.page_size;
      }
    }
  });
}

// Pages in use per run of kPagesRun, a wave each.
__global__ __launch_bounds__(kThreads) void compact_count_kernel(PagesArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t run = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t p0 = run * kPagesRun;
  if (p0 >= a.pages) return;
  int32_t n = 0;
#pragma unroll
  for (int i = 0; i < kPagesRun / 64; ++i) {
    const int64_t p = p0 + i * 64 + lane;
    n += __popcll(__ballot(p < a.pages && a.refs[min(p, (int64_t)a.pages - 1)] > 0));
  }
  if (lane == 0) a.ws_runs[run] = n;
}

// Ranks: of the pages in use from U on, and of the free places below U.
// ws_list: a move's rank, -1 of a page that stays, -2 of one that is free.
__global__ __launch_bounds__(kThreads) void compact_rank_kernel(PagesArgs a) {
  __shared__ int32_t parts[3][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t runs = (a.pages + kPagesRun - 1) / kPagesRun;
  const int32_t run0 = blockIdx.x * 4;
  int32_t all = 0, before = 0;
  for (int32_t i = tid; i < runs; i += kThreads) {
    const int32_t x = a.ws_runs[i];
    all += x;
    if (i < run0) before += x;
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
  const int32_t run = run0 + wave;
  if (run >= runs) return;
  for (int32_t i = run0; i < run; ++i) before += a.ws_runs[i];
  const unsigned long long below = (1ull << lane) - 1;
#pragma unroll 4
  for (int i = 0; i < kPagesRun / 64; ++i) {
    const int32_t p = run * kPagesRun + i * 64 + lane;
    const bool is_used = p < a.pages && a.refs[min(p, a.pages - 1)] > 0;
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

// A workgroup copies pieces of 16 KB, key pools and value pools of all layers.
constexpr int kPiece = 16384;
__global__ __launch_bounds__(kThreads) void copy_pages_kernel(CopyPagesArgs a, int64_t items, int32_t pieces) {
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

}  // namespace

hipError_t launch_update_pages(const PagesArgs &a, hipStream_t stream) {
  hipError_t e = copy_refs(a, stream);
  if (e != hipSuccess || a.rows == 0) return e;
  hipLaunchKernelGGL(update_drop_kernel, dim3((unsigned)a.rows), dim3(kThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || !a.need_len) return e;
  hipLaunchKernelGGL(update_take_kernel, dim3(1), dim3(kTakeThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(update_assign_kernel, dim3((unsigned)a.rows), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_fork_pages(const PagesArgs &a, hipStream_t stream) {
  hipError_t e = copy_refs(a, stream);
  if (e != hipSuccess || a.rows + a.sources == 0) return e;
  hipLaunchKernelGGL(fork_rows_kernel, dim3((unsigned)(a.sources + a.rows)), dim3(kThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.rows == 0) return e;
  hipLaunchKernelGGL(fork_take_kernel, dim3(1), dim3(kTakeThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_compact_pages(const PagesArgs &a, hipStream_t stream) {
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
  hipLaunchKernelGGL(copy_pages_kernel, dim3(grid), dim3(kThreads), 0, stream, a, items, pieces);
  return hipGetLastError();
}

}  // namespace adaserve
