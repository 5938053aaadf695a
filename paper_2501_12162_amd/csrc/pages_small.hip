// The pages of a small cache on gfx950, one workgroup and one launch a call: the
// reference counts lie in LDS from the beginning to the end, so the steps of a call
// follow each other by barriers instead of launches.  Same results as pages.hip.  On
// the device: a step of 24 rows of 256 entries, 4096 pages 8.0 us; 128 rows of 40 entries
// forked to 128, 3200 pages 9.4; 600 pages of 8 rows of 60 compacted 3.0.
#include "device_common.h"
#include "pages.h"

namespace adaserve {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kMostWords = kSmallPages / 64;
constexpr int kWordsPerLane = (kMostWords + 63) / 64;
static_assert(kSmallRows <= kThreads, "a thread per row");

__device__ __forceinline__ bool in_pool(const PagesArgs &a, int32_t p) { return p >= 0 && p < a.pages; }

__device__ __forceinline__ void load_refs(const PagesArgs &a, int32_t *refs) {
  for (int32_t p = threadIdx.x; p < a.pages; p += kThreads) refs[p] = a.refs[p];
}

__device__ __forceinline__ void store_refs(const PagesArgs &a, const int32_t *refs) {
  for (int32_t p = threadIdx.x; p < a.pages; p += kThreads) a.new_refs[p] = refs[p];
}

// Pages as bits, and how many there are in the words before each.
struct PageBits {
  unsigned long long word[kMostWords];
  int32_t before[kMostWords + 1];   // the last one: all of them

  // Of the pages with which(refs[p]); the first wave adds up.  Barriers around it are the caller's.
  template <class Which>
  __device__ __forceinline__ void set(const int32_t *refs, int32_t pages, Which which) {
    const int lane = threadIdx.x & 63;
    const int32_t words = (pages + 63) / 64;
    for (int32_t i = threadIdx.x >> 6; i < words; i += kWaves) {
      const int32_t p = i * 64 + lane;
      const unsigned long long w = __ballot(p < pages && which(refs[min(p, pages - 1)]));
      if (lane == 0) word[i] = w;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
      int32_t n[kWordsPerLane], sum = 0;
#pragma unroll
      for (int k = 0; k < kWordsPerLane; ++k) {
        const int32_t i = lane * kWordsPerLane + k;
        n[k] = i < words ? __popcll(word[i]) : 0;
        sum += n[k];
      }
      int32_t upto = (int32_t)wave_inclusive_scan(sum);
      if (lane == 63) before[kMostWords] = upto;
#pragma unroll
      for (int k = kWordsPerLane - 1; k >= 0; --k) {
        upto -= n[k];
        if (lane * kWordsPerLane + k < words) before[lane * kWordsPerLane + k] = upto;
      }
    }
    __syncthreads();
  }
  __device__ __forceinline__ int32_t all() const { return before[kMostWords]; }
  __device__ __forceinline__ int32_t rank(int32_t p) const {
    return before[p / 64] + __popcll(word[p / 64] & ((1ull << (p % 64)) - 1));
  }
  // The rank-th page (rank < all()).
  __device__ __forceinline__ int32_t at(int32_t rank, int32_t pages) const {
    int32_t lo = 0, hi = (pages + 63) / 64;
    while (hi - lo > 1) {
      const int32_t mid = (lo + hi) / 2;
      if (before[mid] <= rank) lo = mid;
      else hi = mid;
    }
    rank -= before[lo];
    unsigned long long w = word[lo];
    int32_t p = lo * 64;
#pragma unroll
    for (int half = 32; half >= 1; half /= 2) {
      const int32_t n = __popcll(w & ((1ull << half) - 1));
      if (rank >= n) {
        rank -= n;
        w >>= half;
        p += half;
      }
    }
    return p;
  }
};

// f(row, entry, value) of all entries of a table, a thread's next four loaded together.
template <class F>
__device__ __forceinline__ void for_entries(const int32_t *table, int32_t rows, int32_t stride, F f) {
  constexpr int kAtOnce = 4;
  const uint32_t n = (uint32_t)rows * (uint32_t)stride, wide = (uint32_t)stride;
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kAtOnce * kThreads) {
    int32_t x[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) x[k] = table[min(i0 + k * kThreads, n - 1)];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const uint32_t i = i0 + k * kThreads, r = i / wide;
      if (i < n) f((int32_t)r, (int32_t)(i - r * wide), x[k]);
    }
  }
}

// want[r] becomes the sum of the rows before r; by the first wave, up to its own barrier.
__device__ __forceinline__ void sum_wants(int32_t *want, int32_t rows) {
  if (threadIdx.x < 64) {
    int64_t sum = 0;
    for (int32_t r0 = 0; r0 < rows; r0 += 64) {
      const int32_t r = r0 + threadIdx.x, x = r < rows ? want[r] : 0;
      const int64_t upto = wave_inclusive_scan(x);
      if (r < rows) want[r] = (int32_t)(sum + upto - x);
      sum += __shfl(upto, 63, 64);
    }
  }
  __syncthreads();
}

__global__ __launch_bounds__(kThreads) void update_small_kernel(PagesArgs a) {
  extern __shared__ int32_t refs[];
  __shared__ PageBits bits;
  __shared__ int32_t want[kSmallUpdateRows], from[kSmallUpdateRows], to[kSmallUpdateRows], first[kSmallUpdateRows],
      last[kSmallUpdateRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t ps = a.page_size;
  load_refs(a, refs);
  if (tid < a.rows) {
    // entries [from, to) go, [first, last) are to have pages
    const int32_t c = a.context_len[tid];
    int32_t f = 0, l = 0;
    from[tid] = c < 0 ? 0 : (int32_t)(((int64_t)a.sinks + ps - 1) / ps);
    to[tid] = c < 0 ? a.stride : a.window > 0 && c >= a.window ? (c - a.window + 1) / ps : 0;
    if (a.need_len && c >= 0) {
      const int32_t need = a.need_len[tid];
      f = min((int32_t)(((int64_t)c + ps - 1) / ps), a.stride);
      l = need > 0 ? max(f, min((int32_t)(((int64_t)need + ps - 1) / ps), a.stride)) : f;
    }
    first[tid] = f;
    last[tid] = l;
    want[tid] = 0;
  }
  __syncthreads();
  const bool same = a.new_table == a.table;
  for_entries(a.table, a.rows, a.stride, [&](int32_t r, int32_t e, int32_t p) {
    const bool has = in_pool(a, p), gone = e >= from[r] && e < to[r];
    if (gone && has) atomicAdd(&refs[p], -1);
    if (gone || !same) a.new_table[(int64_t)r * a.stride + e] = gone ? -1 : p;
    if (e >= first[r] && e < last[r] && !has) atomicAdd(&want[r], 1);   // (none of them is gone: the window ends before)
  });
  __syncthreads();
  if (a.need_len) {
    bits.set(refs, a.pages, [](int32_t n) { return n <= 0; });
    sum_wants(want, a.rows);
    const int32_t got = a.pages > 0 ? bits.all() : 0;
    for (int32_t r = wave; r < a.rows; r += kWaves) {
      const int32_t c = a.context_len[r], need = a.need_len[r];
      if (c < 0) {
        if (lane == 0) a.capacity[r] = 0;
        continue;
      }
      int32_t missing = a.stride, rank0 = want[r];
      // (from the entry that holds some of the c tokens on nothing has gone: the window ends before it)
      for (int32_t e0 = min(c / ps, a.stride); e0 < last[r]; e0 += 64) {
        const int32_t e = e0 + lane;
        const bool without = e < last[r] && !in_pool(a, a.table[(int64_t)r * a.stride + e]);
        const unsigned long long wants = __ballot(without && e >= first[r]);
        const int32_t rank = rank0 + __popcll(wants & ((1ull << lane) - 1));
        const bool taken = without && e >= first[r] && rank < got;
        if (taken) {
          const int32_t p = bits.at(rank, a.pages);
          refs[p] = 1;
          a.new_table[(int64_t)r * a.stride + e] = p;
        }
        const unsigned long long lacks = __ballot(without && !taken);
        if (lacks && missing == a.stride) missing = e0 + __ffsll(lacks) - 1;
        rank0 += __popcll(wants);
      }
      if (lane == 0) {
        const int64_t at = max((int64_t)c, (int64_t)missing * ps);
        a.capacity[r] = (int32_t)(need > c && at < need ? at : need);
      }
    }
    __syncthreads();
  }
  store_refs(a, refs);
}

__global__ __launch_bounds__(kThreads) void fork_small_kernel(PagesArgs a) {
  extern __shared__ int32_t refs[];
  __shared__ PageBits bits;
  __shared__ int32_t want[kSmallRows], takers[kSmallRows], first[kSmallRows], tokens[kSmallRows], source[kSmallRows];
  const int tid = threadIdx.x;
  const int32_t ps = a.page_size;
  load_refs(a, refs);
  if (tid < a.sources) {
    takers[tid] = 0;
    first[tid] = a.rows;
    tokens[tid] = (int32_t)min((int64_t)max(a.context_len[tid], 0), (int64_t)a.stride * ps);
  }
  int32_t mine = tid < a.rows ? a.source[tid] : -1;   // (a thread per row, too)
  if (mine < 0 || mine >= a.sources) mine = -1;
  if (tid < a.rows) source[tid] = mine;
  __syncthreads();
  if (mine >= 0) {
    atomicAdd(&takers[mine], 1);
    atomicMin(&first[mine], tid);
  }
  __syncthreads();
  for_entries(a.table, a.sources, a.stride, [&](int32_t s, int32_t e, int32_t p) {
    const int32_t more = e < tokens[s] / ps ? takers[s] - 1 : takers[s] > 0 ? 0 : -1;
    if (in_pool(a, p) && more != 0) atomicAdd(&refs[p], more);
  });
  // a row's own entry of the partly filled page, where it needs one, is written at the end
  int32_t c = 0, from = -1;
  bool copy = false;
  if (mine >= 0) {
    c = tokens[mine];
    if (c % ps != 0 && first[mine] != tid) from = a.table[(int64_t)mine * a.stride + c / ps];
    copy = in_pool(a, from);
  }
  if (tid < a.rows) want[tid] = copy;
  __syncthreads();
  const uint32_t n = (uint32_t)a.rows * (uint32_t)a.stride, wide = (uint32_t)a.stride;
#pragma unroll 4
  for (uint32_t i = tid; i < n; i += kThreads) {
    const int32_t r = (int32_t)(i / wide), e = (int32_t)(i - r * wide), s = source[r];
    const int32_t whole = s >= 0 ? tokens[s] / ps : 0, upto = s < 0 ? 0 : first[s] == r ? a.stride : whole;
    if (!(want[r] && e == whole)) a.new_table[i] = e < upto ? a.table[(int64_t)s * a.stride + e] : -1;   // (no old row: no read)
  }
  __syncthreads();
  bits.set(refs, a.pages, [](int32_t n) { return n <= 0; });
  sum_wants(want, a.rows);
  if (tid < a.rows) {
    int32_t page = -1;
    if (copy && want[tid] < bits.all()) {
      page = bits.at(want[tid], a.pages);
      refs[page] = 1;
    }
    if (copy) a.new_table[(int64_t)tid * a.stride + c / ps] = page;
    a.copy_src[tid] = page >= 0 ? from : -1;
    a.copy_dst[tid] = page;
    a.new_len[tid] = copy && page < 0 ? c / ps * ps : c;
  }
  __syncthreads();
  store_refs(a, refs);
}

__global__ __launch_bounds__(kThreads) void compact_small_kernel(PagesArgs a) {
  extern __shared__ int32_t refs[];
  int32_t *const place = refs + a.pages, *const holes = place + a.pages;
  __shared__ PageBits bits;
  const int tid = threadIdx.x;
  load_refs(a, refs);
  __syncthreads();
  bits.set(refs, a.pages, [](int32_t n) { return n > 0; });
  const int32_t used = a.pages > 0 ? bits.all() : 0;
  const int32_t front = used < a.pages ? bits.rank(used) : used, moves = used - front;   // in use below U
  for (int32_t p = tid; p < used; p += kThreads)
    if (refs[p] <= 0) holes[p - bits.rank(p)] = p;
  __syncthreads();
  for (int32_t p = tid; p < a.pages; p += kThreads) {
    int32_t to = refs[p] > 0 ? p : -1;
    if (to >= used) {
      const int32_t i = bits.rank(p) - front;
      to = holes[i];
      a.copy_src[i] = p;
      a.copy_dst[i] = to;
      a.new_refs[to] = refs[p];
    } else if (to >= 0) {
      a.new_refs[p] = refs[p];
    }
    if (p >= used) a.new_refs[p] = 0;
    place[p] = to;
    a.new_place[p] = to;
    if (p >= moves) a.copy_src[p] = a.copy_dst[p] = -1;
  }
  if (tid == 0) {
    a.counts[0] = used;
    a.counts[1] = moves;
  }
  __syncthreads();
  for (int64_t i = tid; i < (int64_t)a.rows * a.stride; i += kThreads) {
    const int32_t p = a.table[i];
    a.new_table[i] = in_pool(a, p) ? place[p] : p;
  }
}

}  // namespace

hipError_t launch_update_small(const PagesArgs &a, hipStream_t stream) {
  hipLaunchKernelGGL(update_small_kernel, dim3(1), dim3(kThreads), (unsigned)a.pages * 4, stream, a);
  return hipGetLastError();
}

hipError_t launch_fork_small(const PagesArgs &a, hipStream_t stream) {
  hipLaunchKernelGGL(fork_small_kernel, dim3(1), dim3(kThreads), (unsigned)a.pages * 4, stream, a);
  return hipGetLastError();
}

hipError_t launch_compact_small(const PagesArgs &a, hipStream_t stream) {
  hipLaunchKernelGGL(compact_small_kernel, dim3(1), dim3(kThreads), (unsigned)(2 * a.pages + a.pages / 2 + 1) * 4, stream, a);
  return hipGetLastError();
}

}  // namespace adaserve
