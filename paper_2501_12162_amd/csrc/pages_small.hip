// The pages of a small cache on gfx950, one workgroup and one launch a call: the
// reference counts lie in LDS from the beginning to the end, so the steps of a call
// follow each other by barriers instead of launches.  Same results as pages.hip.
#include "device_common.h"
#include "pages.h"

namespace adaserve {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kMostWords = kSmallPages / 64;
static_assert(kSmallPages % 64 == 0 && kMostWords <= 2 * 64, "two words of pages per lane");

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
      const int32_t n0 = 2 * lane < words ? __popcll(word[2 * lane]) : 0;
      const int32_t n1 = 2 * lane + 1 < words ? __popcll(word[2 * lane + 1]) : 0;
      const int32_t upto = (int32_t)wave_inclusive_scan(n0 + n1);
      if (2 * lane < words) before[2 * lane] = upto - n0 - n1;
      if (2 * lane + 1 < words) before[2 * lane + 1] = upto - n1;
      if (lane == 63) before[kMostWords] = upto;
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
  __shared__ int32_t want[kSmallRows];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t ps = a.page_size;
  load_refs(a, refs);
  __syncthreads();
  // a row's entries that are to have pages: [first, last)
  auto range = [&](int32_t c, int32_t need, int32_t &first, int32_t &last) {
    first = min((int32_t)(((int64_t)c + ps - 1) / ps), a.stride);
    last = need > 0 ? min((int32_t)(((int64_t)need + ps - 1) / ps), a.stride) : 0;
    last = max(last, first);
  };
  for (int32_t r = wave; r < a.rows; r += kWaves) {
    const int32_t c = a.context_len[r];
    const int32_t *in = a.table + (int64_t)r * a.stride;
    int32_t *out = a.new_table + (int64_t)r * a.stride;
    int32_t from = 0, to = a.stride, first = 0, last = 0;   // entries [from, to) go
    if (c >= 0) {
      from = (int32_t)(((int64_t)a.sinks + ps - 1) / ps);
      to = a.window > 0 && c >= a.window ? (c - a.window + 1) / ps : 0;
      if (a.need_len) range(c, a.need_len[r], first, last);
    }
    int32_t n = 0;
    for (int32_t e0 = 0; e0 < a.stride; e0 += 64) {
      const int32_t e = e0 + lane;
      if (e < a.stride) {
        const int32_t p = in[e];
        const bool has = in_pool(a, p), gone = e >= from && e < to;
        if (gone && has) atomicAdd(&refs[p], -1);
        if (gone || out != in) out[e] = gone ? -1 : p;
        n += e >= first && e < last && (gone || !has);
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) n += __shfl_xor(n, off, 64);
    if (lane == 0) want[r] = n;
  }
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
      int32_t first, last, missing = a.stride, rank0 = want[r];
      range(c, need, first, last);
      // (from the entry that holds some of the c tokens on nothing has gone: the window ends before it)
      for (int32_t e0 = min(c / ps, a.stride); e0 < last; e0 += 64) {
        const int32_t e = e0 + lane;
        const bool without = e < last && !in_pool(a, a.table[(int64_t)r * a.stride + e]);
        const unsigned long long wants = __ballot(without && e >= first);
        const int32_t rank = rank0 + __popcll(wants & ((1ull << lane) - 1));
        const bool taken = without && e >= first && rank < got;
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
  __shared__ int32_t want[kSmallRows], takers[kSmallRows], first[kSmallRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t ps = a.page_size;
  const int64_t most = (int64_t)a.stride * ps;
  load_refs(a, refs);
  if (tid < a.sources) {
    takers[tid] = 0;
    first[tid] = a.rows;
  }
  __syncthreads();
  const int32_t mine = tid < a.rows ? a.source[tid] : -1;   // (a thread per row, too)
  const bool any = mine >= 0 && mine < a.sources;
  if (any) {
    atomicAdd(&takers[mine], 1);
    atomicMin(&first[mine], tid);
  }
  __syncthreads();
  auto tokens = [&](int32_t s) { return (int32_t)min((int64_t)max(a.context_len[s], 0), most); };
  for (int32_t s = wave; s < a.sources; s += kWaves) {
    const int32_t whole = tokens(s) / ps, n = takers[s];
    for (int32_t e = lane; e < a.stride; e += 64) {
      const int32_t p = a.table[(int64_t)s * a.stride + e], more = e < whole ? n - 1 : n > 0 ? 0 : -1;
      if (in_pool(a, p) && more != 0) atomicAdd(&refs[p], more);
    }
  }
  // a row's own entry of the partly filled page, where it needs one, is written at the end
  int32_t c = 0, from = -1;
  bool copy = false;
  if (any) {
    c = tokens(mine);
    if (c % ps != 0 && first[mine] != tid) from = a.table[(int64_t)mine * a.stride + c / ps];
    copy = in_pool(a, from);
  }
  if (tid < a.rows) want[tid] = copy;
  __syncthreads();
  for (int32_t r = wave; r < a.rows; r += kWaves) {
    const int32_t s = a.source[r];
    const bool ok = s >= 0 && s < a.sources;
    const int32_t whole = ok ? tokens(s) / ps : 0, upto = !ok ? 0 : first[s] == r ? a.stride : whole;
    const int32_t skip = want[r] ? whole : -1;
    for (int32_t e = lane; e < a.stride; e += 64)
      if (e != skip) a.new_table[(int64_t)r * a.stride + e] = e < upto ? a.table[(int64_t)s * a.stride + e] : -1;
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
