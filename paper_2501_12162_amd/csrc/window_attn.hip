// Attention over a window and sinks on gfx950, one wave per (token, query head):
//   out = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale q k_j - m),
// over the positions j <= p with j > p - window or j < sinks.
#include "device_common.h"
#include "kernels.h"
#include "plan.h"
#include "serving.h"
#include "window_rows.h"

namespace adaserve {

namespace {

constexpr int kThreads = kServingThreads;
constexpr int kWaves = kThreads / 64;

// The request of row t: the last r with indptr[r] <= t.
__device__ __forceinline__ int find_request(const int32_t *indptr, int n, int32_t t) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (indptr[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void window_rows_kernel(PagedAttnArgs a, bool decode) {
  __shared__ RowScratch<D> scratch[kWaves];
  constexpr int ESZ = BF16 ? 2 : 4;
  const int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int64_t t = id / a.num_q_heads;
  const int h = (int)(id - t * a.num_q_heads), g = h / a.group;
  if (t >= a.total_tokens) return;
  int r = (int)t;
  int64_t pos = 0;
  char *out = (char *)a.out + id * D * ESZ;
  if (decode) {
    pos = (int64_t)a.context_len[r] - 1;
    if (pos < -1 || pos >= a.max_context) {
      for (int i = threadIdx.x & 63; i < D; i += 64) {
        if (BF16) ((__bf16 *)out)[i] = (__bf16)__builtin_nanf("");
        else ((float *)out)[i] = __builtin_nanf("");
      }
      return;
    }
  } else {
    r = find_request(a.token_indptr, a.num_requests, (int32_t)t);
    pos = (int64_t)a.context_len[r] - (a.token_indptr[r + 1] - t);
  }
  const SeenKeys seen = seen_keys(pos, a.window, a.sinks);
  attend_keys<BF16, D>((const char *)a.q + (t * a.q_stride + (int64_t)h * D) * ESZ, seen.count,
                       [&](int64_t i) { return paged_key(a, r, g, seen.place(i), D * ESZ); }, a.sm_scale, out,
                       scratch[threadIdx.x >> 6]);
}

template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void window_tree_rows_kernel(TreeAttnArgs a) {
  __shared__ RowScratch<D> scratch[kWaves];
  __shared__ int32_t path[kWaves][kMaxTreeNodes];
  constexpr int ESZ = BF16 ? 2 : 4;
  const int wave = threadIdx.x >> 6;
  const int64_t id = (int64_t)blockIdx.x * kWaves + wave;
  const int64_t t = id / a.num_q_heads;
  const int h = (int)(id - t * a.num_q_heads), g = h / a.group;
  if (t >= a.total_nodes) return;
  const int r = find_request(a.node_indptr, a.num_requests, (int32_t)t);
  const int32_t base = a.node_indptr[r], n = min(a.node_indptr[r + 1] - base, kMaxTreeNodes), L = a.prefix_len[r];
  // the path, from the node up (it ends at anything that is not a parent before its child)
  int32_t len = 0;
  for (int32_t v = (int32_t)(t - base); v >= 0 && v < n && len < kMaxTreeNodes;) {
    path[wave][len++] = v;
    const int32_t p = v == 0 ? -1 : a.parent[base + v];
    v = p < v ? p : -1;
  }
  row_sync();
  const int32_t depth = len - 1;
  const SeenKeys seen = seen_keys((int64_t)L + depth, a.window, a.sinks);
  PagedAttnArgs pages{};
  pages.bt_stride = a.bt_stride;
  pages.block_table = a.block_table;
  pages.num_pages = a.num_pages;
  pages.num_kv_heads = a.num_kv_heads;
  pages.k_pages = a.k_pages;
  pages.v_pages = a.v_pages;
  attend_keys<BF16, D>((const char *)a.q + id * D * ESZ, seen.count,
                       [&](int64_t i) {
                         const int64_t place = seen.place(i);   // (from L on: of the path)
                         if (place < L) return paged_key(pages, r, g, place, D * ESZ);
                         const int32_t node = path[wave][depth - (int32_t)(place - L)];
                         const int64_t at = ((int64_t)(base + node) * a.num_kv_heads + g) * D * ESZ;
                         return KeyRows{(const char *)a.k_tree + at, (const char *)a.v_tree + at};
                       },
                       a.sm_scale, (char *)a.out + id * D * ESZ, scratch[wave]);
}

unsigned row_blocks(int64_t rows) { return (unsigned)((rows + kWaves - 1) / kWaves); }

}  // namespace

hipError_t launch_window_rows(const PagedAttnArgs &a, int head_dim, bool bf16, bool decode, hipStream_t stream) {
  const dim3 grid(row_blocks((int64_t)a.total_tokens * a.num_q_heads)), block(kThreads);
  if (bf16 && head_dim == 128) hipLaunchKernelGGL((window_rows_kernel<true, 128>), grid, block, 0, stream, a, decode);
  else if (bf16) hipLaunchKernelGGL((window_rows_kernel<true, 64>), grid, block, 0, stream, a, decode);
  else if (head_dim == 128) hipLaunchKernelGGL((window_rows_kernel<false, 128>), grid, block, 0, stream, a, decode);
  else hipLaunchKernelGGL((window_rows_kernel<false, 64>), grid, block, 0, stream, a, decode);
  return hipGetLastError();
}

hipError_t launch_window_tree_rows(const TreeAttnArgs &a, int head_dim, bool bf16, hipStream_t stream) {
  const dim3 grid(row_blocks((int64_t)a.total_nodes * a.num_q_heads)), block(kThreads);
  if (bf16 && head_dim == 128) hipLaunchKernelGGL((window_tree_rows_kernel<true, 128>), grid, block, 0, stream, a);
  else if (bf16) hipLaunchKernelGGL((window_tree_rows_kernel<true, 64>), grid, block, 0, stream, a);
  else if (head_dim == 128) hipLaunchKernelGGL((window_tree_rows_kernel<false, 128>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((window_tree_rows_kernel<false, 64>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace adaserve
