// Causal attention of packed prompts over the paged cache on gfx950: row i of
// a request's n tokens stands at position c - n + i of its c cached keys and
// sees the keys up to itself.
#include "device_common.h"
#include "paged_rows.h"
#include "plan.h"
#include "serving.h"

namespace adaserve {

namespace {

constexpr int kThreads = 256;

template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void prompt_attn_kernel(PagedAttnArgs a) {
  const int wave = threadIdx.x >> 6;
  const int64_t id = (int64_t)blockIdx.x * (kThreads / 64) + wave;
  const int64_t t = id / a.num_q_heads;
  const int h = (int)(id - t * a.num_q_heads);
  if (t >= a.total_tokens) return;
  int r = 0;
  while (r < a.num_requests && a.token_indptr[r + 1] <= t) ++r;
  if (r >= a.num_requests || a.token_indptr[r] > t) return;
  const int32_t n = a.token_indptr[r + 1] - a.token_indptr[r];
  const int64_t pos = (int64_t)a.context_len[r] - n + (t - a.token_indptr[r]);
  attend_row<BF16, D>(a, r, t, h, pos + 1);
}

}  // namespace

hipError_t launch_prompt_attn(const PagedAttnArgs &a, int head_dim, bool bf16, hipStream_t stream) {
  const int64_t waves = (int64_t)a.total_tokens * a.num_q_heads;
  const dim3 grid((unsigned)((waves + 3) / 4)), block(kThreads);
  if (bf16 && head_dim == 128) hipLaunchKernelGGL((prompt_attn_kernel<true, 128>), grid, block, 0, stream, a);
  else if (bf16) hipLaunchKernelGGL((prompt_attn_kernel<true, 64>), grid, block, 0, stream, a);
  else if (head_dim == 128) hipLaunchKernelGGL((prompt_attn_kernel<false, 128>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((prompt_attn_kernel<false, 64>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace adaserve
