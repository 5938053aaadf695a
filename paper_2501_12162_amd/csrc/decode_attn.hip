// Attention of one new token per request over its paged cache on gfx950.
#include "device_common.h"
#include "paged_rows.h"
#include "plan.h"
#include "serving.h"

namespace adaserve {

namespace {

constexpr int kThreads = 256;

template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void decode_attn_kernel(PagedAttnArgs a) {
  const int wave = threadIdx.x >> 6;
  const int64_t id = (int64_t)blockIdx.x * (kThreads / 64) + wave;
  const int64_t r = id / a.num_q_heads;
  const int h = (int)(id - r * a.num_q_heads);
  if (r >= a.num_requests) return;
  const int32_t len = a.context_len[r];
  if (len < 0 || len > a.max_context) {
    const int lane = threadIdx.x & 63;
    for (int i = lane; i < D; i += 64) {
      if (BF16) ((__bf16 *)a.out)[(r * a.num_q_heads + h) * D + i] = (__bf16)__builtin_nanf("");
      else ((float *)a.out)[(r * a.num_q_heads + h) * D + i] = __builtin_nanf("");
    }
    return;
  }
  attend_row<BF16, D>(a, (int)r, r, h, len);
}

}  // namespace

hipError_t launch_decode_attn(const PagedAttnArgs &a, int head_dim, bool bf16, hipStream_t stream) {
  const int64_t waves = (int64_t)a.num_requests * a.num_q_heads;
  const dim3 grid((unsigned)((waves + 3) / 4)), block(kThreads);
  if (bf16 && head_dim == 128) hipLaunchKernelGGL((decode_attn_kernel<true, 128>), grid, block, 0, stream, a);
  else if (bf16) hipLaunchKernelGGL((decode_attn_kernel<true, 64>), grid, block, 0, stream, a);
  else if (head_dim == 128) hipLaunchKernelGGL((decode_attn_kernel<false, 128>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((decode_attn_kernel<false, 64>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace adaserve
