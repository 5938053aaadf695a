// Attention of one query row over a request's paged keys, by one wave.
#pragma once
#include "device_common.h"
#include "plan.h"
#include "serving.h"

namespace adaserve {

template <bool BF16, int N>
__device__ __forceinline__ void load_row(const void *p, int64_t i, float (&x)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k)
    x[k] = BF16 ? bf16_bits_to_float(((const uint16_t *)p)[i + k]) : ((const float *)p)[i + k];
}

// out[t, h] = attention of q[t, h] over the first `keys` keys of request r;
// lane l holds columns l * D/64 ...  No key: zeros.
template <bool BF16, int D>
__device__ __forceinline__ void attend_row(const PagedAttnArgs &a, int r, int64_t t, int h, int64_t keys) {
  constexpr int N = D / 64;
  const int lane = threadIdx.x & 63;
  const int g = h / a.group;
  float q[N], o[N] = {};
  load_row<BF16>(a.q, t * a.q_stride + (int64_t)h * D + lane * N, q);
  float m = -INFINITY, l = 0.f;
  for (int64_t key = 0; key < keys; ++key) {
    const int64_t e = key / kPageSize;
    const int32_t p = e < a.bt_stride ? a.block_table[(int64_t)r * a.bt_stride + e] : -1;
    float k[N] = {}, v[N] = {};
    if (p >= 0 && p < a.num_pages) {
      const int64_t at = (((int64_t)p * a.num_kv_heads + g) * kPageSize + key % kPageSize) * D + lane * N;
      load_row<BF16>(a.k_pages, at, k);
      load_row<BF16>(a.v_pages, at, v);
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = __builtin_fmaf(q[i], k[i], s);
    s = wave_sum(s) * a.sm_scale;
    const float mn = fmaxf(m, s);
    const float old = m == -INFINITY ? 0.f : __expf(m - mn), w = s == -INFINITY ? 0.f : __expf(s - mn);
    m = mn;
    l = l * old + w;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = o[i] * old + w * v[i];
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const int64_t at = (t * a.num_q_heads + h) * (int64_t)D + lane * N;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (BF16) ((__bf16 *)a.out)[at + i] = (__bf16)(o[i] * inv);
    else ((float *)a.out)[at + i] = o[i] * inv;
  }
}

}  // namespace adaserve
