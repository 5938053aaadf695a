// Attention of one query row over any list of keys, by one wave: what the
// attentions over a window fall back to for single rows.
#pragma once
#include "device_common.h"
#include "plan.h"
#include "serving.h"

namespace adaserve {

// What a row at position `pos` sees: positions [0, sinks) and [lo, pos], in this order.
struct SeenKeys {
  int32_t sinks, lo;
  int64_t count;
  __device__ __forceinline__ int64_t place(int64_t i) const { return i < sinks ? i : lo + (i - sinks); }
};

__device__ __forceinline__ SeenKeys seen_keys(int64_t pos, int32_t window, int32_t sinks) {
  SeenKeys s;
  s.lo = (int32_t)max(pos + 1 - window, (int64_t)0);
  s.sinks = min(sinks, s.lo);
  s.count = pos < 0 ? 0 : s.sinks + (pos + 1 - s.lo);
  return s;
}

// A key's rows; no k: a page that does not exist (score 0, value 0).
struct KeyRows {
  const char *k, *v;
};

__device__ __forceinline__ KeyRows paged_key(const PagedAttnArgs &a, int32_t r, int32_t g, int64_t place, int64_t row_bytes) {
  const int64_t e = place / kPageSize;
  const int32_t p = e < a.bt_stride ? a.block_table[(int64_t)r * a.bt_stride + e] : -1;
  if (p < 0 || p >= a.num_pages) return {nullptr, nullptr};
  const int64_t at = (((int64_t)p * a.num_kv_heads + g) * kPageSize + place % kPageSize) * row_bytes;
  return {(const char *)a.k_pages + at, (const char *)a.v_pages + at};
}

template <int D>
struct RowScratch {   // of a wave, in LDS
  float q[D], w[64];
};

__device__ __forceinline__ void row_sync() {
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// out = attention of the row q over the keys at(0) .. at(count - 1).  A lane
// takes the score of every 64th key, then D / 64 columns of the sum.  A key of
// weight 0 adds nothing; no key: zeros.
template <bool BF16, int D, class At>
__device__ __forceinline__ void attend_keys(const void *q, int64_t count, At at, float sm_scale, void *out, RowScratch<D> &s) {
  constexpr int N = D / 64, ESZ = BF16 ? 2 : 4, EPV = 16 / ESZ;
  const int lane = threadIdx.x & 63;
  auto value = [](const char *p, int i) {
    return BF16 ? bf16_bits_to_float(((const uint16_t *)p)[i]) : ((const float *)p)[i];
  };
  row_sync();   // (the row before is done with the scratch)
#pragma unroll
  for (int i = 0; i < N; ++i) s.q[lane + i * 64] = value((const char *)q, lane + i * 64);
  row_sync();
  float m = -INFINITY, l = 0.f, o[N] = {};
  for (int64_t base = 0; base < count; base += 64) {
    KeyRows key{nullptr, nullptr};
    float x = -INFINITY;
    if (base + lane < count) {
      key = at(base + lane);
      x = 0.f;
      if (key.k) {
#pragma unroll 4
        for (int c = 0; c < D / EPV; ++c) {
          const u32x4 w = *(const u32x4 *)(key.k + c * 16);
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            const float kv = BF16 ? __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16) : __uint_as_float(w[e % 4]);
            x = __builtin_fmaf(s.q[c * EPV + e], kv, x);
          }
        }
        x *= sm_scale;
      }
    }
    float bm = x;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) bm = fmaxf(bm, __shfl_xor(bm, off, 64));
    const float mn = fmaxf(m, bm);
    const float old = m == -INFINITY ? 0.f : expf(m - mn);
    const float w = x == -INFINITY ? 0.f : expf(x - mn);   // (a NaN stays one)
    m = mn;
    l = l * old + wave_sum(w);
    s.w[lane] = w;
    row_sync();
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] *= old;
    for (unsigned long long todo = __ballot(key.v != nullptr && w != 0.f); todo; todo &= todo - 1) {
      const int j = __ffsll(todo) - 1;
      const uint64_t p = (uint64_t)key.v;
      const char *v = (const char *)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(p >> 32), j) << 32) |
                                     (uint32_t)__builtin_amdgcn_readlane((int)p, j));
      const float wj = s.w[j];
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = __builtin_fmaf(wj, value(v, lane + i * 64), o[i]);
    }
    bool nan = true;   // (in all columns: whatever comes, they stay so)
#pragma unroll
    for (int i = 0; i < N; ++i) nan = nan && (l != l || o[i] != o[i]);
    if (__all(nan)) break;
    row_sync();
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;   // (a NaN stays one)
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (BF16) ((__bf16 *)out)[lane + i * 64] = (__bf16)(o[i] * inv);
    else ((float *)out)[lane + i * 64] = o[i] * inv;
  }
}

// out[t, h] = attention of q[t, h], at position `pos` of request r, over a window and sinks.
template <bool BF16, int D>
__device__ __forceinline__ void attend_seen(const PagedAttnArgs &a, int32_t r, int64_t t, int32_t h, int64_t pos,
                                            RowScratch<D> &scratch) {
  constexpr int ESZ = BF16 ? 2 : 4;
  const SeenKeys seen = seen_keys(pos, a.window, a.sinks);
  attend_keys<BF16, D>((const char *)a.q + (t * a.q_stride + (int64_t)h * D) * ESZ, seen.count,
                       [&](int64_t i) { return paged_key(a, r, h / a.group, seen.place(i), D * ESZ); }, a.sm_scale,
                       (char *)a.out + (t * a.num_q_heads + h) * D * ESZ, scratch);
}

}  // namespace adaserve
