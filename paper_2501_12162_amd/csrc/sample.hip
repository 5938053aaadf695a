// Sampling on gfx950: a token per row of logits by temperature, top-k, top-p
// and min-p, from a given uniform number.
//
// With z = (x - max) / T the mass of a token is the whole number
// W = round(2^32 e^z).  Tokens are ordered by logit, the larger first, equal
// ones (+0 = -0) by index.  Top-k keeps the first k; top-p keeps of those the
// tokens whose predecessors' mass is below p times the mass of the k; min-p
// keeps of those the tokens with W >= 2^32 min_p; the first token is always
// kept.  The token drawn is the first, in index order, whose cumulative kept
// mass exceeds u times the kept mass.  Whole-number masses make every sum
// exact and independent of its order (2^20 tokens of 2^32 are below 2^53, so
// also as doubles); the units are fine enough (2.3e-10 of the likeliest
// token's mass) that their rounding is far below that of fp32 sums.
#include <limits.h>

#include "device_common.h"
#include "serving.h"

namespace adaserve {

namespace {

constexpr int kThreads = 1024;
constexpr double kUnit = 4294967296.0;

template <bool BF16>
__device__ __forceinline__ float logit(const SampleArgs &a, int row, int v) {
  const int64_t i = (int64_t)row * a.row_stride + v;
  const float x = BF16 ? bf16_bits_to_float(((const uint16_t *)a.logits)[i]) : ((const float *)a.logits)[i];
  return x + 0.f;   // -0 ranks with +0
}

// Unsigned order of the keys = order of the values.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}

__device__ __forceinline__ uint64_t mass_of(float x, float top, double t) {
  return (uint64_t)__builtin_rint(exp(((double)x - (double)top) / t) * kUnit);
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ uint32_t hist_n[256];
  __shared__ unsigned long long hist_w[256];
  __shared__ unsigned long long scan[kThreads];
  __shared__ uint32_t s_key;
  __shared__ int32_t s_bad, s_token, s_cut;
  __shared__ unsigned long long s_a, s_b, s_c;
  const int row = blockIdx.x, tid = threadIdx.x;
  const float temp = a.temperature ? a.temperature[row] : 1.f;
  int64_t k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f, least = a.min_p ? a.min_p[row] : 0.f, u = a.u[row];
  if (tid == 0) {
    s_key = 0;
    s_bad = !(temp >= 0.f && temp < INFINITY) || p != p || least != least || u != u;
    s_token = INT_MAX;
    s_cut = INT_MAX;
  }
  __syncthreads();
  uint32_t best = 0;
  bool bad = false;
  for (int v = tid; v < a.vocab; v += kThreads) {
    const float x = logit<BF16>(a, row, v);
    bad |= !(x < INFINITY);
    best = max(best, order_key(x));
  }
  atomicMax(&s_key, best);
  if (bad) s_bad = 1;
  __syncthreads();
  const uint32_t top_key = s_key;
  const float top = key_value(top_key);
  if (s_bad || top == -INFINITY) {
    if (tid == 0) a.out_token[row] = -1;
    return;
  }
  if (k <= 0 || k > a.vocab) k = a.vocab;
  if (temp == 0.f || least > 1.f) k = 1;
  const double t = temp == 0.f ? 1.0 : (double)temp;

  // Radix descent over the keys, most significant byte first: by count to the
  // k-th token, then by mass to the last token of the nucleus.
  uint32_t cut = 0;          // keys above it are kept, and `ties` of those equal to it
  int64_t ties = INT_MAX;
  auto descend = [&](bool by_mass, unsigned long long want) {
    // the first bins whose running total reaches `want`
    uint32_t prefix = 0;
    unsigned long long before = 0, have = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kThreads) hist_n[i] = 0, hist_w[i] = 0;
      __syncthreads();
      for (int v = tid; v < a.vocab; v += kThreads) {
        const float x = logit<BF16>(a, row, v);
        const uint32_t key = order_key(x);
        if (shift < 24 && (key >> (shift + 8)) != prefix) continue;
        if (by_mass && key <= cut) continue;   // the ties at the cut are added below
        atomicAdd(&hist_n[(key >> shift) & 255], 1u);
        if (by_mass) atomicAdd(&hist_w[(key >> shift) & 255], (unsigned long long)mass_of(x, top, t));
      }
      __syncthreads();
      if (tid == 0) {
        if (by_mass && (shift == 24 || (cut >> (shift + 8)) == prefix))
          hist_w[(cut >> shift) & 255] += (unsigned long long)ties * mass_of(key_value(cut), top, t);
        int b = 255;
        unsigned long long here = by_mass ? hist_w[b] : hist_n[b];
        while (b > 0 && before + here < want) {
          before += here;
          --b;
          here = by_mass ? hist_w[b] : hist_n[b];
        }
        s_key = (prefix << 8) | (uint32_t)b;
        s_a = before;
        s_b = here;
      }
      __syncthreads();
      prefix = s_key;
      before = s_a;
      have = s_b;
      __syncthreads();
    }
    s_c = have;
    const unsigned long long left = want > before ? want - before : 0;
    return make_ulonglong2(left, prefix);
  };
  if (k < a.vocab) {
    const ulonglong2 d = descend(false, (unsigned long long)k);
    cut = (uint32_t)d.y;
    ties = (int64_t)d.x;
  } else {
    // every token: the cut lies below the smallest key
    cut = 0;
    ties = 0;
  }
  auto total_kept = [&](double w_least) {
    unsigned long long sum = 0;
    for (int v = tid; v < a.vocab; v += kThreads) {
      const float x = logit<BF16>(a, row, v);
      if (order_key(x) <= cut) continue;
      const uint64_t w = mass_of(x, top, t);
      if ((double)w >= w_least) sum += w;
    }
    if (tid == 0) s_a = 0;
    __syncthreads();
    atomicAdd(&s_a, sum);
    __syncthreads();
    unsigned long long all = s_a;
    __syncthreads();
    const uint64_t w = cut ? mass_of(key_value(cut), top, t) : 0;
    if ((double)w >= w_least) all += (unsigned long long)ties * w;
    return all;
  };
  if (p < 1.f) {
    const double want = (double)p * (double)total_kept(0.0);
    const unsigned long long w = want > 1.0 ? (unsigned long long)__builtin_ceil(want) : 1ull;
    const ulonglong2 d = descend(true, w);
    const uint32_t c = (uint32_t)d.y;
    const uint64_t each = mass_of(key_value(c), top, t);
    // each token at the cut whose predecessors' mass is below `want`
    const uint64_t n = each ? (d.x + each - 1) / each : 0;
    if (c != cut || (int64_t)n < ties) {
      cut = c;
      ties = (int64_t)n;
    }
  }
  const double w_least = fmin((double)least, 1.0) * kUnit;
  const unsigned long long kept = total_kept(w_least);
  const double target = fmax((double)u, 0.0) * (double)kept;

  // tokens in index order, kThreads at a time
  unsigned long long run = 0;
  int64_t tie_run = 0;
  for (int v0 = 0; v0 < a.vocab; v0 += kThreads) {
    const int v = v0 + tid;
    const float x = v < a.vocab ? logit<BF16>(a, row, v) : -INFINITY;
    const uint32_t key = order_key(x);
    const bool tie = v < a.vocab && key == cut;
    scan[tid] = tie;
    __syncthreads();
    for (int off = 1; off < kThreads; off <<= 1) {
      const unsigned long long o = tid >= off ? scan[tid - off] : 0;
      __syncthreads();
      scan[tid] += o;
      __syncthreads();
    }
    const int64_t rank = tie_run + (int64_t)scan[tid] - 1;
    tie_run += (int64_t)scan[kThreads - 1];
    __syncthreads();
    uint64_t w = v < a.vocab && (key > cut || (tie && rank < ties)) ? mass_of(x, top, t) : 0;
    if ((double)w < w_least) w = 0;
    scan[tid] = w;
    __syncthreads();
    for (int off = 1; off < kThreads; off <<= 1) {
      const unsigned long long o = tid >= off ? scan[tid - off] : 0;
      __syncthreads();
      scan[tid] += o;
      __syncthreads();
    }
    const unsigned long long upto = run + scan[tid];
    // with u >= 1 nothing exceeds the target and the last kept token is drawn
    if (w && ((double)upto > target || upto == kept)) atomicMin(&s_token, v);
    run += scan[kThreads - 1];
    __syncthreads();
    if (s_token != INT_MAX) break;
  }
  if (tid == 0) a.out_token[row] = s_token == INT_MAX ? -1 : s_token;
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t stream) {
  if (bf16)
    hipLaunchKernelGGL(sample_kernel<true>, dim3((unsigned)a.rows), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(sample_kernel<false>, dim3((unsigned)a.rows), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace adaserve
