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
//
// No sort: a row is cut into parts of 4096 to 32768 logits, so that a single row
// runs on many compute units, and four launches go over them:
//   1. maxima of the parts;
//   2. per part a histogram of (count, mass) over 512 bins of -z log2 e: the one
//      pass that takes an exponential per logit;
//   3. from the row's histogram, the bins in which a filter may cut; every part
//      lists its tokens of those bins, in index order (a bin is a sixteenth of a
//      power of two wide: a few hundred tokens out of 10^5);
//   4. one workgroup per row: the exact cuts among the listed tokens, the kept
//      mass of each part (that of the bins before all cuts from pass 3, the rest
//      from the list), and the draw within the one part that holds it.
// The first three read the row (from HBM once, then out of the caches); pass 2
// is bound by fp64 arithmetic and LDS atomics, the rest by memory and latency.
// Measured, fp32, 250 rows of 128256 (128 MB), all filters: 20 (6.3 TB/s), 37, 35
// and 24 us; one bf16 row: 2.8, 4.9, 10.1 and 15 us, of which 10 or so are launches
// and the rest dependent steps.  250 bf16 rows: the call 102 us.
// A row whose cut bins hold more tokens than the lists take (one of few distinct
// values, or nearly flat) is searched as a whole in pass 4, by its one workgroup: such
// calls take 305 (one bf16 row) to 380 us (250 rows).
#include <limits.h>

#include <type_traits>

#include "device_common.h"
#include "serving.h"

namespace adaserve {

namespace {

constexpr int kThreads = kServingThreads;          // of passes 1 to 3
constexpr int kDrawThreads = kSampleDrawThreads;
constexpr int kBins = kSampleBins;
constexpr double kUnit = 4294967296.0;
// Bins 0 .. 510 cover -z log2 e in [0, 33.01), where masses can be 1 or more;
// the last bin's tokens have none.
constexpr float kBinsPerLog2 = 511.f / 33.01f;
constexpr uint64_t kMassBits = 48, kMassMask = (1ull << kMassBits) - 1;   // a part's mass: at most 32768 2^32

// Unsigned order of the keys = order of the values; -0 ranks with +0.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
constexpr uint32_t kKeyMinusInf = 0x007fffffu;   // order_key(-inf)

// What a row asks for, and its logits' place.
struct Row {
  const char *base;        // its first logit
  int off;                 // elements between the 16-byte line of the first logit and it
  float top;               // largest logit
  uint32_t top_key;
  double rate;             // log2 e / T
  int64_t k;               // 0: off
  double p;                // >= 1: off
  double least;            // least mass (0: off)
  float u;
  int state;               // 0: draw, 1: the first-ranked token, 2: no distribution
};

// -z log2 e of logit x (monotone in x, also in its roundings).
__device__ __forceinline__ double depth_of(const Row &r, float x) {
  return ((double)r.top - (double)x) * r.rate;
}
__device__ __forceinline__ int bin_of(double y) {
  return y < 33.01 ? min((int)((float)y * kBinsPerLog2), kBins - 1) : kBins - 1;
}
// round(2^(32 - y)): 2^f, |f| <= 1/2, by its series to f^11 (error below 2^-46).
// Without branches: from y = 33 on the result rounds to 0 by itself.
__device__ __forceinline__ uint64_t mass_at(double y) {
  // (ln 2)^k / k!, k = 1 .. 11
  constexpr double kSeries[11] = {
    0.6931471805599453, 0.24022650695910072, 0.05550410866482158, 0.009618129107628477,
    0.0013333558146428443, 0.0001540353039338161, 1.5252733804059841e-05, 1.321548679014431e-06,
    1.01780860092397e-07, 7.054911620801123e-09, 4.4455382718708116e-10};
  y = fmin(y, 40.0);
  const double n = __builtin_rint(y), f = n - y;
  double s = kSeries[10];
#pragma unroll
  for (int k = 9; k >= 0; --k) {
    double c = kSeries[k];
    asm("" : "+s"(c));   // stays in scalar registers: the sum needs no copy of it
    s = __builtin_fma(s, f, c);
  }
  s = __builtin_fma(s, f, 1.0);
  // adding 2^52 rounds to a whole number and leaves it in the mantissa
  const double w = __builtin_ldexp(s, 32 - (int)n) + 4503599627370496.0;
  return (uint64_t)__double_as_longlong(w) & ((1ull << 52) - 1);
}
__device__ __forceinline__ uint64_t mass_of(const Row &r, float x) { return mass_at(depth_of(r, x)); }

// Logit vectors: vector v of a row holds elements v * EPV - off .. + EPV - 1, so
// that whole ones are 16-byte lines; f(index, value) for those in the row.
template <bool BF16>
struct Vec {
  static constexpr int EPV = BF16 ? 8 : 4;
  // Loads in flight per thread in passes 1 to 3: 4096 elements, the smallest
  // part, are 4 fp32 vectors per thread and 2 bf16 ones.
  static constexpr int BATCH = BF16 ? 2 : 4;
  float x[EPV];
  int first;   // index of x[0], may lie before the row
  __device__ __forceinline__ void load(const Row &r, int vocab, int v) {
    first = v * EPV - r.off;
    if (first >= 0 && first + EPV <= vocab) {
      const u32x4 w = *(const u32x4 *)(r.base + (int64_t)first * (BF16 ? 2 : 4));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (BF16) {
          x[2 * i] = __uint_as_float(w[i] << 16);
          x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
          x[i] = __uint_as_float(w[i]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPV; ++i) {
        const int e = first + i;
        x[i] = -INFINITY;
        if (e >= 0 && e < vocab)
          x[i] = BF16 ? bf16_bits_to_float(((const uint16_t *)r.base)[e]) : ((const float *)r.base)[e];
      }
    }
  }
  __device__ __forceinline__ bool in(int i, int vocab) const { return (uint32_t)(first + i) < (uint32_t)vocab; }
};

template <bool BF16>
__device__ __forceinline__ float logit_at(const Row &r, int i) {
  return BF16 ? bf16_bits_to_float(((const uint16_t *)r.base)[i]) : ((const float *)r.base)[i];
}

template <bool BF16>
__device__ __forceinline__ Row row_place(const SampleArgs &a, int64_t row) {
  Row r{};
  r.base = (const char *)a.logits + row * a.row_stride * (BF16 ? 2 : 4);
  r.off = (int)((uintptr_t)r.base & 15) / (BF16 ? 2 : 4);
  return r;
}

// The row's parameters and maximum (by every wave of the workgroup).
template <bool BF16>
__device__ __forceinline__ Row load_row(const SampleArgs &a, int64_t row) {
  Row r = row_place<BF16>(a, row);
  const int lane = threadIdx.x & 63;
  uint32_t key = lane < a.parts ? a.ws_max[row * a.parts + lane] : 0;
  const float t = a.temperature ? a.temperature[row] : 1.f, p = a.top_p ? a.top_p[row] : 1.f;
  const float m = a.min_p ? a.min_p[row] : 0.f;
  const int32_t k = a.top_k ? a.top_k[row] : 0;
  r.u = a.u[row];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) key = max(key, (uint32_t)__shfl_xor((int)key, o, 64));
  r.top_key = key;
  r.top = key_value(key);
  const bool bad = key >= 0xff800000u || key <= kKeyMinusInf ||   // (a NaN's part has the largest key)
                   !(t >= 0.f && t < INFINITY) || p != p || m != m || r.u != r.u;
  r.state = bad ? 2 : t == 0.f || k == 1 || m > 1.f || p <= 0.f ? 1 : 0;
  r.rate = 1.4426950408889634074 / (t == 0.f ? 1.0 : (double)t);
  r.k = k >= 1 && k < a.vocab ? k : 0;
  r.p = p;
  r.least = m > 0.f ? (double)m * kUnit : 0.0;
  if (r.least <= 0.5) r.least = 0.0;   // every mass of 1 passes, and a mass of 0 is never drawn
  return r;
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void sample_max_kernel(SampleArgs a) {
  __shared__ uint32_t part_key[kThreads / 64];
  const int64_t row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x - row * a.parts);
  const Row r = row_place<BF16>(a, row);
  const int v0 = part * a.part_vecs;
  uint32_t best = 0;
  Vec<BF16> x[Vec<BF16>::BATCH];
  for (int v = threadIdx.x; v < a.part_vecs; v += Vec<BF16>::BATCH * kThreads) {
#pragma unroll
    for (int h = 0; h < Vec<BF16>::BATCH; ++h) x[h].load(r, v + h * kThreads < a.part_vecs ? a.vocab : 0, v0 + v + h * kThreads);
#pragma unroll
    for (int h = 0; h < Vec<BF16>::BATCH; ++h)
#pragma unroll
      for (int i = 0; i < Vec<BF16>::EPV; ++i)
        best = max(best, x[h].x[i] < INFINITY ? order_key(x[h].x[i]) : 0xffffffffu);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) best = max(best, (uint32_t)__shfl_xor((int)best, o, 64));
  if ((threadIdx.x & 63) == 0) part_key[threadIdx.x >> 6] = best;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) best = max(best, part_key[w]);
    a.ws_max[blockIdx.x] = best;
  }
}

// A bin's word: mass | count << 48.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void sample_hist_kernel(SampleArgs a) {
  __shared__ unsigned long long hist[kBins];
  const int64_t row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x - row * a.parts);
  const Row r = load_row<BF16>(a, row);
  if (r.state) return;
  for (int b = threadIdx.x; b < kBins; b += kThreads) hist[b] = 0;
  __syncthreads();
  const int v0 = part * a.part_vecs;
  Vec<BF16> x[Vec<BF16>::BATCH];
  for (int v = threadIdx.x; v < a.part_vecs; v += Vec<BF16>::BATCH * kThreads) {
#pragma unroll
    for (int h = 0; h < Vec<BF16>::BATCH; ++h) x[h].load(r, v + h * kThreads < a.part_vecs ? a.vocab : 0, v0 + v + h * kThreads);
#pragma unroll
    for (int h = 0; h < Vec<BF16>::BATCH; ++h)
    {
      int b[Vec<BF16>::EPV];
      uint64_t w[Vec<BF16>::EPV];
#pragma unroll
      for (int i = 0; i < Vec<BF16>::EPV; ++i) {
        const double y = depth_of(r, x[h].x[i]);
        b[i] = bin_of(y);
        w[i] = mass_at(y) | (1ull << kMassBits);
      }
#pragma unroll
      for (int i = 0; i < Vec<BF16>::EPV; ++i)
        if (b[i] < kBins - 1) atomicAdd(&hist[b[i]], (unsigned long long)w[i]);
    }
  }
  __syncthreads();
  uint64_t *out = a.ws_hist + (int64_t)blockIdx.x * kBins;
  for (int b = threadIdx.x; b < kBins; b += kThreads) out[b] = hist[b];
}

// Exclusive prefix sum over the workgroup's threads, the total in `total`.
template <int T>
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t *lds, uint64_t &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t x = __shfl_up((unsigned long long)s, o, 64);
    if (lane >= o) s += x;
  }
  if (lane == 63) lds[wave] = s;
  __syncthreads();
  uint64_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < T / 64; ++w) {
    if (w < wave) before += lds[w];
    total += lds[w];
  }
  __syncthreads();
  return before + s - v;
}

// Bins that min-p may cut in: those of tokens whose mass is within 1/2 of the
// least one, and of the roundings beside them.
__device__ __forceinline__ void least_bins(const Row &r, int &lo, int &hi) {
  lo = hi = kBins;
  if (r.least == 0.0) return;
  const double a = 32.0 - log2(r.least + 0.500001), b = 32.0 - log2(fmax(r.least - 0.500001, 1e-9));
  lo = bin_of(fmax(a - 1e-6, 0.0));
  hi = bin_of(b + 1e-6);
}

// The least key whose token lies in bin `bin` or before it (the bins fall as the
// logits rise), by the whole wave, six bits a step.
__device__ __forceinline__ uint32_t least_key(const Row &r, int bin) {
  const int lane = threadIdx.x & 63;
  uint32_t key = 0;
#pragma unroll
  for (int shift = 30; shift >= 0; shift -= 6) {
    // (the first step has two bits only)
    const uint32_t at = key + ((uint32_t)lane << shift);
    const bool in = (shift < 30 || lane < 4) && (at >= r.top_key || bin_of(depth_of(r, key_value(at))) <= bin);
    const unsigned long long hit = __ballot(in);
    // the last key of the step that is not in; the first key of all may be
    const int first = hit ? __ffsll(hit) - 1 : shift < 30 ? 64 : 4;
    if (shift == 0) return key + first;
    key += (uint32_t)max(first - 1, 0) << shift;
  }
  return key;
}

// Logits from `lo` to below `hi`.
struct Span {
  float lo, hi;
  __device__ __forceinline__ uint32_t has(float x) const { return x >= lo && x < hi; }
};

typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));

// (eight workgroups per CU, so that the first steps of some hide behind the loads
// of others: 250 rows of 128256 37 -> 34 us)
template <bool BF16>
__global__ __launch_bounds__(kThreads, 8) void sample_list_kernel(SampleArgs a) {
  static_assert(kBins == 2 * kThreads, "two bins per thread");
  __shared__ uint64_t scan[kThreads / 64];
  __shared__ uint64_t cum_w[kBins + 1];
  __shared__ uint32_t cum_n[kBins + 1];
  __shared__ int cut_k, cut_lo, cut_hi;
  __shared__ Span spans[3];
  const int64_t row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x - row * a.parts);
  const Row r = load_row<BF16>(a, row);
  if (r.state) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const u64x2 own = *(const u64x2 *)(a.ws_hist + (int64_t)blockIdx.x * kBins + 2 * tid);
  // the part's mass in the bins before `floor`
  auto part_mass = [&](int floor) {
    uint64_t total;
    block_scan<kThreads>((2 * tid < floor ? own[0] & kMassMask : 0) + (2 * tid + 1 < floor ? own[1] & kMassMask : 0), scan, total);
    if (tid == 0) a.ws_part_w[blockIdx.x] = total;
  };
  if (!(r.k || r.p < 1.0 || r.least > 0.0)) {   // no filter: nothing to cut
    part_mass(kBins);
    if (lane == 0) a.ws_count[(int64_t)blockIdx.x * (kThreads / 64) + wave] = 0;
    return;
  }
  // the row's histogram and its running sums
  uint64_t w[2] = {0, 0}, n[2] = {0, 0};
  const uint64_t *h = a.ws_hist + row * a.parts * kBins + 2 * tid;
  auto add_parts = [&](int p, auto count) {   // this many loads in flight
    constexpr int C = decltype(count)::value;
    u64x2 x[C];
#pragma unroll
    for (int q = 0; q < C; ++q) x[q] = *(const u64x2 *)(h + (int64_t)(p + q) * kBins);
#pragma unroll
    for (int q = 0; q < C; ++q) {
      w[0] += x[q][0] & kMassMask, n[0] += x[q][0] >> kMassBits;
      w[1] += x[q][1] & kMassMask, n[1] += x[q][1] >> kMassBits;
    }
  };
  int done = 0;
  for (; done + 8 <= a.parts; done += 8) add_parts(done, std::integral_constant<int, 8>{});
  for (; done < a.parts; ++done) add_parts(done, std::integral_constant<int, 1>{});
  uint64_t all_w, all_n;
  const uint64_t before_w = block_scan<kThreads>(w[0] + w[1], scan, all_w);
  const uint64_t before_n = block_scan<kThreads>(n[0] + n[1], scan, all_n);
  cum_w[2 * tid] = before_w, cum_w[2 * tid + 1] = before_w + w[0];
  cum_n[2 * tid] = (uint32_t)before_n, cum_n[2 * tid + 1] = (uint32_t)(before_n + n[0]);
  if (tid == 0) {
    cum_w[kBins] = all_w, cum_n[kBins] = (uint32_t)all_n;
    cut_k = kBins, cut_lo = kBins, cut_hi = -1;
  }
  __syncthreads();
  if (part == 0)
    for (int b = tid; b <= kBins; b += kThreads) {
      a.ws_cum_w[row * (kBins + 1) + b] = cum_w[b];
      a.ws_cum_n[row * (kBins + 1) + b] = cum_n[b];
    }
  // Top-k cuts in the bin that holds the k-th token (none: all tokens with mass
  // are kept); the mass that it keeps lies between that of the bins before it and
  // that with it, and so does where top-p cuts.
  if (r.k)
    for (int b = 2 * tid; b < 2 * tid + 2; ++b)
      if ((int64_t)cum_n[b] < r.k && r.k <= (int64_t)cum_n[b + 1]) cut_k = b;
  __syncthreads();
  const int ck = cut_k;
  if (r.p < 1.0) {
    const double most = r.p * (double)(ck < kBins ? cum_w[ck + 1] : all_w), fewest = r.p * (double)(ck < kBins ? cum_w[ck] : all_w);
    for (int b = 2 * tid; b < 2 * tid + 2; ++b) {
      // the bins whose masses reach from below to at or above a wanted sum of the range
      const double from = (double)cum_w[b], to = (double)cum_w[b + 1];
      if (cum_n[b + 1] > cum_n[b] && from < fmax(most, 1.0) && to >= fewest) {
        atomicMin(&cut_lo, b);
        atomicMax(&cut_hi, b);
      }
    }
  }
  __syncthreads();
  const int plo = cut_lo, phi = cut_hi;
  int mlo, mhi;
  least_bins(r, mlo, mhi);
  // The logits of those bins (of the last one none: it has no mass), so that a
  // token costs comparisons instead of its bin (250 rows of 128256: 41 -> 37 us).
  if (wave < 3) {
    const int lo = wave == 0 ? ck : wave == 1 ? plo : mlo, hi = min(wave == 0 ? ck : wave == 1 ? phi : mhi, kBins - 2);
    Span x{INFINITY, -INFINITY};
    if (lo <= hi) {
      x.lo = key_value(least_key(r, hi));
      x.hi = lo > 0 ? key_value(least_key(r, lo - 1)) : INFINITY;
    }
    if (lane == 0) spans[wave] = x;
  }
  // (the bins from there on that are kept as a whole are listed, too: the cut of
  // top-p lies in [plo, phi], that of top-k, where there is no top-p, in ck)
  part_mass(min(ck, min(plo, mlo)));
  __syncthreads();
  const Span sk = spans[0], sp = spans[1], sm = spans[2];
  // tokens of those bins, in index order; each wave lists those of its quarter
  const int quarter = a.part_vecs / (kThreads / 64);
  const int v0 = part * a.part_vecs + wave * quarter;
  const int64_t slot = (int64_t)blockIdx.x * (kThreads / 64) + wave;
  uint64_t *list = a.ws_list + slot * kSampleListCap;
  uint32_t have = 0;
  for (int vb = 0; vb < quarter; vb += 64 * Vec<BF16>::BATCH) {
      Vec<BF16> x[Vec<BF16>::BATCH];
#pragma unroll
      for (int h = 0; h < Vec<BF16>::BATCH; ++h) {
        const int v = vb + h * 64 + lane;
        x[h].load(r, v < quarter ? a.vocab : 0, v0 + v);
      }
#pragma unroll
      for (int h = 0; h < Vec<BF16>::BATCH; ++h) {
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < Vec<BF16>::EPV; ++i) {
          const float v = x[h].x[i];
          mine |= (sk.has(v) | sp.has(v) | sm.has(v)) << i;
        }
        if (!__any(mine != 0)) continue;
        const int count = __popc(mine);
        int s = count;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int y = __shfl_up(s, o, 64);
          if (lane >= o) s += y;
        }
        uint32_t at = have + s - count;
        have += (uint32_t)__shfl(s, 63, 64);
#pragma unroll
        for (int i = 0; i < Vec<BF16>::EPV; ++i)
          if (mine >> i & 1) {
            if (at < (uint32_t)kSampleListCap) list[at] = (uint64_t)order_key(x[h].x[i]) << 32 | (uint32_t)(x[h].first + i);
            ++at;
          }
      }
    }
  if (lane == 0) a.ws_count[slot] = have;
}

template <bool BF16>
__global__ __launch_bounds__(kDrawThreads) void sample_draw_kernel(SampleArgs a) {
  constexpr int T = kDrawThreads, EPV = Vec<BF16>::EPV;
  __shared__ uint32_t list_key[kSampleList];
  __shared__ int32_t list_idx[kSampleList];
  __shared__ unsigned long long digit_w[2][256];
  __shared__ uint32_t digit_n[2][256];
  __shared__ unsigned long long part_w[kSampleMaxParts];
  __shared__ uint32_t list_at[kSampleMaxParts * 4 + 1];
  __shared__ uint64_t cum_w[kBins + 1];
  __shared__ uint32_t cum_n[kBins + 1];
  __shared__ uint64_t scan[T / 64];
  __shared__ uint64_t s_before, s_sum;
  __shared__ uint32_t s_digit;
  __shared__ int s_bin, s_token;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Row r = load_row<BF16>(a, row);
  if (r.state == 2) {
    if (tid == 0) a.out_token[row] = -1;
    return;
  }
  if (tid == 0) s_token = INT_MAX, s_bin = kBins;
  if (r.state == 1) {
    // the first token of the row's largest logit, in the first part that has it
    int first = a.parts - 1;
    const bool has = lane < a.parts && a.ws_max[row * a.parts + lane] == r.top_key;
    const unsigned long long hit = __ballot(has);
    if (hit) first = __ffsll(hit) - 1;
    __syncthreads();
    int best = INT_MAX;
    for (int v = tid; v < a.part_vecs; v += T) {
      Vec<BF16> x;
      x.load(r, a.vocab, first * a.part_vecs + v);
#pragma unroll
      for (int i = EPV - 1; i >= 0; --i)
        if (x.in(i, a.vocab) && order_key(x.x[i]) == r.top_key) best = min(best, x.first + i);
    }
    if (best != INT_MAX) atomicMin(&s_token, best);
    __syncthreads();
    if (tid == 0) a.out_token[row] = s_token;
    return;
  }
  // the row's running sums (of a row with a filter), and the listed tokens in index order
  for (int b = tid; b <= kBins; b += T) {
    cum_w[b] = a.ws_cum_w[row * (kBins + 1) + b];
    cum_n[b] = a.ws_cum_n[row * (kBins + 1) + b];
  }
  const int lists = a.parts * 4;
  {
    const uint32_t c = tid < lists ? a.ws_count[row * lists + tid] : 0;
    uint64_t all;
    const uint64_t before = block_scan<T>(c, scan, all);
    const uint64_t over = __any(c > (uint32_t)kSampleListCap);
    if (tid <= lists) list_at[tid] = (uint32_t)before;
    if (tid < kSampleMaxParts) part_w[tid] = tid < a.parts ? a.ws_part_w[row * a.parts + tid] : 0;
    if (tid == 0) s_digit = all > (uint64_t)kSampleList;
    __syncthreads();
    if (over && lane == 0) s_digit = 1;
  }
  static_assert(kSampleMaxParts * 4 < T, "one thread per list");
  __syncthreads();
  const bool whole = s_digit != 0;          // the lists do not hold them: the row is searched
  const int listed = whole ? 0 : (int)list_at[lists];
  for (int i = tid; i < listed; i += T) {
    int lo = 0, n = lists;                  // the list that entry i is in
    while (n > 1) {
      const int half = n / 2;
      if ((int)list_at[lo + half] <= i) lo += half, n -= half;
      else n = half;
    }
    const uint64_t e = a.ws_list[(row * lists + lo) * kSampleListCap + (i - (int)list_at[lo])];
    list_key[i] = (uint32_t)(e >> 32);
    list_idx[i] = (int32_t)(uint32_t)e;
  }
  __syncthreads();
  // f(key, index) for every token that may be of interest (all of the row where
  // there are no lists)
  auto each = [&](auto f) {
    if (!whole)
      for (int i = tid; i < listed; i += T) f(list_key[i], list_idx[i]);
    else
      for (int v = tid; v < a.parts * a.part_vecs; v += T) {
        Vec<BF16> x;
        x.load(r, a.vocab, v);
#pragma unroll
        for (int i = 0; i < EPV; ++i)
          if (x.in(i, a.vocab)) f(order_key(x.x[i]), x.first + i);
      }
  };
  auto key_bin = [&](uint32_t key) { return bin_of(depth_of(r, key_value(key))); };

  // Radix descent over the keys of the tokens of bin `bin`, most significant byte
  // first: to the key at which their count (or mass) reaches `want`, `before`
  // being what the larger keys have of it.  Ties of the cut key stand for `ties`
  // tokens.
  uint32_t cut = 0;              // keys above it are kept, and the first `ties` tokens of it
  int64_t ties = 0;
  auto descend = [&](bool by_mass, int bin, uint64_t want, uint64_t &before, uint32_t &found) {
    uint32_t prefix = 0;
    before = 0;
    const uint64_t tie_w = by_mass && ties > 0 && key_bin(cut) == bin ? (uint64_t)ties * mass_of(r, key_value(cut)) : 0;
    if (tid < 256) digit_n[0][tid] = 0, digit_w[0][tid] = 0;
    __syncthreads();
    int at = 0;   // the sums of this digit; the others are cleared meanwhile
    // (of a bf16 key the high half says all)
    for (int shift = 24; shift >= (BF16 ? 16 : 0); shift -= 8, at ^= 1) {
      each([&](uint32_t key, int) {
        if (shift < 24 && (key >> (shift + 8)) != prefix) return;
        if (key_bin(key) != bin) return;
        if (!by_mass) atomicAdd(&digit_n[at][(key >> shift) & 255], 1u);
        else if (key > cut) atomicAdd(&digit_w[at][(key >> shift) & 255], (unsigned long long)mass_of(r, key_value(key)));
      });
      __syncthreads();
      if (tid < 64) {
        // lane l holds digits 255 - 4 l .. 252 - 4 l, the largest first
        const int tie_digit = tie_w && (shift == 24 || (cut >> (shift + 8)) == prefix) ? (int)(cut >> shift) & 255 : -1;
        uint64_t d[4], sum = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int digit = 255 - 4 * lane - q;
          d[q] = by_mass ? digit_w[at][digit] : digit_n[at][digit];
          if (digit == tie_digit) d[q] += tie_w;
          sum += d[q];
        }
        uint64_t s = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const uint64_t y = __shfl_up((unsigned long long)s, o, 64);
          if (lane >= o) s += y;
        }
        // (the last digit that has anything, should the total fall short)
        const unsigned long long reach = __ballot(before + s >= want), some = __ballot(sum > 0);
        const int l = reach ? __ffsll(reach) - 1 : some ? 63 - __clzll(some) : 63;
        if (lane == l) {
          uint64_t upto = before + s - sum;
          int q = 0;
          while (q < 3 && upto + d[q] < want) upto += d[q++];
          s_digit = (uint32_t)(255 - 4 * lane - q);
          s_before = upto;
        }
      } else if (tid >= 256 && tid < 512) {
        digit_n[at ^ 1][tid - 256] = 0, digit_w[at ^ 1][tid - 256] = 0;
      }
      __syncthreads();
      prefix = (prefix << 8) | s_digit;
      before = s_before;
    }
    // low halves: those of u ^ 0x80000000 and of ~u with a zero low half
    found = !BF16 ? prefix : prefix << 16 | (prefix >> 15 ? 0 : 0xffffu);
  };
  // sum over the workgroup of f(key, index), over the tokens of interest
  auto sum_of = [&](auto f) {
    uint64_t v = 0, total;
    each([&](uint32_t key, int i) { v += f(key, i); });
    block_scan<T>(v, scan, total);
    return total;
  };

  uint64_t total = cum_w[kBins];
  int bin_k = kBins;
  if (r.k) {
    for (int b = tid; b < kBins; b += T)
      if ((int64_t)cum_n[b] < r.k && r.k <= (int64_t)cum_n[b + 1]) s_bin = b;
    __syncthreads();
    bin_k = s_bin;
    __syncthreads();
    if (bin_k < kBins) {
      const uint64_t need = (uint64_t)r.k - cum_n[bin_k];
      uint64_t before;
      uint32_t found;
      descend(false, bin_k, need, before, found);
      cut = found;
      ties = (int64_t)(need - before);
      const uint64_t above = sum_of([&](uint32_t key, int) -> uint64_t {
        return key > cut && key_bin(key) == bin_k ? mass_of(r, key_value(key)) : 0;
      });
      total = cum_w[bin_k] + above + (uint64_t)ties * mass_of(r, key_value(cut));
    }
  }
  if (r.p < 1.0) {
    const double wanted = r.p * (double)total;
    const uint64_t want = wanted > 1.0 ? (uint64_t)__builtin_ceil(wanted) : 1;
    if (tid == 0) s_bin = kBins - 1;
    __syncthreads();
    for (int b = tid; b < kBins; b += T)
      if (cum_w[b] < want && want <= cum_w[b + 1]) s_bin = b;
    __syncthreads();
    const int bin_p = min(s_bin, bin_k);
    __syncthreads();
    uint64_t before;
    uint32_t found;
    descend(true, bin_p, want - cum_w[bin_p], before, found);
    const uint64_t each_w = mass_of(r, key_value(found)), left = want - cum_w[bin_p] - before;
    const int64_t n = each_w ? (int64_t)((left + each_w - 1) / each_w) : 0;   // tokens of that key it takes to get there
    if (found > cut || n < ties) {
      cut = found;
      ties = n;
    }
  }
  // the index of the last kept token of the cut's key
  int last_tie = INT_MAX;
  if (cut) {
    const uint64_t equal = sum_of([&](uint32_t key, int) -> uint64_t { return key == cut; });
    if (ties < (int64_t)equal) {
      if (tid == 0) s_bin = -1;
      __syncthreads();
      int64_t run = 0;
      const int items = whole ? a.vocab : listed;
      for (int i0 = 0; i0 < items; i0 += T) {
        const int i = i0 + tid;
        bool tie = false;
        int index = 0;
        if (i < items) {
          index = whole ? i : list_idx[i];
          tie = (whole ? order_key(logit_at<BF16>(r, i)) : list_key[i]) == cut;
        }
        const unsigned long long b = __ballot(tie);
        if (lane == 0) scan[wave] = (uint64_t)__popcll(b);
        __syncthreads();
        int64_t rank = run;
        for (int q = 0; q < T / 64; ++q) {
          if (q < wave) rank += (int64_t)scan[q];
          run += (int64_t)scan[q];
        }
        rank += __popcll(b & ((1ull << lane) - 1));
        if (tie && rank == ties - 1) s_bin = index;
        __syncthreads();
        if (run >= ties) break;
      }
      last_tie = s_bin;
    }
  }
  auto kept = [&](uint32_t key, int i) -> uint64_t {
    if (key < cut || (key == cut && i > last_tie)) return 0;
    const uint64_t w = mass_of(r, key_value(key));
    return (double)w >= r.least ? w : 0;
  };

  // kept mass by part: the bins before all cuts (pass 3), the rest token by token
  if (!whole) {
    for (int i = tid; i < listed; i += T) {
      const uint64_t w = kept(list_key[i], list_idx[i]);
      if (w) atomicAdd(&part_w[(list_idx[i] + r.off) / (a.part_vecs * EPV)], (unsigned long long)w);
    }
  } else {
    __syncthreads();
    if (tid < kSampleMaxParts) part_w[tid] = 0;
    __syncthreads();
    for (int p = 0; p < a.parts; ++p) {
      uint64_t w = 0;
      for (int v = tid; v < a.part_vecs; v += T) {
        Vec<BF16> x;
        x.load(r, a.vocab, p * a.part_vecs + v);
#pragma unroll
        for (int i = 0; i < EPV; ++i)
          if (x.in(i, a.vocab)) w += kept(order_key(x.x[i]), x.first + i);
      }
      atomicAdd(&part_w[p], (unsigned long long)w);
    }
  }
  __syncthreads();
  // the part that holds the target, then the token
  if (tid < 64) {
    const uint64_t w = part_w[lane];
    uint64_t s = w;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t y = __shfl_up((unsigned long long)s, o, 64);
      if (lane >= o) s += y;
    }
    const uint64_t all = __shfl((unsigned long long)s, 63, 64);
    // the first sum above the target; with u >= 1 there is none, and the last token with mass is drawn
    const double target = fmax((double)r.u, 0.0) * (double)all;
    const unsigned long long hit = __ballot(w > 0 && ((double)s > target || s == all));
    const int l = __ffsll(hit) - 1;
    if (lane == l) {
      s_bin = l;
      s_before = s - w;
      s_sum = all;
    }
  }
  __syncthreads();
  const int part = s_bin;
  const uint64_t all = s_sum;
  uint64_t run = s_before;
  const double target = fmax((double)r.u, 0.0) * (double)all;
  const int per = (a.part_vecs + T - 1) / T;      // consecutive vectors per thread
  uint64_t mine = 0;
  for (int q = 0; q < per; ++q) {
    const int v = tid * per + q;
    if (v >= a.part_vecs) break;
    Vec<BF16> x;
    x.load(r, a.vocab, part * a.part_vecs + v);
#pragma unroll
    for (int i = 0; i < EPV; ++i)
      if (x.in(i, a.vocab)) mine += kept(order_key(x.x[i]), x.first + i);
  }
  uint64_t part_total;
  run += block_scan<T>(mine, scan, part_total);
  // the first thread whose tokens take the sum beyond the target looks for the one
  if (tid == 0) s_bin = T;
  __syncthreads();
  const bool here = mine && ((double)(run + mine) > target || run + mine == all);
  const unsigned long long hit = __ballot(here);
  if (hit && lane == __ffsll(hit) - 1) atomicMin(&s_bin, tid);
  __syncthreads();
  if (tid == s_bin) {
    for (int q = 0; q < per && s_token == INT_MAX; ++q) {
      const int v = tid * per + q;
      if (v >= a.part_vecs) break;
      Vec<BF16> x;
      x.load(r, a.vocab, part * a.part_vecs + v);
#pragma unroll
      for (int i = 0; i < EPV; ++i) {
        const uint64_t w = x.in(i, a.vocab) ? kept(order_key(x.x[i]), x.first + i) : 0;
        run += w;
        if (w && s_token == INT_MAX && ((double)run > target || run == all)) s_token = x.first + i;
      }
    }
  }
  __syncthreads();
  if (tid == 0) a.out_token[row] = s_token == INT_MAX ? -1 : s_token;
}

template <bool BF16>
hipError_t launch(const SampleArgs &a, hipStream_t stream) {
  const dim3 parts((unsigned)((int64_t)a.rows * a.parts)), block(kThreads);
  hipLaunchKernelGGL(sample_max_kernel<BF16>, parts, block, 0, stream, a);
  hipLaunchKernelGGL(sample_hist_kernel<BF16>, parts, block, 0, stream, a);
  hipLaunchKernelGGL(sample_list_kernel<BF16>, parts, block, 0, stream, a);
  hipLaunchKernelGGL(sample_draw_kernel<BF16>, dim3((unsigned)a.rows), dim3(kDrawThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t stream) {
  return bf16 ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace adaserve
