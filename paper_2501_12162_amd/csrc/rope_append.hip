// Rotary position embedding of queries and keys, and the append of keys and
// values to the paged cache, on gfx950: what precedes attention in a decoder
// layer, as one pass over the projection's output.
//
// Pair (x1, x2) of a head at position p turns by the angle p f_i:
//   y1 = x1 cos - x2 sin,  y2 = x1 sin + x2 cos.
// p f_i is exact in fp64 (an integer below 2^29 times a 24-bit float) and is
// reduced to a part of a turn there, since fp32 would lose 6e-3 rad of it at
// position 10^5; sine and cosine of the rest are fp32, and so is the turn,
// rounded once to the output type.
//
// Bound by memory: every row is read once and written once (keys a second
// time where k_out is asked for).  A workgroup takes one token: its first wave
// puts the token's sines and cosines into LDS, one angle per lane (every thread
// computing those of its own columns would repeat each once per head, as much
// time as the copy takes), then all move 16-byte pieces, both halves of a pair in
// one thread, so that the outputs may be the inputs.  (Four tokens to a workgroup,
// a wave for the angles of each: 54.5 instead of 48 us on the 9611 tokens below, 9.1
// instead of 6.7 on 1023.)
//
// Measured, bf16, D = 128, 32 + 8 + 8 heads: 9.6 thousand tokens of 8 prompts, 236 MB
// read and written, 48 us, 4.9 TB/s, with inputs that no cache holds (a device
// copy of 1 GiB runs at 5.0), 37 us when the caches hold some of them; 40 thousand
// tokens 5.1 TB/s.  fp32: 92 us, 5.1 TB/s.  One token: 4.1 us in a graph.  Few heads
// leave most of a workgroup without a piece: 8 + 2 + 2 heads 18.5 us, 3.2 TB/s, 4 + 2 + 2 of
// D = 64 16 us, 1.2 TB/s.
#include "device_common.h"
#include "plan.h"
#include "serving.h"

namespace adaserve {

namespace {

constexpr int kThreads = kServingThreads;

// The request that owns token t: the last r with indptr[r] <= t, by the whole
// wave (64 entries per round of loads).  -1 when t is in no request.
__device__ __forceinline__ int find_request(const int32_t *indptr, int B, int32_t t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B + 1;        // the answer + 1 lies in [lo, lo + n]
  while (n > 64) {
    const int step = (n + 63) / 64;
    const int i = lo + lane * step;
    const bool le = lane * step < n && indptr[i] <= t;
    const int c = __popcll(__ballot(le));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    n = min(step, B + 1 - lo);
  }
  const bool le = lane < n && indptr[lo + lane] <= t;
  const int r = lo + __popcll(__ballot(le)) - 1;
  if (r < 0 || r >= B) return -1;
  return indptr[r] <= t && t < indptr[r + 1] ? r : -1;
}

template <bool BF16>
__device__ __forceinline__ void turn(u32x4 &a, u32x4 &b, const float2 *cs) {
  // elements of a and b with equal index are the pairs
  if constexpr (BF16) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a0 = __uint_as_float(a[w] << 16), a1 = __uint_as_float(a[w] & 0xffff0000u);
      const float b0 = __uint_as_float(b[w] << 16), b1 = __uint_as_float(b[w] & 0xffff0000u);
      const float2 t0 = cs[2 * w], t1 = cs[2 * w + 1];
      a[w] = pack_bf16x2(__builtin_fmaf(a0, t0.x, -(b0 * t0.y)), __builtin_fmaf(a1, t1.x, -(b1 * t1.y)));
      b[w] = pack_bf16x2(__builtin_fmaf(a0, t0.y, b0 * t0.x), __builtin_fmaf(a1, t1.y, b1 * t1.x));
    }
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float x = __uint_as_float(a[w]), y = __uint_as_float(b[w]);
      a[w] = __float_as_uint(__builtin_fmaf(x, cs[w].x, -(y * cs[w].y)));
      b[w] = __float_as_uint(__builtin_fmaf(x, cs[w].y, y * cs[w].x));
    }
  }
}

template <bool BF16>
__device__ __forceinline__ void turn_neighbours(u32x4 &a, const float2 *cs) {
  // elements 2i and 2i + 1 of a are the pairs
  if constexpr (BF16) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float x = __uint_as_float(a[w] << 16), y = __uint_as_float(a[w] & 0xffff0000u);
      a[w] = pack_bf16x2(__builtin_fmaf(x, cs[w].x, -(y * cs[w].y)), __builtin_fmaf(x, cs[w].y, y * cs[w].x));
    }
  } else {
#pragma unroll
    for (int w = 0; w < 4; w += 2) {
      const float x = __uint_as_float(a[w]), y = __uint_as_float(a[w + 1]);
      a[w] = __float_as_uint(__builtin_fmaf(x, cs[w / 2].x, -(y * cs[w / 2].y)));
      a[w + 1] = __float_as_uint(__builtin_fmaf(x, cs[w / 2].y, y * cs[w / 2].x));
    }
  }
}

// Workgroups 0 .. tokens - 1 take a token each, the others four requests each,
// whose new lengths they write.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(RopeAppendArgs a, int32_t tokens) {
  constexpr int EPV = BF16 ? 8 : 4;
  constexpr int ESZ = BF16 ? 2 : 4;
  __shared__ float2 cs[kRopeMaxHeadDim / 2];
  __shared__ int64_t page_row;   // row (page, head 0, slot) of the pools, or -1
  __shared__ int32_t owner;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  if ((int64_t)blockIdx.x >= tokens) {
    // new lengths: a request grows by its leading rows whose page exists
    const int64_t r = ((int64_t)blockIdx.x - tokens) * 4 + wave;
    if (r >= a.num_requests) return;
    const int32_t L = a.prefix_len[r];
    const int64_t begin = max(a.token_indptr[r], 0), end = min(a.token_indptr[r + 1], a.num_tokens);
    int64_t n = L >= 0 ? max(end - begin, (int64_t)0) : 0;
    if (n > 0) {
      const int64_t e0 = L / a.page_size, e1 = (L + n - 1) / a.page_size;
      for (int64_t e = e0; e <= e1; e += 64) {
        const int64_t mine = e + lane;
        bool bad = false;
        if (mine <= e1) {
          const int32_t p = mine < a.bt_stride ? a.block_table[r * a.bt_stride + mine] : -1;
          bad = p < 0 || p >= a.num_pages;
        }
        const unsigned long long hit = __ballot(bad);
        if (hit) {
          n = max((e + __ffsll(hit) - 1) * a.page_size - L, (int64_t)0);
          break;
        }
      }
    }
    // cache lengths are int32: the rows of a table never reach past 2^31 - 1
    if (lane == 0) a.new_prefix_len[r] = (int32_t)min((int64_t)L + n, (int64_t)INT32_MAX);
    return;
  }

  const int64_t t = blockIdx.x;
  // its request, position and page
  if (wave == 0) {
    const int r = find_request(a.token_indptr, a.num_requests, (int32_t)t);
    int64_t place = 0, row = -1;
    if (r >= 0) {
      const int32_t L = a.prefix_len[r];
      place = (int64_t)L + (t - a.token_indptr[r]);
      if (a.k_pages && L >= 0) {
        const int64_t e = place / a.page_size;
        const int32_t p = e < a.bt_stride ? a.block_table[(int64_t)r * a.bt_stride + e] : -1;
        if (p >= 0 && p < a.num_pages)
          row = (int64_t)p * a.num_kv_heads * a.page_size + (place - e * a.page_size);
      }
      const int64_t pos = a.positions ? a.positions[t] : place;
      for (int i = lane; i < a.rotary_dim / 2; i += 64) {
        const double turns = (double)pos * (double)a.inv_freq[i] * 0.15915494309189533577;
        float s, c;
        sincospif((float)(2.0 * (turns - __builtin_rint(turns))), &s, &c);
        cs[i] = make_float2(c, s);
      }
    }
    if (lane == 0) {
      owner = r;
      page_row = row;
    }
  }
  __syncthreads();
  if (owner < 0) return;
  const int64_t place_row = page_row;

  // rotated heads: `pairs` pieces of two vectors each, then the vectors past
  // the rotated part, all of one head by neighbouring threads
  const int vecs = a.head_dim / EPV, half = a.rotary_dim / (2 * EPV);
  const int pieces = vecs - half;
  const int hk = a.num_q_heads + a.num_kv_heads;
  const uint32_t items = (uint32_t)hk * pieces;
  const int64_t D = a.head_dim;
  for (uint32_t w = tid; w < items; w += kThreads) {
    const int h = (int)(w / (uint32_t)pieces);
    const int j = (int)w - h * pieces;
    const bool is_q = h < a.num_q_heads;
    const int g = is_q ? h : h - a.num_q_heads;
    const char *src = is_q ? (const char *)a.q + (t * a.q_stride + (int64_t)g * D) * ESZ
                           : (const char *)a.k + (t * a.k_stride + (int64_t)g * D) * ESZ;
    char *dst = is_q ? (char *)a.q_out : (char *)a.k_out;
    if (dst) dst += (t * (is_q ? a.num_q_heads : a.num_kv_heads) + g) * D * ESZ;
    char *page = !is_q && place_row >= 0 ? (char *)a.k_pages + (place_row + (int64_t)g * a.page_size) * D * ESZ : nullptr;
    if (j < half) {
      u32x4 x = *(const u32x4 *)(src + j * 16), y = *(const u32x4 *)(src + (j + half) * 16);
      if (a.interleaved) {
        turn_neighbours<BF16>(x, &cs[j * (EPV / 2)]);
        turn_neighbours<BF16>(y, &cs[(j + half) * (EPV / 2)]);
      } else {
        turn<BF16>(x, y, &cs[j * EPV]);
      }
      if (dst) {
        *(u32x4 *)(dst + j * 16) = x;
        *(u32x4 *)(dst + (j + half) * 16) = y;
      }
      if (page) {
        *(u32x4 *)(page + j * 16) = x;
        *(u32x4 *)(page + (j + half) * 16) = y;
      }
    } else {
      const u32x4 x = *(const u32x4 *)(src + (j + half) * 16);
      if (dst) *(u32x4 *)(dst + (j + half) * 16) = x;
      if (page) *(u32x4 *)(page + (j + half) * 16) = x;
    }
  }
  if (!a.v_pages || place_row < 0) return;
  const uint32_t vitems = (uint32_t)a.num_kv_heads * vecs;
  for (uint32_t w = tid; w < vitems; w += kThreads) {
    const int g = (int)(w / (uint32_t)vecs);
    const int j = (int)w - g * vecs;
    const char *src = (const char *)a.v + (t * a.v_stride + (int64_t)g * D) * ESZ;
    *(u32x4 *)((char *)a.v_pages + (place_row + (int64_t)g * a.page_size) * D * ESZ + j * 16) = *(const u32x4 *)(src + j * 16);
  }
}

}  // namespace

hipError_t launch_rope_append(const RopeAppendArgs &a, bool bf16, hipStream_t stream) {
  const int64_t length_blocks = a.new_prefix_len ? rope_length_blocks(a.num_requests) : 0;
  const bool in_place = a.new_prefix_len && a.new_prefix_len == a.prefix_len;
  auto run = [&](int32_t tokens, int64_t blocks) {
    if (blocks == 0) return hipSuccess;
    if (bf16) hipLaunchKernelGGL(rope_append_kernel<true>, dim3((unsigned)blocks), dim3(kThreads), 0, stream, a, tokens);
    else hipLaunchKernelGGL(rope_append_kernel<false>, dim3((unsigned)blocks), dim3(kThreads), 0, stream, a, tokens);
    return hipGetLastError();
  };
  // lengths written over those that the tokens read wait for a launch of their own
  if (!in_place) return run(a.num_tokens, a.num_tokens + length_blocks);
  const hipError_t e = run(a.num_tokens, a.num_tokens);
  return e != hipSuccess ? e : run(0, length_blocks);
}

}  // namespace adaserve
