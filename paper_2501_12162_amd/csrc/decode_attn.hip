// Attention of one new token per request over its paged cache on gfx950.
//
// The batch's 32-key blocks, request after request, are dealt in equal and
// contiguous shares to as many workgroups per kv-head as the device holds, so
// that all end together whatever the lengths; a workgroup goes from request to
// request, with all query heads of its kv-head as rows, and the runs of a request
// that lies in several shares are joined by a second launch.  The lengths are
// read on the device only: every workgroup finds its share from all of them
// (schedule()), so a captured launch follows them.
//
// Bound by memory: 2 c Hkv D s bytes per request against 4 c Hq D flops.  So
// everything serves to keep loads in flight: no LDS in the loop and no
// barrier; each of a workgroup's four waves walks its own blocks with K and V
// straight in registers, 16 KB of them in flight per wave.
//  * S^T = K Q^T on the matrix cores (16 keys x 16 rows; K as it lies in
//    memory is the A operand, lanes without a row multiply zeros).  A lane then
//    holds 4 keys of each 16 and one row: what P^T as a B operand wants.
//  * O^T += V^T P^T on the matrix cores, too.  A contraction may take its slots
//    in any order and a tile its rows: the lane that holds the weights of 4 keys
//    loads D / 16 columns of those keys' values, and tile c of O^T is column c
//    of each lane's.  fp32 values are operands as they are loaded; of bf16 ones
//    two neighbouring keys are put into a word (one v_perm per pair).  (On the
//    vector ALUs, with a broadcast of every weight, 8 rows took as long as their
//    loads.)
//  * for bf16 values a weight goes into the product as the sum of two bf16 parts,
//    which holds 16 bits of it: the matrix cores wait for memory anyway (with the
//    first part alone the times are the same and the error against fp64 0.0021
//    instead of the output rounding's 0.0017).
//  * exponentials are 2^x of scores in log2 units; the running maximum moves
//    only when it is exceeded by 2^8, which spares the rescaling of the output.
//
// Measured, bf16, D = 128 (a kernel that only reads gets 7.0 TB/s): 64 requests
// of up to 4096 tokens, 64 on 8 heads, 668 MB: 111 us, 6.0 TB/s; 8 requests of
// 32768 tokens, 32 on 8 heads, 1074 MB: 164 us, 6.5 TB/s; one of 1500 tokens: 6.4
// us and 3.2 for the join.  fp32: 32 of the 64 requests 93 us, 5.8 TB/s, 4 of the 8
// 165 us, 6.5 TB/s.  With a unit per run of a request, two rounds of them,
// the first two took 124 and 169 us; with three workgroups per CU (168 registers,
// 8 of them spilled) 130 and 185.  Loading a run's first block before the end of
// the run before gains nothing: 111 and 166.
//
// Over a window and sinks (WINDOW) the shares are of the blocks that are read, the sinks' and
// the window's, numbered through.  64 requests of up to 16384 tokens over 2048, 64 on 8
// heads, 530 MB: 86 us and 5 for the join; one of 20001 over 4096: 8.3 and 3.7.  In fp32 the
// same 64, 1.06 GB: 172 us with the join.
#include <float.h>

#include <type_traits>

#include "device_common.h"
#include "plan.h"
#include "serving.h"

namespace adaserve {

namespace {

constexpr int kThreads = kServingThreads;
constexpr int kWaves = kThreads / 64;
constexpr float kLowest = -FLT_MAX;     // running maximum before any key
constexpr float kRescaleLog2 = 8.f;
constexpr int kPagesPerBlock = kKeysPerBlock / kPageSize;

// The batch's 32-key blocks in one line, request after request; unit u takes
// blocks [lo, hi) of it.
struct DecodeUnit {
  int32_t lo, hi;
  int32_t first;    // first request with a block in it, or an empty one that it owns
  int32_t per;      // blocks per unit
  bool last;        // of the units with work: it owns the empty requests at the end
};

__device__ __forceinline__ int32_t decode_blocks(int32_t len) { return len > 0 ? (len + kKeysPerBlock - 1) / kKeysPerBlock : 0; }

// Over a window: the keys of a request of `len` that are read, numbered through
// (WindowSpan).
template <bool WINDOW>
__device__ __forceinline__ int32_t decode_len(const PagedAttnArgs &a, int32_t len) {
  if (!WINDOW || len <= 0) return len;
  return len - window_span(len - a.window, a.sinks, kKeysPerBlock).shift * kKeysPerBlock;
}

// Unit u, from all lengths: every unit has `per` blocks but for the last one.
// Each thread takes 1 to 4 neighbouring requests (at most kDecodeSplitRequests
// in all); start[] gets each request's first block, len[] its length (-1: out of
// range).  False: no such unit.
template <bool WINDOW>
__device__ __forceinline__ bool schedule(const PagedAttnArgs &a, int32_t u, int32_t *start, int32_t *len, DecodeUnit &un) {
  __shared__ int32_t part[2][kWaves];
  __shared__ int32_t first;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per_thread = (a.num_requests + kThreads - 1) / kThreads;
  int32_t nb[4], mine = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = tid * per_thread + i;
    nb[i] = 0;
    if (i < per_thread && r < a.num_requests) {
      const int32_t x = a.context_len[r], ok = x >= 0 && x <= a.max_context ? x : -1;
      len[r] = ok;
      nb[i] = decode_blocks(decode_len<WINDOW>(a, ok));
    }
    mine += nb[i];
  }
  // the sum over the threads before, and over all
  auto scan = [&](int32_t *parts, int32_t x, int32_t &total) {
    int32_t upto = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int32_t o = __shfl_up(upto, off, 64);
      if (lane >= off) upto += o;
    }
    if (lane == 63) parts[wave] = upto;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) upto += parts[w];
      total += parts[w];
    }
    return upto - x;
  };
  int32_t total, at = scan(part[0], mine, total);
  un.per = max(a.min_blocks, (total + a.units_per_head - 1) / a.units_per_head);
  // Where there are units for it every request begins with one of its own: a unit
  // of two requests takes their runs one after the other (4 requests of 1500
  // tokens, which do not fill the device: 14.3 -> 13.0 us; finding out costs 0.3
  // to 0.5 us, so it is asked only where there are two units per request).
  int32_t step = 1;   // requests begin at multiples of it
  if (a.num_requests > 1 && 2 * a.num_requests <= a.units_per_head) {
    int32_t apart = 0, all;
#pragma unroll
    for (int i = 0; i < 4; ++i) apart += (nb[i] + un.per - 1) / un.per * un.per;
    const int32_t from = scan(part[1], apart, all);
    if (all <= a.units_per_head * un.per) {
      step = un.per;
      at = from;
      total = all;
    }
  }
  auto space = [&](int32_t n) { return (n + step - 1) / step * step; };
  const int32_t units = max(1, (total + un.per - 1) / un.per);
  if (u >= units) return false;
  un.lo = u * un.per;
  un.hi = min(total, un.lo + un.per);
  un.last = u == units - 1;
  // `first`: the one request that is the unit's where the one before is not.  A
  // request with blocks is if it ends behind lo, an empty one from lo on.
  auto is_in = [&](int32_t from, int32_t n) { return n > 0 ? from + n > un.lo : from >= un.lo; };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = tid * per_thread + i;
    if (i < per_thread && r < a.num_requests) {
      start[r] = at;
      if (is_in(at, nb[i])) {
        // (the request before: its space ends at `at`)
        bool before = false;
        if (i > 0) before = is_in(at - space(nb[i - 1]), nb[i - 1]);
        else if (r > 0) {
          const int32_t x = a.context_len[r - 1], n = decode_blocks(decode_len<WINDOW>(a, x <= a.max_context ? x : -1));
          before = is_in(at - space(n), n);
        }
        if (!before) first = r;
      }
      at += space(nb[i]);
    }
  }
  __syncthreads();
  un.first = __builtin_amdgcn_readfirstlane(first);
  return true;
}

// A run of a request's keys.
struct Run {
  int32_t r;
  int32_t k0, k1;     // its keys
  int32_t nb, mine;   // blocks of the wave's size; this wave's: wave, wave + 4, ...
  int32_t slot;       // of the workspace: 2 u + 1 where it begins a request, 2 u where it goes on with one; -1: all of it
  WindowSpan span;    // over a window: where the keys stand in the cache,
  int32_t lo;         // and the window's first one: those from the sinks to it are not seen
};

template <bool BF16, int D, bool WINDOW>
__global__ __launch_bounds__(kThreads, 2) void decode_attn_kernel(PagedAttnArgs a) {
  constexpr int T = BF16 ? 2 : 1;          // 16-key tiles (pages) per block of a wave
  constexpr int KB = T * 16;
  constexpr int EPL = D / 16;              // columns of a lane, tiles of O^T
  constexpr int ESZ = BF16 ? 2 : 4;
  constexpr int NK = D * ESZ / 64;         // 16-byte K loads per lane and tile
  constexpr int LDO = D + 4;
  __shared__ __align__(16) float mo[kWaves][kDecodeRows][LDO];
  __shared__ float mw[kWaves][kDecodeRows], lw[kWaves][kDecodeRows];

  __shared__ int32_t start[kDecodeSplitRequests], lens[kDecodeSplitRequests];
  const int32_t u = (int32_t)(blockIdx.x / a.num_kv_heads);
  const int g = (int)(blockIdx.x - (int64_t)u * a.num_kv_heads);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int quad = lane >> 4, j = lane & 15;
  const int rows = a.group;
  const bool split = a.ws_request != nullptr;
  DecodeUnit un{0, INT32_MAX, u, 0, false};
  if (split && !schedule<WINDOW>(a, u, start, lens, un)) return;

  // The unit's run of request r or of the first one after it that has keys
  // there; the rows of the empty requests on the way become zeros, of lengths
  // out of range NaN.  False: no more.
  auto find_run = [&](int32_t r, Run &run) {
    for (; r < (split ? a.num_requests : u + 1); ++r) {
      int32_t len, from = 0;
      if (split) {
        from = __builtin_amdgcn_readfirstlane(start[r]);
        len = __builtin_amdgcn_readfirstlane(lens[r]);
        if (from >= un.hi && !un.last) return false;
      } else {
        len = a.context_len[r];
        if (len > a.max_context) len = -1;
      }
      if (len <= 0) {
        const float x = len < 0 ? __builtin_nanf("") : 0.f;
        const int64_t at = ((int64_t)r * a.num_q_heads + (int64_t)g * rows) * D;
        for (int i = tid; i < rows * D; i += kThreads) {
          if (BF16) ((__bf16 *)a.out)[at + i] = (__bf16)x;
          else ((float *)a.out)[at + i] = x;
        }
        continue;
      }
      if (WINDOW) {
        const int32_t first = len - a.window;
        run.span = window_span(first, a.sinks, kKeysPerBlock);
        run.lo = first - run.span.shift * kKeysPerBlock;
        len -= run.span.shift * kKeysPerBlock;
      }
      const int32_t end = from + decode_blocks(len);
      const int32_t b0 = max(from, un.lo), b1 = min(end, un.hi);
      run.r = r;
      run.k0 = (b0 - from) * kKeysPerBlock;
      run.k1 = min(len, (b1 - from) * kKeysPerBlock);
      run.nb = (run.k1 - run.k0 + KB - 1) / KB;
      run.mine = run.nb > wave ? (run.nb - wave + kWaves - 1) / kWaves : 0;
      run.slot = b0 > from ? 2 * u : b1 < end ? 2 * u + 1 : -1;
      // the request's units, for the join
      if (split && b0 == from && g == 0 && tid == 0) {
        a.ws_request[2 * r] = u;
        a.ws_request[2 * r + 1] = (end - 1) / un.per - u + 1;
      }
      return true;
    }
    return false;
  };
  Run run, next;
  if (!find_run(un.first, run)) return;

  // page ids: lane i holds that of tile i of this wave's blocks, 64 tiles at a time
  int32_t pages, page_base = 0;
  auto page_ids = [&](const Run &w, int base) -> int32_t {
    const int i = base + lane;                       // tile of the wave
    const int32_t b = wave + (i / T) * kWaves;
    int32_t e = (w.k0 + b * KB) / kPageSize + i % T;
    int32_t p = -1;
    const bool inside = b < w.nb && e * kPageSize < w.k1;
    if (WINDOW) e = w.span.real(e / kPagesPerBlock) * kPagesPerBlock + e % kPagesPerBlock;
    if (inside && e < a.bt_stride) {
      p = a.block_table[(int64_t)w.r * a.bt_stride + e];
      if (p < 0 || p >= a.num_pages) p = -1;
    }
    return p;
  };
  pages = page_ids(run, 0);

  // query rows as the B operand: lane holds row j (none: zeros)
  u32x4 qf[NK];
  auto load_q = [&](int32_t r) {
    const char *qp = (const char *)a.q + ((int64_t)r * a.q_stride + ((int64_t)g * rows + (j < rows ? j : 0)) * D) * ESZ;
#pragma unroll
    for (int c = 0; c < NK; ++c) {
      u32x4 v = *(const u32x4 *)(qp + c * 64 + quad * 16);
      qf[c] = j < rows ? v : u32x4{0, 0, 0, 0};
    }
  };
  load_q(run.r);

  const int64_t page_bytes = (int64_t)a.num_kv_heads * kPageSize * D * ESZ;
  const int64_t head_bytes = (int64_t)g * kPageSize * D * ESZ;
  u32x4 kr[T][NK];
  constexpr int NV = EPL * ESZ / 4;        // 32-bit words of a lane's V slice: 4 or 2 (bf16), 8 or 4 (fp32)
  uint32_t vr[T][4][NV];
  bool have[T];                            // the tile's page exists (of the tiles in kr)
  bool have_v[T];
  auto page_of = [&](int i, int t) { return __builtin_amdgcn_readlane(pages, i * T + t - page_base); };
  // (nothing reads them again: past the caches)
  auto load16 = [&](const char *p) -> u32x4 { return __builtin_nontemporal_load((const u32x4 *)p); };
  auto load8 = [&](const char *p) -> u32x2 { return __builtin_nontemporal_load((const u32x2 *)p); };
  // A missing page reads page 0 (its values are not used): no branch around the loads.
  auto load_k = [&](int i) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int32_t p = page_of(i, t);
      have[t] = p >= 0;
      const char *base = (const char *)a.k_pages + max(p, 0) * page_bytes + head_bytes + j * D * ESZ + quad * 16;
#pragma unroll
      for (int c = 0; c < NK; ++c) kr[t][c] = load16(base + c * 64);
    }
  };
  auto load_v = [&](int i) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int32_t p = page_of(i, t);
      have_v[t] = p >= 0;
      const char *base = (const char *)a.v_pages + max(p, 0) * page_bytes + head_bytes + (quad * 4) * D * ESZ + j * (BF16 ? EPL * 2 : 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (NV == 2) {
          const u32x2 x = load8(base + e * D * ESZ);
          vr[t][e][0] = x[0], vr[t][e][1] = x[1];
        } else {
#pragma unroll
          for (int w = 0; w < NV; w += 4) {
            const u32x4 x = load16(base + e * D * ESZ + (w / 4) * 256);
            vr[t][e][w] = x[0], vr[t][e][w + 1] = x[1], vr[t][e][w + 2] = x[2], vr[t][e][w + 3] = x[3];
          }
        }
      }
    }
  };

  // O^T, row j of the queries: bf16: tile c, element i is column (4 quad + i) EPL + c;
  // fp32: tile 4 h + k, element i is column 64 h + 16 quad + 4 i + k
  f32x4 o[EPL];
  float m, l;   // of row j: the reference in log2 units; this lane's part of the sum
  auto block = [&](int i, auto last) __attribute__((always_inline)) {
    constexpr bool kMore = !decltype(last)::value;
    f32x4 s[T];
    bool hk[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      hk[t] = have[t];
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        if constexpr (BF16) {
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[t][c]),
                                                         __builtin_bit_cast(bf16x8, qf[c]), s[t], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[t][c][e]), __uint_as_float(qf[c][e]), s[t], 0, 0, 0);
        }
      }
    }
    if constexpr (kMore) {
      if ((i + 2) * T - page_base > 64) {
        page_base = (i + 1) * T;
        pages = page_ids(run, page_base);
      }
      load_k(i + 1);
    }
    // s[t][e]: key 16 t + 4 quad + e of the block, row j
    const int32_t left = run.k1 - (run.k0 + (wave + i * kWaves) * KB);   // keys of the block and after
    float p[T][4];
    float bm = kLowest;
    // over a window: the block's keys [cut0, cut1) are not seen
    const int32_t cut0 = WINDOW ? left - run.k1 + a.sinks : 0, cut1 = WINDOW ? left - run.k1 + run.lo : 0;
    const bool edge = left < KB || (WINDOW && cut0 < KB && cut1 > 0);
    auto unseen = [&](int key) { return key >= left || (WINDOW && key >= cut0 && key < cut1); };
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = hk[t] ? s[t][e] * a.scale_log2 : 0.f;
        p[t][e] = !edge || !unseen(t * 16 + quad * 4 + e) ? x : -INFINITY;
        bm = fmaxf(bm, p[t][e]);
      }
    bm = fmaxf(bm, __shfl_xor(bm, 16, 64));
    bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
    const bool up = bm > m + kRescaleLog2 || (m == kLowest && bm > m);
    if (__any(up)) {
      const float mn = up ? bm : m;
      const float al = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= al;
#pragma unroll
      for (int c = 0; c < EPL; ++c) o[c] *= al;
    }
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[t][e] = __builtin_amdgcn_exp2f(p[t][e] - m);
        l += p[t][e];
      }
    // a slot past the run's keys may hold anything
#pragma unroll
    for (int t = 0; t < T; ++t)
      if (edge || !have_v[t]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!have_v[t] || unseen(t * 16 + quad * 4 + e))
#pragma unroll
            for (int w = 0; w < NV; ++w) vr[t][e][w] = 0;
      }
    if constexpr (BF16) {
      // weights as the sum of two bf16 parts
      u32x4 w0, w1;
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const uint32_t x = pack_bf16x2(p[t][e], p[t][e + 1]);
          w0[t * 2 + e / 2] = x;
          w1[t * 2 + e / 2] = pack_bf16x2(p[t][e] - __uint_as_float(x << 16), p[t][e + 1] - __uint_as_float(x & 0xffff0000u));
        }
      const bf16x8 p0 = __builtin_bit_cast(bf16x8, w0), p1 = __builtin_bit_cast(bf16x8, w1);
#pragma unroll
      for (int w = 0; w < NV; ++w) {
        u32x4 lo, hi;
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            lo[t * 2 + e / 2] = __builtin_amdgcn_perm(vr[t][e + 1][w], vr[t][e][w], 0x05040100u);
            hi[t * 2 + e / 2] = __builtin_amdgcn_perm(vr[t][e + 1][w], vr[t][e][w], 0x07060302u);
          }
        o[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), p0, o[2 * w], 0, 0, 0);
        o[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), p0, o[2 * w + 1], 0, 0, 0);
        o[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), p1, o[2 * w], 0, 0, 0);
        o[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), p1, o[2 * w + 1], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int w = 0; w < NV; ++w)
          o[w] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[0][e][w]), p[0][e], o[w], 0, 0, 0);
    }
    if constexpr (kMore) load_v(i + 1);
  };

#pragma unroll 1
  for (;;) {
    if (run.mine > 0) {
      load_k(0);
      load_v(0);
    }
    // the next run and its page ids, before they are used
    const bool more = split && find_run(run.r + 1, next);
    int32_t next_pages = -1;
    if (more) next_pages = page_ids(next, 0);
    m = kLowest;
    l = 0.f;
#pragma unroll
    for (int c = 0; c < EPL; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int i = 0; i < run.mine - 1; ++i) block(i, std::false_type{});
    if (run.mine > 0) block(run.mine - 1, std::true_type{});

    // the four waves
    l = sum_over_lane_rows(l);
    __syncthreads();   // (the run before is read)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < EPL; c += 4)
        *(f32x4 *)&mo[wave][j][BF16 ? (4 * quad + i) * EPL + c : c * 16 + 16 * quad + 4 * i] =
            f32x4{o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]};
    if (quad == 0) {
      mw[wave][j] = m;
      lw[wave][j] = l;
    }
    __syncthreads();
    const int64_t out_row = (int64_t)run.r * a.num_q_heads + (int64_t)g * rows;
    const int64_t slot = (int64_t)run.slot * a.num_q_heads + (int64_t)g * rows;
#pragma unroll 1
    for (int it = tid; it < rows * D; it += kThreads) {
      const int i = it / D, c = it % D;
      float mm = mw[0][i];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, mw[w][i]);
      float den = 0.f, num = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(mw[w][i] - mm);
        den = __builtin_fmaf(f, lw[w][i], den);
        num = __builtin_fmaf(f, mo[w][i][c], num);
      }
      if (run.slot < 0) {
        const float x = num / den;
        if (BF16) ((__bf16 *)a.out)[out_row * D + it] = (__bf16)x;
        else ((float *)a.out)[out_row * D + it] = x;
      } else {
        a.ws_o[(slot + i) * D + c] = num;
        if (c == 0) *(f32x2 *)(a.ws_ml + (slot + i) * 2) = f32x2{mm, den};
      }
    }
    if (!more) return;
    run = next;
    pages = next_pages;
    page_base = 0;
    load_q(run.r);
  }
}

// Joins the runs of a request's row: with reference m over the runs' m_c,
// out = sum 2^(m_c - m) o_c / sum 2^(m_c - m) l_c.  One workgroup per row, its
// four waves taking every fourth run, eight of them in flight (47 runs of a request
// of 6000 tokens: 6.7 -> 3.7 us).
template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void decode_join_kernel(PagedAttnArgs a) {
  constexpr int EPL = D / 64;
  __shared__ float so[kWaves][D], sm[kWaves], sl[kWaves];
  const int64_t row = blockIdx.x;
  const int r = (int)(row / a.num_q_heads), h = (int)(row - (int64_t)r * a.num_q_heads);
  // (in flight together; of a request without keys the second is not written)
  const int32_t len = a.context_len[r], first = a.ws_request[2 * r], chunks = a.ws_request[2 * r + 1];
  if (len <= 0 || len > a.max_context || chunks <= 1) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float m = kLowest, m_sum = kLowest, l = 0.f, o[EPL] = {};
  constexpr int kRuns = 8;   // in flight
  for (int c0 = wave; c0 < chunks; c0 += kRuns * kWaves) {
    f32x2 ml[kRuns];
    float x[kRuns][EPL];
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int c = __builtin_amdgcn_readfirstlane(c0 + i * kWaves);
      ml[i] = f32x2{kLowest, 0.f};
#pragma unroll
      for (int e = 0; e < EPL; ++e) x[i][e] = 0.f;
      if (c < chunks) {
        const int64_t slot = (int64_t)(2 * (first + c) + (c == 0)) * a.num_q_heads + h;
        ml[i] = *(const f32x2 *)(a.ws_ml + slot * 2);
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[i][e] = a.ws_o[slot * D + lane * EPL + e];
      }
    }
#pragma unroll
    for (int i = 0; i < kRuns; ++i) m = fmaxf(m, ml[i][0]);
    // (the sums so far have reference m_sum)
    const float f = __builtin_amdgcn_exp2f(m_sum - m);
    m_sum = m;
    l *= f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[e] *= f;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const float w = __builtin_amdgcn_exp2f(ml[i][0] - m);
      l = __builtin_fmaf(w, ml[i][1], l);
#pragma unroll
      for (int e = 0; e < EPL; ++e) o[e] = __builtin_fmaf(w, x[i][e], o[e]);
    }
  }
  if (lane == 0) sm[wave] = m, sl[wave] = l;
#pragma unroll
  for (int e = 0; e < EPL; ++e) so[wave][lane * EPL + e] = o[e];
  __syncthreads();
  const int c = threadIdx.x;
  if (c >= D) return;
  float mm = sm[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, sm[w]);
  float den = 0.f, num = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float f = __builtin_amdgcn_exp2f(sm[w] - mm);
    den = __builtin_fmaf(f, sl[w], den);
    num = __builtin_fmaf(f, so[w][c], num);
  }
  const float x = num / den;
  if (BF16) ((__bf16 *)a.out)[row * D + c] = (__bf16)x;
  else ((float *)a.out)[row * D + c] = x;
}

template <bool BF16, int D>
hipError_t launch(const PagedAttnArgs &a, hipStream_t stream) {
  const int64_t blocks = (int64_t)a.units_per_head * a.num_kv_heads;
  if (a.window) hipLaunchKernelGGL((decode_attn_kernel<BF16, D, true>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((decode_attn_kernel<BF16, D, false>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.ws_request) return e;
  hipLaunchKernelGGL((decode_join_kernel<BF16, D>), dim3((unsigned)((int64_t)a.num_requests * a.num_q_heads)),
                     dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decode_attn(const PagedAttnArgs &a, int head_dim, bool bf16, hipStream_t stream) {
  if (bf16) return head_dim == 128 ? launch<true, 128>(a, stream) : launch<true, 64>(a, stream);
  return head_dim == 128 ? launch<false, 128>(a, stream) : launch<false, 64>(a, stream);
}

}  // namespace adaserve
