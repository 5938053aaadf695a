// Causal attention of packed prompts over the paged cache on gfx950: row i of
// a request's n tokens stands at position c - n + i of its c cached keys and
// sees the keys up to itself.
//
//   o_i = sum_k w_ik v_k / sum_k w_ik,  w_ik = 2^(c (q_i k_k - m_i)),  c = scale log2 e
// in one pass over the keys; m_i is any reference that keeps the weights in
// range, and cancels.
//
// Bound by the matrix cores: 4 D flops per (row, key) pair, and a key is read
// from memory once per 256 rows, from LDS once per 64.  The rows of a kv-head's
// query heads share its keys, so a tile is 256 / G tokens with all G heads.  S is
// taken transposed (keys by rows): a lane then holds 16 keys of one row, the sum
// of its weights stays in the lane, and P^T is the B operand of O^T = V^T P^T
// after one exchange of halves.  Weights are rounded to bf16 for that product (the
// output is, too); their sum is of the unrounded ones.
//
// Measured, bf16, D = 128, 32 heads on 8: one prompt of 8191 tokens 449 - 468 us
// (over cards), 1.17 - 1.22 PFLOP/s of the pairs seen (a library product of 8192 x 8192
// x 8192 runs at 1.16); 16 ragged prompts of 512 - 2048 tokens 354 - 369 us, 0.83 - 0.87
// PFLOP/s: a tile's start, masked end and output take 8 us, as long as 300 keys of
// the loop and a quarter of the whole (every tile but a workgroup's first waits for
// all of its ring and for the stores of the one before).  fp32, D = 64, 3 prompts of
// up to 700 tokens, 8 on 8 heads: 19.6 us.
#include <float.h>

#include <type_traits>

#include "device_common.h"
#include "lds_dma.h"
#include "paged_rows.h"
#include "plan.h"
#include "serving.h"

namespace adaserve {

namespace {

constexpr int kThreads = kServingThreads;
constexpr int kWaves = 4;
constexpr int kTileRows = kPromptTileRows;

// 16 bytes of zeros: the source of the LDS loads whose key does not exist.
__device__ __align__(16) uint32_t zero_line[4];

__device__ __forceinline__ float fmax3(float x, float y, float z) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z);   // (a NaN passes through)
}

// A unit: one tile of rows (kTileRows, in fp32 16 or 32) of one kv-head's (token, query head in
// group) pairs of a request, row = token * G + head; where the keys are split,
// over those from k0 on.
struct PromptUnit {
  int32_t r, token0, n, ctx, tile, g, k0;
};

// Unit u.  With a table (requests in descending order of tiles) units run from
// the longest tiles to the shortest over the whole batch: level by level of
// the tile's number, all requests that have the level, the kv-heads of a tile
// next to each other, so that with 8 kv-heads each XCD's L2 holds the keys of
// one.  Entry e ends the units of the levels that e + 1 requests have; `e` is
// where the search starts and stays.  With split keys the table holds the
// requests one after another, and a tile's heads come once per chunk.  Without a
// table: request by request, the last tile first.
template <int ROWS>
__device__ __forceinline__ bool find_prompt_unit(const PromptAttnArgs &a, int64_t u, int32_t &e, PromptUnit &un) {
  if (u >= a.units) return false;
  int32_t r = -1, token0 = 0, n = 0, ctx = 0, tile = 0, g = 0, k0 = 0;
  if (a.chunks > 1) {
    const int32_t row = (int32_t)u / a.num_kv_heads, level = row / a.chunks;
    g = (int32_t)u - row * a.num_kv_heads;
    k0 = (row - level * a.chunks) * a.chunk_keys;
    while (e < a.table_count - 1 && a.table[e].unit_end <= level * a.num_kv_heads) ++e;
    tile = a.table[e].unit_end / a.num_kv_heads - 1 - level;
    r = a.table[e].request;
    token0 = a.table[e].token0;
    n = a.table[e].n;
    ctx = a.table[e].ctx;
  } else if (a.table_count > 0) {
    while (e < a.table_count - 1 && a.table[e].unit_end <= u) ++e;
    const int32_t before = e > 0 ? a.table[e - 1].unit_end : 0;
    const int32_t per_level = (e + 1) * a.num_kv_heads;
    const int32_t local = (int32_t)u - before, level = local / per_level, in = local - level * per_level;
    const int32_t rank = in / a.num_kv_heads;
    tile = prompt_tiles(a.table[e].n, a.group, ROWS) - 1 - level;
    g = in - rank * a.num_kv_heads;
    r = a.table[rank].request;
    token0 = a.table[rank].token0;
    n = a.table[rank].n;
    ctx = a.table[rank].ctx;
  } else {
    const int lane = threadIdx.x & 63;
    int64_t base = 0;
    int32_t local = 0;
    for (int r0 = 0; r0 < a.num_requests; r0 += 64) {
      const int i = r0 + lane;
      int64_t units = 0;
      if (i < a.num_requests)
        units = (int64_t)prompt_tiles(max(a.token_indptr[i + 1] - a.token_indptr[i], 0), a.group, ROWS) * a.num_kv_heads;
      const int64_t upto = wave_inclusive_scan(units);
      const unsigned long long hit = __ballot(base + upto > u);
      if (hit) {
        const int f = __ffsll(hit) - 1;
        r = r0 + f;
        local = (int32_t)(u - base - __shfl(upto - units, f, 64));
        break;
      }
      base += __shfl(upto, 63, 64);
    }
    if (r < 0) return false;
    token0 = a.token_indptr[r];
    n = a.token_indptr[r + 1] - token0;
    ctx = a.context_len[r];
    tile = prompt_tiles(n, a.group, ROWS) - 1 - local / a.num_kv_heads;
    g = local % a.num_kv_heads;
  }
  un.r = __builtin_amdgcn_readfirstlane(r);
  un.token0 = __builtin_amdgcn_readfirstlane(token0);
  un.n = __builtin_amdgcn_readfirstlane(n);
  un.ctx = __builtin_amdgcn_readfirstlane(ctx);
  un.tile = __builtin_amdgcn_readfirstlane(tile);
  un.g = __builtin_amdgcn_readfirstlane(g);
  un.k0 = __builtin_amdgcn_readfirstlane(k0);
  return un.tile >= 0 && un.token0 >= 0 && un.n > 0 && un.token0 + un.n <= a.total_tokens;
}

// The unit of workgroup b in round k of a launch of `grid` workgroups that take
// more than one each: odd rounds run backwards (in groups of 8 neighbours, which
// keep their XCD), so that the workgroups' shares of units in descending order
// come out equal.
__device__ __forceinline__ int64_t prompt_round_unit(int64_t b, int64_t k, int64_t grid) {
  const int64_t in = (k & 1) ? (grid / 8 - 1 - b / 8) * 8 + b % 8 : b;
  return k * grid + in;
}

// 64 rows per wave, one wave per SIMD.  The two 32-row halves of a wave run
// half a sub-block apart, so that the matrix products of one half always meet
// the softmax of the other in the instruction stream:
//   phase A of sub-block i: S0(i+1) = K Q0, O0 += V P0(i)  beside  P1(i) from S1(i)
//   phase B:                S1(i+1) = K Q1, O1 += V P1(i)  beside  P0(i+1) from S0(i+1)
// Both halves take the same K and V fragments from registers; the next ones
// are read in phase B as the current ones are used up.
template <int D>
__global__ __launch_bounds__(kThreads, 1) void prompt_attn_bf16_kernel(PromptAttnArgs a) {
  constexpr int KS = D / 16, DT = D / 32, KB = 32, ROWB = D * 2, NCH = D / 8;
  constexpr int BLK = KB * ROWB;
  constexpr int WI = BLK / 1024 / kWaves;
  constexpr int RPI = 1024 / ROWB;
  // Stage i of the ring holds K of sub-block i + 1 and V of sub-block i; three
  // are in flight while one is read.  At 64 KB every place in it is within reach
  // of an LDS instruction's offset.
  constexpr int NST = 4;
  constexpr int STAGE = 2 * BLK;
  constexpr int LPS = 2 * WI;                // loads per wave and stage
  constexpr float kRescaleLog2 = 8.f;
  // The weights 2^(s c - m c) keep the reference m that a row has from its first
  // 32 keys: bf16 and fp32 are as precise at 2^60 as at 1, so no maximum is taken
  // per sub-block.  A row whose sum gets beyond kMost is one whose scores
  // rise by more than 44 nats over those of its first keys; its tile is done
  // again with the maximum taken everywhere.  So is that of a row whose weights
  // reach further than with maxima (2^8 per key) and whose products with the values
  // get beyond kMostOut: |value| * keys < 2^118 keeps both ways' sums, and those
  // of their joined chunks, within fp32.
  constexpr float kMost = 0x1p64f, kMostOut = 0x1p120f;
  __shared__ int redo;
  __shared__ __align__(1024) char ring[NST * STAGE];   // (K of sub-block 0: in the last stage at first)

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.group;
  PromptUnit un;
  int32_t entry = 0;
  int64_t round = 0;
  if (!find_prompt_unit<kTileRows>(a, blockIdx.x, entry, un)) return;

  // what follows from the unit
  int32_t row_end, wrow0, first, k_end, nb, wave_nb, n_full;
  int64_t head_bytes;
  auto derive = [&]() __attribute__((always_inline)) {
    const int32_t row0 = un.tile * kTileRows;
    row_end = min(un.n * G, row0 + kTileRows);
    wrow0 = row0 + wave * 64;
    first = un.ctx - un.n + 1 - un.k0;            // keys (of the unit's) that token 0 sees
    // keys that the tile's (the wave's) last row sees; sub-blocks whose keys the wave's rows all see
    k_end = min(max(0, first + (row_end - 1) / G), a.chunk_keys);
    const int32_t wave_end = wrow0 < row_end ? min(max(0, first + (min(row_end, wrow0 + 64) - 1) / G), a.chunk_keys) : 0;
    nb = (k_end + KB - 1) / KB;
    wave_nb = (wave_end + KB - 1) / KB;
    n_full = min(wave_nb, max(0, first + wrow0 / G) / KB);
    head_bytes = (int64_t)un.g * kPageSize * D * 2;
  };
  derive();

  // Page ids: the DMA rows of a wave lie in one 16-key page of each sub-block.
  // Lane l of `pages` holds that page's id in sub-block `window` + l (-1: none),
  // `pages_after` the 64 sub-blocks after those.
  const int wave_page = (wave * WI * RPI) / kPageSize;
  int32_t pages, pages_after, window;
  // no whole sub-block of the windows so far lacks its page (a last one of at most
  // 16 keys has no second page, which is no reason to leave the common path:
  // 16 ragged prompts, half of them such, 386 -> 364 us)
  bool all_pages;
  auto load_pages = [&](const PromptUnit &of, int base) __attribute__((always_inline)) -> int32_t {
    const int32_t e = of.k0 / kPageSize + (base + lane) * (KB / kPageSize) + wave_page;
    return e < a.bt_stride && e < (of.ctx + kPageSize - 1) / kPageSize ? a.block_table[(int64_t)of.r * a.bt_stride + e] : -1;
  };
  auto take_pages = [&](int32_t ids) __attribute__((always_inline)) {
    pages = ids >= 0 && ids < a.num_pages ? ids : -1;
    all_pages = all_pages && !__any(pages < 0 && window + lane < k_end / KB);
    pages_after = load_pages(un, window + 64);
  };
  auto next_window = [&]() __attribute__((always_inline)) {
    window += 64;
    take_pages(pages_after);
  };

  // Query fragments (B operand of S^T = K Q^T): lane holds row (lane & 31) of
  // each half, head-dim elements ks*16 + (lane >> 5)*8 .. +7.
  bf16x8 qf[2][KS];
  int32_t vis[2];   // keys that the row sees
  auto load_q = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      const int32_t row = min(wrow0 + rt * 32 + (lane & 31), row_end - 1);   // (a row past the end repeats the last)
      const int32_t tok = row / G, head = un.g * G + row - tok * G;
      vis[rt] = min(first + tok, a.chunk_keys);
      const __bf16 *qp = (const __bf16 *)a.q + (int64_t)(un.token0 + tok) * a.q_stride + (int64_t)head * D + half * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[rt][ks] = *(const bf16x8 *)(qp + ks * 16);
    }
  };

  const int slot = ((lane * 16) % ROWB) / 16;
  int dma_row[WI];
  uint32_t page_off[WI];
#pragma unroll
  for (int i = 0; i < WI; ++i) {
    dma_row[i] = (wave * WI + i) * RPI + (lane * 16) / ROWB;
    page_off[i] = (uint32_t)(((dma_row[i] % kPageSize) * D + (slot ^ swizzle<NCH>(dma_row[i])) * 8) * 2);
  }
  const int64_t page_bytes = (int64_t)a.num_kv_heads * kPageSize * D * 2;
  // Sub-blocks are asked for in ascending order.
  auto page_of = [&](int blk) __attribute__((always_inline)) -> int32_t {
    if (blk >= window + 64) next_window();
    return __builtin_amdgcn_readlane(pages, blk - window);
  };
  const uint32_t wave_lds = lds_addr(ring) + wave * WI * 1024;
  const void *zeros = zero_line;
  asm volatile("" : "+s"(zeros));   // (its address is looked up once)
  // Sub-block blk of K or V into LDS at `dst`; rows past the tile's keys and
  // pages that do not exist come from the zero line, so that every stage is the
  // same number of loads.
  auto issue = [&](const void *pool, uint32_t dst, int blk, int32_t page) __attribute__((always_inline)) {
    const int32_t left = page >= 0 ? k_end - blk * KB : 0;
    const char *base = (const char *)pool + (int64_t)max(page, 0) * page_bytes + head_bytes;
#pragma unroll
    for (int i = 0; i < WI; ++i)
      dma16<false>(dma_row[i] < left ? (const void *)(base + page_off[i]) : zeros, dst + i * 1024);
  };
  // Stage i's loads: K first, then V.
  int32_t page = -1;   // of sub-block i (before stage i's loads)
  int32_t page_v = -1;
  auto issue_k = [&](int i) __attribute__((always_inline)) {
    if (i >= nb) return;
    page_v = page;
    page = page_of(i + 1);
    issue(a.k_pages, wave_lds + (i & 3) * STAGE, i + 1, page);
  };
  auto issue_v = [&](int i) __attribute__((always_inline)) {
    if (i < nb) issue(a.v_pages, wave_lds + (i & 3) * STAGE + BLK, i, page_v);
  };

  int koff[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    koff[ks] = (lane & 31) * ROWB + (((ks * 2 + half) ^ swizzle<NCH>(lane & 31)) * 16);
  int voff[DT], voff8[DT];
  {
    const int j16 = lane & 15;
    const int vrow = half * 4 + (j16 >> 2);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const int ch = dt * 4 + ((lane >> 4) & 1) * 2 + ((j16 & 3) >> 1);
      voff[dt] = vrow * ROWB + ((ch ^ swizzle<NCH>(vrow)) * 16) + (j16 & 1) * 8;
      voff8[dt] = (vrow + 8) * ROWB + ((ch ^ swizzle<NCH>(vrow + 8)) * 16) + (j16 & 1) * 8;
    }
  }

  f32x16 o[2][DT];
  // References are in units of q k; before any key -1e30 in log2 units, below
  // every score whatever the scale.
  const float c = a.scale_log2, up_raw = kRescaleLog2 / c, lowest = fmaxf(-1e30f / c, -FLT_MAX);
  float lsum[2], m_ref[2];

  bf16x8 kf[KS], vf[2 * DT];
  auto read_k = [&](const char *kst, int ks) { kf[ks] = *(const bf16x8 *)(kst + koff[ks]); };
  auto read_v = [&](const char *vst, int x) {   // x = h * DT + dt
    const int h = x / DT, dt = x % DT;
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(vst + voff[dt] + h * 16 * ROWB));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(vst + voff8[dt] + h * 16 * ROWB));
    vf[x] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto mask = [&](f32x16 &x, int rt, int blk) {
    const int32_t left = vis[rt] - blk * KB - half * 4;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = (i >> 2) * 8 + (i & 3) < left ? x[i] : -INFINITY;
  };
  auto rowmax = [&](const f32x16 &x) {
    float m0 = x[0], m1 = x[1];
#pragma unroll
    for (int i = 2; i < 14; i += 4) {
      m0 = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m0, x[i]), x[i + 2]);
      m1 = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m1, x[i + 1]), x[i + 3]);
    }
    m0 = __builtin_elementwise_maximum(m0, x[14]);
    return max_over_halves(__builtin_elementwise_maximum(__builtin_elementwise_maximum(m0, m1), x[15]));
  };
  // Takes row half rt's reference up to the maximum bm of sub-block scores where
  // that is more than 2^8 above it.
  auto rescale = [&](int rt, float bm) __attribute__((always_inline)) {
    const bool up = bm > m_ref[rt] + up_raw;
    if (__any(up)) {
      const float mn = up ? bm : m_ref[rt];
      const float al = __builtin_amdgcn_exp2f((m_ref[rt] - mn) * c);
      m_ref[rt] = mn;
      lsum[rt] *= al;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[rt][dt] *= al;
    }
  };
  auto probs = [&](int rt, const f32x16 &x, bf16x8 (&pk)[2]) __attribute__((always_inline)) {
    const float mc = m_ref[rt] * c;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[h * 8 + 2 * e], c, -mc));
        const float y1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[h * 8 + 2 * e + 1], c, -mc));
        lsum[rt] += y0 + y1;
        w[e] = pack_bf16x2(y0, y1);
      }
      pk[h] = __builtin_bit_cast(bf16x8, w);
    }
  };
  f32x16 s0, s1;
  bf16x8 p0[2], p1[2];
  bool careful = false;   // the tile is done again, with maxima
  // One phase: half `rt` takes its products (scores of the next sub-block into
  // sx, O += V P of this one), the other half its weights (from sy, sub-block
  // yblk).  `src` with kDma: the wave's part of a K or V sub-block, loaded to LDS
  // at `dst`.
  auto phase = [&](auto half_c, f32x16 &sx, const bf16x8 (&px)[2], f32x16 &sy, bf16x8 (&py)[2], int yblk, auto masked,
                   const char *kst, const char *vst, auto dma, const char *src, uint32_t dst) __attribute__((always_inline)) {
    constexpr int rt = decltype(half_c)::value;
    constexpr int ry = 1 - rt;
    constexpr bool kRead = rt == 1;
    constexpr bool kMasked = decltype(masked)::value;
    constexpr bool kDma = decltype(dma)::value;
    constexpr int SLOTS = KS + 2 * DT;   // matrix instructions
    if constexpr (kMasked) mask(sy, ry, yblk);
    if (kMasked && careful) rescale(ry, rowmax(sy));
    // A slot is one matrix instruction and the vector work that issues while it
    // runs: one step each of a few weights (scale; exponential; sum and
    // rounding), none of which waits for another, and two LDS reads.  The empty
    // asm statements and scheduling barriers keep that order: the compiler would
    // gather the instructions by kind.  (Sums by
    // v_dot2_f32_bf16 would take the matrix unit from the products.)
    const float mc = m_ref[ry] * c;
    float z[16], l2[2] = {lsum[ry], 0.f};
    uint32_t w[8];
    sx = f32x16{};
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      if (j < KS) {
        sx = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j], qf[rt][j], sx, 0, 0, 0);
      } else {
        const int x = j - KS;
        o[rt][x % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[x], px[x / DT], o[rt][x % DT], 0, 0, 0);
      }
      if constexpr (kDma) {
        if (j >= 1 && j <= WI) dma16_off<false>(src, page_off[j - 1], dst + (j - 1) * 1024);
      }
      // scaled by the end of slot j: the first `to` scores; exponentials are a slot
      // behind, sums and roundings two
      const auto to = [](int j) { return j < 0 ? 0 : (j + 1) * 16 / (SLOTS - 2) + 1 < 16 ? (j + 1) * 16 / (SLOTS - 2) + 1 : 16; };
#pragma unroll
      for (int t = to(j - 3); t < to(j - 2); ++t) {
        l2[t & 1] += z[t];
        asm volatile("" : "+v"(l2[t & 1]));
        if (t & 1) {
          w[t / 2] = pack_bf16x2(z[t - 1], z[t]);
          asm volatile("" : "+v"(w[t / 2]));
        }
      }
#pragma unroll
      for (int t = to(j - 2); t < to(j - 1); ++t) {
        z[t] = __builtin_amdgcn_exp2f(z[t]);
        asm volatile("" : "+v"(z[t]));
      }
#pragma unroll
      for (int t = to(j - 1); t < to(j); ++t) {
        z[t] = __builtin_fmaf(sy[t], c, -mc);
        asm volatile("" : "+v"(z[t]));
      }
      if constexpr (kRead) {
        // the fragments whose last use is behind
        if (j < KS) read_k(kst, j);
        else read_v(vst, j - KS);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    py[0] = __builtin_bit_cast(bf16x8, (u32x4{w[0], w[1], w[2], w[3]}));
    py[1] = __builtin_bit_cast(bf16x8, (u32x4{w[4], w[5], w[6], w[7]}));
    lsum[ry] = l2[0] + l2[1];
    asm volatile("" : "+v"(py[0]), "+v"(py[1]), "+v"(lsum[ry]));
    __builtin_amdgcn_sched_barrier(0);
  };
  using Zero = std::integral_constant<int, 0>;
  using One = std::integral_constant<int, 1>;
  using Yes = std::true_type;
  using No = std::false_type;

  // Sub-block i, all of whose keys the wave's rows see, as they do those of
  // sub-block i + 1, and all loads on the way of whole sub-blocks.  X = i mod 4.
  // Phase B opens with the barrier after which stage i + 1 has landed (the two
  // after it may fly) and stage i, which every wave has read, is refilled.
  auto full_sub = [&](int i, auto slot_c) __attribute__((always_inline)) {
    constexpr int X = decltype(slot_c)::value, Y = (X + 1) & 3, Z = (X + 3) & 3;
    // (past the tile's keys any page will do: nothing reads those stages)
    const char *src = (const char *)a.v_pages + (int64_t)max(page_v, 0) * page_bytes + head_bytes;
    phase(Zero{}, s0, p0, s1, p1, i, No{}, nullptr, nullptr, Yes{}, src, wave_lds + Z * STAGE + BLK);
    page_v = page;
    page = __builtin_amdgcn_readlane(pages, i + 5 - window);
    src = (const char *)a.k_pages + (int64_t)max(page, 0) * page_bytes + head_bytes;
    wait_loads_barrier<2 * LPS>();
    phase(One{}, s1, p1, s0, p0, i + 1, No{}, ring + Y * STAGE, ring + Y * STAGE + BLK, Yes{}, src, wave_lds + X * STAGE);
  };
  auto any_sub = [&](int i) __attribute__((always_inline)) {
    issue_v(i + 3);
    if (i < wave_nb) phase(Zero{}, s0, p0, s1, p1, i, Yes{}, nullptr, nullptr, No{}, nullptr, 0);
    if (i + 3 < nb) wait_loads_barrier<2 * LPS>();
    else if (i + 2 < nb) wait_loads_barrier<LPS>();
    else wait_loads_barrier<0>();
    issue_k(i + 4);
    const char *nxt = ring + ((i + 1) & 3) * STAGE;
    if (i < wave_nb) phase(One{}, s1, p1, s0, p0, i + 1, Yes{}, nxt, nxt + BLK, No{}, nullptr, 0);
  };
  // A row that holds a NaN before any key is hidden from it has it from a key
  // that it sees.
  bool had_nan[2] = {false, false};
  auto is_nan = [&](int rt) {
    float x = lsum[rt];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) x = __builtin_elementwise_maximum(x, o[rt][dt][i]);
    x = max_over_halves(x);
    return x != x;
  };
  // The unit's first loads (`ids`: its first page ids): queries, then K of
  // sub-block 0, stages 0 to 2 and K of stage 3 once sub-block 0's is used.
  auto start = [&](int32_t ids) __attribute__((always_inline)) {
    load_q();
    window = 0;
    all_pages = true;
    take_pages(ids);
    if (nb > 0) {
      page = page_of(0);
      issue(a.k_pages, wave_lds + 3 * STAGE, 0, page);
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        issue_k(i);
        issue_v(i);
      }
    }
  };
  bool fresh = true;   // no store since the unit's loads
  if (tid == 0) redo = 0;
  start(load_pages(un, 0));
#pragma unroll 1
  for (;;) {
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      lsum[rt] = 0.f;
      m_ref[rt] = lowest;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[rt][dt] = f32x16{};
    }
    if (fresh && nb >= 3) wait_loads_barrier<2 * LPS>();
    else if (fresh && nb == 2) wait_loads_barrier<LPS>();
    else wait_loads_barrier<0>();
    if (wave_nb > 0) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) read_k(ring + 3 * STAGE, ks);
      s0 = f32x16{};
      s1 = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[0][ks], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[1][ks], s1, 0, 0, 0);
      }
      mask(s0, 0, 0);
      mask(s1, 1, 0);
      rescale(0, rowmax(s0));
      rescale(1, rowmax(s1));
      probs(0, s0, p0);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) read_k(ring, ks);
#pragma unroll
      for (int x = 0; x < 2 * DT; ++x) read_v(ring + BLK, x);
    }
    wait_loads_barrier<15>();   // (every wave has read K of sub-block 0)
    issue_k(3);
    // the next unit and its first page ids, long before they are used
    PromptUnit next;
    int32_t next_ids = -1;
    const bool more = a.units > gridDim.x &&
                      find_prompt_unit<kTileRows>(a, prompt_round_unit(blockIdx.x, round + 1, gridDim.x), entry, next);
    if (more) next_ids = load_pages(next, 0);
    int i = 0;
#pragma unroll 1
    while (i < nb) {
      if (!careful && (i & 3) == 0) {
#pragma unroll 1
        for (; i + 4 < n_full && (k_end % KB == 0 || i + 8 < k_end / KB); i += 4) {
          if (i + 8 >= window + 64) break;   // (the other path moves the window)
          if (!all_pages) break;
          full_sub(i, std::integral_constant<int, 0>{});
          full_sub(i + 1, std::integral_constant<int, 1>{});
          full_sub(i + 2, std::integral_constant<int, 2>{});
          full_sub(i + 3, std::integral_constant<int, 3>{});
        }
      }
      if (i == n_full) {   // hidden keys from here on
        had_nan[0] = is_nan(0);
        had_nan[1] = is_nan(1);
      }
      any_sub(i++);
    }
    if (!careful) {
      bool beyond = !(lsum[0] < kMost) || !(lsum[1] < kMost);
      // (rarely: 2 x 16 DT comparisons)
      const float fair = 0x1p8f * (float)k_end;
      if (__any(fmaxf(lsum[0], lsum[1]) > fair)) {
#pragma unroll
        for (int rt = 0; rt < 2; ++rt)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 16; ++j) beyond = beyond || !(fabsf(o[rt][dt][j]) < kMostOut);
      }
      if (__any(beyond) && lane == 0) redo = 1;
    }
    __syncthreads();   // every wave is done with the ring, too
    if (redo) {
      __syncthreads();
      if (tid == 0) redo = 0;
      careful = true;
      fresh = true;
      start(load_pages(un, 0));
      continue;
    }
    // the next unit's loads, then this one's output
    const PromptUnit done = un;
    const int32_t done_end = row_end, done_row0 = wrow0;
    const int32_t done_vis[2] = {vis[0], vis[1]};
    if (more) {
      ++round;
      un = next;
      derive();
      start(next_ids);
      careful = false;
      fresh = false;
    }
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      const int32_t row = done_row0 + rt * 32 + (lane & 31);
      const bool ok = row < done_end;
      const float l_tot = sum_over_halves(lsum[rt]);
      const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
      const int32_t tok = ok ? row / G : 0, head = done.g * G + (ok ? row - tok * G : 0);
      // A key that the row does not see has weight 0, and 0 times an infinite
      // value is NaN: such rows are taken again, key by key.
      const bool again = ok && is_nan(rt) && !had_nan[rt];
      if (a.chunks > 1) {
        // the chunk's part: sums, and (reference in log2 units, sum of weights);
        // an infinite reference has the join take the row again
        const int64_t slot = (int64_t)blockIdx.x * kTileRows + (row - done.tile * kTileRows);
        if (ok) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
              *(f32x4 *)(a.ws_o + slot * D + dt * 32 + i * 2 + half * 4) =
                  f32x4{o[rt][dt][i], o[rt][dt][i + 1], o[rt][dt][i + 2], o[rt][dt][i + 3]};
          if (half == 0) *(f32x2 *)(a.ws_ml + slot * 2) = f32x2{again ? INFINITY : m_ref[rt] * c, l_tot};
        }
        continue;
      }
      __bf16 *dst = (__bf16 *)a.out + ((int64_t)(done.token0 + tok) * a.num_q_heads + head) * D;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
          const uint32_t x0 = pack_bf16x2(o[rt][dt][i] * inv, o[rt][dt][i + 1] * inv);
          const uint32_t x1 = pack_bf16x2(o[rt][dt][i + 2] * inv, o[rt][dt][i + 3] * inv);
          const uint32_t y0 = pack_bf16x2(o[rt][dt][i + 4] * inv, o[rt][dt][i + 5] * inv);
          const uint32_t y1 = pack_bf16x2(o[rt][dt][i + 6] * inv, o[rt][dt][i + 7] * inv);
          const auto r0 = __builtin_amdgcn_permlane32_swap(x0, y0, false, false);
          const auto r1 = __builtin_amdgcn_permlane32_swap(x1, y1, false, false);
          if (ok && !again) *(u32x4 *)(dst + dt * 32 + i * 2 + half * 8) = u32x4{r0[0], r1[0], r0[1], r1[1]};
        }
      unsigned long long todo = __ballot(again) & 0xffffffffull;
      while (todo) {
        const int l = __ffsll(todo) - 1;
        todo &= todo - 1;
        attend_row<true, D>(a, done.r, done.token0 + __shfl(tok, l, 64), __shfl(head, l, 64), __shfl(done_vis[rt], l, 64));
      }
    }
    if (!more) return;
  }
}

// Joins the chunks of split keys: with m the largest reference of the row's
// chunks, out = sum 2^(m_c - m) o_c / sum 2^(m_c - m) l_c.  One wave per row.
template <int D>
__global__ __launch_bounds__(kThreads) void prompt_join_kernel(PromptAttnArgs a) {
  constexpr int EPL = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int32_t t = __builtin_amdgcn_readfirstlane((int32_t)(id / a.num_q_heads));
  const int32_t h = __builtin_amdgcn_readfirstlane((int32_t)(id - (int64_t)t * a.num_q_heads));
  if (t >= a.total_tokens) return;
  int e = -1;
  for (int i0 = 0; i0 < a.table_count; i0 += 64) {
    const int i = i0 + lane;
    const unsigned long long hit =
        __ballot(i < a.table_count && t >= a.table[i].token0 && t < a.table[i].token0 + a.table[i].n);
    if (hit) {
      e = i0 + __ffsll(hit) - 1;
      break;
    }
  }
  if (e < 0) return;
  const int32_t g = h / a.group, row = (t - a.table[e].token0) * a.group + (h - g * a.group);
  const int32_t tile = row / kTileRows;
  const int32_t level = a.table[e].unit_end / a.num_kv_heads - 1 - tile;
  const int32_t seen = max(0, a.table[e].ctx - a.table[e].n + 1 + (t - a.table[e].token0));
  const int32_t chunks = min(a.chunks, (seen + a.chunk_keys - 1) / a.chunk_keys);
  float m = -1e30f, l = 0.f, o[EPL] = {};
  for (int c = 0; c < chunks; ++c) {
    const int64_t slot = (((int64_t)level * a.chunks + c) * a.num_kv_heads + g) * kTileRows + (row - tile * kTileRows);
    const f32x2 ml = *(const f32x2 *)(a.ws_ml + slot * 2);
    float x[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = a.ws_o[slot * D + lane * EPL + i];
    const float mn = fmaxf(m, ml[0]);
    const float f = __builtin_amdgcn_exp2f(m - mn), w = __builtin_amdgcn_exp2f(ml[0] - mn);
    m = mn;
    l = l * f + w * ml[1];
#pragma unroll
    for (int i = 0; i < EPL; ++i) o[i] = o[i] * f + w * x[i];
  }
  if (m == INFINITY) {
    attend_row<true, D>(a, a.table[e].request, t, h, seen);
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;   // (a NaN stays one)
  __bf16 *dst = (__bf16 *)a.out + id * D + lane * EPL;
#pragma unroll
  for (int i = 0; i < EPL; ++i) dst[i] = (__bf16)(o[i] * inv);
}

// fp32: one workgroup per tile of 16 RB rows, its four waves taking a quarter of
// the tile's keys each and joining in LDS.  S^T = K Q^T and O^T = V^T P^T run on
// v_mfma_f32_16x16x4_f32; both contractions may take their slots in any order,
// so every lane loads 16 contiguous bytes of K and V straight into the operand
// registers and P needs no exchange: slot q of QK step (c, e) is head-dim
// element 16 c + 4 q + e, slot q of PV step e is key 4 q + e, and O^T tile (h, k)
// holds the columns 64 h + 4 j + k.  Every tile reads its keys for itself, one page
// ahead, 8 flops a byte with 16 rows and 16 with 32, so two row tiles share each
// operand where there are enough tiles to fill the device.  Bound by the fp32 matrix
// rate (a sixteenth of bf16's) and the waits for those loads together: 2 prompts of
// 1500 tokens (32 heads on 8, D = 128) 351 us, 105 TFLOP/s (a library product: 154),
// matrix cores busy 0.70 of the time and 7.5 TB/s out of the L2s; the 3 prompts
// above 0.41 and 8.6 TB/s.
template <int D, int RB>
__global__ __launch_bounds__(kThreads) void prompt_attn_f32_kernel(PromptAttnArgs a) {
  constexpr int RT = 16 * RB;
  constexpr int NC = D / 16;      // 16-byte K loads per lane and page
  constexpr int NH = D / 64;      // 16-byte V loads per lane and key
  constexpr int LDO = D + 4;
  __shared__ __align__(16) float mo[kWaves * RT * LDO];
  __shared__ float mw[kWaves][RT], lw[kWaves][RT];
  __shared__ int taken[RT];
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, j = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.group;

  // The longest first, in rounds that run back and forth, so that the CUs'
  // shares are alike (request by request: 24.0 instead of 19.5 us)
  PromptUnit un;
  int32_t entry = 0;
  const int64_t round = blockIdx.x / kPromptGrid;
  if (!find_prompt_unit<RT>(a, prompt_round_unit(blockIdx.x - round * kPromptGrid, round, kPromptGrid), entry, un)) return;
  const int r = __builtin_amdgcn_readfirstlane(un.r);
  const int32_t token0 = un.token0, n = un.n, ctx = un.ctx, tile = un.tile, g = un.g;
  const int32_t row0 = tile * RT, row_end = min(n * G, row0 + RT);
  const int32_t first = ctx - n + 1;
  const int32_t k_end = max(0, first + (row_end - 1) / G);
  const int32_t n_full = max(0, first + row0 / G) / 16;   // pages that all rows see
  const int32_t nb = (k_end + 15) / 16;
  const int32_t b0 = (int32_t)((int64_t)nb * wave / kWaves), b1 = (int32_t)((int64_t)nb * (wave + 1) / kWaves);

  f32x4 qf[RB][NC];
  int32_t vis[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int32_t row = min(row0 + rb * 16 + j, row_end - 1), tok = row / G, head = g * G + row - tok * G;
    vis[rb] = first + tok;
    const float *qp = (const float *)a.q + (int64_t)(token0 + tok) * a.q_stride + (int64_t)head * D + q * 4;
#pragma unroll
    for (int c = 0; c < NC; ++c) qf[rb][c] = *(const f32x4 *)(qp + c * 16);
  }
  // lane i holds the id of page page_base + i (-1: none)
  int32_t page_base = b0, pages = -1;
  auto load_pages = [&]() {
    const int b = page_base + lane;
    pages = -1;
    if (b < nb && b < a.bt_stride) {
      const int32_t p = a.block_table[(int64_t)r * a.bt_stride + b];
      if (p >= 0 && p < a.num_pages) pages = p;
    }
  };
  load_pages();
  auto page_of = [&](int b) -> int32_t {
    if (b >= page_base + 64) {
      page_base = b;
      load_pages();
    }
    return __builtin_amdgcn_readlane(pages, b - page_base);
  };
  // a missing page reads page 0, whose scores and values are not used
  f32x4 kr[NC], vr[4][NH];
  auto load_k = [&](int32_t page) {
    const float *p = (const float *)a.k_pages + (((int64_t)max(page, 0) * a.num_kv_heads + g) * kPageSize + j) * D + q * 4;
#pragma unroll
    for (int c = 0; c < NC; ++c) kr[c] = *(const f32x4 *)(p + c * 16);
  };
  auto load_v = [&](int32_t page) {
    const float *p = (const float *)a.v_pages + (((int64_t)max(page, 0) * a.num_kv_heads + g) * kPageSize + q * 4) * D + j * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int h = 0; h < NH; ++h) vr[e][h] = *(const f32x4 *)(p + e * D + h * 64);
  };
  f32x4 o[RB][NH][4];
  float m[RB], l[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m[rb] = -1e30f;
    l[rb] = 0.f;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[rb][h][k] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto is_nan = [&](int rb) {
    float x = l[rb];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) x = __builtin_elementwise_maximum(x, o[rb][h][k][i]);
    x = max_over_lane_rows(x);
    return x != x;
  };
  bool had_nan[RB] = {};
  int32_t page = -1;
  if (b0 < b1) {
    page = page_of(b0);
    load_k(page);
    load_v(page);
  }
  for (int b = b0; b < b1; ++b) {
    if (b == n_full || (b == b0 && b > n_full))
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) had_nan[rb] = is_nan(rb);
    const int32_t next = page_of(min(b + 1, b1 - 1));
    f32x4 s[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          s[rb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[c][e], qf[rb][c][e], s[rb], 0, 0, 0);
    load_k(next);
    // s[rb][e]: key 4 q + e of the page, row j; in log2 units from here on
    const bool masked = b >= n_full, none = page < 0;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = none ? 0.f : s[rb][e] * a.scale_log2;
        s[rb][e] = !masked || b * 16 + q * 4 + e < vis[rb] ? x : -INFINITY;
      }
      const float bm = max_over_lane_rows(fmax3(s[rb][0], s[rb][1], __builtin_elementwise_maximum(s[rb][2], s[rb][3])));
      if (__any(bm > m[rb])) {
        const float mn = bm > m[rb] ? bm : m[rb], al = __builtin_amdgcn_exp2f(m[rb] - mn);
        m[rb] = mn;
        l[rb] *= al;
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[rb][h][k] *= al;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[rb][e] = __builtin_amdgcn_exp2f(s[rb][e] - m[rb]);
        l[rb] += s[rb][e];
      }
    }
    // a slot past the tile's keys may hold anything
    if (none || b * 16 + 16 > k_end) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int h = 0; h < NH; ++h)
          if (none || b * 16 + q * 4 + e >= k_end) vr[e][h] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            o[rb][h][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[e][h][k], s[rb][e], o[rb][h][k], 0, 0, 0);
    load_v(next);
    page = next;
  }
  if (tid < RT) taken[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int rl = rb * 16 + j;
    const float ls = sum_over_lane_rows(l[rb]);
    // a key that the row does not see has weight 0, and 0 times an infinite value
    // is NaN: such rows are taken again, key by key
    if (b1 > n_full && is_nan(rb) && !had_nan[rb]) taken[rl] = 1;
    if (q == 0) {
      mw[wave][rl] = m[rb];
      lw[wave][rl] = ls;
    }
    float *dst = mo + (wave * RT + rl) * LDO;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4 *)(dst + h * 64 + q * 16 + i * 4) = f32x4{o[rb][h][0][i], o[rb][h][1][i], o[rb][h][2][i], o[rb][h][3][i]};
  }
  __syncthreads();
  for (int it = tid; it < RT * (D / 4); it += kThreads) {
    const int rl = it / (D / 4), col = it % (D / 4) * 4;
    const int row = row0 + rl;
    if (row >= row_end || taken[rl]) continue;
    float mm = mw[0][rl];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, mw[w][rl]);
    float den = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float wt = __builtin_amdgcn_exp2f(mw[w][rl] - mm);
      den = __builtin_fmaf(wt, lw[w][rl], den);
      acc += *(const f32x4 *)(mo + (w * RT + rl) * LDO + col) * wt;
    }
    const int tok = row / G, head = g * G + row - tok * G;
    f32x4 res = {0.f, 0.f, 0.f, 0.f};
    if (den != 0.f) res = acc / den;   // (a NaN stays one)
    *(f32x4 *)((float *)a.out + ((int64_t)(token0 + tok) * a.num_q_heads + head) * D + col) = res;
  }
  for (int rl = wave; rl < RT && row0 + rl < row_end; rl += kWaves)
    if (taken[rl]) {
      const int tok = (row0 + rl) / G, head = g * G + row0 + rl - tok * G;
      attend_row<false, D>(a, r, token0 + tok, head, first + tok);
    }
}

template <int D, int RB>
void launch_prompt_f32(const PromptAttnArgs &a, int64_t units, hipStream_t stream) {
  const int64_t blocks = (units + kPromptGrid - 1) / kPromptGrid * kPromptGrid;   // whole rounds
  hipLaunchKernelGGL((prompt_attn_f32_kernel<D, RB>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_prompt_attn(const PromptAttnArgs &a, int head_dim, bool bf16, hipStream_t stream) {
  const dim3 block(kThreads);
  if (bf16) {
    const dim3 grid((unsigned)a.grid);
    if (head_dim == 128) hipLaunchKernelGGL((prompt_attn_bf16_kernel<128>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((prompt_attn_bf16_kernel<64>), grid, block, 0, stream, a);
    if (a.chunks > 1) {
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      const dim3 rows((unsigned)(((int64_t)a.total_tokens * a.num_q_heads + kWaves - 1) / kWaves));
      if (head_dim == 128) hipLaunchKernelGGL((prompt_join_kernel<128>), rows, block, 0, stream, a);
      else hipLaunchKernelGGL((prompt_join_kernel<64>), rows, block, 0, stream, a);
    }
    return hipGetLastError();
  }
  if (head_dim == 128) {
    if (a.f32_rows == 32) launch_prompt_f32<128, 2>(a, a.units, stream);
    else launch_prompt_f32<128, 1>(a, a.units, stream);
  } else {
    if (a.f32_rows == 32) launch_prompt_f32<64, 2>(a, a.units, stream);
    else launch_prompt_f32<64, 1>(a, a.units, stream);
  }
  return hipGetLastError();
}

}  // namespace adaserve
