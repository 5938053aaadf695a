// Causal attention of packed prompts over the paged cache on gfx950: row i of
// a request's n tokens stands at position c - n + i of its c cached keys and
// sees the keys up to itself.
#include <type_traits>

#include "device_common.h"
#include "lds_dma.h"
#include "paged_rows.h"
#include "plan.h"
#include "serving.h"

namespace adaserve {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;

// 16 bytes of zeros: the source of the LDS loads whose key does not exist.
__device__ __align__(16) uint32_t zero_line[4];

// A workgroup's tile: rows row0 .. row0 + tile_rows - 1 of one kv-head's
// (token, query head in group) pairs of a request, row = token * G + head.
struct PromptUnit {
  int32_t r, token0, n, ctx, tile, g;
};

// Units are numbered request by request (in the table's order), the last tile
// first (it has the most keys) and the kv-heads of a tile next to each other,
// so that with 8 kv-heads each XCD's L2 holds the keys of one.
__device__ __forceinline__ bool find_prompt_unit(const PagedAttnArgs &a, int64_t u, PromptUnit &un) {
  int32_t r = -1, token0 = 0, n = 0, ctx = 0;
  int64_t local = 0;
  const int lane = threadIdx.x & 63;
  if (a.table_count > 0) {
    int64_t before = 0;
    bool ok = false;
    for (int i0 = 0; i0 < a.table_count; i0 += 64) {
      const int i = i0 + lane;
      const int32_t end = i < a.table_count ? a.table[i].unit_end : INT32_MAX;
      const unsigned long long hit = __ballot((int64_t)end > u);
      if (hit) {
        const int e = i0 + __ffsll(hit) - 1;
        if (e >= a.table_count) return false;
        before = e > 0 ? a.table[e - 1].unit_end : 0;
        r = a.table[e].request;
        token0 = a.table[e].token0;
        n = a.table[e].n;
        ctx = a.table[e].ctx;
        ok = true;
        break;
      }
    }
    if (!ok) return false;
    local = u - before;
  } else {
    int64_t base = 0;
    for (int r0 = 0; r0 < a.num_requests; r0 += 64) {
      const int i = r0 + lane;
      int64_t units = 0;
      if (i < a.num_requests)
        units = (int64_t)prompt_tiles(a.token_indptr[i + 1] - a.token_indptr[i], a.group, a.tile_rows) * a.num_kv_heads;
      const int64_t upto = wave_inclusive_scan(units);
      const unsigned long long hit = __ballot(base + upto > u);
      if (hit) {
        const int f = __ffsll(hit) - 1;
        r = r0 + f;
        local = u - base - __shfl(upto - units, f, 64);
        break;
      }
      base += __shfl(upto, 63, 64);
    }
    if (r < 0) return false;
    token0 = a.token_indptr[r];
    n = a.token_indptr[r + 1] - token0;
    ctx = a.context_len[r];
  }
  un.r = __builtin_amdgcn_readfirstlane(r);
  un.token0 = __builtin_amdgcn_readfirstlane(token0);
  un.n = __builtin_amdgcn_readfirstlane(n);
  un.ctx = __builtin_amdgcn_readfirstlane(ctx);
  const int32_t l = __builtin_amdgcn_readfirstlane((int32_t)local);
  const int32_t tiles = prompt_tiles(un.n, a.group, a.tile_rows);
  un.tile = tiles - 1 - l / a.num_kv_heads;
  un.g = l % a.num_kv_heads;
  return un.tile >= 0 && un.token0 >= 0 && un.token0 + un.n <= a.total_tokens;
}

// One wave per row tile of 32 RT rows; four of them share K and V in LDS.
template <int D, int RT>
__global__ __launch_bounds__(kThreads, RT == 2 ? 1 : 2) void prompt_attn_bf16_kernel(PagedAttnArgs a) {
  constexpr int KS = D / 16;                 // matrix k-steps over the head dim
  constexpr int DT = D / 32;                 // 32-wide output tiles over the head dim
  constexpr int KB = 32;                     // keys per sub-block
  constexpr int ROWB = D * 2;
  constexpr int NCH = D / 8;
  constexpr int BLK = KB * ROWB;             // bytes of K (or V) per sub-block
  constexpr int WI = BLK / 1024 / kWaves;    // loads per wave and sub-block
  constexpr int RPI = 1024 / ROWB;           // key rows per load
  constexpr int NST = RT == 2 ? 3 : 2;       // stages of 64 keys
  constexpr int STAGE = 4 * BLK;             // K sub-blocks 2s+1, 2s+2, V sub-blocks 2s, 2s+1
  constexpr int LPS = 4 * WI;                // loads per wave and stage
  constexpr float kRescaleLog2 = 8.f;
  __shared__ __align__(1024) char ring[NST * STAGE];

  PromptUnit un;
  if (!find_prompt_unit(a, blockIdx.x, un)) return;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.group, g = un.g;
  const int32_t M = un.n * G, row0 = un.tile * a.tile_rows, row_end = min(M, row0 + a.tile_rows);
  const int32_t first = un.ctx - un.n + 1;   // keys that token 0 sees
  // keys that the tile's (the wave's) last row sees, and those that all its rows see
  const int32_t k_end = max(0, first + (row_end - 1) / G);
  const int32_t wrow0 = row0 + wave * 32 * RT;
  const bool wave_live = wrow0 < row_end;
  const int32_t wave_end = wave_live ? max(0, first + (min(row_end, wrow0 + 32 * RT) - 1) / G) : 0;
  const int32_t nb = (k_end + KB - 1) / KB, wave_nb = (wave_end + KB - 1) / KB;
  const int32_t n_full = max(0, first + row0 / G) / KB;

  // Page ids: the DMA rows of a wave lie in one 16-key page of each sub-block;
  // lane l of pgv[i] holds that page's id in sub-block page_base + 64 i + l.
  const int wave_page = (wave * WI * RPI) / kPageSize;
  int32_t pgv[4], page_base = 0;
  auto load_pages = [&](int base) {
    page_base = base;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int32_t blk = base + i * 64 + lane;
      const int32_t e = blk * (KB / kPageSize) + wave_page;
      int32_t p = -1;
      if (blk < nb && e < a.bt_stride) {
        p = a.block_table[(int64_t)un.r * a.bt_stride + e];
        if (p < 0 || p >= a.num_pages) p = -1;
      }
      pgv[i] = p;
    }
  };
  load_pages(0);

  // Query fragments (B operand of S^T = K Q^T): lane holds row (lane & 31) of
  // each 32, head-dim elements ks*16 + half*8 .. +7.
  int32_t row[RT], vis[RT];
  bf16x8 qf[RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    row[rt] = wrow0 + rt * 32 + (lane & 31);
    const bool ok = row[rt] < row_end;
    const int32_t tok = ok ? row[rt] / G : 0, head = g * G + (ok ? row[rt] - tok * G : 0);
    vis[rt] = ok ? first + tok : 0;
    const __bf16 *qp = (const __bf16 *)a.q + (int64_t)(un.token0 + tok) * a.q_stride + (int64_t)head * D + half * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 v = {};
      if (ok) v = *(const bf16x8 *)(qp + ks * 16);
      qf[rt][ks] = v;
    }
  }

  const int slot = ((lane * 16) % ROWB) / 16;
  int dma_row[WI];
  uint32_t page_off[WI];
#pragma unroll
  for (int i = 0; i < WI; ++i) {
    dma_row[i] = (wave * WI + i) * RPI + (lane * 16) / ROWB;
    page_off[i] = (uint32_t)(((dma_row[i] % kPageSize) * D + (slot ^ swizzle<NCH>(dma_row[i])) * 8) * 2);
  }
  const int64_t page_bytes = (int64_t)a.num_kv_heads * kPageSize * D * 2;
  const int64_t head_bytes = (int64_t)g * kPageSize * D * 2;
  auto page_of = [&](int blk) -> int32_t {
    const int l = (blk - page_base) & 63, hi = (blk - page_base) >> 6;
    const int32_t p0 = __builtin_amdgcn_readlane(pgv[0], l), p1 = __builtin_amdgcn_readlane(pgv[1], l);
    const int32_t p2 = __builtin_amdgcn_readlane(pgv[2], l), p3 = __builtin_amdgcn_readlane(pgv[3], l);
    return blk >= nb ? -1 : hi == 0 ? p0 : hi == 1 ? p1 : hi == 2 ? p2 : p3;
  };
  // Sub-block blk of K or V into `dst`; rows past the tile's keys and pages
  // that do not exist come from the zero line, so that every stage is the same
  // number of loads.
  auto issue = [&](const void *pool, char *dst, int blk, int32_t page) {
    const int32_t p = __builtin_amdgcn_readfirstlane(page);
    const int32_t left = p >= 0 ? k_end - blk * KB : 0;
    const char *base = (const char *)pool + (int64_t)max(p, 0) * page_bytes + head_bytes;
    const uint32_t lds = lds_addr(dst) + wave * WI * 1024;
    if (left >= KB) {
#pragma unroll
      for (int i = 0; i < WI; ++i) dma16_off<false>(base, page_off[i], lds + i * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < WI; ++i)
        dma16<false>(dma_row[i] < left ? (const void *)(base + page_off[i]) : (const void *)zero_line, lds + i * 1024);
    }
  };
  int32_t page_v = -1;   // of the next stage's first V sub-block
  auto issue_stage = [&](int s, char *st) {
    if (2 * s + 2 - page_base >= 256) load_pages(2 * s);
    const int32_t p0 = page_v, p1 = page_of(2 * s + 1), p2 = page_of(2 * s + 2);
    issue(a.k_pages, st, 2 * s + 1, p1);
    issue(a.v_pages, st + 2 * BLK, 2 * s, p0);
    issue(a.k_pages, st + BLK, 2 * s + 2, p2);
    issue(a.v_pages, st + 3 * BLK, 2 * s + 1, p1);
    page_v = p2;
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

  f32x16 o[RT][DT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[rt][dt] = f32x16{};
  const float c = a.scale_log2, up_raw = kRescaleLog2 / c;
  float lsum[RT], m_ref[RT], bm[RT];
  f32x16 s[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) lsum[rt] = 0.f, m_ref[rt] = -1e30f, bm[rt] = 0.f;

  // S^T of one sub-block: s[i] is key (i >> 2)*8 + half*4 + (i & 3) of the lane's row.
  auto scores = [&](const char *kst, f32x16 (&x)[RT]) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) x[rt] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 kf = *(const bf16x8 *)(kst + koff[ks]);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) x[rt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[rt][ks], x[rt], 0, 0, 0);
    }
  };
  auto mask = [&](f32x16 (&x)[RT], int blk) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int32_t left = vis[rt] - blk * KB - half * 4;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[rt][i] = (i >> 2) * 8 + (i & 3) < left ? x[rt][i] : -INFINITY;
    }
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
  auto rescale = [&]() {
    bool up = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) up |= bm[rt] > m_ref[rt] + up_raw;
    if (__any(up)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float mn = bm[rt] > m_ref[rt] + up_raw ? bm[rt] : m_ref[rt];
        const float al = __builtin_amdgcn_exp2f((m_ref[rt] - mn) * c);
        m_ref[rt] = mn;
        lsum[rt] *= al;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[rt][dt] *= al;
      }
    }
  };
  auto probs = [&](int rt, const f32x16 &x, bf16x8 (&pk)[2]) {
    const float mc = m_ref[rt] * c;
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[h * 8 + 2 * e], c, -mc));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[h * 8 + 2 * e + 1], c, -mc));
        const bf16x2 pp = __builtin_convertvector((f32x2{p0, p1}), bf16x2);
        lsum[rt] = __builtin_amdgcn_fdot2_f32_bf16(pp, ones, lsum[rt], false);
        w[e] = __builtin_bit_cast(uint32_t, pp);
      }
      pk[h] = __builtin_bit_cast(bf16x8, w);
    }
  };
  auto pv = [&](const char *vst, const bf16x8 (&pk)[RT][2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(vst + voff[dt] + h * 16 * ROWB));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(vst + voff8[dt] + h * 16 * ROWB));
        const bf16x8 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pk[rt][h], o[rt][dt], 0, 0, 0);
      }
  };
  // Sub-block i: its weights, the next one's scores, its product with V; the
  // next scores are masked and reduced last, while the products run.
  auto sub_block = [&](int i, const char *kst, const char *vst, auto masked) {
    rescale();
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 pk[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) probs(rt, s[rt], pk[rt]);
    __builtin_amdgcn_sched_barrier(0);
    // (past the last sub-block K is zeros, and these scores go unused)
    scores(kst, s);
    __builtin_amdgcn_sched_barrier(0);
    pv(vst, pk);
    if constexpr (decltype(masked)::value) mask(s, i + 1);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) bm[rt] = rowmax(s[rt]);
    __builtin_amdgcn_sched_barrier(0);
  };

  wait_vmcnt<0>();   // page ids and queries, before the counted loads
  const int ns = (nb + 1) / 2;
  if (ns > 0) {
    // K of sub-block 0 waits in the last stage, which is refilled at step 0
    const int32_t p0 = page_of(0);
    issue(a.k_pages, ring + (NST - 1) * STAGE, 0, p0);
    page_v = p0;
    issue_stage(0, ring);
    if (NST == 3 && ns > 1) {
      issue_stage(1, ring + STAGE);
      wait_loads_barrier<2 * LPS>();
    } else {
      wait_loads_barrier<LPS>();
    }
    if (wave_nb > 0) {
      scores(ring + (NST - 1) * STAGE, s);
      if (n_full == 0) mask(s, 0);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) bm[rt] = rowmax(s[rt]);
    }
  }
  using Yes = std::true_type;
  using No = std::false_type;
  int cs = 0;
  for (int st = 0; st < ns; ++st) {
    // this stage has landed (the next may fly), and every wave is done with
    // the one before, which is refilled
    if (NST == 3 && st + 1 < ns) wait_loads_barrier<LPS>();
    else wait_loads_barrier<0>();
    const int fill = st + NST - 1;
    if (fill < ns) issue_stage(fill, ring + (cs == 0 ? NST - 1 : cs - 1) * STAGE);
    const char *cur = ring + cs * STAGE;
    const int i = 2 * st;
    if (i + 2 < n_full) {
      sub_block(i, cur, cur + 2 * BLK, No{});
      sub_block(i + 1, cur + BLK, cur + 3 * BLK, No{});
    } else {
#pragma unroll 1
      for (int k = 0; k < 2; ++k)
        if (i + k < wave_nb) sub_block(i + k, cur + k * BLK, cur + (2 + k) * BLK, Yes{});
    }
    cs = cs == NST - 1 ? 0 : cs + 1;
  }
  if (!wave_live) return;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const bool ok = row[rt] < row_end;
    const float l_tot = sum_over_halves(lsum[rt]);
    const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
    const int32_t tok = ok ? row[rt] / G : 0, head = g * G + (ok ? row[rt] - tok * G : 0);
    // A key that the row does not see has weight 0, and 0 times an infinite
    // value is NaN: such rows are taken again, key by key.
    float nan = l_tot;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) nan = __builtin_elementwise_maximum(nan, o[rt][dt][i]);
    const bool again = ok && max_over_halves(nan) != max_over_halves(nan);
    __bf16 *dst = (__bf16 *)a.out + ((int64_t)(un.token0 + tok) * a.num_q_heads + head) * D;
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
      attend_row<true, D>(a, un.r, un.token0 + __shfl(tok, l, 64), __shfl(head, l, 64), __shfl(vis[rt], l, 64));
    }
  }
}

template <int D>
__global__ __launch_bounds__(kThreads) void prompt_attn_f32_kernel(PagedAttnArgs a) {
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
  attend_row<false, D>(a, r, t, h, pos + 1);
}

}  // namespace

hipError_t launch_prompt_attn(const PagedAttnArgs &a, int head_dim, bool bf16, hipStream_t stream) {
  const dim3 block(kThreads);
  if (bf16) {
    const dim3 grid((unsigned)a.units);
    if (head_dim == 128) hipLaunchKernelGGL((prompt_attn_bf16_kernel<128, 1>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((prompt_attn_bf16_kernel<64, 1>), grid, block, 0, stream, a);
    return hipGetLastError();
  }
  const int64_t waves = (int64_t)a.total_tokens * a.num_q_heads;
  const dim3 grid((unsigned)((waves + 3) / 4));
  if (head_dim == 128) hipLaunchKernelGGL((prompt_attn_f32_kernel<128>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((prompt_attn_f32_kernel<64>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace adaserve
