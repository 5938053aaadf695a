// Host side of the serving operators' entry points (rotary append, prompt and
// decode attention, sampling): argument validation, which runs before any HIP
// call, and the launches.
#include "serving.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "adaserve.h"
#include "host_device.h"
#include "host_plan.h"
#include "plan.h"

namespace {

using namespace adaserve;

int32_t elem_size(int32_t dtype) { return dtype == ADASERVE_BF16 ? 2 : 4; }

struct Range {
  const char *begin, *end;
};

// Bytes of `rows` rows of `row` elements, `stride` elements apart.
Range rows_range(const void *p, int64_t rows, int64_t stride, int64_t row, int32_t esz) {
  const char *b = (const char *)p;
  if (!p || rows <= 0 || row <= 0) return {b, b};
  return {b, b + ((rows - 1) * stride + row) * esz};
}

bool overlap(const Range &a, const Range &b) { return a.begin < b.end && b.begin < a.end; }

// What the attention entry points share: head layout, type, pages and scale.
int32_t validate_paged(int32_t num_requests, int32_t num_pages, int32_t bt_stride, int32_t hq, int32_t hkv,
                       int32_t head_dim, int32_t page_size, float sm_scale, int32_t dtype) {
  if (num_requests < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_requests %d < 0", num_requests);
  if (num_pages < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_pages %d < 0", num_pages);
  if (bt_stride < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "block_table_stride %d < 0", bt_stride);
  if (hq <= 0 || hkv <= 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "head counts must be positive (%d, %d)", hq, hkv);
  if (hq % hkv != 0)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_q_heads %d is not a multiple of num_kv_heads %d", hq, hkv);
  if (hq / hkv > 16) return fail(ADASERVE_ERR_UNSUPPORTED, "head group %d > 16", hq / hkv);
  if (hq > kMaxHeads) return fail(ADASERVE_ERR_UNSUPPORTED, "num_q_heads %d > %d", hq, kMaxHeads);
  if (dtype != ADASERVE_F32 && dtype != ADASERVE_BF16)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "dtype %d is neither F32 nor BF16", dtype);
  if (head_dim != 64 && head_dim != 128) return fail(ADASERVE_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", head_dim);
  if (page_size != kPageSize) return fail(ADASERVE_ERR_UNSUPPORTED, "page_size %d (supported: 16)", page_size);
  if (!std::isfinite(sm_scale)) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "sm_scale is not finite");
  if (dtype == ADASERVE_BF16 && !(sm_scale > 0.f))
    return fail(ADASERVE_ERR_UNSUPPORTED, "sm_scale %g: the BF16 path needs sm_scale > 0", (double)sm_scale);
  return ADASERVE_OK;
}

// HIP launches fewer than 2^32 threads.
int32_t validate_launch(const char *what, int64_t blocks, int64_t threads) {
  if (blocks * threads >> 32)
    return fail(ADASERVE_ERR_UNSUPPORTED, "%s: %lld workgroups of %lld threads exceed a launch", what, (long long)blocks,
                (long long)threads);
  return ADASERVE_OK;
}

// `rows` rows `stride` elements apart stay within what a pointer reaches (and their byte count within 64 bits).
int32_t validate_span(const char *name, int64_t rows, int64_t stride) {
  constexpr int64_t kMostElements = (int64_t)1 << 48;
  if (rows > 1 && stride > kMostElements / (rows - 1))
    return fail(ADASERVE_ERR_UNSUPPORTED, "%s: %lld rows %lld elements apart span more than 2^48 elements", name,
                (long long)rows, (long long)stride);
  return ADASERVE_OK;
}

// `rows` rows of `row` elements, `stride` elements apart, readable in 16-byte pieces.
int32_t validate_rows(const char *name, const void *p, int64_t rows, int64_t stride, int64_t row, int32_t esz) {
  if (stride < row) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "%s_row_stride %lld < %lld", name, (long long)stride, (long long)row);
  if (stride > (int64_t)1 << 40) return fail(ADASERVE_ERR_UNSUPPORTED, "%s_row_stride %lld > 2^40", name, (long long)stride);
  if (!aligned(p, 16) || (stride * esz) % 16 != 0)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "%s must be 16-byte aligned with rows a multiple of 16 bytes apart", name);
  return validate_span(name, rows, stride);
}

// Shape checks of prompt attention that the workspace query shares.
int32_t validate_prompt(int32_t num_requests, const int32_t *indptr, const int32_t *ctx, int32_t bt_stride_or_neg,
                        int32_t hq, int64_t &total, int64_t &most_context) {
  total = most_context = 0;
  if (num_requests == 0) return ADASERVE_OK;
  if (!indptr || !ctx) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "host mirrors must not be NULL");
  if (indptr[0] != 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "token_indptr[0] = %d, expected 0", indptr[0]);
  for (int32_t r = 0; r < num_requests; ++r) {
    if (indptr[r + 1] < indptr[r])
      return fail(ADASERVE_ERR_INVALID_ARGUMENT, "token_indptr decreases at request %d", r);
    const int32_t c = ctx[r];
    if (c < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "context_len[%d] = %d < 0", r, c);
    if (c > kMaxPrefixLen) return fail(ADASERVE_ERR_UNSUPPORTED, "context_len[%d] = %d (max %d)", r, c, kMaxPrefixLen);
    if (bt_stride_or_neg >= 0 && ceil_div(c, kPageSize) > bt_stride_or_neg)
      return fail(ADASERVE_ERR_INVALID_ARGUMENT, "context_len[%d] = %d needs %d pages > block_table_stride %d", r, c,
                  ceil_div(c, kPageSize), bt_stride_or_neg);
    if (c > most_context) most_context = c;
  }
  total = indptr[num_requests];
  if (total * hq > INT32_MAX)
    return fail(ADASERVE_ERR_UNSUPPORTED, "%lld tokens of %d query heads exceed 2^31 - 1 rows", (long long)total, hq);
  return ADASERVE_OK;
}

// The units of a prompt attention call, and the table that orders them; more
// requests than it holds are found by a scan on the device, in their own order.
// Several units per workgroup, each workgroup taking every kPromptGrid-th,
// hide the loads that open a unit behind the end of the one before (16 ragged
// prompts of 636-2012 tokens 369 -> 355 us, one of 8191 468 -> 463); that needs
// units in descending order of keys, which the table gives where all rows have as
// many cached keys before them.
struct PromptPlan {
  int64_t units = 0;
  int32_t chunks = 1, chunk_keys = INT32_MAX;
  bool in_order = false;     // every row has about as many cached keys before its request's rows
  size_t ml_bytes = 0, ws_bytes = 0;
};

// Few tiles over many keys (a small chunk of a long prompt) leave compute units
// idle, so their keys are split and joined by a second launch.  Priced by a
// tile's time over k keys, kTileUs + k * kKeyUs, in rounds of kPromptGrid tiles,
// and by the join's traffic: tiles write and the join reads D + 2 floats per row.
// (64 rows over 8064 keys, 64 heads on 8: 167 us whole, 37 split; one row 157 and
// 27; 2000 rows of a prompt, 504 tiles, stay whole: 69.)
// Over a window a tile's keys are those of its rows' windows.
PromptPlan prompt_plan(int32_t num_requests, const int32_t *indptr, const int32_t *ctx, int32_t hq, int32_t hkv,
                       int32_t head_dim, int32_t window, int32_t sinks, bool bf16) {
  constexpr double kTileUs = 9.0, kJoinUs = 6.0, kJoinBytesPerUs = 4e6;
  constexpr int32_t kLeastKeys = 256, kMostChunks = 64;
  const double key_us = 0.022 * head_dim / 128;
  PromptPlan p;
  int32_t keys = 0;
  int64_t least = INT32_MAX, most = 0;
  for (int32_t r = 0; r < num_requests; ++r) {
    const int32_t n = indptr[r + 1] - indptr[r];
    if (n == 0) continue;
    p.units += (int64_t)prompt_tiles(n, hq / hkv, kPromptTileRows) * hkv;
    least = std::min<int64_t>(least, ctx[r] - n);
    most = std::max<int64_t>(most, ctx[r] - n);
    keys = std::max(keys, ctx[r]);
  }
  if (window) keys = window_keys(keys, window, sinks, kPromptTileRows / (hq / hkv) + 1);
  p.in_order = most - least <= 128 || (window && least >= window);
  if (!bf16 || num_requests > kPromptTable || p.units == 0 || p.units >= 2 * kPromptGrid) return p;
  const double row_bytes = 2.0 * (head_dim * 4 + 8) * indptr[num_requests] * hq;
  double best = 0.95 * std::ceil((double)p.units / kPromptGrid) * (kTileUs + keys * key_us);
  const int64_t units = p.units;
  for (int32_t c = 2; c <= kMostChunks; ++c) {
    const int32_t chunk = (ceil_div(keys, c) + 127) / 128 * 128;
    if (chunk < kLeastKeys) break;
    const int32_t chunks = ceil_div(keys, chunk);
    const double us = std::ceil((double)(units * chunks) / kPromptGrid) * (kTileUs + chunk * key_us) + kJoinUs +
                      row_bytes * chunks / kJoinBytesPerUs;
    if (us < best) {
      best = us;
      p.chunks = chunks;
      p.chunk_keys = chunk;
    }
  }
  if (p.chunks > 1) {
    p.units = units * p.chunks;
    p.ml_bytes = round_up((size_t)p.units * kPromptTileRows * 8, 256);
    p.ws_bytes = p.ml_bytes + (size_t)p.units * kPromptTileRows * head_dim * 4;
  }
  return p;
}

void fill_prompt(PromptAttnArgs &a, const PromptPlan &p, const int32_t *indptr, const int32_t *ctx, int32_t tile_rows,
                 void *workspace) {
  const bool split = p.chunks > 1;
  int32_t count = 0;
  if (a.num_requests <= kPromptTable)
    for (int32_t r = 0; r < a.num_requests; ++r) {
      const int32_t n = indptr[r + 1] - indptr[r];
      if (n == 0) continue;
      int32_t i = count++;
      if (!split)
        for (; i > 0 && (a.table[i - 1].n < n || (a.table[i - 1].n == n && a.table[i - 1].ctx < ctx[r])); --i)
          a.table[i] = a.table[i - 1];
      a.table[i] = {0, r, indptr[r], n, ctx[r]};
    }
  int64_t end = 0;
  for (int32_t i = 0; i < count; ++i) {
    const int32_t tiles = prompt_tiles(a.table[i].n, a.group, tile_rows);
    const int32_t below = i + 1 < count ? prompt_tiles(a.table[i + 1].n, a.group, tile_rows) : 0;
    end += (split ? (int64_t)tiles : (int64_t)(tiles - below) * (i + 1)) * a.num_kv_heads;
    a.table[i].unit_end = (int32_t)end;
  }
  a.table_count = count;
  a.units = p.units;
  a.chunks = p.chunks;
  a.chunk_keys = p.chunk_keys;
  a.grid = (int32_t)p.units;
  if (!split && count > 0 && p.units > kPromptGrid && p.in_order) a.grid = kPromptGrid;
  if (split) {
    a.ws_ml = (float *)workspace;
    a.ws_o = (float *)((char *)workspace + p.ml_bytes);
  }
}

int32_t validate_pages(bool any_key, const void *k_pages, const void *v_pages, int32_t num_pages, const int32_t *table) {
  if (any_key && (!k_pages || !v_pages || !table))
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "k_pages, v_pages and block_table are required when a context is non-empty");
  if (any_key && num_pages < 1)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_pages must be >= 1 when a context is non-empty");
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16))
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "k_pages and v_pages must be 16-byte aligned");
  return ADASERVE_OK;
}

int32_t validate_workspace(const void *workspace, size_t given, size_t need) {
  if (need == 0) return ADASERVE_OK;
  if (!workspace || given < need)
    return fail(ADASERVE_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace ? given : (size_t)0, need);
  if (!aligned(workspace, 256)) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "workspace must be 256-byte aligned");
  return ADASERVE_OK;
}

int32_t validate_decode(int32_t num_requests, int32_t hq, int32_t hkv, int32_t max_context, int32_t bt_stride_or_neg) {
  if (max_context < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "max_context %d < 0", max_context);
  if (max_context > kMaxPrefixLen) return fail(ADASERVE_ERR_UNSUPPORTED, "max_context %d > %d", max_context, kMaxPrefixLen);
  if (bt_stride_or_neg >= 0 && ceil_div(max_context, kPageSize) > bt_stride_or_neg)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "max_context %d needs %d pages > block_table_stride %d", max_context,
                ceil_div(max_context, kPageSize), bt_stride_or_neg);
  if ((int64_t)num_requests * hq > INT32_MAX)
    return fail(ADASERVE_ERR_UNSUPPORTED, "%d requests of %d query heads exceed 2^31 - 1 rows", num_requests, hq);
  // (one workgroup each at most, and per query head in the join, of at most kDecodeSplitRequests)
  return validate_launch("decode attention", (int64_t)num_requests * hkv, kServingThreads);
}

int32_t validate_sample(int32_t num_rows, int32_t vocab, int32_t dtype) {
  if (num_rows < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_rows %d < 0", num_rows);
  if (vocab < 1 || vocab > kSampleMaxVocab)
    return fail(vocab < 1 ? ADASERVE_ERR_INVALID_ARGUMENT : ADASERVE_ERR_UNSUPPORTED, "vocab %d outside [1, %d]",
                vocab, kSampleMaxVocab);
  if (dtype != ADASERVE_F32 && dtype != ADASERVE_BF16)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "dtype %d is neither F32 nor BF16", dtype);
  const int64_t parts = sample_plan(num_rows, vocab, dtype == ADASERVE_BF16).parts;
  const int32_t st = validate_launch("sampling", num_rows * parts, kServingThreads);
  return st != ADASERVE_OK ? st : validate_launch("sampling", num_rows, kSampleDrawThreads);
}

// Prompt attention; over a window where there is one.
int32_t prompt_attn_impl(int32_t num_requests, const int32_t *token_indptr, const int32_t *token_indptr_host,
                         const void *q, int64_t q_row_stride, const void *k_pages, const void *v_pages,
                         int32_t num_pages, const int32_t *block_table, int32_t block_table_stride,
                         const int32_t *context_len, const int32_t *context_len_host, int32_t num_q_heads,
                         int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t window, int32_t sinks,
                         float sm_scale, int32_t dtype, void *out, void *workspace, size_t workspace_bytes,
                         void *stream) {
  int32_t st = validate_paged(num_requests, num_pages, block_table_stride, num_q_heads, num_kv_heads, head_dim,
                              page_size, sm_scale, dtype);
  if (st != ADASERVE_OK) return st;
  int64_t total, most;
  st = validate_prompt(num_requests, token_indptr_host, context_len_host, block_table_stride, num_q_heads, total, most);
  if (st != ADASERVE_OK) return st;
  if (total == 0) return ADASERVE_OK;
  if (sees_all(window, sinks, most)) window = sinks = 0;
  if (!token_indptr || !q || !out || !context_len)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "a required device pointer is NULL");
  st = validate_rows("q", q, total, q_row_stride, (int64_t)num_q_heads * head_dim, elem_size(dtype));
  if (st != ADASERVE_OK) return st;
  if (!aligned(out, 16)) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "out must be 16-byte aligned");
  st = validate_pages(most > 0, k_pages, v_pages, num_pages, block_table);
  if (st != ADASERVE_OK) return st;
  const PromptPlan plan = prompt_plan(num_requests, token_indptr_host, context_len_host, num_q_heads, num_kv_heads,
                                      head_dim, window, sinks, dtype == ADASERVE_BF16);
  st = validate_workspace(workspace, workspace_bytes, plan.ws_bytes);
  if (st != ADASERVE_OK) return st;
  PromptAttnArgs a{};
  a.num_requests = num_requests;
  a.token_indptr = token_indptr;
  a.context_len = context_len;
  a.block_table = block_table;
  a.bt_stride = block_table_stride;
  a.num_pages = num_pages;
  a.q = q;
  a.q_stride = q_row_stride;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.out = out;
  a.total_tokens = (int32_t)total;
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = num_kv_heads;
  a.group = num_q_heads / num_kv_heads;
  a.sm_scale = sm_scale;
  a.scale_log2 = sm_scale * 1.4426950408889634f;
  a.window = window;
  a.sinks = sinks;
  if (dtype == ADASERVE_BF16) {
    fill_prompt(a, plan, token_indptr_host, context_len_host, kPromptTileRows, workspace);
  } else {
    // 32-row tiles read each key half as often, 16-row tiles put more units to work: 2250 tiles of 32
    // (2 prompts of up to 1500 tokens, D = 128) 301 against 341 us, 1800 (8 of up to 300) 88 against 83
    for (a.f32_rows = 32;; a.f32_rows = 16) {
      a.units = 0;
      for (int32_t r = 0; r < num_requests; ++r)
        a.units += (int64_t)prompt_tiles(token_indptr_host[r + 1] - token_indptr_host[r], a.group, a.f32_rows) * num_kv_heads;
      if (a.units >= 2048 || a.f32_rows == 16) break;
    }
    PromptPlan tiles;
    tiles.units = a.units;
    fill_prompt(a, tiles, token_indptr_host, context_len_host, a.f32_rows, nullptr);
  }
  // (the join's rows: below 2^17, those of 512 tiles)
  st = validate_launch("prompt attention", dtype == ADASERVE_BF16 ? a.grid : round_up(a.units, kPromptGrid), kServingThreads);
  if (st != ADASERVE_OK) return st;
  st = check_device();
  if (st != ADASERVE_OK) return st;
  return launch_status(launch_prompt_attn(a, head_dim, dtype == ADASERVE_BF16, (hipStream_t)stream),
                       "prompt attention launch");
}

// Single-token attention; over a window where there is one.
int32_t decode_attn_impl(int32_t num_requests, const void *q, int64_t q_row_stride, const void *k_pages,
                         const void *v_pages, int32_t num_pages, const int32_t *block_table,
                         int32_t block_table_stride, const int32_t *context_len, int32_t max_context,
                         int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                         int32_t window, int32_t sinks, float sm_scale, int32_t dtype, void *out, void *workspace,
                         size_t workspace_bytes, void *stream) {
  int32_t st = validate_paged(num_requests, num_pages, block_table_stride, num_q_heads, num_kv_heads, head_dim,
                              page_size, sm_scale, dtype);
  if (st != ADASERVE_OK) return st;
  st = validate_decode(num_requests, num_q_heads, num_kv_heads, max_context, block_table_stride);
  if (st != ADASERVE_OK) return st;
  if (num_requests == 0) return ADASERVE_OK;
  if (sees_all(window, sinks, max_context)) window = sinks = 0;
  if (!q || !out || !context_len) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "a required device pointer is NULL");
  st = validate_rows("q", q, num_requests, q_row_stride, (int64_t)num_q_heads * head_dim, elem_size(dtype));
  if (st != ADASERVE_OK) return st;
  if (!aligned(out, 16)) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "out must be 16-byte aligned");
  st = validate_pages(max_context > 0, k_pages, v_pages, num_pages, block_table);
  if (st != ADASERVE_OK) return st;
  const DecodePlan plan = decode_plan(num_requests, num_q_heads, num_kv_heads, head_dim,
                                      window ? window_keys(max_context, window, sinks, 1) : max_context);
  st = validate_workspace(workspace, workspace_bytes, plan.ws_bytes);
  if (st != ADASERVE_OK) return st;
  st = check_device();
  if (st != ADASERVE_OK) return st;
  PagedAttnArgs a{};
  a.num_requests = num_requests;
  a.context_len = context_len;
  a.block_table = block_table;
  a.bt_stride = block_table_stride;
  a.num_pages = num_pages;
  a.q = q;
  a.q_stride = q_row_stride;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.out = out;
  a.total_tokens = num_requests;
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = num_kv_heads;
  a.group = num_q_heads / num_kv_heads;
  a.max_context = max_context;
  a.units_per_head = plan.units_per_head;
  a.min_blocks = kDecodeMinBlocks;
  if (plan.split) {
    a.ws_request = (int32_t *)workspace;
    a.ws_ml = (float *)((char *)workspace + plan.ml_offset);
    a.ws_o = (float *)((char *)workspace + plan.o_offset);
  }
  a.sm_scale = sm_scale;
  a.scale_log2 = sm_scale * 1.4426950408889634f;
  a.window = window;
  a.sinks = sinks;
  return launch_status(launch_decode_attn(a, head_dim, dtype == ADASERVE_BF16, (hipStream_t)stream),
                       "decode attention launch");
}

}  // namespace

extern "C" {

int32_t adaserve_rope_append_kv(int32_t num_requests, int32_t num_tokens, const int32_t *token_indptr,
                                const int32_t *prefix_len, const int32_t *positions, const void *q,
                                int64_t q_row_stride, const void *k, int64_t k_row_stride, const void *v,
                                int64_t v_row_stride, const float *inv_freq, int32_t rotary_dim, int32_t interleaved,
                                int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                                int32_t dtype, void *q_out, void *k_out, void *k_pages, void *v_pages,
                                int32_t num_pages, const int32_t *block_table, int32_t block_table_stride,
                                int32_t *new_prefix_len, void *stream) {
  if (num_requests < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_requests %d < 0", num_requests);
  if (num_tokens < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_tokens %d < 0", num_tokens);
  if (dtype != ADASERVE_F32 && dtype != ADASERVE_BF16)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "dtype %d is neither F32 nor BF16", dtype);
  const int32_t esz = elem_size(dtype);
  if (head_dim < 1) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "head_dim %d < 1", head_dim);
  if (head_dim > kRopeMaxHeadDim || (head_dim * esz) % 16 != 0)
    return fail(ADASERVE_ERR_UNSUPPORTED, "head_dim %d: rows must be a multiple of 16 bytes, of at most %d elements",
                head_dim, kRopeMaxHeadDim);
  if (rotary_dim < 0 || rotary_dim > head_dim)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "rotary_dim %d outside [0, head_dim = %d]", rotary_dim, head_dim);
  if ((rotary_dim * esz) % 32 != 0)
    return fail(ADASERVE_ERR_UNSUPPORTED, "rotary_dim %d: rotated parts must be a multiple of 32 bytes", rotary_dim);
  if (interleaved != 0 && interleaved != 1)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "interleaved %d is neither 0 nor 1", interleaved);
  if (num_kv_heads < 1 || (q && num_q_heads < 1))
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "head counts must be positive (%d, %d)", num_q_heads, num_kv_heads);
  if (num_kv_heads > kMaxHeads || (q && num_q_heads > kMaxHeads))
    return fail(ADASERVE_ERR_UNSUPPORTED, "more than %d heads (%d, %d)", kMaxHeads, num_q_heads, num_kv_heads);
  if (page_size < 1) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "page_size %d < 1", page_size);
  if (num_pages < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "num_pages %d < 0", num_pages);
  if (block_table_stride < 0) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "block_table_stride %d < 0", block_table_stride);
  if ((q == nullptr) != (q_out == nullptr)) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "q and q_out go together");
  if ((k_pages == nullptr) != (v_pages == nullptr))
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "k_pages and v_pages go together");
  const bool append = k_pages != nullptr;
  if (!append && new_prefix_len) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "new_prefix_len needs pages to append to");
  if (num_requests == 0) return ADASERVE_OK;
  if (!token_indptr || !prefix_len) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "a required device pointer is NULL");
  if (append && (!new_prefix_len || (block_table_stride > 0 && !block_table)))
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "an append needs block_table and new_prefix_len");
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(q_out, 16) || !aligned(k_out, 16))
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "q_out, k_out, k_pages and v_pages must be 16-byte aligned");
  const int64_t q_row = (int64_t)num_q_heads * head_dim, kv_row = (int64_t)num_kv_heads * head_dim;
  const Range lens_in = {(const char *)prefix_len, (const char *)(prefix_len + num_requests)};
  const Range lens_out = {(const char *)new_prefix_len, (const char *)new_prefix_len + (append ? 4ll * num_requests : 0)};
  if (new_prefix_len != prefix_len && overlap(lens_in, lens_out))
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "new_prefix_len overlaps prefix_len without being it");
  if (num_tokens > 0) {
    if (rotary_dim > 0 && !inv_freq) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "inv_freq is NULL");
    if (!q && !k) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "neither q nor k is given");
    if (append && (!k || !v)) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "an append needs k and v");
    if (k_out && !k) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "k_out needs k");
    if (k && !k_out && !append) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "k has neither k_out nor pages to go to");
    if (q) {
      const int32_t st = validate_rows("q", q, num_tokens, q_row_stride, q_row, esz);
      if (st != ADASERVE_OK) return st;
    }
    if (k) {
      const int32_t st = validate_rows("k", k, num_tokens, k_row_stride, kv_row, esz);
      if (st != ADASERVE_OK) return st;
    }
    if (append) {
      const int32_t st = validate_rows("v", v, num_tokens, v_row_stride, kv_row, esz);
      if (st != ADASERVE_OK) return st;
    }
    // an output is its own input or apart from every input
    const Range qi = rows_range(q, num_tokens, q_row_stride, q_row, esz), ki = rows_range(k, num_tokens, k_row_stride, kv_row, esz);
    const Range vi = rows_range(append ? v : nullptr, num_tokens, v_row_stride, kv_row, esz);
    const Range qo = rows_range(q_out, num_tokens, q_row, q_row, esz), ko = rows_range(k_out, num_tokens, kv_row, kv_row, esz);
    const bool q_same = q_out == q && q_row_stride == q_row, k_same = k_out == k && k_row_stride == kv_row;
    if ((overlap(qo, qi) && !q_same) || overlap(qo, ki) || overlap(qo, vi) || (overlap(ko, ki) && !k_same) ||
        overlap(ko, qi) || overlap(ko, vi) || overlap(qo, ko))
      return fail(ADASERVE_ERR_INVALID_ARGUMENT, "q_out or k_out overlaps an input without being it (dense rows), or the other");
  }
  const int64_t length_blocks = append ? rope_length_blocks(num_requests) : 0;
  int32_t st = validate_launch("rotary append", new_prefix_len == prefix_len ? std::max<int64_t>(num_tokens, length_blocks)
                                                                              : num_tokens + length_blocks, kServingThreads);
  if (st != ADASERVE_OK) return st;
  st = check_device();
  if (st != ADASERVE_OK) return st;
  RopeAppendArgs a{};
  a.num_requests = num_requests;
  a.num_tokens = num_tokens;
  a.token_indptr = token_indptr;
  a.prefix_len = prefix_len;
  a.positions = positions;
  a.q = q;
  a.k = k;
  a.v = append ? v : nullptr;
  a.q_stride = q_row_stride;
  a.k_stride = k_row_stride;
  a.v_stride = v_row_stride;
  a.inv_freq = inv_freq;
  a.rotary_dim = rotary_dim;
  a.interleaved = interleaved;
  a.num_q_heads = q ? num_q_heads : 0;
  a.num_kv_heads = k ? num_kv_heads : 0;
  a.head_dim = head_dim;
  a.page_size = page_size;
  a.q_out = q_out;
  a.k_out = k_out;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.num_pages = num_pages;
  a.block_table = block_table;
  a.bt_stride = block_table_stride;
  a.new_prefix_len = new_prefix_len;
  return launch_status(launch_rope_append(a, dtype == ADASERVE_BF16, (hipStream_t)stream), "rotary append launch");
}

size_t adaserve_prompt_attn_workspace_bytes(int32_t num_requests, const int32_t *token_indptr_host,
                                            const int32_t *context_len_host, int32_t num_q_heads, int32_t num_kv_heads,
                                            int32_t head_dim, int32_t page_size, int32_t dtype) {
  int64_t total, most;
  if (validate_paged(num_requests, 0, 0, num_q_heads, num_kv_heads, head_dim, page_size, 1.f, dtype) != ADASERVE_OK ||
      validate_prompt(num_requests, token_indptr_host, context_len_host, -1, num_q_heads, total, most) != ADASERVE_OK)
    return SIZE_MAX;
  return prompt_plan(num_requests, token_indptr_host, context_len_host, num_q_heads, num_kv_heads, head_dim, 0, 0,
                     dtype == ADASERVE_BF16)
      .ws_bytes;
}

int32_t adaserve_prompt_attn(int32_t num_requests, const int32_t *token_indptr, const int32_t *token_indptr_host,
                             const void *q, int64_t q_row_stride, const void *k_pages, const void *v_pages,
                             int32_t num_pages, const int32_t *block_table, int32_t block_table_stride,
                             const int32_t *context_len, const int32_t *context_len_host, int32_t num_q_heads,
                             int32_t num_kv_heads, int32_t head_dim, int32_t page_size, float sm_scale, int32_t dtype,
                             void *out, void *workspace, size_t workspace_bytes, void *stream) {
  return prompt_attn_impl(num_requests, token_indptr, token_indptr_host, q, q_row_stride, k_pages, v_pages, num_pages,
                          block_table, block_table_stride, context_len, context_len_host, num_q_heads, num_kv_heads,
                          head_dim, page_size, 0, 0, sm_scale, dtype, out, workspace, workspace_bytes, stream);
}

size_t adaserve_window_prompt_attn_workspace_bytes(int32_t num_requests, const int32_t *token_indptr_host,
                                                   const int32_t *context_len_host, int32_t num_q_heads,
                                                   int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                                                   int32_t window, int32_t sinks, int32_t dtype) {
  int64_t total, most;
  if (validate_window(window, sinks) != ADASERVE_OK ||
      validate_paged(num_requests, 0, 0, num_q_heads, num_kv_heads, head_dim, page_size, 1.f, dtype) != ADASERVE_OK ||
      validate_prompt(num_requests, token_indptr_host, context_len_host, -1, num_q_heads, total, most) != ADASERVE_OK)
    return SIZE_MAX;
  if (sees_all(window, sinks, most)) window = sinks = 0;
  return prompt_plan(num_requests, token_indptr_host, context_len_host, num_q_heads, num_kv_heads, head_dim, window, sinks,
                     dtype == ADASERVE_BF16)
      .ws_bytes;
}

int32_t adaserve_window_prompt_attn(int32_t num_requests, const int32_t *token_indptr,
                                    const int32_t *token_indptr_host, const void *q, int64_t q_row_stride,
                                    const void *k_pages, const void *v_pages, int32_t num_pages,
                                    const int32_t *block_table, int32_t block_table_stride,
                                    const int32_t *context_len, const int32_t *context_len_host, int32_t num_q_heads,
                                    int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t window,
                                    int32_t sinks, float sm_scale, int32_t dtype, void *out, void *workspace,
                                    size_t workspace_bytes, void *stream) {
  const int32_t st = validate_window(window, sinks);
  if (st != ADASERVE_OK) return st;
  return prompt_attn_impl(num_requests, token_indptr, token_indptr_host, q, q_row_stride, k_pages, v_pages, num_pages,
                          block_table, block_table_stride, context_len, context_len_host, num_q_heads, num_kv_heads,
                          head_dim, page_size, window, sinks, sm_scale, dtype, out, workspace, workspace_bytes, stream);
}

size_t adaserve_decode_attn_workspace_bytes(int32_t num_requests, int32_t max_context, int32_t num_q_heads,
                                            int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t dtype) {
  if (validate_paged(num_requests, 0, 0, num_q_heads, num_kv_heads, head_dim, page_size, 1.f, dtype) != ADASERVE_OK ||
      validate_decode(num_requests, num_q_heads, num_kv_heads, max_context, -1) != ADASERVE_OK)
    return SIZE_MAX;
  return decode_plan(num_requests, num_q_heads, num_kv_heads, head_dim, max_context).ws_bytes;
}

int32_t adaserve_decode_attn(int32_t num_requests, const void *q, int64_t q_row_stride, const void *k_pages,
                             const void *v_pages, int32_t num_pages, const int32_t *block_table,
                             int32_t block_table_stride, const int32_t *context_len, int32_t max_context,
                             int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                             float sm_scale, int32_t dtype, void *out, void *workspace, size_t workspace_bytes,
                             void *stream) {
  return decode_attn_impl(num_requests, q, q_row_stride, k_pages, v_pages, num_pages, block_table, block_table_stride,
                          context_len, max_context, num_q_heads, num_kv_heads, head_dim, page_size, 0, 0, sm_scale,
                          dtype, out, workspace, workspace_bytes, stream);
}

size_t adaserve_window_decode_attn_workspace_bytes(int32_t num_requests, int32_t max_context, int32_t num_q_heads,
                                                   int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                                                   int32_t window, int32_t sinks, int32_t dtype) {
  if (validate_window(window, sinks) != ADASERVE_OK ||
      validate_paged(num_requests, 0, 0, num_q_heads, num_kv_heads, head_dim, page_size, 1.f, dtype) != ADASERVE_OK ||
      validate_decode(num_requests, num_q_heads, num_kv_heads, max_context, -1) != ADASERVE_OK)
    return SIZE_MAX;
  const int32_t keys = sees_all(window, sinks, max_context) ? max_context : window_keys(max_context, window, sinks, 1);
  return decode_plan(num_requests, num_q_heads, num_kv_heads, head_dim, keys).ws_bytes;
}

int32_t adaserve_window_decode_attn(int32_t num_requests, const void *q, int64_t q_row_stride, const void *k_pages,
                                    const void *v_pages, int32_t num_pages, const int32_t *block_table,
                                    int32_t block_table_stride, const int32_t *context_len, int32_t max_context,
                                    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                                    int32_t window, int32_t sinks, float sm_scale, int32_t dtype, void *out,
                                    void *workspace, size_t workspace_bytes, void *stream) {
  const int32_t st = validate_window(window, sinks);
  if (st != ADASERVE_OK) return st;
  return decode_attn_impl(num_requests, q, q_row_stride, k_pages, v_pages, num_pages, block_table, block_table_stride,
                          context_len, max_context, num_q_heads, num_kv_heads, head_dim, page_size, window, sinks,
                          sm_scale, dtype, out, workspace, workspace_bytes, stream);
}

size_t adaserve_sample_workspace_bytes(int32_t num_rows, int32_t vocab, int32_t dtype) {
  if (validate_sample(num_rows, vocab, dtype) != ADASERVE_OK) return SIZE_MAX;
  return sample_plan(num_rows, vocab, dtype == ADASERVE_BF16).bytes;
}

int32_t adaserve_sample(const void *logits, int64_t row_stride, int32_t num_rows, int32_t vocab, int32_t dtype,
                        const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                        const float *u, int32_t *out_token, void *workspace, size_t workspace_bytes, void *stream) {
  int32_t st = validate_sample(num_rows, vocab, dtype);
  if (st != ADASERVE_OK) return st;
  if (row_stride < vocab)
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "row_stride %lld < vocab %d", (long long)row_stride, vocab);
  if (num_rows == 0) return ADASERVE_OK;
  if (!logits || !u || !out_token) return fail(ADASERVE_ERR_INVALID_ARGUMENT, "a required device pointer is NULL");
  if (!aligned(logits, elem_size(dtype)) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) ||
      !aligned(min_p, 4) || !aligned(u, 4) || !aligned(out_token, 4))
    return fail(ADASERVE_ERR_INVALID_ARGUMENT, "a pointer is not aligned to its elements");
  st = validate_span("logits", num_rows, row_stride);
  if (st != ADASERVE_OK) return st;
  const SamplePlan plan = sample_plan(num_rows, vocab, dtype == ADASERVE_BF16);
  st = validate_workspace(workspace, workspace_bytes, plan.bytes);
  if (st != ADASERVE_OK) return st;
  st = check_device();
  if (st != ADASERVE_OK) return st;
  SampleArgs a{};
  a.logits = logits;
  a.row_stride = row_stride;
  a.rows = num_rows;
  a.vocab = vocab;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.u = u;
  a.out_token = out_token;
  a.parts = plan.parts;
  a.part_vecs = plan.part_vecs;
  char *ws = (char *)workspace;
  a.ws_hist = (uint64_t *)ws;
  a.ws_cum_w = (uint64_t *)(ws + plan.cum_w);
  a.ws_cum_n = (uint32_t *)(ws + plan.cum_n);
  a.ws_max = (uint32_t *)(ws + plan.max);
  a.ws_part_w = (uint64_t *)(ws + plan.part_w);
  a.ws_count = (uint32_t *)(ws + plan.count);
  a.ws_list = (uint64_t *)(ws + plan.list);
  return launch_status(launch_sample(a, dtype == ADASERVE_BF16, (hipStream_t)stream), "sampling launch");
}

}  // extern "C"
