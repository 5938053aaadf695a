// Internal interface between the host entry points of the serving operators
// (serving.cpp) and their gfx950 kernels: what fills the paged cache
// (rope_append.hip), attention of prompts and of single tokens over it
// (prompt_attn.hip, decode_attn.hip) and sampling (sample.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "plan.h"

namespace adaserve {

constexpr int kMaxHeads = 4096;          // of one kind, in the serving operators
constexpr int kServingThreads = 256;     // of a workgroup, but in sampling's last pass
constexpr int kSampleDrawThreads = 1024;
constexpr int kRopeMaxHeadDim = 512;

struct RopeAppendArgs {
  int32_t num_requests;
  int32_t num_tokens;
  const int32_t *token_indptr;   // [B + 1]
  const int32_t *prefix_len;     // [B]
  const int32_t *positions;      // [num_tokens], or null: the cache positions
  const void *q, *k, *v;         // rows q_stride, k_stride, v_stride elements apart; null: none
  int64_t q_stride, k_stride, v_stride;
  const float *inv_freq;         // [rotary_dim / 2]
  int32_t rotary_dim;
  int32_t interleaved;
  int32_t num_q_heads;           // 0 without q
  int32_t num_kv_heads;          // 0 without k
  int32_t head_dim;
  int32_t page_size;
  void *q_out;                   // [num_tokens, Hq, D]
  void *k_out;                   // [num_tokens, Hkv, D], or null
  void *k_pages, *v_pages;       // [num_pages, Hkv, page_size, D], or null: no append
  int32_t num_pages;
  const int32_t *block_table;    // [B, bt_stride]
  int32_t bt_stride;
  int32_t *new_prefix_len;       // [B], or null
};

// Workgroups that write the new lengths, a wave per request.
inline int64_t rope_length_blocks(int32_t num_requests) { return ((int64_t)num_requests + 3) / 4; }

hipError_t launch_rope_append(const RopeAppendArgs &a, bool bf16, hipStream_t stream);

// The requests of a prompt attention call in descending order of tiles.
constexpr int kPromptTileRows = 256;   // 4 waves x 64 rows
constexpr int kPromptGrid = 256;       // workgroups on the device at a time: one per CU
constexpr int kPromptTable = 128;
struct PromptEntry {
  int32_t unit_end;   // exclusive end of the units of the levels that this and the requests before it have
  int32_t request;
  int32_t token0;     // token_indptr[request]
  int32_t n, ctx;     // its rows and its keys
};

// Row tiles of n tokens with `group` query heads per kv-head.
ADASERVE_HD int32_t prompt_tiles(int32_t n, int32_t group, int32_t tile_rows) {
  return (int32_t)(((int64_t)n * group + tile_rows - 1) / tile_rows);
}

struct PagedAttnArgs {
  int32_t num_requests;
  const int32_t *token_indptr;   // [B + 1] (prompt attention)
  const int32_t *context_len;    // [B]
  const int32_t *block_table;    // [B, bt_stride]
  int32_t bt_stride;
  int32_t num_pages;
  const void *q;                 // [T, Hq, D], rows q_stride elements apart
  int64_t q_stride;
  const void *k_pages, *v_pages; // [num_pages, Hkv, 16, D]
  void *out;                     // [T, Hq, D]
  int32_t total_tokens;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;                 // Hq / Hkv
  float sm_scale;
  float scale_log2;              // sm_scale * log2(e)
  int32_t window, sinks;         // a row sees the newest `window` positions and the first `sinks` (window 0: all)
  // prompt attention
  int64_t units;                 // tiles of all heads, times chunks
  int32_t chunks;                // most chunks of keys per tile: 1 unless there are few tiles
  int32_t chunk_keys;            // keys per chunk (INT32_MAX: all)
  int32_t grid;                  // workgroups: one per unit, or kPromptGrid
  int32_t f32_rows;              // rows per F32 tile: 16 or 32
  int32_t table_count;           // entries used in table[] (0: the device arrays are scanned)
  // decode attention (DecodePlan); prompt attention with split keys: sums and
  // references of [units, kPromptTileRows] rows in ws_o and ws_ml
  int32_t max_context;
  int32_t units_per_head;
  int32_t min_blocks;
  int32_t *ws_request;           // [B, 2] first unit, units; null: a unit is a request
  float *ws_ml;                  // [units, 2, Hq, 2] reference, sum
  float *ws_o;                   // [units, 2, Hq, D] weighted sums of V
};

// (apart, since the launches of decode attention need not carry its 2.5 KB)
struct PromptAttnArgs : PagedAttnArgs {
  PromptEntry table[kPromptTable];
};

// Decode attention's work, from sizes alone.  Per kv-head the batch's 32-key
// blocks are dealt in equal, contiguous shares to as many units as the device
// holds at a time, so that all end together whatever the lengths; a unit goes
// from request to request, and a request in several units is joined by a second
// launch.  Requests of one short run each, and more of them than the scan takes,
// are units themselves.
constexpr int kDecodeRows = 16;              // most query heads per kv-head: the columns of a matrix tile
// One block per wave: in a graph, 32 heads on 8, a request of 1500 tokens 8.7 us and
// of 6000 12.3; with shares of 8 blocks and more 9.5 and 10.9, of 2 and more 8.5 and 11.7.
constexpr int kDecodeMinBlocks = 4;
constexpr int kDecodeUnits = 512;            // on the device: two workgroups per CU
constexpr int kDecodeSplitRequests = 1024;

struct DecodePlan {
  int32_t units_per_head;
  bool split;
  int64_t ml_offset, o_offset;
  size_t ws_bytes;
};

inline DecodePlan decode_plan(int32_t B, int32_t hq, int32_t hkv, int32_t head_dim, int32_t max_context) {
  DecodePlan p{};
  const int64_t blocks = (max_context + 31) / 32;
  p.split = blocks > kDecodeMinBlocks && B <= kDecodeSplitRequests;
  p.units_per_head = B;
  if (p.split) {
    int64_t units = kDecodeUnits / hkv;
    const int64_t most = B * ((blocks + kDecodeMinBlocks - 1) / kDecodeMinBlocks);
    if (units > most) units = most;
    if (units < 1) units = 1;
    p.units_per_head = (int32_t)units;
    const size_t slots = (size_t)units * 2 * hq;
    p.ml_offset = ((int64_t)B * 8 + 255) / 256 * 256;
    p.o_offset = p.ml_offset + (int64_t)((slots * 8 + 255) / 256 * 256);
    p.ws_bytes = (size_t)p.o_offset + slots * head_dim * 4;
  }
  return p;
}

hipError_t launch_prompt_attn(const PromptAttnArgs &a, int head_dim, bool bf16, hipStream_t stream);
hipError_t launch_decode_attn(const PagedAttnArgs &a, int head_dim, bool bf16, hipStream_t stream);

constexpr int kSampleMaxVocab = 1 << 20;   // sums of 2^32 per token stay below 2^53

constexpr int kSampleBins = 512;
constexpr int kSampleMaxParts = 64;
constexpr int kSampleList = 8192;           // listed tokens of a row that pass 4 holds in LDS
constexpr int kSampleListCap = 512;         // tokens in the list of a quarter of a part

struct SampleArgs {
  const void *logits;            // [rows, row_stride]
  int64_t row_stride;
  int32_t rows;
  int32_t vocab;
  const float *temperature;      // [rows] each, or null: 1, off, off, off
  const int32_t *top_k;
  const float *top_p;
  const float *min_p;
  const float *u;                // [rows]
  int32_t *out_token;            // [rows]
  int32_t parts;                 // parts of a row (SamplePlan)
  int32_t part_vecs;             // 16-byte vectors per part
  uint32_t *ws_max;              // [rows, parts] largest key (all ones: a NaN or +inf)
  uint64_t *ws_hist;             // [rows, parts, bins] mass | count << 48
  uint64_t *ws_cum_w;            // [rows, bins + 1] mass of the bins before
  uint32_t *ws_cum_n;            // [rows, bins + 1] tokens of the bins before
  uint64_t *ws_part_w;           // [rows, parts] mass of the bins before all cuts
  uint32_t *ws_count;            // [rows, parts, 4] listed tokens
  uint64_t *ws_list;             // [rows, parts, 4, kSampleListCap] key << 32 | index
};

// Parts of 4096 to 32768 logits: a few rows are cut finely, to run on many
// compute units; many rows coarsely, since pass 3 adds up a row's histograms in
// every part.  At most 64 parts (2^20 logits and up to 7 before the row).
struct SamplePlan {
  int32_t parts, part_vecs;
  size_t cum_w, cum_n, max, part_w, count, list, bytes;   // offsets; the histograms come first
};

inline SamplePlan sample_plan(int32_t rows, int32_t vocab, bool bf16) {
  const int32_t epv = bf16 ? 8 : 4;
  int32_t elements = rows <= 16 ? 4096 : rows <= 64 ? 8192 : 16384;
  while (elements < 32768 && (int64_t)(vocab + epv - 1 + elements - 1) / elements > kSampleMaxParts) elements *= 2;
  SamplePlan p;
  p.part_vecs = elements / epv;
  p.parts = (vocab + epv - 1 + elements - 1) / elements;
  const size_t all = (size_t)rows * p.parts;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  p.cum_w = up(all * kSampleBins * 8);
  p.cum_n = p.cum_w + up((size_t)rows * (kSampleBins + 1) * 8);
  p.max = p.cum_n + up((size_t)rows * (kSampleBins + 1) * 4);
  p.part_w = p.max + up(all * 4);
  p.count = p.part_w + up(all * 8);
  p.list = p.count + up(all * 4 * 4);
  p.bytes = rows ? p.list + up(all * 4 * kSampleListCap * 8) : 0;
  return p;
}

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t stream);

}  // namespace adaserve
