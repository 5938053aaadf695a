// Internal interface between the host entry points of the serving operators
// (serving.cpp) and their gfx950 kernels: what fills the paged cache
// (rope_append.hip), attention of prompts and of single tokens over it
// (prompt_attn.hip, decode_attn.hip) and sampling (sample.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace adaserve {

constexpr int kMaxHeads = 4096;          // of one kind, in the serving operators
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
  int32_t num_kv_heads;
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

hipError_t launch_rope_append(const RopeAppendArgs &a, bool bf16, hipStream_t stream);

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
  int32_t max_context;           // (decode attention)
  float sm_scale;
  float scale_log2;              // sm_scale * log2(e)
};

hipError_t launch_prompt_attn(const PagedAttnArgs &a, int head_dim, bool bf16, hipStream_t stream);
hipError_t launch_decode_attn(const PagedAttnArgs &a, int head_dim, bool bf16, hipStream_t stream);

constexpr int kSampleMaxVocab = 1 << 20;   // sums of 2^32 per token stay below 2^53

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
};

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t stream);

}  // namespace adaserve
