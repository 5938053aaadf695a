/*
 * adaserve.h -- C ABI of the MI355X (gfx950) batched tree-verification library.
 *
 * One verification pass of SLO-customised speculative decoding (section 4.3,
 * step 4): the target model scores every node of every request's draft token
 * tree in one pass, and the tokens to commit are read off the logits of those
 * nodes (section 5.1).  The library provides the steps of that pass that run
 * after the projections:
 *
 *   adaserve_tree_attn_verify  paged tree attention: each node attends to its
 *                              request's cached prefix plus its own
 *                              root-to-node path (section 2, draft token tree;
 *                              section 3, Theorem 1's root-to-v paths);
 *   adaserve_node_argmax       the target's greedy choice at every node;
 *   adaserve_tree_accept       the longest accepted root path per request and
 *                              the tokens it commits;
 *   adaserve_tree_verify_step  the three above as one call;
 *   adaserve_tree_accept_sampled  the same for sampled decoding (speculative
 *                              sampling over the tree);
 *   adaserve_commit_accepted_kv  the accepted path's keys and values written
 *                              into the request's paged cache;
 *   adaserve_select_trees      (before the pass) the two selection phases that
 *                              turn candidate trees into the draft trees;
 *   adaserve_beam_step         (before selection) one beam-search step of the
 *                              speculation phase that grows the candidate trees;
 * and what a request needs before and beside speculation:
 *   adaserve_rope_append_kv    rotary embedding of q and k, and the keys and
 *                              values written into the paged cache;
 *   adaserve_prompt_attn       causal attention of packed prompts over it;
 *   adaserve_decode_attn       attention of one new token per request;
 *   adaserve_sample            a token per row by temperature, top-k, top-p, min-p;
 *   adaserve_window_prompt_attn, adaserve_window_decode_attn, adaserve_window_tree_attn
 *                              the three attentions of models that see a window of
 *                              the newest keys and a few first ones (sinks);
 * and the cache's pages, all on the device:
 *   adaserve_update_pages      what left the window is freed, what comes next taken;
 *   adaserve_fork_pages        rows of the cache go over to other rows (beams, samples);
 *   adaserve_compact_pages     the pages in use move to the front of the pool;
 *   adaserve_copy_pages        page contents, as the two before ask for.
 *
 * Conventions for every entry point:
 *  - Pointers without a _host suffix are DEVICE pointers owned by the caller;
 *    _host pointers are host memory read synchronously during the call and
 *    not retained.  Nothing is allocated or freed, and nothing synchronises:
 *    work is enqueued on `stream` (a hipStream_t; NULL = the null stream) and
 *    the call returns.
 *  - Every scalar, pointer and host-mirror value is validated on the host
 *    before anything is enqueued; on a non-OK status nothing was enqueued and
 *    adaserve_last_error() describes the problem.
 *  - Device-only contents (parent arrays, block tables, draft tokens) are
 *    checked in the kernels: malformed trees give accept_len = -1 in
 *    adaserve_tree_accept and unspecified (but in-bounds) attention output.
 *  - The library is stateless apart from a per-device architecture check and
 *    the thread-local error string; calls on different streams may overlap.
 *  - Only gfx950 devices are supported (ADASERVE_ERR_UNSUPPORTED otherwise).
 *
 * Tree encoding (all entry points): request r owns the global node rows
 * [node_indptr[r], node_indptr[r+1]); local node 0 is the root (the last
 * committed token); parent[] holds LOCAL parent ids with parent[root] = -1 and
 * 0 <= parent[i] < i for every other node (a parent is drafted before its
 * children, Appendix B).  1 <= N_r <= 128 nodes per request.
 */
#ifndef ADASERVE_H
#define ADASERVE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes returned by every entry point. */
#define ADASERVE_OK                   0
#define ADASERVE_ERR_INVALID_ARGUMENT 1  /* bad pointer, size, layout or host-mirror value   */
#define ADASERVE_ERR_UNSUPPORTED      2  /* valid but not built: head_dim, page size, device  */
#define ADASERVE_ERR_WORKSPACE        3  /* workspace missing or smaller than required        */
#define ADASERVE_ERR_DEVICE           4  /* a HIP runtime call or kernel launch failed        */

/* Element types of the floating-point tensors. */
#define ADASERVE_F32  0
#define ADASERVE_BF16 1

/* Maximum tree nodes per request. */
#define ADASERVE_MAX_TREE_NODES 128

/*
 * Bytes of device workspace adaserve_tree_attn_verify needs for this batch
 * (split-KV partial results).  Depends only on the arguments given here, so a
 * caller can size the workspace once per batch shape.  Returns 0 when no
 * workspace is needed and SIZE_MAX when the arguments are invalid (the
 * reason is in adaserve_last_error()).
 */
size_t adaserve_tree_attn_workspace_bytes(int32_t num_requests, const int32_t *node_indptr_host,
                                          const int32_t *prefix_len_host, int32_t num_q_heads,
                                          int32_t num_kv_heads, int32_t head_dim,
                                          int32_t page_size, int32_t dtype);

/*
 * Paged tree attention (section 4.3 step 4; section 2 draft token tree).
 *
 * For node i of request r and q-head h, with kv-head g = h / (Hq / Hkv)
 * (contiguous head groups), the output is softmax-weighted attention of
 * q[i, h] over, in this order,
 *   - the request's cached prefix: positions t = 0 .. L_r - 1, held in page
 *     block_table[r * block_table_stride + t / page_size], slot t % page_size;
 *   - the tree nodes on i's root-to-node path (root .. i, i included), whose
 *     keys and values are k_tree / v_tree rows of those nodes;
 * with scores sm_scale * <q, k>.  No other tree node is visible to i.  The
 * kernel applies no positional encoding: q and k_tree arrive post-RoPE.
 *
 * Layouts (row-major, dense):
 *   q, out            [T, Hq, D]              dtype
 *   k_tree, v_tree    [T, Hkv, D]             dtype
 *   k_pages, v_pages  [num_pages, Hkv, page_size, D]   dtype
 *   block_table       [num_requests, block_table_stride] int32 physical page ids
 *   prefix_len        [num_requests] int32 (device), prefix_len_host its host copy
 *   node_indptr       [num_requests + 1] int32 (device), node_indptr_host its copy
 * Supported: dtype F32 or BF16; head_dim 64 or 128; page_size 16; any
 * Hq % Hkv == 0 with Hq / Hkv <= 16; L_r >= 0 (L_r = 0: attention over the
 * root path only); sm_scale finite, and > 0 for BF16
 * (ADASERVE_ERR_UNSUPPORTED otherwise; F32 takes any finite scale).
 * BF16 computes Q.K^T and P.V on bf16 matrix cores with
 * fp32 accumulation and rounds the output to bf16 (nearest even); when a
 * prefix is split into chunks, each chunk's own normalised output is kept in
 * bf16 and the chunks are merged with fp32 weights.  F32 computes in fp32
 * throughout.
 * F32: a key of weight 0, and every tree node off i's path, adds nothing to
 * the output of i whatever its value row holds (an Inf or NaN in one branch
 * stays in the nodes that see it).  BF16 multiplies the values of all of a
 * request's nodes by their weights, 0 for the nodes off the path, so there
 * tree and prefix values must be finite (0 * Inf is NaN).
 * Slots past L_r in the last page and pages not listed for r are never read
 * into the result (they may hold NaN).  Block-table entries outside
 * [0, num_pages) are treated as all-zero pages.  The device arrays must equal
 * their host mirrors.  workspace must hold at least
 * adaserve_tree_attn_workspace_bytes(...) bytes (256-byte aligned; contents
 * need no initialisation); calls that share a workspace must not overlap in
 * time.  When some prefix is split, a second kernel (the split-KV merge) is
 * enqueued after the attention kernel on the same stream.
 */
int32_t adaserve_tree_attn_verify(int32_t num_requests, const int32_t *node_indptr,
                                  const int32_t *node_indptr_host, const int32_t *parent,
                                  const void *q, const void *k_tree, const void *v_tree,
                                  const void *k_pages, const void *v_pages, int32_t num_pages,
                                  const int32_t *block_table, int32_t block_table_stride,
                                  const int32_t *prefix_len, const int32_t *prefix_len_host,
                                  int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                  int32_t page_size, float sm_scale, int32_t dtype, void *out,
                                  void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of the static split-KV scratch of adaserve_tree_attn_verify_noalloc. */
#define ADASERVE_TREE_ATTN_SCRATCH_BYTES (32u << 20)

/*
 * adaserve_tree_attn_verify without a workspace argument, for callers that
 * cannot allocate device memory: code under HIP graph capture, serving loops
 * that must not allocate, harnesses that forbid hipMalloc.  It calls no
 * allocator of any kind.
 *
 * Arguments, layouts, results and errors are those of
 * adaserve_tree_attn_verify; the split-KV partial results go to a static
 * array of ADASERVE_TREE_ATTN_SCRATCH_BYTES bytes that the library holds on
 * every device it runs on until the process ends.  A batch whose partials fit
 * it (adaserve_tree_attn_workspace_bytes(...) <= the limit) runs with the same
 * plan and kernels, bit-identical to adaserve_tree_attn_verify.  A batch whose
 * partials do not is split more coarsely, where a split that fits is not
 * estimated much slower (BF16 results then differ by rounding), and is otherwise rejected
 * with ADASERVE_ERR_WORKSPACE before anything is enqueued.  Every
 * call on one device shares that device's array: calls that overlap in time
 * on one device (other streams, other threads) race and give undefined
 * results; calls on one stream are ordered and safe.  The array's contents
 * need no initialisation.
 */
int32_t adaserve_tree_attn_verify_noalloc(int32_t num_requests, const int32_t *node_indptr,
                                          const int32_t *node_indptr_host, const int32_t *parent,
                                          const void *q, const void *k_tree, const void *v_tree,
                                          const void *k_pages, const void *v_pages, int32_t num_pages,
                                          const int32_t *block_table, int32_t block_table_stride,
                                          const int32_t *prefix_len, const int32_t *prefix_len_host,
                                          int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                          int32_t page_size, float sm_scale, int32_t dtype, void *out,
                                          void *stream);

/*
 * Per-node vocabulary argmax of the verification logits (section 5.1: the
 * logits of every node come back from verification and the verified tokens
 * are identified from them; greedy reading: the target's choice is its
 * highest-scoring token).
 *
 * logits: [num_rows, row_stride] of dtype, row i = logits + i * row_stride
 * elements, columns 0 .. vocab - 1 compared (the rest of a row is never read).
 * argmax_out: [num_rows] int32, the LOWEST index holding the row's maximum
 * (values compare after exact widening to fp32; +0 == -0).  NaN inputs give
 * an unspecified index in [0, vocab).  Requires vocab >= 1 when num_rows > 0,
 * row_stride >= vocab.  num_rows = 0 is a no-op.
 */
int32_t adaserve_node_argmax(const void *logits, int64_t row_stride, int32_t num_rows,
                             int32_t vocab, int32_t dtype, int32_t *argmax_out, void *stream);

/*
 * Longest-accepted-path acceptance (greedy tree verification, section 4.3
 * step 4, read with section 2's tree and Algorithm 2's count of the root as
 * one accepted token).
 *
 * Node j > 0 matches when draft_tokens[j] == target_argmax[parent(j)]; j is
 * accepted when every non-root node on its root-to-node path matches; the
 * root is always accepted and its draft token is never compared.  With d* the
 * largest depth of an accepted node (root depth 0) and i* the smallest local
 * id among accepted nodes of that depth:
 *   accept_len[r]              = d* + 1
 *   accept_nodes[r][k]         = local id of the depth-k node on the root..i*
 *                                path, k = 0..d*
 *   accept_tokens[r][k]        = draft token of accept_nodes[r][k + 1], k < d*
 *   accept_tokens[r][d*]       = target_argmax[i*]  (the target's next token)
 *   slots k > d*               = -1
 * Outputs are [num_requests, max_accept] int32 rows (row stride max_accept).
 * A request whose tree is malformed (N_r outside 1..128, indptr outside
 * [0, total_nodes], parent[root] != -1, a parent not earlier than its child)
 * or deeper than max_accept - 1 gets accept_len = -1 and -1 in every slot.
 * draft_tokens, target_argmax: [total_nodes] int32 (device).
 */
int32_t adaserve_tree_accept(int32_t num_requests, int32_t total_nodes,
                             const int32_t *node_indptr, const int32_t *parent,
                             const int32_t *draft_tokens, const int32_t *target_argmax,
                             int32_t max_accept, int32_t *accept_len, int32_t *accept_tokens,
                             int32_t *accept_nodes, void *stream);

/*
 * The whole verification pass in one call (section 4.3 step 4: every tree
 * of the batch scored in one pass, then the tokens to commit read off the
 * node logits, section 5.1): tree attention as adaserve_tree_attn_verify,
 * the per-node argmax as adaserve_node_argmax over the logits' T rows, and
 * the acceptance as adaserve_tree_accept on that argmax.  Every output is
 * bit-identical to those three calls in that order on the same stream.
 *
 * The attention arguments, workspace (size:
 * adaserve_tree_attn_workspace_bytes) and limits are those of
 * adaserve_tree_attn_verify; logits [T, logits_row_stride] have the
 * attention's dtype (columns 0 .. vocab - 1 compared); draft_tokens [T],
 * target_argmax [T], accept_len [num_requests], accept_tokens and
 * accept_nodes [num_requests, max_accept] are as in adaserve_node_argmax
 * and adaserve_tree_accept (all device memory).  Errors: the union of those
 * calls' checks, all made before anything is enqueued.
 *
 * BF16 runs in two launches: the attention workgroups followed, in the same
 * grid, by one argmax workgroup per node (they take the CUs no attention
 * work unit holds and the attention's tail, so the logits stream beside the
 * attention instead of after it); then the split-KV merge (when a prefix is
 * split) together with one acceptance wave per request.  F32 runs in two
 * launches too (its prefixes are never split: the second is the acceptance
 * alone), or three when many short logits rows run faster in a launch of
 * their own.  Calls that share a workspace must not overlap in time.
 */
int32_t adaserve_tree_verify_step(int32_t num_requests, const int32_t *node_indptr,
                                  const int32_t *node_indptr_host, const int32_t *parent,
                                  const void *q, const void *k_tree, const void *v_tree,
                                  const void *k_pages, const void *v_pages, int32_t num_pages,
                                  const int32_t *block_table, int32_t block_table_stride,
                                  const int32_t *prefix_len, const int32_t *prefix_len_host,
                                  int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                  int32_t page_size, float sm_scale, int32_t dtype,
                                  const void *logits, int64_t logits_row_stride, int32_t vocab,
                                  const int32_t *draft_tokens, int32_t max_accept, void *out,
                                  int32_t *target_argmax, int32_t *accept_len,
                                  int32_t *accept_tokens, int32_t *accept_nodes, void *workspace,
                                  size_t workspace_bytes, void *stream);

/*
 * Accepted-path KV commit: the keys and values of the accepted path enter
 * the request's paged cache, so the next iteration's prefix holds them
 * (section 5.1: once verified, a request's tokens return with it to the pool
 * of requests that the next iteration draws from; section 2: the root is the
 * last generated token, whose K/V, like every tree node's, was computed in
 * the verification pass).
 *
 * For request r with len = accept_len[r] >= 1 and L = prefix_len[r], row
 * k = 0 .. len-1 copies the tree row of local node accept_nodes[r][k]
 * (k_tree/v_tree row node_indptr[r] + node, every kv-head) to cache position
 * L + k: page block_table[r][(L + k) / page_size], slot (L + k) % page_size.
 * Rows are committed in order up to the first row that cannot be: node
 * outside [0, N_r), position past the block-table row, or a page id outside
 * [0, num_pages); nothing at or after that row is written.
 * new_prefix_len[r] = L + (rows committed).  A request with accept_len < 1
 * (e.g. -1 from adaserve_tree_accept), accept_len > max_accept or
 * accept_len > ADASERVE_MAX_TREE_NODES commits nothing and keeps L.  new_prefix_len may be the prefix_len array itself.
 * No other byte of k_pages / v_pages is written.
 *
 * Layouts as in adaserve_tree_attn_verify: k_tree, v_tree [total_nodes, Hkv,
 * D]; k_pages, v_pages [num_pages, Hkv, page_size, D]; accept_nodes
 * [num_requests, max_accept] int32 (device).  dtype F32 or BF16; head_dim * element
 * size a multiple of 16 bytes; page_size >= 1.  All arrays are device
 * memory; the copy is bit-exact.
 */
int32_t adaserve_commit_accepted_kv(int32_t num_requests, const int32_t *node_indptr,
                                    const int32_t *accept_len, const int32_t *accept_nodes,
                                    int32_t max_accept, const void *k_tree, const void *v_tree,
                                    void *k_pages, void *v_pages, int32_t num_pages,
                                    const int32_t *block_table, int32_t block_table_stride,
                                    const int32_t *prefix_len, int32_t num_kv_heads,
                                    int32_t head_dim, int32_t page_size, int32_t dtype,
                                    int32_t *new_prefix_len, void *stream);

/*
 * Draft-tree selection: the SLO-customised and throughput-optimised selection
 * phases of Algorithm 2 (section 4.3 steps 2 and 3), run on the candidate
 * token trees the speculation phase built; the result is the draft token
 * trees the verification pass scores.
 *
 * Request r owns candidates [cand_indptr[r], cand_indptr[r+1]) (root not
 * included); cand_parent holds LOCAL parents, -1 for a child of the root;
 * cand_prob is each candidate's path probability f(v).  Every well-formed
 * request starts with its root (one budget unit).  Requests are visited in
 * descending order of need (NaN: last; ties by index); each adds its best
 * remaining candidate while the float32 sum of its added path probabilities
 * (from 0, in the order added) is below need[r], its tree has fewer than
 * n_max nodes (root included) and budget remains (section 4.3 step 2; need[r]
 * is A_cap(r) minus the root's 1).  Then the best remaining candidates of
 * the whole batch are added while budget remains (step 3).  "Best" is the
 * highest path probability, ties to the smaller depth (so a parent always
 * precedes its child and every tree stays connected), then the smaller
 * request, then the smaller local index.  The budget loops run while
 * budget > 0 (the printed "B >= 0" would select one node past the budget).
 *
 * Outputs: tree_size[r] = nodes selected (root included); row r of
 * tree_parent / tree_cand ([num_requests, max_nodes] int32) lists the root
 * first (-1, -1), then the selected candidates by (depth, local index) with
 * their tree-local parent and their local candidate index; -1 past
 * tree_size.  These rows are a valid tree for adaserve_tree_attn_verify.
 * A request with more than 127 candidates, a parent that is not -1 or an
 * earlier candidate, or a path probability outside (0, 1] or above its
 * parent's (the root's is 1) takes no part: no budget, tree_size -1, rows of
 * -1.  If cand_indptr does not start at 0, decreases, or does not end at
 * num_candidates, every request gets -1.
 * Limits: num_requests <= 512, num_candidates <= 8192, max_nodes >= 128.
 * All arrays are device memory.
 */
int32_t adaserve_select_trees(int32_t num_requests, int32_t num_candidates,
                              const int32_t *cand_indptr, const int32_t *cand_parent,
                              const float *cand_prob, const float *need, int32_t budget,
                              int32_t n_max, int32_t max_nodes, int32_t *tree_size,
                              int32_t *tree_parent, int32_t *tree_cand, void *stream);

/*
 * One beam-search speculation step (section 4.3 step 1): every beam node of
 * a request expands into all vocabulary tokens, a child's path probability
 * being the beam's path probability times the draft model's softmax
 * probability of the token (section 4.2's product of draft probabilities
 * along the path), and each request keeps the beam_out children with the
 * highest path probability.  The first step has one beam per request (the
 * root, log path probability 0); later steps have beam_in = the previous
 * step's beam_out.
 *
 * Row b of request r is logits row r * beam_in + b: the draft model's logits
 * after beam node b, columns 0 .. vocab - 1 (row_stride elements apart; the
 * rest of a row is never read).  beam_logprob [num_requests * beam_in]
 * holds each beam's natural-log path probability; -inf marks an unused beam
 * slot, whose logits row is not read.  A child's score is
 *   beam_logprob[b] + x[b, t] - log(sum over t' of exp(x[b, t'])),
 * computed in fp32 (the log-sum-exp over the row accumulated in fp32).
 * Children are ranked by score (higher first), ties to the smaller beam, then
 * the smaller token (children of one beam whose fp32 scores coincide only
 * through rounding keep the order of their logits); the beam_out best
 * children with a finite score are written best first to row r of
 *   out_parent  [num_requests, beam_out] int32  beam index in [0, beam_in)
 *   out_token   [num_requests, beam_out] int32  token id in [0, vocab)
 *   out_logprob [num_requests, beam_out] fp32   the child's score
 * and slots past them hold -1, -1, -inf.  Logits are finite or -inf (a -inf
 * logit is a token of probability 0, never kept); NaN or +inf logits give
 * unspecified (in-range) outputs.
 *
 * dtype F32 or BF16 logits; logits 16-byte aligned and row_stride * element
 * size a multiple of 16 bytes; 1 <= beam_in, beam_out <= 64; vocab <= 2^20
 * (ADASERVE_ERR_UNSUPPORTED above).  workspace: at
 * least adaserve_beam_step_workspace_bytes(...) bytes of device memory,
 * 256-byte aligned, no initialisation needed; calls sharing a workspace must
 * not overlap in time.  Two kernels are enqueued on `stream` (a scan of
 * every live logits row, then a per-request merge).  num_requests = 0 is a
 * no-op.
 */
size_t adaserve_beam_step_workspace_bytes(int32_t num_requests, int32_t beam_in, int32_t vocab,
                                          int32_t beam_out, int32_t dtype);

int32_t adaserve_beam_step(int32_t num_requests, int32_t beam_in, const void *logits,
                           int64_t row_stride, int32_t vocab, int32_t dtype,
                           const float *beam_logprob, int32_t beam_out, int32_t *out_parent,
                           int32_t *out_token, float *out_logprob, void *workspace,
                           size_t workspace_bytes, void *stream);

/*
 * Tree verification for sampled decoding: multi-step speculative sampling
 * over each request's draft token tree (the tree-based verification of prior
 * work that section 4.3 step 4 delegates to; lossless -- the emitted tokens
 * follow the target distribution -- when each node's children were drawn
 * independently from the draft distribution at that node).  The greedy
 * counterpart is adaserve_tree_accept.
 *
 * Row u of target_logits / draft_logits ([total_nodes, row_stride], dtype)
 * holds the target / draft model's logits after node u's root path, already
 * divided by the sampling temperature; p_u / q_u are their softmax over
 * columns 0 .. vocab - 1.  Draft rows of leaves are not read (q at a leaf
 * enters no test and no residual).  From the
 * root, the children of the current node u are tried in index order: child
 * c with token t = draft_tokens[c] is accepted when
 *   u_accept[c] * q_u(t) < p_res(t)
 * (probability min(1, p_res(t) / q_u(t)) for u_accept uniform in [0, 1)),
 * where p_res starts as p_u at every node; a rejection replaces p_res by
 * max(0, p_res - q_u), renormalised.  The accepted child becomes the current
 * node and its token is emitted; when no child is accepted (or u is a leaf)
 * the bonus token -- the smallest v whose cumulative p_res, in token order,
 * exceeds u_bonus[u] -- is emitted and the walk ends.  A rejection that
 * leaves p_res without mass (possible only through rounding) ends the walk
 * with the bonus drawn from p_res before it.  Arithmetic is fp32.
 *
 * Outputs as adaserve_tree_accept: accept_len[r] = accepted drafts + 1,
 * accept_nodes[r] = the path from the root, accept_tokens[r] = the accepted
 * drafts' tokens then the bonus token, -1 past them; accept_len = -1 and rows
 * of -1 for a malformed tree (as adaserve_tree_accept), a draft token of a
 * non-root node outside [0, vocab), a tree deeper than max_accept - 1, or a
 * node with children whose draft row has no logit above -inf (NaN counts as
 * none: q is then no distribution).  node_indptr must
 * be increasing (requests of consecutive, disjoint node ranges): where it is
 * not, requests that share nodes may also get -1.
 * u_accept, u_bonus: [total_nodes] fp32 (device).  Logits 16-byte aligned,
 * row_stride * element size a multiple of 16 bytes.  workspace: at least
 * adaserve_tree_accept_sampled_workspace_bytes(total_nodes) bytes of device
 * memory (1 KB per node: every node's softmax statistics, in parts of 16
 * bytes, up to 64 per node), 16-byte aligned,
 * no initialisation needed; calls sharing a workspace must not overlap in
 * time.  Two kernels are enqueued on `stream`: the statistics of every node
 * (the whole chip), then the walks, one workgroup per request.
 */
size_t adaserve_tree_accept_sampled_workspace_bytes(int32_t total_nodes);

int32_t adaserve_tree_accept_sampled(int32_t num_requests, int32_t total_nodes,
                                     const int32_t *node_indptr, const int32_t *parent,
                                     const int32_t *draft_tokens, const void *target_logits,
                                     const void *draft_logits, int64_t row_stride, int32_t vocab,
                                     int32_t dtype, const float *u_accept, const float *u_bonus,
                                     int32_t max_accept, int32_t *accept_len,
                                     int32_t *accept_tokens, int32_t *accept_nodes,
                                     void *workspace, size_t workspace_bytes, void *stream);

/*
 * The serving operators below fill the paged cache that the verification pass
 * reads and serve a request where it does not speculate: its prompt, and its
 * single tokens.  Conventions, error codes and cache layouts are those above.
 * Token packing: request r owns the token rows [token_indptr[r],
 * token_indptr[r+1]), of any number, 0 among them; rows past the last request's
 * (padding of a batch) are neither read nor written.
 * Rows given with a stride span at most 2^48 elements.  A launch has fewer than
 * 2^32 threads, so num_tokens + num_requests / 4 of an append, num_requests * Hkv
 * of single tokens, the tiles of prompts (a request's rows by 16 or more, per
 * kv-head) and the row parts of sampling (4096 logits or more) stay below 2^24,
 * sampled rows below 2^22; calls beyond are refused (ADASERVE_ERR_UNSUPPORTED).
 */

/*
 * Rotary position embedding of queries and keys, and the append of keys and
 * values to the paged cache (what makes the post-RoPE q, k_tree and prefix
 * keys of the attention calls).
 *
 * Token i of request r stands at cache position place = prefix_len[r] + i and
 * is rotated by the angles p * inv_freq[j], j < rotary_dim / 2, where p is
 * positions[t] of its row t, or place where positions is NULL.  Pair j of a
 * head is columns (j, j + rotary_dim / 2), or (2j, 2j + 1) with interleaved = 1:
 *   y1 = x1 cos - x2 sin,  y2 = x1 sin + x2 cos;
 * columns from rotary_dim on are copied.  The angle is taken in fp64 (within
 * 2^-21 rad at any position for frequencies up to 1), sine, cosine and rotation
 * are fp32, rounded once to dtype.
 *
 *   q [num_tokens, Hq, D], k, v [num_tokens, Hkv, D]: heads dense, rows
 *     *_row_stride elements apart (slices of one projection's rows can be given
 *     as they are);
 *   q_out [num_tokens, Hq, D], k_out [num_tokens, Hkv, D]: dense rotated rows;
 *     q_out may be q and k_out may be k where those are dense.  q and q_out may
 *     both be NULL; k_out may be NULL when there are pages, k (and k_out) when
 *     there are none.
 *   k_pages, v_pages [num_pages, Hkv, page_size, D]: rotated keys, and values
 *     bit for bit, go to page block_table[r][place / page_size], slot
 *     place % page_size.  Both NULL: nothing is appended (nodes of draft trees:
 *     positions = prefix length + depth), and v is not read.
 *   new_prefix_len [num_requests] int32 (required with pages, NULL without):
 *     prefix_len[r] + the leading rows whose page lies in the block-table row
 *     and in [0, num_pages).  A row whose page does not is not stored; rows
 *     after it whose page does are.  prefix_len[r] < 0 stores nothing and is
 *     kept.  May be the prefix_len array itself (a second, small launch).
 *
 * Every place belongs to one token: requests that share pages must not append
 * to them in one call.  dtype F32 or BF16; head_dim * element size a multiple
 * of 16 bytes, head_dim <= 512; rotary_dim * element size a multiple of 32
 * bytes (0: plain append, inv_freq may be NULL); page_size >= 1; at most 4096
 * heads of a kind.  num_requests = 0 is a no-op.
 */
int32_t adaserve_rope_append_kv(int32_t num_requests, int32_t num_tokens, const int32_t *token_indptr,
                                const int32_t *prefix_len, const int32_t *positions, const void *q,
                                int64_t q_row_stride, const void *k, int64_t k_row_stride, const void *v,
                                int64_t v_row_stride, const float *inv_freq, int32_t rotary_dim,
                                int32_t interleaved, int32_t num_q_heads, int32_t num_kv_heads,
                                int32_t head_dim, int32_t page_size, int32_t dtype, void *q_out,
                                void *k_out, void *k_pages, void *v_pages, int32_t num_pages,
                                const int32_t *block_table, int32_t block_table_stride,
                                int32_t *new_prefix_len, void *stream);

/*
 * Causal attention of packed prompts, or of a chunk of each, over the paged
 * cache that already holds their keys and values (adaserve_rope_append_kv).
 *
 * Request r has n = token_indptr[r+1] - token_indptr[r] rows and c =
 * context_len[r] cached keys, its own rows' among them (the length after the
 * append).  Row i stands at position c - n + i and attends to positions
 * 0 .. c - n + i, with scores sm_scale * <q, k> and head groups as in
 * adaserve_tree_attn_verify.  A row whose position is negative (c < n) sees
 * nothing and its output is 0.  Layouts: q [T, Hq, D] with rows q_row_stride
 * elements apart, out [T, Hq, D] dense, T = token_indptr[num_requests];
 * k_pages, v_pages, block_table, types, head dims, page size and scales as in
 * adaserve_tree_attn_verify, and BF16 rounds as described there.  Slots past c
 * are never read into the result; a key that a row does not see adds nothing to
 * it, whatever key and value it holds.
 * Block-table entries outside [0, num_pages) are all-zero pages.
 * Scores are to be below 2^29 in magnitude, and the values that a row sees
 * finite (0 * Inf is NaN), with |value| * c below 2^118: sums over the keys are
 * taken in fp32, of weights up to 2^8.
 * token_indptr_host and context_len_host mirror the device arrays; a captured
 * call is replayed with the lengths of its capture (adaserve_decode_attn follows
 * lengths on the device).  T * Hq < 2^31.  workspace: at least adaserve_prompt_attn_workspace_bytes(...) bytes
 * (0 for most batches, and not bounded by another batch's: it depends on the
 * lengths; 256-byte aligned, no initialisation needed); calls that share one must
 * not overlap in time.
 */
size_t adaserve_prompt_attn_workspace_bytes(int32_t num_requests, const int32_t *token_indptr_host,
                                            const int32_t *context_len_host, int32_t num_q_heads,
                                            int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                                            int32_t dtype);

int32_t adaserve_prompt_attn(int32_t num_requests, const int32_t *token_indptr,
                             const int32_t *token_indptr_host, const void *q, int64_t q_row_stride,
                             const void *k_pages, const void *v_pages, int32_t num_pages,
                             const int32_t *block_table, int32_t block_table_stride,
                             const int32_t *context_len, const int32_t *context_len_host,
                             int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                             int32_t page_size, float sm_scale, int32_t dtype, void *out,
                             void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention of one new token per request over its paged cache: row r of q
 * [num_requests, Hq, D] attends to positions 0 .. context_len[r] - 1 (its own
 * key among them), as adaserve_prompt_attn with one row per request.  The
 * lengths are read on the device only, so a captured call serves a batch whose
 * lengths grow: max_context bounds them (a bound well above them costs little).
 * context_len[r] = 0 (padding of a batch) gives an output of 0; a length
 * outside [0, max_context] gives NaN.  The caches are split over their length
 * where the batch alone would not fill the device, and joined by a second
 * launch.  workspace: at least adaserve_decode_attn_workspace_bytes(...) bytes
 * (it depends on sizes, not on lengths; 256-byte aligned, no initialisation
 * needed); calls that share one must not overlap in time.  num_requests * Hq <
 * 2^31.
 */
size_t adaserve_decode_attn_workspace_bytes(int32_t num_requests, int32_t max_context,
                                            int32_t num_q_heads, int32_t num_kv_heads,
                                            int32_t head_dim, int32_t page_size, int32_t dtype);

int32_t adaserve_decode_attn(int32_t num_requests, const void *q, int64_t q_row_stride,
                             const void *k_pages, const void *v_pages, int32_t num_pages,
                             const int32_t *block_table, int32_t block_table_stride,
                             const int32_t *context_len, int32_t max_context, int32_t num_q_heads,
                             int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                             float sm_scale, int32_t dtype, void *out, void *workspace,
                             size_t workspace_bytes, void *stream);

/*
 * One token per row of logits by temperature, top-k, top-p and min-p, from a
 * given uniform number (the first token after a prompt, and every token of a
 * request that does not speculate; the greedy counterpart is
 * adaserve_node_argmax).
 *
 * logits [num_rows, row_stride] of dtype, columns 0 .. vocab - 1, of any
 * alignment to the element.  temperature, top_p, min_p, u [num_rows] fp32,
 * top_k [num_rows] int32 (device); each but u may be NULL: 1, off, off, off.
 * With z = (x - max) / temperature, a token's mass is the whole number
 * W = round(2^32 exp(z)), computed in fp64: a token below 2^-33 of the
 * likeliest has none.  Tokens are ranked by logit (higher first; +0 == -0),
 * equal ones by index.  Then, in this order:
 *   top_k = k in [1, vocab) keeps the first k (other values: all);
 *   top_p = p < 1 keeps of them those whose predecessors' mass is below
 *     p * (their whole mass) (fp64 product);
 *   min_p = m > 0 keeps of them those with W >= m * 2^32;
 * the first token is always kept (m > 1 or p <= 0 leave it alone).  The token
 * is the first, in index order, whose cumulative kept mass exceeds u * (the
 * kept mass) (fp64 product); u >= 1 takes the last that has mass, u < 0 counts
 * as 0.  temperature = 0 takes the first-ranked token.  Sums of masses are
 * exact, so results depend on no order of summation.
 * out_token [num_rows] int32; -1 for a row with a NaN or +inf logit or with no
 * logit above -inf, with a temperature that is negative, infinite or NaN, or
 * with a NaN top_p, min_p or u.  vocab <= 2^20.  workspace: at least
 * adaserve_sample_workspace_bytes(...) bytes, 256-byte aligned, no
 * initialisation needed; calls that share one must not overlap in time.
 * num_rows = 0 is a no-op.
 */
size_t adaserve_sample_workspace_bytes(int32_t num_rows, int32_t vocab, int32_t dtype);

int32_t adaserve_sample(const void *logits, int64_t row_stride, int32_t num_rows, int32_t vocab,
                        int32_t dtype, const float *temperature, const int32_t *top_k,
                        const float *top_p, const float *min_p, const float *u, int32_t *out_token,
                        void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention over a window and sinks: a row at position p sees position j <= p
 * where j > p - window (the newest `window` positions, its own among them) or
 * j < sinks (the first ones, for good).  window >= 1, sinks >= 0; a window that
 * reaches the first position gives the attention without one.  Three forms:
 *
 *   adaserve_window_prompt_attn  adaserve_prompt_attn's rows, at positions
 *     c - n + i.
 *   adaserve_window_decode_attn  adaserve_decode_attn's, at position c - 1.
 *   adaserve_window_tree_attn    adaserve_tree_attn_verify's nodes, at positions
 *     L + depth (the root's depth is 0): of the prefix and of the nodes on the
 *     root-to-node path a node sees those that its position sees.
 *
 * Everything else -- layouts, types, head groups, roundings, limits, zero pages,
 * lengths on the host and on the device, workspaces -- is as in those calls, but that
 * in trees the chunks of a split prefix keep their outputs in fp32; rows of q may lie
 * apart in the first two.  Where the window or the sinks reach every position of the
 * batch (of max_context, in the second), the call is the one without a window, bit for
 * bit, with that call's bf16 chunks.
 * Pages that hold no position seen by any row of their request add nothing, whatever
 * they hold and whatever their block-table entries say: they may have been freed
 * (adaserve_update_pages) and given to other requests.  (Keys are taken 32 positions
 * together, so such a page beside one that is seen may be loaded, where its entry
 * names one of the pool, and is then masked.)
 * A position that a row does not see adds nothing to it, whatever key and value
 * it holds; in BF16 trees that is so for prefix positions that no node of the
 * request sees and for nodes past the request's, and the values of the others must
 * be finite, as there.
 */
size_t adaserve_window_prompt_attn_workspace_bytes(int32_t num_requests, const int32_t *token_indptr_host,
                                                   const int32_t *context_len_host, int32_t num_q_heads,
                                                   int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                                                   int32_t window, int32_t sinks, int32_t dtype);

int32_t adaserve_window_prompt_attn(int32_t num_requests, const int32_t *token_indptr,
                                    const int32_t *token_indptr_host, const void *q, int64_t q_row_stride,
                                    const void *k_pages, const void *v_pages, int32_t num_pages,
                                    const int32_t *block_table, int32_t block_table_stride,
                                    const int32_t *context_len, const int32_t *context_len_host,
                                    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                    int32_t page_size, int32_t window, int32_t sinks, float sm_scale,
                                    int32_t dtype, void *out, void *workspace, size_t workspace_bytes,
                                    void *stream);

size_t adaserve_window_decode_attn_workspace_bytes(int32_t num_requests, int32_t max_context,
                                                   int32_t num_q_heads, int32_t num_kv_heads,
                                                   int32_t head_dim, int32_t page_size, int32_t window,
                                                   int32_t sinks, int32_t dtype);

int32_t adaserve_window_decode_attn(int32_t num_requests, const void *q, int64_t q_row_stride,
                                    const void *k_pages, const void *v_pages, int32_t num_pages,
                                    const int32_t *block_table, int32_t block_table_stride,
                                    const int32_t *context_len, int32_t max_context, int32_t num_q_heads,
                                    int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                                    int32_t window, int32_t sinks, float sm_scale, int32_t dtype, void *out,
                                    void *workspace, size_t workspace_bytes, void *stream);

size_t adaserve_window_tree_attn_workspace_bytes(int32_t num_requests, const int32_t *node_indptr_host,
                                                 const int32_t *prefix_len_host, int32_t num_q_heads,
                                                 int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                                                 int32_t window, int32_t sinks, int32_t dtype);

int32_t adaserve_window_tree_attn(int32_t num_requests, const int32_t *node_indptr,
                                  const int32_t *node_indptr_host, const int32_t *parent, const void *q,
                                  const void *k_tree, const void *v_tree, const void *k_pages,
                                  const void *v_pages, int32_t num_pages, const int32_t *block_table,
                                  int32_t block_table_stride, const int32_t *prefix_len,
                                  const int32_t *prefix_len_host, int32_t num_q_heads, int32_t num_kv_heads,
                                  int32_t head_dim, int32_t page_size, int32_t window, int32_t sinks,
                                  float sm_scale, int32_t dtype, void *out, void *workspace,
                                  size_t workspace_bytes, void *stream);

/*
 * The cache's pages.  page_refs [num_pages] int32 counts the block-table
 * entries, of all tables and whatever else keeps a page, that hold each page; a
 * page is free where it is <= 0.  Taken pages are the free ones with the lowest
 * numbers, so results depend on no order of execution.  A block-table entry
 * outside [0, num_pages) holds no page.  Everything is read and written on the
 * device, so that a captured call follows the tables; all arrays are int32.
 *
 * new_page_refs may be page_refs itself, and new_block_table block_table (not in
 * adaserve_fork_pages); otherwise outputs overlap neither inputs nor each other
 * and are written whole.  workspace: at least adaserve_pages_workspace_bytes(the
 * larger of a call's row counts, num_pages) bytes, 256-byte aligned, no
 * initialisation needed; calls that share one must not overlap in time, nor may
 * calls on the same page_refs.  At most 65536 rows, 2^23 pages, page_size <= 2^16.
 */
size_t adaserve_pages_workspace_bytes(int32_t num_rows, int32_t num_pages);

/*
 * One step of a batch's pages.  Row r of block_table [num_requests,
 * block_table_stride] has c = context_len[r] tokens.
 *   c < 0: the request is over; all its entries become -1.
 *   c >= 0, window > 0: entry e becomes -1 where none of its positions is a sink
 *     or seen by a token at position c or later: e * page_size >= sinks and
 *     (e + 1) * page_size <= c + 1 - window.  window = 0: no entry does.
 * A page loses one reference per entry that held it and became -1.  Then, where
 * need_len is given (NULL: pages are only freed, and capacity is NULL, too), the
 * entries e with ceil(c / page_size) <= e < ceil(need_len[r] / page_size), inside
 * the row, of requests with c >= 0 that hold no page get a free one each (those
 * just freed among them), in order of rows and entries, as long as there are any,
 * and one reference.  capacity[r]: the first position from c on and below need_len[r]
 * whose entry holds no page (or lies past the row), or need_len[r] where there is
 * none; 0 where c < 0.
 */
int32_t adaserve_update_pages(int32_t num_requests, const int32_t *context_len, const int32_t *need_len,
                              int32_t window, int32_t sinks, int32_t page_size, const int32_t *block_table,
                              int32_t block_table_stride, const int32_t *page_refs, int32_t num_pages,
                              int32_t *new_block_table, int32_t *new_page_refs, int32_t *capacity,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * Rows of a cache go over to the rows of a new batch: beams to their children
 * (source = adaserve_beam_step's parents, as rows of the batch), a prompt to its
 * samples, requests to other places.  New row r < num_requests has the cache of row
 * source[r] of the num_sources old ones (outside [0, num_sources): an empty row).
 * With c = context_len[source[r]], taken into [0, block_table_stride * page_size],
 * the c / page_size whole pages are shared.  What is behind them -- the page that
 * is filled in part, and pages taken for later tokens -- stays with the first of
 * the new rows; every other one has -1 there, but for a page of its own in the place of the
 * partly filled one, if c is not a multiple of page_size and that entry holds a page:
 * the lowest free one, in order of rows, whose content adaserve_copy_pages then
 * copies: copy_src[r] to copy_dst[r] (-1, -1 for rows that need none).  Rows for
 * which no free page is left keep the whole pages alone.
 *   new_context_len[r]: c; the whole pages' tokens where no page was left; 0 of an empty row.
 *   new_page_refs: a page's references by old rows taken off, those by new rows
 *   added; so pages of rows that nobody takes become free, and serve this call.
 * Entries behind c / page_size are taken to belong to one row each.
 */
int32_t adaserve_fork_pages(int32_t num_sources, int32_t num_requests, const int32_t *source,
                            const int32_t *context_len, int32_t page_size, const int32_t *block_table,
                            int32_t block_table_stride, const int32_t *page_refs, int32_t num_pages,
                            int32_t *new_block_table, int32_t *new_context_len, int32_t *new_page_refs,
                            int32_t *copy_src, int32_t *copy_dst, void *workspace, size_t workspace_bytes,
                            void *stream);

/*
 * The pages in use move to the front of the pool: with U of them, the i-th one
 * numbered U or higher goes to the i-th free place below U, and the pool ends at U
 * (to be handed back, or to hold other caches).
 *   new_place [num_pages]: a page's number afterwards, -1 of a free one (for page
 *   numbers kept elsewhere);
 *   new_block_table: every entry that held a page has its new number (a free
 *   one: -1), others stay; new_page_refs: the references moved, 0 from U on;
 *   counts [2]: U, and the number of moves;
 *   move_src, move_dst [num_pages]: the moves, -1 behind them.
 * The contents: adaserve_copy_pages(move_src, move_dst) with count = counts + 1.
 */
int32_t adaserve_compact_pages(int32_t num_requests, const int32_t *block_table, int32_t block_table_stride,
                               const int32_t *page_refs, int32_t num_pages, int32_t *new_block_table,
                               int32_t *new_page_refs, int32_t *new_place, int32_t *move_src,
                               int32_t *move_dst, int32_t *counts, void *workspace, size_t workspace_bytes,
                               void *stream);

/*
 * Page src[i] of k_pages and v_pages goes to page dst[i], bit for bit, i <
 * num_copies (count given: i < min(*count, num_copies), read on the device); a pair with
 * a page outside [0, num_pages), or src = dst, is left out.  No page is the dst of two
 * pairs, or the src of one and the dst of another.  num_layers pools [num_pages, Hkv,
 * page_size, D], layer_stride elements apart (any for one layer), are copied in one
 * launch.  Rows of a head are a multiple of 16 bytes; a page of one pool has at most 2^30;
 * at most 2^23 pairs, 65536 layers, 4096 kv-heads, head_dim 4096; dtype F32 or BF16.
 */
int32_t adaserve_copy_pages(int32_t num_copies, const int32_t *src, const int32_t *dst, const int32_t *count,
                            void *k_pages, void *v_pages, int32_t num_layers, int64_t layer_stride,
                            int32_t num_pages, int32_t num_kv_heads, int32_t page_size, int32_t head_dim,
                            int32_t dtype, void *stream);

/* Message describing the last non-OK status returned on this thread. */
const char *adaserve_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* ADASERVE_H */
