/*
 * ssa_sparse.h - attention over the blocks of the paged KV cache that each query
 * selects by a cheap score.
 *
 * A request's cached keys cost every later iteration (SlidingServe, Tab. 1, x5); a
 * row of a long context gives nearly all of its attention weight to few of them.
 * Cache positions are taken in blocks of B = 16, 32, 64 or 128 (block b holds
 * positions b B .. b B + B - 1 of its request), and a row looks at some blocks only:
 *   1. ssa_block_summary keeps, per block, kv head and dim, the highest and the
 *      lowest value of the block's keys (after any append);
 *   2. ssa_block_scores bounds every row's logits in a block by them;
 *   3. ssa_block_select lists, per row and kv head, the first blocks, the last ones
 *      and those of the highest bounds;
 *   4. ssa_sparse_attention is softmax attention over the keys of the listed blocks.
 * A row at position p = u_i + j (ssa.h) sees blocks 0 .. p / B, and of the last one
 * the keys up to p.
 *
 * Conventions, layouts and error codes as in ssa.h; in addition
 *   summary  bf16 [num_pages, Hkv, 2, D]: the highest, then the lowest values of the
 *            block that begins in this page (the B / P - 1 pages between hold nothing)
 *   scores   fp32 [T, Hkv, max_blocks], max_blocks from the plan
 *   blocks   int32 [T, Hkv, top_blocks]: block indexes, -1 for none
 * Plans are blobs as in ssa.h: filled on the host, read by the kernels through
 * plan_dev (a device copy, or the pinned host buffer itself).  A kernel that finds
 * another plan at plan_dev than the host checked reads its header alone and writes
 * nothing.
 * Pointers to queries, pools, summaries, scores, outputs and workspaces are 16-byte
 * aligned, plan_dev is 8-byte aligned.
 * Results do not depend on the order in which workgroups run.  All calls can be
 * captured into a HIP graph; the plan at plan_dev must then stay as it is for the
 * replays.
 */
#ifndef SSA_SPARSE_H
#define SSA_SPARSE_H

#include <stddef.h>
#include <stdint.h>

#include "ssa.h"
#include "ssa_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Summaries of the blocks that hold new tokens of the batch (positions u_i .. u_i +
 * c_i - 1), each over all its keys up to u_i + c_i - 1.  The keys must be in the cache
 * (ssa_kv_append, ssa_append_attention or a RoPE + append ran before on the stream).
 * Blocks before u_i / B are left as they are, as is what lies behind the last one.
 * Requests that share pages of the cache share whole blocks of them: a block has one
 * summary, with its first page.
 * After a call that moved or dropped keys (ssa_evict_compact, rejected tokens), a plan
 * of the changed positions makes the summaries anew; a plan of c_i = all, u_i = 0 makes
 * all of them.
 *   plan_host, plan_dev   ssa_plan's, as ssa_kv_append
 *   block_keys            B
 *   summary               values compare as bf16 numbers, -0 below +0; a NaN among the
 *                         keys is the highest or, with its sign set, the lowest value
 * Errors: NULL, the shape errors, PLAN_MISMATCH, ARG (block_keys; a misaligned
 * pointer), HIP.
 */
int ssa_block_summary(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                      int32_t block_keys, const uint16_t* k_cache, const int32_t* block_table,
                      uint16_t* summary, void* stream);

/*
 * What a batch's rows look at.
 *   block_keys     B: 16, 32, 64 or 128
 *   top_blocks     blocks a row and kv head looks at, at most
 *   sink_blocks    of those the first ones of the request that are always among them, >= 0
 *   recent_blocks  and the last ones, the row's own block among them, >= 1;
 *                  sink_blocks + recent_blocks <= top_blocks <= 32768
 */
typedef struct ssa_sparse_config {
  int32_t block_keys;
  int32_t top_blocks;
  int32_t sink_blocks;
  int32_t recent_blocks;
} ssa_sparse_config;

/*
 * Plan of the three calls below for the batch (q_len, ctx_len), host only.
 *   ws_bytes    the workspace of ssa_sparse_attention
 *   max_blocks  blocks of a row of scores: those of the longest request with a new
 *               token, rounded up to a multiple of four (at least four)
 * Errors: those of ssa_plan_size (without TUNING); SHAPE also for Hq D > 2^24; LENGTH
 * also for a request of more than 32768 blocks, for Hkv max_blocks > 2^24, and where the
 * plan would pass 2 GiB or a launch 2^31 workgroups; ARG (config); PLAN_SIZE (plan_bytes too
 * small).
 */
int ssa_sparse_plan_size(const ssa_shape* shape, const ssa_sparse_config* config,
                         const int32_t* q_len_host, const int32_t* ctx_len_host, int32_t num_reqs,
                         size_t* plan_bytes, size_t* ws_bytes, int32_t* max_blocks);
int ssa_sparse_plan(const ssa_shape* shape, const ssa_sparse_config* config,
                    const int32_t* q_len_host, const int32_t* ctx_len_host, int32_t num_reqs,
                    void* plan_host, size_t plan_bytes);

/*
 * For every new row at position p, kv head and block b <= p / B: the highest over the
 * kv head's query heads of
 *   sum over dims d of max(q_d, 0) high_d + min(q_d, 0) low_d
 * with the block's summary, in fp32 from the bf16 products: no key of the block has a
 * larger <q, k>.  Other scores are left as they are.  A NaN (0 times an infinite high or
 * low value is one) counts only where all heads have one.
 *   q            as ssa_mixed_attention
 *   block_table  entries b B / P of a request's row, b <= (u_i + c_i - 1) / B, are read
 * Errors: NULL, the shape errors, PLAN_MISMATCH, ARG (a misaligned pointer or plan), HIP.
 */
int ssa_block_scores(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const uint16_t* q, const uint16_t* summary, const int32_t* block_table,
                     float* scores, void* stream);

/*
 * The blocks that every row and kv head looks at: of its n = p / B + 1 blocks the first
 * sink_blocks, the last recent_blocks and of the others those of the highest scores,
 * min(n, top_blocks) in all, ascending, and -1 behind them.  Of equal scores the lowest
 * index stays first; a NaN counts as +infinity (what is not a number in a block's keys
 * shows in the output, as it would without a selection); -0 equals +0.
 * Errors: NULL, the shape errors, PLAN_MISMATCH, ARG (a misaligned pointer or plan), HIP.
 */
int ssa_block_select(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const float* scores, int32_t* blocks, void* stream);

/*
 * Attention of every new row over the blocks that its list names for each kv head:
 * out as ssa_mixed_attention, over the keys t <= p of those blocks alone.
 *   blocks     [T, Hkv, top_blocks] of ssa_block_select, or any lists: in any order, an
 *              entry outside 0 .. p / B names no block, a block named twice counts
 *              twice.  A row and kv head without any key gives zeros.
 *   block_table  as ssa_mixed_attention; only entries of named blocks are read
 *   out        another buffer than q
 *   workspace  ws_bytes of the plan.  Its first 4096 bytes hold tickets: zero before the
 *              first call (a zeroed allocation) and zero again after every call, whatever
 *              the plan.  Calls that share a workspace must be ordered on one stream.
 * Errors: NULL, the shape errors, PLAN_MISMATCH, WORKSPACE, ARG (a misaligned pointer or
 * plan), HIP.
 */
int ssa_sparse_attention(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                         const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                         const int32_t* block_table, const int32_t* blocks, uint16_t* out,
                         void* workspace, size_t ws_bytes, void* stream);

/*
 * What a decoder layer does for long contexts.  Each part may be left out (NULL).
 *   rope      as ssa_rope_append_as: the layer's cos_sin has rows of rope->rotary_dim then
 *   shift_host, shift_dev   as ssa_rope_append_shifted (ssa_evict.h)
 *   summary, block_keys     after RoPE and append, ssa_block_summary of the new keys
 *   plan_host, plan_dev     ssa_sparse_plan of the same batch as the layer's plan: its rows
 *            attend over the blocks that they select (ssa_block_scores, ssa_block_select,
 *            ssa_sparse_attention), not over all keys.  Then summary (of the plan's
 *            block_keys), scores, blocks and the workspace have to be there; scores and blocks
 *            hold what the two calls gave.  Without, attention is ssa_mixed_attention: a
 *            prompt may run so, with its summaries kept for the rows that follow.
 *   workspace ssa_sparse_attention's, not the layer's
 */
typedef struct ssa_layer_sparse {
  const ssa_rope_form* rope;
  const int32_t* shift_host;
  const int32_t* shift_dev;
  uint16_t* summary;
  const void* plan_host;
  const void* plan_dev;
  float* scores;
  int32_t* blocks;
  void* workspace;
  size_t ws_bytes;
  int32_t block_keys;
} ssa_layer_sparse;

/*
 * ssa_layer_forward with `sparse`'s parts, in the same launches but for RoPE and attention.
 * Without any of them, out and the caches are bit for bit those of ssa_layer_forward.
 * Everything is validated before the first launch.
 * Errors: those of ssa_layer_forward and of the calls that stand for the parts; NULL
 * (sparse); ARG also where block_keys is not the plan's; PLAN_MISMATCH also where the two
 * plans are not of the same batch (q_len and ctx_len of every request).
 */
int ssa_layer_forward_sparse(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                             const ssa_layer_weights* w, const ssa_layer_sparse* sparse,
                             const uint16_t* x, uint16_t* out, uint16_t* k_cache, uint16_t* v_cache,
                             const int32_t* block_table, void* workspace, size_t ws_bytes,
                             void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SSA_SPARSE_H */
