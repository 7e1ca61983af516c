/*
 * ssa_evict.h - eviction from the paged KV cache by accumulated attention
 * weight: how much every cached key was attended to, which keys of a request
 * stay, and the move of those to fewer pages.
 *
 * A request's cache grows by c_i keys an iteration (SlidingServe, Sec. 3.2),
 * and with it the cost of every later one (Tab. 1, x5).  A program that bounds
 * the cache of long requests
 *   1. keeps a score per cached key and kv head: the attention weights that the
 *      key got, summed over rows and the kv head's query heads
 *      (ssa_key_scores beside any attention call, or ssa_decode_scored, which
 *      is the attention of a pure-decode batch and gives the scores as well);
 *   2. when a request is over its budget, lists the keys that stay, per kv head
 *      (ssa_evict_select);
 *   3. moves them to new pages (ssa_evict_compact) and frees the old ones; from
 *      then on the request's u_i is the number of kept keys;
 *   4. rotates later tokens at their true positions, which are no longer their
 *      cache indexes (ssa_rope_append_shifted).
 *
 * Conventions, layouts and error codes as in ssa.h; in addition
 *   scores   fp32 [num_pages, Hkv, P]: the score of the key in the same page,
 *            kv head and slot of k_cache.
 * Plans are blobs as in ssa.h: filled on the host, read by the kernels through
 * plan_dev (a device copy, or the pinned host buffer itself).  A kernel that
 * finds another plan at plan_dev than the host checked writes nothing.  These
 * plans are position-independent but not interchangeable with ssa_plan's.
 * Workspaces need no clearing: a call reads nothing of them that it has not
 * written itself.  Calls that share a workspace must be ordered on one stream.
 * Pointers to queries, pools, scores, outputs and workspaces are 16-byte aligned,
 * plan_dev is 8-byte aligned.
 * Results do not depend on the order in which workgroups run (no atomics on
 * outputs).  All calls can be captured into a HIP graph; the plan at plan_dev
 * must then stay as it is for the replays.
 */
#ifndef SSA_EVICT_H
#define SSA_EVICT_H

#include <stddef.h>
#include <stdint.h>

#include "ssa.h"
#include "ssa_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Plan of ssa_key_scores and ssa_decode_scored for the batch (q_len, ctx_len),
 * host only.
 *   last_rows  of a request's c_i new rows only the last min(c_i, last_rows) add
 *              their weights (the end of a prompt as the window that votes);
 *              0: all of them
 *   ws_bytes   the workspace of the calls with this plan.  The attention logits
 *              of requests with one counted row take 4 Hq bytes per key of it.
 * Errors: those of ssa_plan_size (without TUNING); SHAPE also for Hq D > 2^24;
 * LENGTH also for more than 2^28 counted rows times heads of a group, and where the
 * plan would pass 2 GiB; ARG (last_rows < 0); PLAN_SIZE (plan_bytes too small).
 */
int ssa_score_plan_size(const ssa_shape* shape, const int32_t* q_len_host,
                        const int32_t* ctx_len_host, int32_t num_reqs, int32_t last_rows,
                        size_t* plan_bytes, size_t* ws_bytes);
int ssa_score_plan(const ssa_shape* shape, const int32_t* q_len_host, const int32_t* ctx_len_host,
                   int32_t num_reqs, int32_t last_rows, void* plan_host, size_t plan_bytes);

/*
 * Attention weights of a hybrid batch, summed per key and kv head.  For every
 * request with c_i > 0, key t < u_i + c_i and kv head h:
 *   scores_out = decay * scores_in [t < u_i only] +
 *                sum over counted rows j >= t - u_i and query heads of h of
 *                softmax_t(scale * <q_j, k_t>)
 * in fp32 (logits accumulated in fp32 from the bf16 products, softmax over the
 * keys 0 .. u_i + j that row j sees).  A key of this iteration (t >= u_i) has no
 * earlier score: what scores_in holds there is not read.
 *   q, k_cache, block_table: as ssa_mixed_attention; the batch's own keys must
 *   be in the cache (ssa_kv_append, ssa_append_attention or ssa_rope_append ran
 *   before on the stream), and the table's entries as ssa_check_block_table of
 *   the batch's ssa_plan checks them.
 *   scores_in   may be NULL (all zero; decay is then unused) or scores_out
 *   decay       finite, >= 0
 *   Requests with c_i = 0, slots past a request's last key and other pages are
 *   left as they are.  Pages must not be shared between requests with c_i > 0.
 * Errors: NULL, the shape errors, PLAN_MISMATCH, WORKSPACE, ARG (decay; a
 * misaligned pointer or plan), HIP.
 */
int ssa_key_scores(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                   const uint16_t* q, const uint16_t* k_cache, const int32_t* block_table,
                   const float* scores_in, float decay, float* scores_out, void* workspace,
                   size_t ws_bytes, void* stream);

/*
 * Attention of a pure-decode batch (every c_i <= 1) that also gives its weights:
 * out as ssa_mixed_attention, scores_out as ssa_key_scores, with keys and values
 * read once.  The new tokens' keys and values must be in the cache.
 * Errors: those of ssa_key_scores; ARG also where the plan has a c_i > 1.
 */
int ssa_decode_scored(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                      const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                      const int32_t* block_table, const float* scores_in, float decay,
                      float* scores_out, uint16_t* out, void* workspace, size_t ws_bytes,
                      void* stream);

/*
 * Plan of an eviction, host only.  Request i has kv_len[i] keys in the cache and
 * keeps n_i = min(kv_len[i], budget[i]) of them per kv head: the first `sink`, the
 * last `recent`, and of the others those with the highest scores.
 * Errors: NULL, the shape errors; LENGTH (a negative length or budget, or a sum
 * of lengths beyond 2^30); PAGES (a request longer than its block-table row);
 * ARG (sink or recent negative, or sink + recent > n_i for a request that loses
 * keys); PLAN_SIZE.
 */
int ssa_evict_plan_size(const ssa_shape* shape, const int32_t* kv_len_host,
                        const int32_t* budget_host, int32_t num_reqs, int32_t sink,
                        int32_t recent, size_t* plan_bytes, size_t* ws_bytes);
int ssa_evict_plan(const ssa_shape* shape, const int32_t* kv_len_host, const int32_t* budget_host,
                   int32_t num_reqs, int32_t sink, int32_t recent, void* plan_host,
                   size_t plan_bytes);

/*
 * The kept keys of every request and kv head: keep, int32, holds per request
 * Hkv lists of n_i cache indexes, ascending, one after another (request i's
 * lists start at Hkv * (n_0 + ... + n_{i-1})).  Of equal scores the lowest index
 * stays first; a NaN counts as -infinity; -0 equals +0.  A request that keeps all
 * its keys lists 0 .. n_i - 1.  Requests of more than 8192 keys most of whose scores
 * are equal, or nearly, take time with the square of their length (131072 equal
 * scores: 0.6 ms; spread ones: 0.03 ms).
 * Errors: NULL, the shape errors, PLAN_MISMATCH, WORKSPACE, ARG (a misaligned
 * pointer or plan), HIP.
 */
int ssa_evict_select(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const float* scores, const int32_t* block_table, int32_t* keep,
                     void* workspace, size_t ws_bytes, void* stream);

/*
 * Moves the kept keys, values and scores of every request that loses keys to its
 * new pages: kept key r of kv head h goes to page new_table[i][r / P], slot r % P
 * (new_table: int32 [num_reqs, max_pages_per_req], of which the first
 * ceil(n_i / P) entries of such a request are read).  Bits are moved unchanged;
 * the old pages, the slots behind the last kept key and the requests that keep
 * everything (n_i = kv_len[i], their rows of new_table unread) are left as they
 * are.  The new pages must be pages that no table names otherwise, each once
 * (ssa_check_evict_tables).  An index of keep outside [0, kv_len[i]) is not
 * followed: its slot is left as it is.
 *   scores may be NULL (none are kept).
 * Errors: NULL, the shape errors, PLAN_MISMATCH, ARG (a misaligned pool or plan), HIP.
 */
int ssa_evict_compact(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                      const int32_t* keep, const int32_t* block_table, const int32_t* new_table,
                      uint16_t* k_cache, uint16_t* v_cache, float* scores, void* stream);

/*
 * Optional host-side check of the tables before ssa_evict_select (new_table_host
 * may then be NULL) and ssa_evict_compact, on host copies: every entry that the
 * kernels read is a page of the pool, and no new page is named twice or is an
 * old page of any request of the plan.
 * Errors: NULL, the shape errors, PLAN_MISMATCH, PAGES.
 */
int ssa_check_evict_tables(const ssa_shape* shape, const void* plan_host,
                           const int32_t* block_table_host, const int32_t* new_table_host);

/*
 * ssa_rope_append (ssa_layer.h) for requests that have lost keys: the new token
 * in cache index u_i + j is rotated at position u_i + j + shift[i], shift[i] being
 * the keys that request i has lost so far.  Everything else, the slot included,
 * is as ssa_rope_append.  plan_host, plan_dev: ssa_plan's.
 *   shift_host  int32 [num_reqs], >= 0, checked here
 *   shift_dev   the same values where the device can read them
 * Errors: those of ssa_rope_append; ARG also for a negative shift or a position
 * u_i + j + shift[i] >= max_position.
 */
int ssa_rope_append_shifted(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                            const uint16_t* qkv, const float* cos_sin, int32_t max_position,
                            const int32_t* shift_host, const int32_t* shift_dev, uint16_t* q_out,
                            uint16_t* k_cache, uint16_t* v_cache, const int32_t* block_table,
                            void* stream);

/*
 * What a decoder layer does beside ssa_layer_forward for requests that are evicted
 * from.  Either part may be left out (NULL).
 *   score_plan_host, score_plan_dev   ssa_score_plan of the same batch as the layer's
 *            plan; after RoPE and append, the layer's rows add their weights as
 *            ssa_key_scores (scores_in, decay, scores_out: as there)
 *   score_workspace   of the score plan; not the layer's
 *   shift_host, shift_dev   as ssa_rope_append_shifted
 */
typedef struct ssa_layer_eviction {
  const void* score_plan_host;
  const void* score_plan_dev;
  const float* scores_in;
  float* scores_out;
  void* score_workspace;
  size_t score_ws_bytes;
  const int32_t* shift_host;
  const int32_t* shift_dev;
  float decay;
} ssa_layer_eviction;

/*
 * ssa_layer_forward with `eviction`'s parts: the same launches with the shifted
 * positions, and ssa_key_scores of the rotated queries before attention.  Without
 * shifts, out and the caches are bit for bit those of ssa_layer_forward.
 * Everything is validated before the first launch.
 * Errors: those of ssa_layer_forward, ssa_key_scores and ssa_rope_append_shifted;
 * NULL (eviction); PLAN_MISMATCH also where the two plans are not of the same batch
 * (q_len and ctx_len of every request).
 */
int ssa_layer_forward_evicting(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                               const ssa_layer_weights* w, const ssa_layer_eviction* eviction,
                               const uint16_t* x, uint16_t* out, uint16_t* k_cache,
                               uint16_t* v_cache, const int32_t* block_table, void* workspace,
                               size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SSA_EVICT_H */
