/*
 * paged_attn_tokens.h -- operators that choose tokens of a paged context, in
 * the C ABI of paged_attn.h (same library, same conventions for errors,
 * ownership, streams and device data):
 *
 *   - attention of a tree of drafted tokens over a context and their ancestors,
 *   - bounds of each block's keys, the choice of the blocks whose keys can score
 *     highest for a query, and decode attention over chosen blocks,
 *   - decode attention that adds its weights to running totals per token, and
 *     the choice of the tokens with the largest totals,
 *   - the move of chosen tokens to the front of their sequences, which takes
 *     rejected drafts and evicted tokens out of the cache.
 *
 * They are for serving: none has a backward pass, as the library has none.  Calls that may
 * run at the same time, replays of captured graphs among them, need a workspace each.
 * Device data is clamped as everywhere: lengths into [0, max_context_len], ids
 * into the pool, rows into total_q.
 */
#ifndef PAGED_ATTN_TOKENS_H
#define PAGED_ATTN_TOKENS_H

#include "paged_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------
 * A tree of drafted tokens.
 *
 * The last L_b tokens of sequence b (their K and V in the cache, n_b =
 * context_lens[b] with them) are nodes of a tree whose root is the context
 * before them: node i stands in slot n_b - L_b + i, and parents[q_start[b] + i]
 * is the node that it continues, or -1 for the context.  A node's query row sees
 * the n_b - L_b resident tokens, its ancestors and itself:
 *     s = scale * <q, K_g[t]>,  s = softcap * tanh(s / softcap) where softcap > 0,
 * softmax over those.  (Siblings have the same position: rows are rotated before,
 * see the positions of paged_attn_rope_append.)  What a row does not see changes
 * no bit of it; infinities and NaN that it sees act as in paged_attn_extend_biased.
 * ------------------------------------------------------------------------- */

/* Most nodes of one sequence. */
enum { PA_TREE_MAX_NODES = 256 };

/* Bytes of the workspace of a tree's attention; it depends on these arguments alone. */
int paged_attn_tree_workspace_size(const pa_kv_pool *pool, int32_t batch, int32_t num_q_heads,
                                   int32_t max_context_len, int32_t max_nodes, size_t *bytes_out);

/* Attention of the nodes of a batch's trees.
 *   pool             head_dim 64 or 128
 *   q                device bf16 [total_q][num_q_heads][head_dim], 16-byte aligned
 *   q_start          device int32 [batch + 1], nondecreasing from 0: sequence b's
 *                    nodes are rows q_start[b] .. q_start[b+1] - 1
 *   total_q          rows of q, parents and out; rows behind the last sequence are
 *                    left as they are
 *   parents          device int32 [total_q], each below its own node; one that is
 *                    not, or is negative, stands for the context
 *   block_tables, bt_stride, context_lens, batch, scale
 *                    as in paged_attn_decode
 *   num_q_heads      any multiple of the pool's num_kv_heads
 *   softcap          0 (none) or positive, as in paged_attn_decode_biased
 *   max_context_len  below 2^30
 *   max_nodes        bound of L_b, 0 .. PA_TREE_MAX_NODES (more: PA_EUNSUPPORTED), at
 *                    most max_context_len (or 1)
 *   workspace        device, 16-byte aligned, of workspace_bytes, at least
 *                    paged_attn_tree_workspace_size; its content is not kept.
 *                    Calls that may run at the same time need one each
 *   out              device bf16 [total_q][num_q_heads][head_dim], 16-byte aligned */
int paged_attn_extend_tree(const pa_kv_pool *pool, const void *q, const int32_t *q_start,
                           int32_t total_q, const int32_t *parents, const int32_t *block_tables,
                           int32_t bt_stride, const int32_t *context_lens, int32_t batch,
                           int32_t num_q_heads, float scale, float softcap,
                           int32_t max_context_len, int32_t max_nodes, void *workspace,
                           size_t workspace_bytes, void *out, void *stream);

/* ---------------------------------------------------------------------------
 * Attention over chosen blocks.
 *
 * The bounds of a block are the least and the greatest value of each dimension
 * over the keys of its tokens, per KV head:
 *     bounds[block][g][0][d] = min K,   bounds[block][g][1][d] = max K,
 * bf16 [num_blocks][num_kv_heads][2][head_dim], beside the pools (so shared
 * blocks share them).  No key of block j can score higher for query head h than
 * sum_d max(q_hd lo_d, q_hd hi_d), that is q_hd hi_d where q_hd > 0, q_hd lo_d where
 * q_hd < 0 and 0 where q_hd = 0; the sum of that over the heads of a KV head is the block's score, and
 * each (sequence, KV head) attends to
 *     its first_blocks first and last_blocks last blocks, and the blocks of the
 *     highest scores among the others, max_blocks in all
 * or to all where it has no more.  Scores are sums in 64 bits, off by parts of 2^-53 of
 * their largest terms where bf16 values lie too far apart for an exact sum, and equal
 * ones go to the lower block: the choice is exact for the scores so computed, which do
 * not depend on a block's place.  A score of NaN counts as the highest.  A dimension that
 * holds NaN in every token of a block bounds nothing: lo is +infinity and hi -infinity
 * there, and the block's score -infinity (or NaN).  (With a negative scale the bound would
 * be the other end's.)
 * ------------------------------------------------------------------------- */

/* Bounds of the blocks that hold the tokens first_tokens[b] .. n_b - 1, of the
 * tokens that a block has (NaN among them left out).
 *   bounds           device bf16 as above, 16-byte aligned, written
 *   block_tables, bt_stride, context_lens, batch, max_context_len
 *                    as in paged_attn_decode
 *   first_tokens     device int32 [batch], or NULL: n_b - max_new
 *   max_new          bound of n_b - first_tokens[b], >= 0; of more, the last
 *                    max_new tokens' blocks are done
 * A block that several sequences of the batch share must be full in each that
 * has it done. */
int paged_attn_block_bounds(const pa_kv_pool *pool, void *bounds, const int32_t *block_tables,
                            int32_t bt_stride, const int32_t *first_tokens,
                            const int32_t *context_lens, int32_t batch, int32_t max_context_len,
                            int32_t max_new, void *stream);

/* Bytes of the workspace of a choice of blocks. */
int paged_attn_select_workspace_size(const pa_kv_pool *pool, int32_t batch,
                                     int32_t max_context_len, int32_t max_blocks,
                                     size_t *bytes_out);

/* The blocks that each sequence's new token attends to, per KV head.
 *   q                device bf16 [batch][num_q_heads][head_dim], 16-byte aligned
 *   bounds           as above: those of the blocks between the first and the last
 *                    ones are read
 *   num_q_heads      any multiple of the pool's num_kv_heads
 *   first_blocks     >= 0
 *   last_blocks      >= 1 (the block of the token itself)
 *   max_blocks       at least first_blocks + last_blocks
 *   workspace        device, 16-byte aligned, at least
 *                    paged_attn_select_workspace_size; its content is not kept
 *   selected         device int32 [batch][num_kv_heads][max_blocks]: the blocks'
 *                    places in the table's row, ascending, then -1
 * Others as in paged_attn_decode; max_context_len below 2^30. */
int paged_attn_select_blocks(const pa_kv_pool *pool, const void *q, const void *bounds,
                             const int32_t *block_tables, int32_t bt_stride,
                             const int32_t *context_lens, int32_t batch, int32_t num_q_heads,
                             int32_t max_context_len, int32_t first_blocks, int32_t last_blocks,
                             int32_t max_blocks, void *workspace, size_t workspace_bytes,
                             int32_t *selected, void *stream);

/* Bytes of the workspace of attention over chosen blocks. */
int paged_attn_selected_workspace_size(const pa_kv_pool *pool, int32_t batch, int32_t num_q_heads,
                                       int32_t max_blocks, size_t *bytes_out);

/* One decode step over chosen blocks: softmax over the tokens t < n_b of the
 * blocks that selected lists for the (sequence, KV head).
 *   selected         device int32 [batch][num_kv_heads][max_blocks], of
 *                    paged_attn_select_blocks or the caller's own: places in the
 *                    table's row in any order.  One outside [0, ceil(n_b / 16))
 *                    is passed over; a block listed twice counts twice
 *   max_blocks       >= 0; 0 gives zeros
 *   workspace        device, 16-byte aligned, at least
 *                    paged_attn_selected_workspace_size; its content is not kept
 *   out              device bf16 [batch][num_q_heads][head_dim], 16-byte aligned;
 *                    a row without tokens is zeros
 * Others as in paged_attn_select_blocks and paged_attn_decode. */
int paged_attn_decode_selected(const pa_kv_pool *pool, const void *q, const int32_t *block_tables,
                               int32_t bt_stride, const int32_t *context_lens, int32_t batch,
                               int32_t num_q_heads, float scale, int32_t max_context_len,
                               const int32_t *selected, int32_t max_blocks, void *workspace,
                               size_t workspace_bytes, void *out, void *stream);

/* ---------------------------------------------------------------------------
 * Attention weights per token, and eviction by them.
 * ------------------------------------------------------------------------- */

/* Bytes of the workspace of a decode that keeps weights: the scores of a step, fp32 per
 * token and row of a tile of 4 (at most four query heads per KV head) or 8 rows, and
 * partial results.  With G query heads per KV head the scores take, of the K and V
 * that they are of, 4 / head_dim (G <= 4) or 8 ceil(G / 8) / head_dim: 3.1 or 6.3 % at
 * head_dim 128 and 6.3 or 12.5 % at 64 up to G = 8, twice 8's share up to 16, and so on;
 * in all they are of max_context_len tokens of every sequence. */
int paged_attn_weights_workspace_size(const pa_kv_pool *pool, int32_t batch, int32_t num_q_heads,
                                      int32_t max_context_len, size_t *bytes_out);

/* One decode step as paged_attn_decode's, whose softmax weights, summed over all
 * query heads, are added to a total per token:
 *     totals_out[b][t] = decay * totals[b][t] + sum_h softmax_t(scale <q_h, K_g[t]>)
 * for t < n_b; what lies behind is left as it is.
 *   num_q_heads      any multiple of the pool's num_kv_heads
 *   decay            finite
 *   totals           device fp32 [batch][totals_stride], or NULL: zeros (a decay of
 *                    0 still multiplies what is there)
 *   totals_out       the same layout; totals itself (in place), or overlapping no input
 *   totals_stride    at least max_context_len
 *   workspace        device, 16-byte aligned, at least
 *                    paged_attn_weights_workspace_size; its content is not kept
 *   out              device bf16 [batch][num_q_heads][head_dim], 16-byte aligned
 * Others as in paged_attn_decode; max_context_len below 2^30. */
int paged_attn_decode_weights(const pa_kv_pool *pool, const void *q, const int32_t *block_tables,
                              int32_t bt_stride, const int32_t *context_lens, int32_t batch,
                              int32_t num_q_heads, float scale, int32_t max_context_len,
                              float decay, const float *totals, float *totals_out,
                              int64_t totals_stride, void *workspace, size_t workspace_bytes,
                              void *out, void *stream);

/* The tokens of each sequence that stay when it is cut to `keep` tokens: its
 * first_tokens[b] first and its `recent` last ones, and those of the largest
 * totals among the others, `keep` in all (more only where the first and the last
 * ones are more), or all where it has no more.  Equal totals go to the lower
 * token; NaN counts as the largest.
 *   totals           device fp32 [batch][totals_stride], totals_stride >= max_context_len
 *   first_tokens     device int32 [batch], or NULL: 0
 *   context_lens     device int32 [batch]
 *   recent, keep     >= 0
 *   kept             device int32 [batch][kept_stride]: the tokens that stay behind
 *                    the first ones, as token - first_tokens[b], ascending, then -1
 *   kept_stride      at least min(max(keep, recent), max_context_len)
 *   kept_lens        device int32 [batch]: how many */
int paged_attn_keep_heaviest(const float *totals, int64_t totals_stride,
                             const int32_t *first_tokens, const int32_t *context_lens,
                             int32_t batch, int32_t max_context_len, int32_t recent, int32_t keep,
                             int32_t *kept, int32_t kept_stride, int32_t *kept_lens, void *stream);

/* Moves chosen tokens of each sequence together: for j < kept_lens[b], the K and
 * V rows (and the total) of token first_tokens[b] + kept[b][j] become those of
 * token first_tokens[b] + j, all as if read before any is written.  What stood
 * behind the moved ones is no longer the sequence's.
 *
 * After a tree's attention first_tokens is n_b - L_b and kept the nodes of the
 * accepted path; for an eviction both are those of paged_attn_keep_heaviest.
 * In place a sequence's rows move one round after the other, by one workgroup per KV
 * head and pool: right for an accepted path, slow for the eviction of few long
 * sequences (16384 of 30000 tokens of one, 8 KV heads of 128: 837 us, to other blocks 41).
 *   block_tables     device int32 [batch][bt_stride], of the tokens as they are
 *   dst_tables       device int32 [batch][dst_stride], of the tokens as they will
 *                    be: blocks that hold no token which this call reads, but for
 *                    the one in which first_tokens[b] lies, which may be the same;
 *                    or NULL (dst_stride 0), or block_tables itself with its
 *                    bt_stride: in place
 *   first_tokens     device int32 [batch], or NULL: 0.  Tokens before it stay.  A
 *                    sequence of fewer tokens (a padded slot of none) keeps what it
 *                    has and nothing of it moves
 *   context_lens     device int32 [batch], before the move
 *   kept             device int32 [batch][kept_stride], each row ascending without
 *                    equal ones (else what the moved tokens hold is unspecified)
 *   kept_lens        device int32 [batch]
 *   totals, totals_out  device fp32 [batch][totals_stride] (>= max_context_len), or
 *                    both NULL: moved with the tokens; the first ones' are copied and
 *                    those of the tokens behind the moved ones, up to n_b, become 0.
 *                    The same pointer (in place), or not overlapping
 *   new_lens         device int32 [batch], or NULL: first_tokens[b] + kept_lens[b], or
 *                    context_lens[b] where that is below first_tokens[b]; may be
 *                    context_lens, and no other array of the call (PA_EINVAL)
 * A block that a row of dst_tables (or block_tables, in place) writes belongs to
 * that sequence alone.  dst_stride need not reach max_context_len: tokens whose place
 * is beyond that table are not moved. */
int paged_attn_compact(const pa_kv_pool *pool, const int32_t *block_tables, int32_t bt_stride,
                       const int32_t *dst_tables, int32_t dst_stride, const int32_t *first_tokens,
                       const int32_t *context_lens, int32_t batch, int32_t max_context_len,
                       const int32_t *kept, int32_t kept_stride, const int32_t *kept_lens,
                       const float *totals, float *totals_out, int64_t totals_stride,
                       int32_t *new_lens, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PAGED_ATTN_TOKENS_H */
