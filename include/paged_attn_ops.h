/*
 * paged_attn_ops.h -- the operators around the paged cache's attention, in the
 * C ABI of paged_attn.h (same library, same conventions for errors, ownership,
 * streams and device data):
 *
 *   - norm of each head's query and key row with the rotation to its position,
 *   - the same with keys and values written into the paged cache, for single
 *     tokens and for chunks,
 *   - decode and extend attention whose scores are capped by a tanh, biased by
 *     distance, or masked by a sliding window, documents or a prefix.
 *
 * They are for serving: none has a backward pass, as the library has none.
 */
#ifndef PAGED_ATTN_OPS_H
#define PAGED_ATTN_OPS_H

#include "paged_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of rows (the cache is bf16 always). */
enum { PA_BF16 = 0, PA_FP16 = 1, PA_FP32 = 2 };

/* ---------------------------------------------------------------------------
 * Rotary positions.
 *
 * The first rotary_dim values of a head's row form pairs, and the pair i of a
 * row at position t turns by the angle t * freqs[i] (RoFormer, arXiv
 * 2104.09864):
 *     (a, b) -> magnitude * (a cos - b sin, b cos + a sin).
 * ------------------------------------------------------------------------- */

/* Which values form pair i (0 <= i < rotary_dim / 2). */
enum {
  PA_ROPE_HALF = 0,        /* i and i + rotary_dim / 2 */
  PA_ROPE_INTERLEAVED = 1  /* 2i and 2i + 1 */
};

/* How the frequencies are scaled for contexts beyond the trained one. */
enum {
  PA_ROPE_UNSCALED = 0, /* f_i = base^(-2i / rotary_dim) */
  PA_ROPE_LINEAR = 1,   /* f_i / factor: interpolated positions */
  PA_ROPE_NTK = 2,      /* base * factor^(rotary_dim / (rotary_dim - 2)) for base */
  PA_ROPE_BANDS = 3,    /* by the turns c_i = original_context * f_i / (2 pi): f_i / factor below `low`
                           turns, f_i above `high`, linear in c_i between */
  PA_ROPE_YARN = 4      /* f_i / factor and f_i blended by a ramp over i between the pairs that turn `high`
                           and `low` times in original_context; magnitude 0.1 ln(factor) + 1 (YaRN, arXiv
                           2309.00071, which uses low 1 and high 32) */
};

/* The rotary_dim / 2 frequencies (radians per position) and the magnitude of a
 * scaling, in host memory, for pa_rope_create.
 *   rotary_dim        even, 0 .. 256
 *   base              > 1
 *   factor            > 0; read by all scalings but PA_ROPE_UNSCALED
 *   original_context  > 0, low, high with 0 < low < high: PA_ROPE_BANDS, PA_ROPE_YARN
 *   freqs_out         [rotary_dim / 2] (may be NULL where that is 0)
 *   magnitude_out     1 but for PA_ROPE_YARN */
int pa_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor,
                        double original_context, double low, double high, double *freqs_out,
                        double *magnitude_out);

/* A rotation: host metadata only, like the pool handle.  Any frequencies may
 * be given, those of pa_rope_frequencies or the caller's own.
 *   head_dim    a multiple of 16, 16 .. 256
 *   rotary_dim  a multiple of 16, 0 .. head_dim; 0: no rotation (norms alone)
 *   layout      PA_ROPE_HALF or PA_ROPE_INTERLEAVED
 *   freqs       [rotary_dim / 2] finite values, copied
 *   magnitude   finite in fp32; multiplies the rotated values
 *   out         receives the handle; untouched on error */
typedef struct pa_rope pa_rope;
int pa_rope_create(int32_t head_dim, int32_t rotary_dim, int32_t layout, const double *freqs,
                   double magnitude, pa_rope **out);

/* Destroy a handle.  NULL is a no-op. */
int pa_rope_destroy(pa_rope *rope);

/* Norm and rotation of the q and k rows of a batch of tokens, in one launch:
 * for every token and head
 *     y = x * weight / sqrt(mean(x^2) + eps)     (weight NULL: y = x),
 * then the pairs of y turn to the token's position.  Sums and products are
 * fp32, rounded once to the rows' type; values that are neither normed nor
 * rotated keep their bits.
 *   q, k          device rows of dtype, 16-byte aligned: head h of token t begins
 *                 at q + t * q_stride + h * head_dim.  Rows of a packed projection
 *                 are given by their offsets and its stride.  Either may be NULL
 *                 with 0 heads
 *   *_stride      elements from token to token, at least heads * head_dim, a
 *                 multiple of 16 bytes
 *   num_q_heads, num_kv_heads  >= 0
 *   q_weight, k_weight  device fp32 [head_dim], 16-byte aligned, or NULL: no norm
 *   eps           >= 0, added to the mean square
 *   dtype         PA_BF16, PA_FP16 or PA_FP32
 *   positions     device int32 [tokens]
 *   tokens        0 (a no-op) .. 2^26 - 64
 *   q_out, k_out  rows like q and k; each may be its input itself (same pointer
 *                 and stride), else they overlap no input */
int paged_attn_norm_rope(const pa_rope *rope, const void *q, int64_t q_stride, int32_t num_q_heads,
                         const float *q_weight, const void *k, int64_t k_stride,
                         int32_t num_kv_heads, const float *k_weight, float eps, int32_t dtype,
                         const int32_t *positions, int32_t tokens, void *q_out,
                         int64_t q_out_stride, void *k_out, int64_t k_out_stride, void *stream);

/* The same for the new tokens of a batch, with their K and V rows written into
 * the paged cache: token i of sequence b's chunk of L_b tokens takes slot
 * t = n_b - L_b + i (n_b = context_lens[b], the chunk included),
 *     K pool[block_tables[b][t / 16]][g][t % 16][:] = normed, rotated k row,
 *     V pool[...]                                   = v row, as it is,
 * and the normed, rotated q row goes to q_out for paged_attn_extend, the
 * decodes, or their biased forms.  K, V and q_out are bf16, rounded once.
 *   pool          geometry and K/V device pools (written); head_dim as rope's
 *   q, k, v       device rows of dtype as in paged_attn_norm_rope (k and v of the
 *                 pool's num_kv_heads); q may be NULL with num_q_heads 0
 *   positions     device int32 [total_q] to rotate by, or NULL: the slot t
 *   q_start       device int32 [batch + 1], nondecreasing from 0: sequence b's
 *                 rows are q_start[b] .. q_start[b+1] - 1; or NULL: row b is
 *                 sequence b's single new token
 *   total_q       rows of q, k, v and q_out, 0 .. 2^26 - 64; rows behind the last sequence are
 *                 neither read into anything nor written
 *   block_tables  device int32 [batch][bt_stride]; the blocks of the new slots
 *                 must belong to sequence b alone (see paged_attn_append_kv)
 *   context_lens  device int32 [batch]
 *   q_out         device bf16 [total_q][num_q_heads][head_dim], 16-byte aligned;
 *                 overlaps no input
 * Device data is clamped: lengths into [0, 16 * bt_stride], chunks into their
 * lengths (a longer one appends its first n_b rows), ids into the pool. */
int paged_attn_rope_append(const pa_kv_pool *pool, const pa_rope *rope, const void *q,
                           int64_t q_stride, int32_t num_q_heads, const float *q_weight,
                           const void *k, int64_t k_stride, const float *k_weight, const void *v,
                           int64_t v_stride, float eps, int32_t dtype, const int32_t *positions,
                           const int32_t *q_start, int32_t total_q, const int32_t *block_tables,
                           int32_t bt_stride, const int32_t *context_lens, int32_t batch,
                           void *q_out, void *stream);

/* ---------------------------------------------------------------------------
 * Attention with capped, biased or masked scores.
 *
 * For a query row of head h at position p and token t of its sequence:
 *     s = scale * <q, K_g[t]>
 *     s = softcap * tanh(s / softcap)         where softcap > 0
 *     s = s - slopes[h] * |p - t|             where slopes is given
 * and the row attends to the tokens first <= t < end, with softmax over them:
 *     first = max(0, first_tokens[row], p - window + 1 where window > 0)
 *     end   = p + 1, or for an extend with prefix_lens max(p + 1, min(prefix_lens[b], n_b)).
 * So first_tokens holds the start of each row's document in a sequence packed
 * from documents, window is a sliding window (the row's own token and the
 * window - 1 before it), and a prefix sees itself whole.  A row that sees
 * nothing gives zeros.  What hidden tokens hold (NaN and infinities too) changes
 * no bit of a row.  An infinity or NaN in V that a row does see, a NaN among its
 * scores, and +infinity there without a softcap (under one it is the cap) make
 * its outputs infinite or NaN; a score of -infinity weighs nothing, and a row of
 * those alone gives zeros.  Weights reach the matrix cores to about 2^-17, as
 * everywhere in this library; sums are fp32.
 * ------------------------------------------------------------------------- */

/* Bytes of the workspace of a biased decode (max_chunk 1) or extend: room for
 * the partial results of rows whose tokens are split over workgroups, 0 where
 * none are.  It depends on these arguments alone.  The arguments are those of
 * the call; window as there. */
int paged_attn_biased_workspace_size(const pa_kv_pool *pool, int32_t batch, int32_t num_q_heads,
                                     int32_t max_context_len, int32_t max_chunk, int32_t window,
                                     size_t *bytes_out);

/* One decode step (one new token per sequence, at position n_b - 1, its K and V
 * in the cache already) with these scores.
 *   pool             head_dim 64 or 128
 *   q, block_tables, bt_stride, context_lens, batch, scale, max_context_len
 *                    as in paged_attn_decode; max_context_len below 2^30
 *   num_q_heads      any multiple of the pool's num_kv_heads
 *   softcap          0 (none) or positive, finite (PA_EUNSUPPORTED where its
 *                    ratio to scale leaves the range of fp32)
 *   slopes           device fp32 [num_q_heads], or NULL
 *   window           0 (none) or positive
 *   first_tokens     device int32 [batch], or NULL
 *   workspace        device, 16-byte aligned, of workspace_bytes, at least
 *                    paged_attn_biased_workspace_size; its content is not kept.
 *                    Calls that may run at the same time need one each
 *   out              device bf16 [batch][num_q_heads][head_dim], 16-byte aligned */
int paged_attn_decode_biased(const pa_kv_pool *pool, const void *q, const int32_t *block_tables,
                             int32_t bt_stride, const int32_t *context_lens, int32_t batch,
                             int32_t num_q_heads, float scale, float softcap, const float *slopes,
                             int32_t window, const int32_t *first_tokens, int32_t max_context_len,
                             void *workspace, size_t workspace_bytes, void *out, void *stream);

/* Attention of each sequence's chunk of new tokens (their K and V in the cache
 * already) with these scores; as paged_attn_extend, for head_dim 64 too, any
 * number of query heads per KV head and contexts below 2^30 tokens.
 *   q, q_start, total_q, block_tables, bt_stride, context_lens, batch, scale,
 *   max_context_len, max_chunk, out     as in paged_attn_extend; rows of out
 *                    behind the last sequence are left as they are
 *   softcap, slopes, window, workspace, workspace_bytes  as in paged_attn_decode_biased
 *   first_tokens     device int32 [total_q], or NULL
 *   prefix_lens      device int32 [batch], or NULL */
int paged_attn_extend_biased(const pa_kv_pool *pool, const void *q, const int32_t *q_start,
                             int32_t total_q, const int32_t *block_tables, int32_t bt_stride,
                             const int32_t *context_lens, int32_t batch, int32_t num_q_heads,
                             float scale, float softcap, const float *slopes, int32_t window,
                             const int32_t *first_tokens, const int32_t *prefix_lens,
                             int32_t max_context_len, int32_t max_chunk, void *workspace,
                             size_t workspace_bytes, void *out, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PAGED_ATTN_OPS_H */
