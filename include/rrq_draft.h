/*
 * rrq_draft.h - C ABI of librrq.so, continued: what a decoder that drafts tokens
 * with a short prefix of its packages and checks them with a longer one runs
 * beside the calls of rrq_serve.h.
 *
 * The conventions of rrq.h and rrq_serve.h hold for every call here.
 */
#ifndef RRQ_DRAFT_H
#define RRQ_DRAFT_H

#include "rrq_serve.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How a row is normalised, mean over the row's elements:
 *   RRQ_NORM_RMS    x / sqrt(mean(x^2) + eps)
 *   RRQ_NORM_LAYER  (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps) */
enum rrq_norm_kind {
    RRQ_NORM_NONE = 0,
    RRQ_NORM_RMS = 1,
    RRQ_NORM_LAYER = 2
};

/*
 * rrq_norm - the norms around a block (host memory, read during the call).
 *
 *   weight, bias  device, float [hidden], of the next block's norm; NULL: 1, 0.
 *   post_weight   device, float [hidden], of the norm of the block's output; NULL: 1.
 *   kind          RRQ_NORM_RMS or _LAYER.
 *   post          how the block's output is normalised: any of rrq_norm_kind.
 *   eps           >= 0, finite.
 *   scale         of what is added to the residual; finite.
 * Arrays 4-byte aligned.
 */
typedef struct rrq_norm {
    const float *weight;
    const float *bias;
    const float *post_weight;
    int32_t kind;
    int32_t post;
    float eps;
    float scale;
} rrq_norm;

/*
 * rrq_block_norm - from one block of a decoder to the next, a row at a time:
 *     y' = post(y) post_weight                   (y itself without a post norm)
 *     h = residual + scale (gate y')             (no gate: 1)
 *     out = kind(h) weight + bias
 *
 *   residual   device, residual_dtype (RRQ_F32 or RRQ_BF16) [n_rows][hidden],
 *              residual_stride elements between rows.
 *   y          device, y_dtype [n_rows][hidden], y_stride: the block's output. NULL:
 *              h is the residual (no gate, no post norm then; h is not written).
 *   gate       device, y_dtype, or NULL: [n_rows][hidden] with gate_stride, or for
 *              gate_stride 0 one row for all.
 *   n_rows     0..2^26 (0 enqueues nothing); hidden 1..65536; strides hidden..2^36
 *              (a single row's is not used).
 *   out        device, out_dtype [n_rows][hidden] contiguous (written).
 *   h          device, residual_dtype [n_rows][hidden] contiguous (written if y is
 *              given). May be the residual itself, where that is contiguous.
 * Buffers are aligned to their types; nothing else may overlap.
 *
 * Arithmetic: binary32 throughout, the mean before the squares of the differences
 * to it, h rounded only where it is written (out comes from the unrounded one).
 * Sums of squares have to stay in binary32's range (elements up to 2^55): a row
 * past it, or one that holds an infinity or a NaN, gives unspecified values in
 * that row alone.
 *
 * Returns RRQ_OK, or RRQ_ERR_NULL / _ALIGN / _SHAPE / _DTYPE / _FORMAT (an unknown
 * kind) with nothing enqueued, or RRQ_ERR_HIP.
 */
int rrq_block_norm(const rrq_norm *norm, const void *residual, int32_t residual_dtype,
                   int64_t residual_stride, const void *y, int32_t y_dtype, int64_t y_stride,
                   const void *gate, int64_t gate_stride, int64_t n_rows, int64_t hidden,
                   void *out, int32_t out_dtype, void *h, hipStream_t stream);

/* Which channels a pair i of a rotation of rot_dim channels consists of. */
enum rrq_rotary_layout {
    RRQ_ROTARY_HALF = 0,            /* i and i + rot_dim / 2 */
    RRQ_ROTARY_INTERLEAVED = 1      /* 2 i and 2 i + 1 */
};

/*
 * rrq_rotary - rotary positions (host memory, read during the call).
 *
 *   frequencies  device, double [rot_dim / 2], 8-byte aligned: pair i of a token at
 *                position p turns by the angle p frequencies[i] (radians). Any
 *                schedule for long contexts is a choice of frequencies.
 *   amplitude    factor of cosines and sines; finite.
 *   rot_dim      the first rot_dim channels of a head are rotated, a multiple of 8,
 *                8..head_dim; the others stay.
 *   layout       enum rrq_rotary_layout.
 */
typedef struct rrq_rotary {
    const double *frequencies;
    double amplitude;
    int32_t rot_dim;
    int32_t layout;
} rrq_rotary;

/*
 * rrq_cache_append - rotate the batch's queries and keys to their positions, and
 * quantise keys and values into their pages.
 *
 *   positions  device, int32 [n_tokens], 4-byte aligned: the position each row is
 *              rotated to (drafted tokens of a tree: by their depth), of any sign.
 *              NULL: the row's place in its sequence.
 *   Q          device, dtype (RRQ_F32 or RRQ_BF16) [n_tokens][n_heads][head_dim], K
 *              and V as for rrq_cache_write, of the same dtype: columns of one
 *              fused projection, with strides in elements; 16-byte aligned, strides
 *              multiples of 16 bytes.
 *   n_heads    query heads, 1..2^16 (any number).
 *   Q_out      device, dtype [n_tokens][n_heads][head_dim] contiguous, 16-byte
 *              aligned (written): the queries rotated. May be Q itself, where that is
 *              contiguous, and overlaps nothing else. Rows outside
 *              offsets[0]..offsets[n_seqs]-1 are not written.
 *
 * With c = fl(amplitude cos t), s = fl(amplitude sin t) of the angle t in 64 bits,
 * fl() one binary32 rounding, a pair (x, y) becomes
 *   fl(fl(x c) - fl(y s)), fl(fl(y c) + fl(x s)),
 * rounded to dtype in Q_out; keys go on in binary32, and keys and values are written
 * as rrq_cache_write does. Angles up to 2^50 (NaN beyond or for frequencies that are
 * not finite: unspecified codes, as for keys that are not finite).
 *
 * Returns as rrq_cache_write (_FORMAT for an unknown layout as well).
 */
int rrq_cache_append(const rrq_cache *cache, const rrq_batch *batch, const rrq_rotary *rotary,
                     const int32_t *positions, const void *Q, const void *K, const void *V,
                     int32_t dtype, int64_t q_token_stride, int64_t q_head_stride,
                     int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                     int64_t v_head_stride, int32_t n_heads, void *Q_out, hipStream_t stream);

/*
 * rrq_tree_attention - softmax attention of drafted tokens over the cache, as
 * rrq_cache_attention, but of its step's own rows a row sees those that its bits say
 * (its path from the tree's root). A sequence's rows of the batch are at positions
 * start = length - n_b on in the cache; row i of them sees
 *   - position j < start, for window > 0 only if j > p_i - window;
 *   - the step's row j (at start + j) if bit j of row i of `seen` is set, whatever
 *     the window; a row sees itself by its own bit alone. Bits of n_b and more play
 *     no part, rows past the bits are not seen.
 * A row that sees nothing gives zeros. All positions below the length have to have
 * been written, the step's rows that no bit names included: those have no weight, but
 * their codes are multiplied by it, and what a slot held before may be no number.
 *
 *   seen       device, uint64 [n_tokens][seen_words], 8-byte aligned: bit j is bit
 *              j % 64 of word j / 64.
 *   seen_words 1..2^20.
 *   positions  device, int32 [n_tokens], 4-byte aligned: p_i, which a window counts
 *              from (a drafted token's depth in its tree, not its row). NULL: the
 *              row's place start + i. Not read without a window.
 *   The other arguments, and the workspace (rrq_cache_attention_workspace), as for
 *   rrq_cache_attention; and its arithmetic.
 *
 * Returns as rrq_cache_attention.
 */
int rrq_tree_attention(const rrq_cache *cache, const rrq_batch *batch, const void *Q,
                       int32_t q_dtype, int64_t q_token_stride, int64_t q_head_stride,
                       int32_t n_heads, float scale, const uint64_t *seen, int64_t seen_words,
                       const int32_t *positions, int64_t window, void *out, int32_t out_dtype,
                       void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * rrq_verify_drafts - which drafted tokens the target accepts, and the token that
 * follows them, from given random numbers.
 *
 * Rows offsets[b] .. offsets[b+1]-1 of the logits are sequence b's: row 0 is its last
 * committed token, row j > 0 the drafted token tokens[j], a child of row parents[j].
 * p_i is the softmax of row i's logits over the temperature (a temperature of 0: 1 for
 * the first of the largest logits). A walk starts at row 0 and ends after max_accept
 * drafts at the latest. At row i its children are tried in the order of their rows:
 *   - with the draft's distributions (a chain; q_j, the softmax of draft row j - 1 over
 *     the draft's temperature, is what token j was drawn from): accepted if
 *     u_j q_j(t_j) < p_i(t_j); else the walk ends, and the next token is drawn from the
 *     positive part of p_i - q_j (from p_i where that is nothing);
 *   - without: accepted if u_j w < p_i(t_j), where w is what p_i has left: 1 at first,
 *     a rejected token's probability is taken out (and is 0 for a sibling with the same
 *     token). After the last child the walk ends, and the next token is drawn from what
 *     is left.
 * Where the walk ends at a row without children, or after max_accept drafts, the next
 * token is drawn from its p. Drawn is the first token whose running sum, over the
 * tokens in order, exceeds u_0 times the whole; for a temperature of 0 it is the
 * likeliest token of the row. At a temperature of 0 draft is not read.
 *
 *   logits     device, dtype (RRQ_F32 or RRQ_BF16) [n_rows][vocab], row_stride
 *              elements between rows, aligned to its type.
 *   tokens     device, int64 [n_rows], of rows 0 without meaning. One outside the
 *              vocabulary is rejected.
 *   offsets    device, int32 [n_seqs + 1], ascending (clamped to 0..n_rows).
 *   uniforms   device, float [n_rows], in [0, 1): u_j.
 *   parents    device, int32 [n_rows], by rows within the sequence, 0 <= parents[j] < j
 *              (another row is no one's child); NULL: a chain, j - 1.
 *   draft      device, dtype [n_seqs][max_accept][vocab] with strides in elements, or
 *              NULL. Not together with parents. Rows of absent drafts are not read.
 *              A row of -inf, or one that holds a NaN or +inf, rejects its token, and
 *              the next one is drawn from p.
 *   temperature, draft_temperature  2^-64 .. 2^64; temperature may be 0.
 *   max_accept 0..2^20.
 *   counts     device, int32 [n_seqs] (written): accepted drafts.
 *   following  device, int64 [n_seqs] (written): the next token; -1 for a sequence
 *              without rows, or that ends at a row without a distribution. Where a row's
 *              drafts are all that it leaves possible, and the sum's last digits reject
 *              them all, the last of them that has any probability. A row of -inf,
 *              or one that holds a NaN or +inf, accepts nothing and gives -1. At a
 *              temperature of 0 infinities are numbers as others and a NaN is less
 *              than any: of a row of -inf the first token is accepted or given, and
 *              only a row of nothing but NaN gives -1.
 *   paths      device, int32 [n_seqs][max_accept + 1] (written): row 0, then the
 *              accepted rows, then -1.
 *   n_rows     0..2^23; vocab 1..2^30; row_stride >= vocab; n_seqs 0..2^20 (0: nothing
 *              is enqueued); (n_rows + n_seqs (max_accept + 1)) ceil(vocab / 4096) < 2^24.
 *   workspace  device, 16-byte aligned, workspace_bytes of at least
 *              rrq_verify_drafts_workspace's value. Its content is of no use before or
 *              after the call; calls that may run at the same time need their own.
 * int64 arrays 8-byte aligned, int32 and float arrays 4-byte.
 *
 * Arithmetic: the next token is drawn in 64 bits; a row's sum behind an acceptance has
 * binary32 exponentials and is good to 2^-24 as a rule, to 18 x 2^-24 at worst. Results
 * are deterministic.
 *
 * Returns RRQ_OK, or RRQ_ERR_NULL / _ALIGN / _SHAPE / _DTYPE / _WORKSPACE with nothing
 * enqueued, or RRQ_ERR_HIP.
 */
int rrq_verify_drafts(const void *logits, int32_t dtype, int64_t n_rows, int64_t vocab,
                      int64_t row_stride, const int64_t *tokens, const int32_t *offsets,
                      int64_t n_seqs, const float *uniforms, const int32_t *parents,
                      const void *draft, int64_t draft_seq_stride, int64_t draft_row_stride,
                      double temperature, double draft_temperature, int32_t max_accept,
                      int32_t *counts, int64_t *following, int32_t *paths, void *workspace,
                      size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace rrq_verify_drafts needs (host only); draft_rows: n_seqs times
 * max_accept with a draft, else 0. */
int rrq_verify_drafts_workspace(int64_t n_rows, int64_t vocab, int64_t n_seqs, int64_t draft_rows,
                                size_t *workspace_bytes);

#ifdef __cplusplus
}
#endif

#endif /* RRQ_DRAFT_H */
