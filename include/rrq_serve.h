/*
 * rrq_serve.h - C ABI of librrq.so, continued: what a decoder served from RRQ
 * packages runs beside rrq_linear. A paged key/value cache held in 8 bits
 * (written from the linear layer's output, read back, attended over) and the
 * scoring of tokens from the head's logits.
 *
 * The conventions of rrq.h hold for every call here: device pointers owned by
 * the caller, work enqueued on `stream` without waiting, arguments checked
 * before anything is enqueued, status codes of enum rrq_status, nothing
 * allocated, no mutable state in the library. The descriptors (struct
 * rrq_cache, struct rrq_batch) are host memory, read during the call only.
 *
 * Index data lives on the device (page table, lengths, offsets) and is not
 * checked by the host: the kernels take an entry that is out of range as
 * absent. A page number outside 0..n_pages-1, or a position at or past
 * max_pages * page_size, is neither read nor written; offsets are clamped to
 * 0..n_tokens.
 */
#ifndef RRQ_SERVE_H
#define RRQ_SERVE_H

#include "rrq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* 8-bit code of a cached value: value = code * scale. */
enum rrq_code_type {
    RRQ_CODE_INT8 = 0,  /* two's complement, -127..127 */
    RRQ_CODE_FP8 = 1    /* e4m3 (4 exponent bits, 3 mantissa bits, no infinities), up to 448 */
};

/*
 * rrq_cache - one layer's key/value cache: n_pages pages of page_size tokens.
 * The block of one page and one kv head has one scale for its keys and one
 * for its values.
 *
 *   k_codes   device, [n_pages][n_kv_heads][page_size][head_dim], 16-byte aligned.
 *   v_codes   device, [n_pages][n_kv_heads][head_dim][page_size], 16-byte aligned
 *             (both products of attention then read runs of bytes).
 *   k_scales, v_scales  device, float [n_pages][n_kv_heads], 4-byte aligned.
 *             Scales of pages in use are finite and 0 or more, as rrq_cache_write
 *             leaves them; with others, what is read from or attended over
 *             their page and head is unspecified.
 *   n_pages   >= 1.
 *   n_kv_heads 1..1024.
 *   head_dim  64, 128 or 256.
 *   page_size 16, 32, 64 or 128.
 *   code_type enum rrq_code_type.
 *
 * The buffers need no initial value: what a page held before a sequence's
 * first token in it is never used.
 */
typedef struct rrq_cache {
    uint8_t *k_codes;
    uint8_t *v_codes;
    float *k_scales;
    float *v_scales;
    int64_t n_pages;
    int32_t n_kv_heads;
    int32_t head_dim;
    int32_t page_size;
    int32_t code_type;
} rrq_cache;

/*
 * rrq_batch - which tokens of which sequences a call works on. Rows
 * offsets[b] .. offsets[b+1]-1 of the call's dense tensors are the last
 * n_b = offsets[b+1] - offsets[b] tokens of sequence b, at positions
 * lengths[b] - n_b .. lengths[b] - 1; n_b may differ from sequence to
 * sequence and may be 0.
 *
 *   page_table  device, int32 [n_seqs][table_stride]: entry j of row b is the
 *               page holding positions j * page_size .. of sequence b; the
 *               first max_pages entries of a row may be read, as far as the
 *               sequence's length reaches. A page that is written belongs to
 *               one sequence.
 *   lengths     device, int32 [n_seqs]: tokens of the sequence, this call's
 *               included (below 0: none). Attention sees the first 2^31 - 4096.
 *   offsets     device, int32 [n_seqs + 1], ascending.
 *   table_stride, max_pages  1 <= max_pages <= table_stride.
 *   n_seqs      0..2^20 (0: the call enqueues nothing).
 *   n_tokens    rows of the call's dense tensors, 0..2^26.
 * All three arrays 4-byte aligned.
 */
typedef struct rrq_batch {
    const int32_t *page_table;
    const int32_t *lengths;
    const int32_t *offsets;
    int64_t table_stride;
    int64_t max_pages;
    int64_t n_seqs;
    int64_t n_tokens;
} rrq_batch;

/*
 * rrq_cache_write - quantise the keys and values of the batch's tokens into
 * their pages.
 *
 *   K, V       device, dtype (RRQ_F32 or RRQ_BF16) [n_tokens][n_kv_heads][head_dim]
 *              with the given strides in elements between tokens and between
 *              heads (a head's values are contiguous): columns of a fused q/k/v
 *              output of rrq_linear are written without a copy. 16-byte
 *              aligned, strides multiples of 16 bytes.
 *
 * Per touched page, kv head, and keys or values, with c_max = 127 (int8) or
 * 448 (fp8), f the slot of the call's first token in the page and fl() one
 * binary32 rounding:
 *   a = max |x| over the call's tokens in the page;
 *   s_n = fl(a fl(1/c_max)); s_o = the stored scale if f > 0, else 0;
 *   s = max(s_o, s_n), 0 if that is below 2^-126; inv = fl(1/s), 0 for s = 0;
 *   new codes E(fl(x inv)); codes of the slots before f, if s > s_o > 0,
 *   E(fl(c fl(s_o inv))); s is stored.
 * E rounds to nearest, ties to even: to an integer clamped to -127..127, or
 * to an e4m3 value clamped to -448..448. A call repeated on the same tokens
 * leaves the same codes.
 * Precondition: finite K and V; otherwise the touched page and head hold
 * unspecified codes and scales (nothing outside them is touched).
 *
 * Returns RRQ_OK, or RRQ_ERR_NULL / _ALIGN / _SHAPE / _DTYPE / _FORMAT (an
 * unknown code_type) with nothing enqueued, or RRQ_ERR_HIP.
 */
int rrq_cache_write(const rrq_cache *cache, const rrq_batch *batch, const void *K, const void *V,
                    int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                    int64_t v_token_stride, int64_t v_head_stride, hipStream_t stream);

/*
 * rrq_cache_read - the batch's tokens read back: fl(c s), as binary32 or
 * rounded to bfloat16 (nearest-even).
 *
 *   K_out, V_out  device, out_dtype [n_tokens][n_kv_heads][head_dim] contiguous,
 *                 16-byte aligned (written). Rows of a page number out of
 *                 range are zeros; rows outside offsets[0]..offsets[n_seqs]-1,
 *                 or without a position in the table, are not written.
 *
 * Returns as rrq_cache_write.
 */
int rrq_cache_read(const rrq_cache *cache, const rrq_batch *batch, void *K_out, void *V_out,
                   int32_t out_dtype, hipStream_t stream);

/*
 * rrq_cache_attention - softmax attention of the batch's tokens over their
 * sequences' cached keys and values (written before, this call's tokens
 * included):
 *     out_i = sum_j p_ij v_j,  p_i = softmax over j of scale (q_i . k_j)
 * with k_j, v_j = code * scale, j over the positions of the row's sequence
 * below its length; if causal, j <= pos_i; if window > 0, j > pos_i - window.
 * Query head h reads kv head h / (n_heads / n_kv_heads). A row that sees no
 * position gives zeros.
 *
 *   Q          device, q_dtype (RRQ_F32 or RRQ_BF16) [n_tokens][n_heads][head_dim]
 *              with strides in elements (a head's values contiguous),
 *              16-byte aligned, strides multiples of 16 bytes.
 *   n_heads    a multiple of n_kv_heads, up to 2^16; n_tokens * n_heads / n_kv_heads
 *              <= 2^26.
 *   scale      finite.
 *   causal     0 or 1.
 *   window     0 (none) or the number of positions a token sees, its own the
 *              last.
 *   out        device, out_dtype [n_tokens][n_heads][head_dim] contiguous,
 *              16-byte aligned (written): rows of rrq_linear's X. Rows outside
 *              offsets[0]..offsets[n_seqs]-1 are not written.
 *   workspace  device, 16-byte aligned, workspace_bytes of at least
 *              rrq_cache_attention_workspace's value (NULL if that is 0). Its
 *              content is of no use before or after the call; calls that may
 *              run at the same time need their own.
 *
 * Arithmetic: codes are exact, products are summed in binary32, and so is the
 * softmax's sum. The other operands are rounded according to the result. For
 * bfloat16 (8 bits): queries to 11 significant bits relative to their row's
 * largest (bfloat16 ones are exact), the softmax's weights, each with its block's
 * value scale, to 11 bits before the second product, and those below 2^-20 of
 * the row's largest to 2^-31 of it. For binary32 both go in as two parts of 11
 * bits: 22 bits, and 2^-39 of the row's largest weight (at about twice the
 * products' time, where those bound the call). (Value scales of one sequence and
 * head are taken to lie within a factor of 2^100 of each other; smaller ones
 * count as at that distance.) Results are deterministic for one shape of call;
 * they may differ in the last bits between calls of another batch.
 *
 * Returns RRQ_OK, or RRQ_ERR_NULL / _ALIGN / _SHAPE / _DTYPE / _FORMAT /
 * _WORKSPACE with nothing enqueued, or RRQ_ERR_HIP.
 */
int rrq_cache_attention(const rrq_cache *cache, const rrq_batch *batch, const void *Q,
                        int32_t q_dtype, int64_t q_token_stride, int64_t q_head_stride,
                        int32_t n_heads, float scale, int32_t causal, int64_t window, void *out,
                        int32_t out_dtype, void *workspace, size_t workspace_bytes,
                        hipStream_t stream);

/*
 * rrq_cache_attention_workspace - bytes of workspace rrq_cache_attention
 * needs for this cache, batch and n_heads (host only; the batch's device
 * arrays are not read, its sizes are). Returns RRQ_OK or an argument error.
 */
int rrq_cache_attention_workspace(const rrq_cache *cache, const rrq_batch *batch, int32_t n_heads,
                                  size_t *workspace_bytes);

/* Alternatives rrq_token_logprobs returns at most. */
#define RRQ_MAX_TOP 32

/*
 * rrq_token_logprobs - for each row of logits x: the log probability of a
 * given token, the entropy of the distribution (both natural), and the n_top
 * likeliest tokens with their log probabilities.
 *     lse = log sum_v exp(x_v);  logprob = x_target - lse;
 *     entropy = lse - sum_v exp(x_v - lse) x_v.
 *
 *   logits     device, dtype (RRQ_F32 or RRQ_BF16) [n_rows][vocab], row_stride
 *              elements between rows, aligned to its type.
 *   n_rows     0..2^23 (0 enqueues nothing); vocab 1..2^30; row_stride >= vocab.
 *   targets    device, int64 [n_rows]; a target outside 0..vocab-1 (an ignored
 *              position) gives 0. NULL: no target, logprobs is not written.
 *   n_top      0..RRQ_MAX_TOP, at most vocab.
 *   logprobs   device, float [n_rows] (written if targets is given).
 *   entropy    device, float [n_rows] (written) or NULL.
 *   top_ids    device, int64 [n_rows][n_top] (written if n_top > 0), by logit
 *              descending, equal logits by index ascending; a NaN counts as
 *              less than every number.
 *   top_logprobs  device, float [n_rows][n_top] (written if n_top > 0).
 *   workspace  as for rrq_cache_attention; rrq_token_logprobs_workspace.
 * Float arrays 4-byte aligned, int64 arrays 8-byte aligned.
 *
 * A logit of -inf has probability 0 and adds nothing to the entropy. A row of
 * -inf only gives log probabilities -inf and entropy 0; a row that holds a
 * NaN or +inf gives NaN (its top_ids stay ordered as above).
 * Arithmetic: differences to the largest logit, exponentials and sums in
 * binary32.
 *
 * Returns RRQ_OK, or RRQ_ERR_NULL / _ALIGN / _SHAPE / _DTYPE / _WORKSPACE
 * with nothing enqueued, or RRQ_ERR_HIP.
 */
int rrq_token_logprobs(const void *logits, int32_t dtype, int64_t n_rows, int64_t vocab,
                       int64_t row_stride, const int64_t *targets, int32_t n_top,
                       float *logprobs, float *entropy, int64_t *top_ids, float *top_logprobs,
                       void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace rrq_token_logprobs needs (host only). */
int rrq_token_logprobs_workspace(int64_t n_rows, int64_t vocab, int32_t n_top,
                                 size_t *workspace_bytes);

#ifdef __cplusplus
}
#endif

#endif /* RRQ_SERVE_H */
