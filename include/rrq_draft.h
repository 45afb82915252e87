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

#ifdef __cplusplus
}
#endif

#endif /* RRQ_DRAFT_H */
