// C ABI of librrq.so declared in include/rrq_serve.h: argument validation,
// workspace sizes and HIP error mapping. Every entry point validates its
// arguments before enqueueing anything and never throws.

#include "rrq_serve.h"

#include <cmath>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "rrq_serve_check.h"
#include "rrq_serve_launch.h"

using namespace rrq_detail;

extern "C" int rrq_cache_write(const rrq_cache *cache, const rrq_batch *batch, const void *K,
                               const void *V, int32_t dtype, int64_t k_token_stride,
                               int64_t k_head_stride, int64_t v_token_stride,
                               int64_t v_head_stride, hipStream_t stream)
{
    int st = check_cache(cache, true);
    if (st == RRQ_OK) st = check_batch(batch, true);
    if (st != RRQ_OK) return st;
    if (!known_dtype(dtype)) return RRQ_ERR_DTYPE;
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return RRQ_OK;
    st = check_rows(K, dtype, k_token_stride, k_head_stride);
    if (st == RRQ_OK) st = check_rows(V, dtype, v_token_stride, v_head_stride);
    if (st != RRQ_OK) return st;
    CacheWrite a = {*cache, *batch, K, V, k_token_stride, k_head_stride, v_token_stride,
                    v_head_stride};
    return status(launch_cache_write(a, dtype == RRQ_BF16, stream));
}

extern "C" int rrq_cache_read(const rrq_cache *cache, const rrq_batch *batch, void *K_out,
                              void *V_out, int32_t out_dtype, hipStream_t stream)
{
    int st = check_cache(cache, true);
    if (st == RRQ_OK) st = check_batch(batch, true);
    if (st != RRQ_OK) return st;
    if (!known_dtype(out_dtype)) return RRQ_ERR_DTYPE;
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return RRQ_OK;
    if (!K_out || !V_out) return RRQ_ERR_NULL;
    if (!aligned(K_out, 16) || !aligned(V_out, 16)) return RRQ_ERR_ALIGN;
    CacheRead a = {*cache, *batch, K_out, V_out};
    return status(launch_cache_read(a, out_dtype == RRQ_BF16, stream));
}

extern "C" int rrq_cache_attention_workspace(const rrq_cache *cache, const rrq_batch *batch,
                                             int32_t n_heads, size_t *workspace_bytes)
{
    if (!workspace_bytes) return RRQ_ERR_NULL;
    int st = check_cache(cache, false);
    if (st == RRQ_OK) st = check_batch(batch, false);
    if (st == RRQ_OK) st = check_heads(cache, batch, n_heads);
    if (st != RRQ_OK) return st;
    *workspace_bytes = 0;
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return RRQ_OK;
    // without a window: with one, no call takes more key ranges
    *workspace_bytes = attend_bytes(cache, batch, n_heads,
                                    attend_plan(*cache, *batch, n_heads, 0).splits);
    return RRQ_OK;
}

extern "C" int rrq_cache_attention(const rrq_cache *cache, const rrq_batch *batch, const void *Q,
                                   int32_t q_dtype, int64_t q_token_stride,
                                   int64_t q_head_stride, int32_t n_heads, float scale,
                                   int32_t causal, int64_t window, void *out, int32_t out_dtype,
                                   void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    Attend a = {};
    AttendPlan plan = {};
    const AttendCall call = {Q, out, workspace, q_token_stride, q_head_stride, window,
                             workspace_bytes, scale, q_dtype, out_dtype, n_heads, causal};
    const int st = prepare_attend(cache, batch, call, a, plan);
    if (st != RRQ_OK || plan.splits == 0) return st;
    return status(launch_attend(a, plan, stream));
}

namespace {

int check_logprobs(int64_t n_rows, int64_t vocab, int32_t n_top)
{
    if (n_rows < 0 || n_rows > (int64_t(1) << 23) || vocab < 1 || vocab > (int64_t(1) << 30))
        return RRQ_ERR_SHAPE;
    if (n_top < 0 || n_top > RRQ_MAX_TOP || n_top > vocab) return RRQ_ERR_SHAPE;
    return RRQ_OK;
}

size_t logprobs_bytes(int64_t n_rows, int64_t vocab, int32_t n_top)
{
    return n_rows == 0 ? 0
                       : (size_t)n_rows *
                             logprobs_row_bytes(logprobs_segments(n_rows, vocab), n_top);
}

}  // namespace

extern "C" int rrq_token_logprobs_workspace(int64_t n_rows, int64_t vocab, int32_t n_top,
                                            size_t *workspace_bytes)
{
    if (!workspace_bytes) return RRQ_ERR_NULL;
    const int st = check_logprobs(n_rows, vocab, n_top);
    if (st != RRQ_OK) return st;
    *workspace_bytes = logprobs_bytes(n_rows, vocab, n_top);
    return RRQ_OK;
}

extern "C" int rrq_token_logprobs(const void *logits, int32_t dtype, int64_t n_rows, int64_t vocab,
                                  int64_t row_stride, const int64_t *targets, int32_t n_top,
                                  float *logprobs, float *entropy, int64_t *top_ids,
                                  float *top_logprobs, void *workspace, size_t workspace_bytes,
                                  hipStream_t stream)
{
    const int st = check_logprobs(n_rows, vocab, n_top);
    if (st != RRQ_OK) return st;
    if (row_stride < vocab || row_stride > (int64_t(1) << 36)) return RRQ_ERR_SHAPE;
    if (!known_dtype(dtype)) return RRQ_ERR_DTYPE;
    if (n_rows == 0) return RRQ_OK;
    if (!logits || (targets && !logprobs) || (n_top > 0 && (!top_ids || !top_logprobs)))
        return RRQ_ERR_NULL;
    if (!aligned(logits, dtype == RRQ_F32 ? 4 : 2) || !aligned(targets, 8) ||
        !aligned(logprobs, 4) || !aligned(entropy, 4) ||
        (n_top > 0 && (!aligned(top_ids, 8) || !aligned(top_logprobs, 4))))
        return RRQ_ERR_ALIGN;
    const size_t need = logprobs_bytes(n_rows, vocab, n_top);
    if (need > 0) {
        if (!workspace) return RRQ_ERR_NULL;
        if (!aligned(workspace, 16)) return RRQ_ERR_ALIGN;
        if (workspace_bytes < need) return RRQ_ERR_WORKSPACE;
    }
    Logprobs a = {};
    a.logits = logits;
    a.targets = targets;
    a.logprobs = logprobs;
    a.entropy = entropy;
    a.top_logprobs = top_logprobs;
    a.top_ids = top_ids;
    a.workspace = workspace;
    a.n_rows = n_rows;
    a.vocab = vocab;
    a.row_stride = row_stride;
    a.n_top = n_top;
    a.segments = logprobs_segments(n_rows, vocab);
    return status(launch_logprobs(a, dtype == RRQ_BF16, stream));
}
