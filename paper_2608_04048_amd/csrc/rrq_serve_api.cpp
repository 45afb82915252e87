// C ABI of librrq.so declared in include/rrq_serve.h: argument validation,
// workspace sizes and HIP error mapping. Every entry point validates its
// arguments before enqueueing anything and never throws.

#include "rrq_serve.h"

#include <cmath>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "rrq_serve_launch.h"

namespace {

using namespace rrq_detail;

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// The cache's sizes, and (buffers) its pointers.
int check_cache(const rrq_cache *c, bool buffers)
{
    if (!c) return RRQ_ERR_NULL;
    if (c->code_type != RRQ_CODE_INT8 && c->code_type != RRQ_CODE_FP8) return RRQ_ERR_FORMAT;
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return RRQ_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return RRQ_ERR_SHAPE;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
        return RRQ_ERR_SHAPE;
    // byte offsets into the codes fit in int64
    if (c->n_pages > INT64_MAX / ((int64_t)c->n_kv_heads * c->head_dim * c->page_size))
        return RRQ_ERR_SHAPE;
    if (!buffers) return RRQ_OK;
    if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return RRQ_ERR_NULL;
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, 4) ||
        !aligned(c->v_scales, 4))
        return RRQ_ERR_ALIGN;
    return RRQ_OK;
}

int check_batch(const rrq_batch *b, bool buffers)
{
    if (!b) return RRQ_ERR_NULL;
    if (b->n_seqs < 0 || b->n_seqs > (int64_t(1) << 20) || b->n_tokens < 0 ||
        b->n_tokens > (int64_t(1) << 26))
        return RRQ_ERR_SHAPE;
    if (b->n_seqs == 0) return RRQ_OK;
    if (b->max_pages < 1 || b->table_stride < b->max_pages ||
        b->table_stride > (int64_t(1) << 40))
        return RRQ_ERR_SHAPE;
    if (!buffers) return RRQ_OK;
    if (!b->page_table || !b->lengths || !b->offsets) return RRQ_ERR_NULL;
    if (!aligned(b->page_table, 4) || !aligned(b->lengths, 4) || !aligned(b->offsets, 4))
        return RRQ_ERR_ALIGN;
    return RRQ_OK;
}

// Dense rows read with caller's strides: 16-byte aligned pieces.
int check_rows(const void *p, int32_t dtype, int64_t token, int64_t head)
{
    const int64_t per = dtype == RRQ_F32 ? 4 : 8;       // elements in 16 bytes
    if (!p) return RRQ_ERR_NULL;
    if (token < 0 || head < 0 || token > (int64_t(1) << 32) || head > (int64_t(1) << 32))
        return RRQ_ERR_SHAPE;
    if (!aligned(p, 16) || token % per != 0 || head % per != 0) return RRQ_ERR_ALIGN;
    return RRQ_OK;
}

bool known_dtype(int32_t t) { return t == RRQ_F32 || t == RRQ_BF16; }

int status(hipError_t e) { return e == hipSuccess ? RRQ_OK : RRQ_ERR_HIP; }

int check_heads(const rrq_cache *c, const rrq_batch *b, int32_t n_heads)
{
    if (n_heads < 1 || n_heads > (1 << 16) || n_heads % c->n_kv_heads != 0) return RRQ_ERR_SHAPE;
    if (b->n_tokens * (n_heads / c->n_kv_heads) > (int64_t(1) << 26)) return RRQ_ERR_SHAPE;
    return RRQ_OK;
}

// Workspace of attention: each split's output (binary32) and its maximum and
// sum, per row.
size_t attend_bytes(const rrq_cache *c, const rrq_batch *b, int32_t n_heads, int splits)
{
    if (splits == 1) return 0;
    return (size_t)splits * (size_t)b->n_tokens * (size_t)n_heads * ((size_t)c->head_dim + 2) * 4;
}

}  // namespace

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
    int st = check_cache(cache, true);
    if (st == RRQ_OK) st = check_batch(batch, true);
    if (st == RRQ_OK) st = check_heads(cache, batch, n_heads);
    if (st != RRQ_OK) return st;
    if (!known_dtype(q_dtype) || !known_dtype(out_dtype)) return RRQ_ERR_DTYPE;
    if (!std::isfinite(scale) || (causal != 0 && causal != 1) || window < 0) return RRQ_ERR_SHAPE;
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return RRQ_OK;
    st = check_rows(Q, q_dtype, q_token_stride, q_head_stride);
    if (st != RRQ_OK) return st;
    if (!out) return RRQ_ERR_NULL;
    if (!aligned(out, 16)) return RRQ_ERR_ALIGN;
    Attend a = {};
    a.cache = *cache;
    a.batch = *batch;
    a.Q = Q;
    a.q_token = q_token_stride;
    a.q_head = q_head_stride;
    a.out = out;
    a.window = window;
    a.scale = scale;
    a.n_heads = n_heads;
    a.ratio = n_heads / cache->n_kv_heads;
    a.causal = causal;
    a.q_bf16 = q_dtype == RRQ_BF16;
    a.out_bf16 = out_dtype == RRQ_BF16;
    const AttendPlan plan = attend_plan(*cache, *batch, n_heads, window);
    a.n_splits = plan.splits;
    a.target = plan.target;
    a.min_tiles = plan.min_tiles;
    a.lds_rows = plan.lds_rows;
    const size_t need = attend_bytes(cache, batch, n_heads, a.n_splits);
    if (need > 0) {
        if (!workspace) return RRQ_ERR_NULL;
        if (!aligned(workspace, 16)) return RRQ_ERR_ALIGN;
        if (workspace_bytes < need) return RRQ_ERR_WORKSPACE;
        a.part_o = static_cast<float *>(workspace);
        a.part_ml = a.part_o + (size_t)a.n_splits * batch->n_tokens * n_heads * cache->head_dim;
    }
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
