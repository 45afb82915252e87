// Argument checks, and what calls of attention prepare, shared by the C ABI layers of rrq_serve.h and rrq_draft.h.
#pragma once

#include <cmath>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "rrq_serve_launch.h"

namespace rrq_detail {

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// The cache's sizes, and (buffers) its pointers.
inline int check_cache(const rrq_cache *c, bool buffers)
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

inline int check_batch(const rrq_batch *b, bool buffers)
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
inline int check_rows(const void *p, int32_t dtype, int64_t token, int64_t head)
{
    const int64_t per = dtype == RRQ_F32 ? 4 : 8;       // elements in 16 bytes
    if (!p) return RRQ_ERR_NULL;
    if (token < 0 || head < 0 || token > (int64_t(1) << 32) || head > (int64_t(1) << 32))
        return RRQ_ERR_SHAPE;
    if (!aligned(p, 16) || token % per != 0 || head % per != 0) return RRQ_ERR_ALIGN;
    return RRQ_OK;
}

inline bool known_dtype(int32_t t) { return t == RRQ_F32 || t == RRQ_BF16; }

inline int status(hipError_t e) { return e == hipSuccess ? RRQ_OK : RRQ_ERR_HIP; }

inline int check_heads(const rrq_cache *c, const rrq_batch *b, int32_t n_heads)
{
    if (n_heads < 1 || n_heads > (1 << 16) || n_heads % c->n_kv_heads != 0) return RRQ_ERR_SHAPE;
    if (b->n_tokens * (n_heads / c->n_kv_heads) > (int64_t(1) << 26)) return RRQ_ERR_SHAPE;
    return RRQ_OK;
}

// Workspace of attention: each split's output (binary32) and its maximum and
// sum, per row.
inline size_t attend_bytes(const rrq_cache *c, const rrq_batch *b, int32_t n_heads, int splits)
{
    if (splits == 1) return 0;
    return (size_t)splits * (size_t)b->n_tokens * (size_t)n_heads * ((size_t)c->head_dim + 2) * 4;
}

// A call's arguments besides its cache and batch.
struct AttendCall {
    const void *Q;
    void *out, *workspace;
    int64_t q_token_stride, q_head_stride, window;
    size_t workspace_bytes;
    float scale;
    int32_t q_dtype, out_dtype, n_heads, causal;
};

// Checks a call's arguments and fills in what the launch takes. plan.splits stays 0
// for a call that has nothing to do.
inline int prepare_attend(const rrq_cache *cache, const rrq_batch *batch, const AttendCall &c,
                          Attend &a, AttendPlan &plan, bool tree = false)
{
    int st = check_cache(cache, true);
    if (st == RRQ_OK) st = check_batch(batch, true);
    if (st == RRQ_OK) st = check_heads(cache, batch, c.n_heads);
    if (st != RRQ_OK) return st;
    if (!known_dtype(c.q_dtype) || !known_dtype(c.out_dtype)) return RRQ_ERR_DTYPE;
    if (!std::isfinite(c.scale) || (c.causal != 0 && c.causal != 1) || c.window < 0)
        return RRQ_ERR_SHAPE;
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return RRQ_OK;
    st = check_rows(c.Q, c.q_dtype, c.q_token_stride, c.q_head_stride);
    if (st != RRQ_OK) return st;
    if (!c.out) return RRQ_ERR_NULL;
    if (!aligned(c.out, 16)) return RRQ_ERR_ALIGN;
    a.cache = *cache;
    a.batch = *batch;
    a.Q = c.Q;
    a.q_token = c.q_token_stride;
    a.q_head = c.q_head_stride;
    a.out = c.out;
    // (lengths and positions have 32 bits: a longer window hides no key, and its sums
    // with them would pass 64)
    const int64_t window = c.window < (int64_t(1) << 33) ? c.window : int64_t(1) << 33;
    a.window = window;
    a.scale = c.scale;
    a.n_heads = c.n_heads;
    a.ratio = c.n_heads / cache->n_kv_heads;
    a.causal = c.causal;
    a.q_bf16 = c.q_dtype == RRQ_BF16;
    a.out_bf16 = c.out_dtype == RRQ_BF16;
    AttendPlan p = attend_plan(*cache, *batch, c.n_heads, window, tree);
    if (tree) {
        // the workspace is that of the other calls on this batch
        const int most = attend_plan(*cache, *batch, c.n_heads, 0).splits;
        if (p.splits > most) p.splits = most;
    }
    a.n_splits = p.splits;
    a.target = p.target;
    a.min_tiles = p.min_tiles;
    a.lds_rows = p.lds_rows;
    const size_t need = attend_bytes(cache, batch, c.n_heads, a.n_splits);
    if (need > 0) {
        if (!c.workspace) return RRQ_ERR_NULL;
        if (!aligned(c.workspace, 16)) return RRQ_ERR_ALIGN;
        if (c.workspace_bytes < need) return RRQ_ERR_WORKSPACE;
        a.part_o = static_cast<float *>(c.workspace);
        a.part_ml =
            a.part_o + (size_t)a.n_splits * batch->n_tokens * c.n_heads * cache->head_dim;
    }
    plan = p;
    return RRQ_OK;
}

}  // namespace rrq_detail
