// C ABI of librrq.so declared in include/rrq_draft.h: argument validation,
// workspace sizes and HIP error mapping. Every entry point validates its
// arguments before enqueueing anything and never throws.

#include "rrq_draft.h"

#include <cmath>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "rrq_draft_launch.h"
#include "rrq_serve_check.h"

using namespace rrq_detail;

namespace {

uintptr_t size_of(int32_t dtype) { return dtype == RRQ_F32 ? 4 : 2; }

// Stride between rows of `width` elements.
bool row_stride_fits(int64_t stride, int64_t width)
{
    return stride >= width && stride <= (int64_t(1) << 36);
}

}  // namespace

extern "C" int rrq_block_norm(const rrq_norm *norm, const void *residual, int32_t residual_dtype,
                              int64_t residual_stride, const void *y, int32_t y_dtype,
                              int64_t y_stride, const void *gate, int64_t gate_stride,
                              int64_t n_rows, int64_t hidden, void *out, int32_t out_dtype,
                              void *h, hipStream_t stream)
{
    if (!norm) return RRQ_ERR_NULL;
    if ((norm->kind != RRQ_NORM_RMS && norm->kind != RRQ_NORM_LAYER) ||
        norm->post < RRQ_NORM_NONE || norm->post > RRQ_NORM_LAYER)
        return RRQ_ERR_FORMAT;
    if (n_rows < 0 || n_rows > (int64_t(1) << 26) || hidden < 1 || hidden > kNormHidden)
        return RRQ_ERR_SHAPE;
    if (!std::isfinite(norm->eps) || norm->eps < 0 || !std::isfinite(norm->scale))
        return RRQ_ERR_SHAPE;
    if (!known_dtype(residual_dtype) || !known_dtype(out_dtype) || !known_dtype(y_dtype))
        return RRQ_ERR_DTYPE;
    if (!y && (gate || norm->post != RRQ_NORM_NONE)) return RRQ_ERR_SHAPE;
    if (n_rows > 1) {
        if (!row_stride_fits(residual_stride, hidden)) return RRQ_ERR_SHAPE;
        if (y && !row_stride_fits(y_stride, hidden)) return RRQ_ERR_SHAPE;
        if (gate && gate_stride != 0 && !row_stride_fits(gate_stride, hidden))
            return RRQ_ERR_SHAPE;
    }
    if (n_rows == 0) return RRQ_OK;
    if (!residual || !out || (y && !h)) return RRQ_ERR_NULL;
    if (!aligned(residual, size_of(residual_dtype)) || !aligned(h, size_of(residual_dtype)) ||
        !aligned(y, size_of(y_dtype)) || !aligned(gate, size_of(y_dtype)) ||
        !aligned(out, size_of(out_dtype)) || !aligned(norm->weight, 4) ||
        !aligned(norm->bias, 4) || !aligned(norm->post_weight, 4))
        return RRQ_ERR_ALIGN;
    BlockNorm a = {};
    a.norm = *norm;
    a.residual = residual;
    a.y = y;
    a.gate = gate;
    a.out = out;
    a.h = h;
    a.r_stride = residual_stride;
    a.y_stride = y_stride;
    a.gate_stride = gate_stride;
    a.n_rows = n_rows;
    a.hidden = (int32_t)hidden;
    a.out_bf16 = out_dtype == RRQ_BF16;
    return status(launch_block_norm(a, residual_dtype == RRQ_BF16, y_dtype == RRQ_BF16, stream));
}

extern "C" int rrq_cache_append(const rrq_cache *cache, const rrq_batch *batch,
                                const rrq_rotary *rotary, const int32_t *positions, const void *Q,
                                const void *K, const void *V, int32_t dtype,
                                int64_t q_token_stride, int64_t q_head_stride,
                                int64_t k_token_stride, int64_t k_head_stride,
                                int64_t v_token_stride, int64_t v_head_stride, int32_t n_heads,
                                void *Q_out, hipStream_t stream)
{
    int st = check_cache(cache, true);
    if (st == RRQ_OK) st = check_batch(batch, true);
    if (st != RRQ_OK) return st;
    if (!rotary) return RRQ_ERR_NULL;
    if (rotary->layout != RRQ_ROTARY_HALF && rotary->layout != RRQ_ROTARY_INTERLEAVED)
        return RRQ_ERR_FORMAT;
    if (rotary->rot_dim < 8 || rotary->rot_dim > cache->head_dim || rotary->rot_dim % 8 != 0 ||
        !std::isfinite(rotary->amplitude) || n_heads < 1 || n_heads > (1 << 16))
        return RRQ_ERR_SHAPE;
    if (!known_dtype(dtype)) return RRQ_ERR_DTYPE;
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return RRQ_OK;
    if (!rotary->frequencies) return RRQ_ERR_NULL;
    if (!aligned(rotary->frequencies, 8) || !aligned(positions, 4)) return RRQ_ERR_ALIGN;
    st = check_rows(Q, dtype, q_token_stride, q_head_stride);
    if (st == RRQ_OK) st = check_rows(K, dtype, k_token_stride, k_head_stride);
    if (st == RRQ_OK) st = check_rows(V, dtype, v_token_stride, v_head_stride);
    if (st != RRQ_OK) return st;
    if (!Q_out) return RRQ_ERR_NULL;
    if (!aligned(Q_out, 16)) return RRQ_ERR_ALIGN;
    CacheAppend a = {};
    a.cache = *cache;
    a.batch = *batch;
    a.K = K;
    a.V = V;
    a.Q = Q;
    a.Q_out = Q_out;
    a.frequencies = rotary->frequencies;
    a.positions = positions;
    a.amplitude = rotary->amplitude;
    a.k_token = k_token_stride;
    a.k_head = k_head_stride;
    a.v_token = v_token_stride;
    a.v_head = v_head_stride;
    a.q_token = q_token_stride;
    a.q_head = q_head_stride;
    a.n_heads = n_heads;
    a.rot = rotary->rot_dim;
    a.interleaved = rotary->layout == RRQ_ROTARY_INTERLEAVED;
    return status(launch_cache_append(a, dtype == RRQ_BF16, stream));
}

extern "C" int rrq_tree_attention(const rrq_cache *cache, const rrq_batch *batch, const void *Q,
                                  int32_t q_dtype, int64_t q_token_stride, int64_t q_head_stride,
                                  int32_t n_heads, float scale, const uint64_t *seen,
                                  int64_t seen_words, const int32_t *positions, int64_t window,
                                  void *out, int32_t out_dtype, void *workspace,
                                  size_t workspace_bytes, hipStream_t stream)
{
    Attend a = {};
    AttendPlan plan = {};
    const AttendCall call = {Q, out, workspace, q_token_stride, q_head_stride, window,
                             workspace_bytes, scale, q_dtype, out_dtype, n_heads, 0};
    const int st = prepare_attend(cache, batch, call, a, plan, true);
    if (st != RRQ_OK) return st;
    if (seen_words < 1 || seen_words > (int64_t(1) << 20)) return RRQ_ERR_SHAPE;
    if (plan.splits == 0) return RRQ_OK;
    if (!seen) return RRQ_ERR_NULL;
    if (!aligned(seen, 8) || !aligned(positions, 4)) return RRQ_ERR_ALIGN;
    a.seen = seen;
    a.seen_words = (int32_t)seen_words;
    a.positions = positions;
    return status(launch_attend(a, plan, stream));
}

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int check_verify(int64_t n_rows, int64_t vocab, int64_t n_seqs, int64_t draft_rows)
{
    if (n_rows < 0 || n_rows > (int64_t(1) << 23) || vocab < 1 || vocab > (int64_t(1) << 30) ||
        n_seqs < 0 || n_seqs > (int64_t(1) << 20) || draft_rows < 0)
        return RRQ_ERR_SHAPE;
    // workgroups of the launches
    if (draft_rows > (int64_t(1) << 24) ||
        (n_rows + draft_rows + n_seqs) * ceil_div(vocab, kVerifyDrawBlock) >= (int64_t(1) << 24))
        return RRQ_ERR_SHAPE;
    return RRQ_OK;
}

size_t sums_bytes(int64_t n_rows, int64_t vocab, int64_t draft_rows)
{
    return (size_t)(n_rows + draft_rows) * (size_t)ceil_div(vocab, verify_segment(n_rows + draft_rows, vocab)) *
           sizeof(VerifySum);
}

size_t verify_bytes(int64_t n_rows, int64_t vocab, int64_t n_seqs, int64_t draft_rows)
{
    return sums_bytes(n_rows, vocab, draft_rows) + (size_t)n_seqs * sizeof(VerifyChoice) +
           (size_t)n_seqs * (size_t)ceil_div(vocab, kVerifyDrawBlock) * sizeof(VerifyBlock);
}

bool temperature_fits(double t) { return t >= 0x1p-64 && t <= 0x1p64; }

}  // namespace

extern "C" int rrq_verify_drafts_workspace(int64_t n_rows, int64_t vocab, int64_t n_seqs,
                                           int64_t draft_rows, size_t *workspace_bytes)
{
    if (!workspace_bytes) return RRQ_ERR_NULL;
    const int st = check_verify(n_rows, vocab, n_seqs, draft_rows);
    if (st != RRQ_OK) return st;
    *workspace_bytes = n_seqs == 0 ? 0 : verify_bytes(n_rows, vocab, n_seqs, draft_rows);
    return RRQ_OK;
}

extern "C" int rrq_verify_drafts(const void *logits, int32_t dtype, int64_t n_rows, int64_t vocab,
                                 int64_t row_stride, const int64_t *tokens,
                                 const int32_t *offsets, int64_t n_seqs, const float *uniforms,
                                 const int32_t *parents, const void *draft,
                                 int64_t draft_seq_stride, int64_t draft_row_stride,
                                 double temperature, double draft_temperature, int32_t max_accept,
                                 int32_t *counts, int64_t *following, int32_t *paths,
                                 void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (max_accept < 0 || max_accept > (1 << 20)) return RRQ_ERR_SHAPE;
    if (max_accept == 0) draft = nullptr;
    // (n_seqs is checked below; the product stays in range before that)
    const int64_t draft_rows =
        draft && n_seqs >= 0 && n_seqs <= (int64_t(1) << 20) ? n_seqs * max_accept : 0;
    const int st = check_verify(n_rows, vocab, n_seqs, draft_rows);
    if (st != RRQ_OK) return st;
    if (n_rows > 1 && (row_stride < vocab || row_stride > (int64_t(1) << 36)))
        return RRQ_ERR_SHAPE;
    if (!known_dtype(dtype)) return RRQ_ERR_DTYPE;
    if (temperature != 0.0 && !temperature_fits(temperature)) return RRQ_ERR_SHAPE;
    if (draft && (parents || (temperature != 0.0 && !temperature_fits(draft_temperature))))
        return RRQ_ERR_SHAPE;
    if (draft && (draft_seq_stride < 0 || draft_row_stride < 0 ||
                  draft_seq_stride > (int64_t(1) << 40) || draft_row_stride > (int64_t(1) << 36)))
        return RRQ_ERR_SHAPE;
    if (n_seqs == 0) return RRQ_OK;
    if (!offsets || !counts || !following || !paths) return RRQ_ERR_NULL;
    if (n_rows > 0 && (!logits || !tokens || !uniforms)) return RRQ_ERR_NULL;
    if (!aligned(logits, size_of(dtype)) || !aligned(draft, size_of(dtype)) ||
        !aligned(tokens, 8) || !aligned(offsets, 4) || !aligned(uniforms, 4) ||
        !aligned(parents, 4) || !aligned(counts, 4) || !aligned(following, 8) ||
        !aligned(paths, 4))
        return RRQ_ERR_ALIGN;
    if (!workspace) return RRQ_ERR_NULL;
    if (!aligned(workspace, 16)) return RRQ_ERR_ALIGN;
    if (workspace_bytes < verify_bytes(n_rows, vocab, n_seqs, draft_rows))
        return RRQ_ERR_WORKSPACE;
    Verify a = {};
    a.logits = logits;
    a.draft = temperature == 0.0 ? nullptr : draft;
    a.tokens = tokens;
    a.offsets = offsets;
    a.parents = parents;
    a.uniforms = uniforms;
    a.counts = counts;
    a.paths = paths;
    a.following = following;
    char *at = static_cast<char *>(workspace);
    a.sums = reinterpret_cast<VerifySum *>(at);
    at += sums_bytes(n_rows, vocab, draft_rows);
    a.choices = reinterpret_cast<VerifyChoice *>(at);
    a.blocks = reinterpret_cast<VerifyBlock *>(at + (size_t)n_seqs * sizeof(VerifyChoice));
    a.n_rows = n_rows;
    a.n_seqs = n_seqs;
    a.vocab = vocab;
    a.row_stride = row_stride;
    a.draft_seq_stride = draft_seq_stride;
    a.draft_row_stride = draft_row_stride;
    a.segment = verify_segment(n_rows + draft_rows, vocab);
    a.inv_temperature = temperature == 0.0 ? 0.0 : 1.0 / temperature;
    a.inv_draft_temperature = a.draft ? 1.0 / draft_temperature : 1.0;
    a.max_accept = max_accept;
    a.segments = (int32_t)ceil_div(vocab, a.segment);
    a.draw_segments = (int32_t)ceil_div(vocab, kVerifyDrawBlock);
    a.bf16 = dtype == RRQ_BF16;
    return status(launch_verify(a, stream));
}
