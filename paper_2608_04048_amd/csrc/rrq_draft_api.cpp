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
