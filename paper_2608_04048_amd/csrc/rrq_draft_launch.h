// Internal launch interface between the C ABI layer of rrq_draft.h
// (rrq_draft_api.cpp) and its kernels. Arguments are already validated.
#pragma once

#include "rrq_draft.h"
#include "rrq_serve_launch.h"

namespace rrq_detail {

// Longest row of the norm: 1024 threads of 8 pieces of 8 elements hold it.
constexpr int64_t kNormHidden = 65536;

struct BlockNorm {
    rrq_norm norm;
    const void *residual, *y, *gate;
    void *out, *h;
    int64_t r_stride, y_stride, gate_stride, n_rows;
    int32_t hidden, out_bf16;
};
hipError_t launch_block_norm(const BlockNorm &a, bool r_bf16, bool y_bf16, hipStream_t stream);

}  // namespace rrq_detail
