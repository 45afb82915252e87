// From one block of a decoder to the next (rrq_draft.h: rrq_block_norm):
// post norm, gate, residual scale and addition, and the next block's norm, with
// one read of every operand and one write of the results.
//
// One workgroup takes a row and holds it, so that the mean and then the squares of the
// differences to it are summed from the exact elements: in registers up to 32768
// columns; of eight pieces a thread, 185 to 527 of the compiler's registers are in
// scratch memory.
//
// Memory bounds many rows: 16384 of 4096 (bfloat16 residual and result, binary32
// output of the block) 117 us, 5.7 TB/s; with a gate of rows and a post norm, 16384 of
// 5120, 234 us, 5.0. Longer rows, as the first without the gate (with a post norm): 4096
// of 12288 106 us (116), 4.7 TB/s; 2048 of 20000 98 (108), 4.2; 1024 of 32768 77 (84), 4.4;
// past that scratch memory sets the time: 1024 of 40000 173 (198), 2.4, of 65536 257 (295),
// 2.6. Few rows are latency: one of 4096 2.8 us, 300 of 5120 with gate,
// post norm and layer norm (three sums) 8.1 us where their bytes need 4.6.
#include <hip/hip_runtime.h>

#include "rrq_draft_launch.h"
#include "rrq_serve_device.h"
#include "rrq_wave.h"

namespace rrq_detail {
namespace {

constexpr int kPiece = 8;       // elements of a thread's contiguous piece

// Rows may start at any multiple of their type: 16-byte accesses without that
// alignment.
struct __attribute__((packed, aligned(2))) Wide {
    uint32_t w[4];
};

// n elements (kPiece, or fewer at a row's end: the others are 0) from x on.
template <bool BF16>
__device__ __forceinline__ void load_piece(const void *base, int64_t at, int n, float (&v)[kPiece])
{
    if (n >= kPiece) {
        if (BF16) {
            const Wide w = *reinterpret_cast<const Wide *>(static_cast<const uint16_t *>(base) + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[2 * e] = __uint_as_float(w.w[e] << 16);
                v[2 * e + 1] = __uint_as_float(w.w[e] & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const Wide w =
                    *reinterpret_cast<const Wide *>(static_cast<const float *>(base) + at + 4 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * i + e] = __uint_as_float(w.w[e]);
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        v[e] = 0.0f;
        if (e < n)
            v[e] = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(base)[at + e]
                                          << 16)
                        : static_cast<const float *>(base)[at + e];
    }
}

__device__ __forceinline__ void store_piece(void *base, bool bf16, int64_t at, int n,
                                            const float (&v)[kPiece])
{
    if (n >= kPiece) {
        if (bf16) {
            Wide w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w.w[e] = bf16_pair(v[2 * e], v[2 * e + 1]);
            *reinterpret_cast<Wide *>(static_cast<uint16_t *>(base) + at) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                Wide w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w.w[e] = __float_as_uint(v[4 * i + e]);
                *reinterpret_cast<Wide *>(static_cast<float *>(base) + at + 4 * i) = w;
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < kPiece; ++e)
        if (e < n) {
            if (bf16)
                static_cast<uint16_t *>(base)[at + e] = (uint16_t)bf16_bits(v[e]);
            else
                static_cast<float *>(base)[at + e] = v[e];
        }
}

// Sum over the workgroup. `lds` is this sum's own: no barrier guards it.
__device__ __forceinline__ float block_sum(float a, float *lds)
{
    a = wave_sum(a);
    const int waves = blockDim.x / 64;
    if (waves == 1) return a;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    a = lds[0];
    for (int w = 1; w < waves; ++w) a += lds[w];
    return a;
}

// Norms the row's elements v (0 past its end) in place: without the weights.
// n_of(c): elements of piece c that the row has.
template <int CH, typename N>
__device__ __forceinline__ void normalise(float (&v)[CH][kPiece], int kind, float inv_n, float eps,
                                          float *lds, N n_of)
{
    if (kind == RRQ_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < kPiece; ++e) s += v[c][e];
        const float mean = block_sum(s, lds) * inv_n;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < kPiece; ++e) v[c][e] = e < n_of(c) ? v[c][e] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < kPiece; ++e) s = __builtin_fmaf(v[c][e], v[c][e], s);
    const float f = 1.0f / sqrtf(block_sum(s, lds + 16) * inv_n + eps);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < kPiece; ++e) v[c][e] *= f;
}

// CH: pieces a thread holds.
template <int CH, bool R16, bool Y16>
__global__ __launch_bounds__(1024) void block_norm_kernel(BlockNorm a)
{
    __shared__ float lds[64];
    const int64_t row = a.row0 + blockIdx.x;
    const int N = a.hidden;
    const float inv_n = 1.0f / (float)N;
    auto first = [&](int c) { return kPiece * (int)(c * blockDim.x + threadIdx.x); };
    auto n_of = [&](int c) { return N - first(c); };    // (more than kPiece: a whole piece)

    // What a row of few pieces needs is on its way before the first sum; longer rows
    // would not have the registers.
    constexpr bool kAhead = CH <= 2;
    float h[CH][kPiece], y[CH][kPiece], g[CH][kPiece], w[CH][kPiece], p[CH][kPiece];
    const bool post = a.norm.post != RRQ_NORM_NONE;
    auto load_post = [&](int c) { load_piece<false>(a.norm.post_weight, first(c), n_of(c), p[c]); };
    auto load_gate = [&](int c) {
        load_piece<Y16>(a.gate, row * a.gate_stride + first(c), n_of(c), g[c]);
    };
    auto load_weight = [&](int c) { load_piece<false>(a.norm.weight, first(c), n_of(c), w[c]); };
    if (a.y) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            load_piece<Y16>(a.y, row * a.y_stride + first(c), n_of(c), y[c]);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
        load_piece<R16>(a.residual, row * a.r_stride + first(c), n_of(c), h[c]);
    if (kAhead) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (a.gate) load_gate(c);
            if (a.norm.post_weight) load_post(c);
            if (a.norm.weight) load_weight(c);
        }
    }
    if (a.y) {
        if (post) {
            normalise(y, a.norm.post, inv_n, a.norm.eps, lds, n_of);
            if (a.norm.post_weight) {
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    if (!kAhead) load_post(c);
#pragma unroll
                    for (int e = 0; e < kPiece; ++e) y[c][e] *= p[c][e];
                }
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (a.gate) {
                if (!kAhead) load_gate(c);
#pragma unroll
                for (int e = 0; e < kPiece; ++e) y[c][e] *= g[c][e];
            }
#pragma unroll
            for (int e = 0; e < kPiece; ++e) h[c][e] += y[c][e] * a.norm.scale;
            store_piece(a.h, R16, row * N + first(c), n_of(c), h[c]);
        }
    }
    normalise(h, a.norm.kind, inv_n, a.norm.eps, lds + 32, n_of);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (a.norm.weight) {
            if (!kAhead) load_weight(c);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) h[c][e] *= w[c][e];
        }
        if (a.norm.bias) {
            load_piece<false>(a.norm.bias, first(c), n_of(c), w[c]);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) h[c][e] += w[c][e];
        }
        store_piece(a.out, a.out_bf16, row * N + first(c), n_of(c), h[c]);
    }
}

template <int CH>
hipError_t norm_pieces(BlockNorm a, bool r_bf16, bool y_bf16, unsigned threads,
                       hipStream_t stream)
{
    // (a grid has 2^32 threads at most)
    constexpr int64_t kMost = 1 << 20;
    for (a.row0 = 0; a.row0 < a.n_rows; a.row0 += kMost) {
        const unsigned grid = (unsigned)(a.n_rows - a.row0 < kMost ? a.n_rows - a.row0 : kMost);
        if (r_bf16 && y_bf16)
            block_norm_kernel<CH, true, true><<<grid, threads, 0, stream>>>(a);
        else if (r_bf16)
            block_norm_kernel<CH, true, false><<<grid, threads, 0, stream>>>(a);
        else if (y_bf16)
            block_norm_kernel<CH, false, true><<<grid, threads, 0, stream>>>(a);
        else
            block_norm_kernel<CH, false, false><<<grid, threads, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_block_norm(const BlockNorm &a, bool r_bf16, bool y_bf16, hipStream_t stream)
{
    // One piece a thread as far as 1024 threads reach: 300 rows of 5120, gated with a
    // post norm, 8.1 us (8.5 with two), 16384 of them 234 (302).
    const int pieces = (a.hidden + kPiece - 1) / kPiece;
    const int ch = pieces <= 1024 ? 1 : (pieces <= 2048 ? 2 : (pieces <= 4096 ? 4 : 8));
    const unsigned threads = ((pieces + ch - 1) / ch + 63) / 64 * 64;
    switch (ch) {
    case 1: return norm_pieces<1>(a, r_bf16, y_bf16, threads, stream);
    case 2: return norm_pieces<2>(a, r_bf16, y_bf16, threads, stream);
    case 4: return norm_pieces<4>(a, r_bf16, y_bf16, threads, stream);
    default: return norm_pieces<8>(a, r_bf16, y_bf16, threads, stream);
    }
}

}  // namespace rrq_detail
