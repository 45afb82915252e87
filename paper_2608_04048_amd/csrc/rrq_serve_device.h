// Device helpers shared by the cache and attention kernels: the batch's
// sequences, and 8-bit codes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rrq_serve.h"

namespace rrq_detail {
namespace {

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Row numbers fit in 32 bits (n_tokens <= 2^26, times the query heads of a kv
// head as well).
__device__ __forceinline__ int clamp_row(const rrq_batch &b, int i)
{
    const int o = b.offsets[i];
    return o < 0 ? 0 : (o > b.n_tokens ? (int)b.n_tokens : o);
}

// The sequence that owns work slot u, where sequence b's slots start at
// f(b) = (offsets[b] * mul >> shift) + extra * b. Every lane of the wave calls
// it; each step compares 64 sequences at once, so up to 64 sequences cost one
// load.
__device__ __forceinline__ int find_sequence(const rrq_batch &b, int u, int mul, int shift,
                                             int extra)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = (int)b.n_seqs;
    while (n > 1) {
        const int step = (n + 63) >> 6;
        const int i = lane * step;
        const bool below =
            i < n && ((clamp_row(b, lo + i) * mul) >> shift) + extra * (lo + i) <= u;
        const int c = __popcll(__ballot(below));
        const int at = c > 0 ? (c - 1) * step : 0;
        lo += at;
        n = n - at < step ? n - at : step;
    }
    return lo;
}

// Eight codes (two words) as binary16, exactly. int8: with the sign bit
// turned over a code is u = c + 128, the bits 0x6400 | u are 1024 + u, and
// subtracting 1152 leaves c.
template <int CODE>
__device__ __forceinline__ void codes_f16(uint32_t w, f16x2 &a, f16x2 &b)
{
    if (CODE == RRQ_CODE_INT8) {
        const uint32_t x = w ^ 0x80808080u;
        const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
        const uint32_t p = __builtin_amdgcn_perm(x, 0x64646464u, 0x00050004u);
        const uint32_t q = __builtin_amdgcn_perm(x, 0x64646464u, 0x00070006u);
        a = __builtin_bit_cast(f16x2, p) - bias;
        b = __builtin_bit_cast(f16x2, q) - bias;
    } else {
        a = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
        b = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
    }
}

template <int CODE>
__device__ __forceinline__ f16x8 codes_f16(uint32_t w0, uint32_t w1)
{
    f16x2 a, b, c, d;
    codes_f16<CODE>(w0, a, b);
    codes_f16<CODE>(w1, c, d);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Four codes as binary32.
template <int CODE>
__device__ __forceinline__ f32x4 codes_f32(uint32_t w)
{
    if (CODE == RRQ_CODE_INT8)
        return f32x4{(float)(int8_t)(w & 255), (float)(int8_t)((w >> 8) & 255),
                     (float)(int8_t)((w >> 16) & 255), (float)(int8_t)(w >> 24)};
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

// Four scaled values to codes: nearest-even, clamped.
template <int CODE>
__device__ __forceinline__ uint32_t encode4(f32x4 y)
{
    if (CODE == RRQ_CODE_INT8) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float r = fminf(fmaxf(__builtin_rintf(y[i]), -127.0f), 127.0f);
            w |= ((uint32_t)(int32_t)r & 255u) << (8 * i);
        }
        return w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fminf(fmaxf(y[i], -448.0f), 448.0f);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    return (uint32_t)w;
}

// bfloat16 bits, nearest-even (a NaN stays one).
__device__ __forceinline__ uint32_t bf16_bits(float x)
{
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    return bf16_bits(lo) | (bf16_bits(hi) << 16);
}

}  // namespace
}  // namespace rrq_detail
