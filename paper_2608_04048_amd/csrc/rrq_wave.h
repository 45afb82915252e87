// Sums and maxima over the lanes of a wave: neighbours within rows of 16 lanes by data
// parallel operands, rows by the swaps of lane 16 and lane 32. Every lane has the
// result. A step is two or three instructions where a shuffle through LDS waits some 100
// cycles.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rrq_detail {
namespace {

constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E;             // within four lanes
constexpr int kDppHalfMirror = 0x141, kDppMirror = 0x140;   // within eight, sixteen
constexpr int kDppShift = 0x110;                            // by + n lanes of a row
constexpr int kDppLast15 = 0x142, kDppLast31 = 0x143;       // a row's last lane to the next

template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint32_t dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, true);
}
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ float dpp(float x)
{
    return __uint_as_float(dpp<CTRL, ROWS>(__float_as_uint(x)));
}
__device__ __forceinline__ double of_words(uint32_t lo, uint32_t hi)
{
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ double dpp(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return of_words(dpp<CTRL, ROWS>((uint32_t)b), dpp<CTRL, ROWS>((uint32_t)(b >> 32)));
}

// The values of a lane and of the lane 16 (32) away, in the same order for both.
template <int LANES>
__device__ __forceinline__ void both(uint32_t x, uint32_t &a, uint32_t &b)
{
    const auto r = LANES == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false)
                               : __builtin_amdgcn_permlane32_swap(x, x, false, false);
    a = r[0];
    b = r[1];
}
template <int LANES>
__device__ __forceinline__ void both(float x, float &a, float &b)
{
    uint32_t p, q;
    both<LANES>(__float_as_uint(x), p, q);
    a = __uint_as_float(p);
    b = __uint_as_float(q);
}
template <int LANES>
__device__ __forceinline__ void both(double x, double &a, double &b)
{
    const uint64_t w = __builtin_bit_cast(uint64_t, x);
    uint32_t pl, ql, ph, qh;
    both<LANES>((uint32_t)w, pl, ql);
    both<LANES>((uint32_t)(w >> 32), ph, qh);
    a = of_words(pl, ph);
    b = of_words(ql, qh);
}

// Over 16 lanes (a row), and over all.
template <typename T>
__device__ __forceinline__ T row_total(T x)
{
    x += dpp<kDppXor1>(x);
    x += dpp<kDppXor2>(x);
    x += dpp<kDppHalfMirror>(x);
    return x + dpp<kDppMirror>(x);
}
template <typename T>
__device__ __forceinline__ T wave_sum(T x)
{
    T a, b;
    both<16>(row_total(x), a, b);
    both<32>(a + b, a, b);
    return a + b;
}
__device__ __forceinline__ float row_max(float x)
{
    x = fmaxf(x, dpp<kDppXor1>(x));
    x = fmaxf(x, dpp<kDppXor2>(x));
    x = fmaxf(x, dpp<kDppHalfMirror>(x));
    return fmaxf(x, dpp<kDppMirror>(x));
}
__device__ __forceinline__ float wave_max(float x)
{
    float a, b;
    both<16>(row_max(x), a, b);
    both<32>(fmaxf(a, b), a, b);
    return fmaxf(a, b);
}

// Sum of the lanes up to this one.
__device__ __forceinline__ double wave_scan(double x)
{
    x += dpp<kDppShift + 1>(x);
    x += dpp<kDppShift + 2>(x);
    x += dpp<kDppShift + 4>(x);
    x += dpp<kDppShift + 8>(x);
    x += dpp<kDppLast15, 0xA>(x);       // rows 1 and 3 get the row before
    return x + dpp<kDppLast31, 0xC>(x); // rows 2 and 3 the half before
}

}  // namespace
}  // namespace rrq_detail
