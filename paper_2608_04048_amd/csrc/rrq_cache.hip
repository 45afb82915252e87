// The 8-bit key/value cache: quantising tokens as they are written, and
// reading them back (rrq_serve.h: rrq_cache_write, rrq_cache_read).
//
// One workgroup owns one page of one kv head and either its keys or its
// values, so every code and the scale of the block have one writer and a
// page that already holds tokens can be rescaled in place without atomics.
//
// Memory bounds long calls: per value 4 or 2 bytes in and 1 out, or the
// reverse. 8713 bfloat16 tokens of seven prompts (8 kv heads of 128): write
// 13.4 us (4.0 TB/s), read 12.2 us (4.4 TB/s); 130000 tokens read in 177 us (4.5
// TB/s; a large device copy makes 4.67). The last tokens of 24 sequences: 5.2
// and 4.5 us, a launch and one chain of dependent loads.
#include "rrq_cache_device.h"

namespace rrq_detail {
namespace {

template <int D, int CODE, bool BF16>
__global__ __launch_bounds__(1024) void cache_write_kernel(CacheWrite a)
{
    __shared__ float lds[16];
    const int H = a.cache.n_kv_heads, P = a.cache.page_size;
    const int head = blockIdx.y >> 1;
    PageSlot p;
    if (!find_page(a.cache, a.batch, blockIdx.x, p)) return;
    if (p.page < 0 || p.page >= a.cache.n_pages) return;
    const int64_t block = p.page * H + head;
    const int t = threadIdx.x;
    if (!(blockIdx.y & 1)) {
        uint32_t *codes = reinterpret_cast<uint32_t *>(a.cache.k_codes + block * P * D);
        float *scale = a.cache.k_scales + block;
        constexpr int TPT = D / 4;                       // threads a token
        const int tokens = blockDim.x / TPT;             // tokens a pass
        const int c = t % TPT, slot0 = t / TPT;
        f32x4 x[kTok];
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < kTok; ++i) {
            const int slot = slot0 + i * tokens;
            x[i] = load4<BF16>(a.K, (p.row0 + p.near(slot)) * a.k_token + head * a.k_head + 4 * c);
        }
        const float stored = p.lo > 0 ? *scale : 0.0f;
#pragma unroll
        for (int i = 0; i < kTok; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fabsf(x[i][e]));
        amax = block_max(amax, lds);
        float inv, ratio;
        const float s = block_scale<CODE>(amax, stored, inv, ratio);
#pragma unroll
        for (int i = 0; i < kTok; ++i) {
            const int slot = slot0 + i * tokens;
            if (slot >= p.lo && slot < p.hi)
                codes[slot * TPT + c] = encode4<CODE>(x[i] * inv);
            else if (slot < p.lo && ratio >= 0.0f)
                codes[slot * TPT + c] =
                    encode4<CODE>(codes_f32<CODE>(codes[slot * TPT + c]) * ratio);
        }
        if (t == 0) *scale = s;     // after the barrier of block_max: every thread has read it
    } else {
        write_values<D, CODE, BF16>(a, p, head, lds);
    }
}

template <int D, int CODE, bool BF16>
__global__ __launch_bounds__(1024) void cache_read_kernel(CacheRead a)
{
    const int H = a.cache.n_kv_heads, P = a.cache.page_size;
    const int head = blockIdx.y >> 1;
    PageSlot p;
    if (!find_page(a.cache, a.batch, blockIdx.x, p)) return;
    const bool there = p.page >= 0 && p.page < a.cache.n_pages;
    const int64_t block = (there ? p.page : 0) * H + head;
    const int t = threadIdx.x;
    if (!(blockIdx.y & 1)) {
        const uint32_t *codes = reinterpret_cast<const uint32_t *>(a.cache.k_codes + block * P * D);
        const float s = there ? a.cache.k_scales[block] : 0.0f;
        constexpr int TPT = D / 4;
        const int tokens = blockDim.x / TPT;
        const int c = t % TPT, slot0 = t / TPT;
#pragma unroll
        for (int i = 0; i < kTok; ++i) {
            const int slot = slot0 + i * tokens;
            if (slot < p.lo || slot >= p.hi) continue;
            const f32x4 y = there ? codes_f32<CODE>(codes[slot * TPT + c]) * s : f32x4{0, 0, 0, 0};
            const int64_t at = ((p.row0 + slot - p.lo) * H + head) * D + 4 * c;
            if (BF16)
                *reinterpret_cast<u32x2v *>(static_cast<uint16_t *>(a.K) + at) =
                    u32x2v{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])};
            else
                *reinterpret_cast<f32x4 *>(static_cast<float *>(a.K) + at) = y;
        }
    } else {
        const uint8_t *codes = a.cache.v_codes + block * P * D;
        const float s = there ? a.cache.v_scales[block] : 0.0f;
        constexpr int TPR = D / 2;
        const int c = t % TPR, slot0 = (t / TPR) * kRun;
        if (slot0 >= p.hi || slot0 + kRun <= p.lo) return;
        u32x4v w[2] = {};
        if (there) {
            w[0] = *reinterpret_cast<const u32x4v *>(codes + 2 * c * P + slot0);
            w[1] = *reinterpret_cast<const u32x4v *>(codes + (2 * c + 1) * P + slot0);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 y0 = codes_f32<CODE>(w[0][q]) * s, y1 = codes_f32<CODE>(w[1][q]) * s;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int slot = slot0 + 4 * q + i;
                if (slot < p.lo || slot >= p.hi) continue;
                const int64_t at = ((p.row0 + slot - p.lo) * H + head) * D + 2 * c;
                const float v0 = there ? y0[i] : 0.0f, v1 = there ? y1[i] : 0.0f;
                if (BF16)
                    *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(a.V) + at) =
                        bf16_pair(v0, v1);
                else
                    *reinterpret_cast<f32x2 *>(static_cast<float *>(a.V) + at) = f32x2{v0, v1};
            }
        }
    }
}

template <int D, int CODE>
hipError_t write_dim(const CacheWrite &a, bool bf16, dim3 grid, dim3 block, hipStream_t stream)
{
    if (bf16)
        cache_write_kernel<D, CODE, true><<<grid, block, 0, stream>>>(a);
    else
        cache_write_kernel<D, CODE, false><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

template <int D, int CODE>
hipError_t read_dim(const CacheRead &a, bool bf16, dim3 grid, dim3 block, hipStream_t stream)
{
    if (bf16)
        cache_read_kernel<D, CODE, true><<<grid, block, 0, stream>>>(a);
    else
        cache_read_kernel<D, CODE, false><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

#define RRQ_CACHE_DISPATCH(fn)                                                               \
    const dim3 block(block_threads(a.cache));                                                \
    const dim3 grid((unsigned)cache_page_slots(a.batch, a.cache.page_size),                  \
                    2 * a.cache.n_kv_heads);                                                 \
    if (a.cache.code_type == RRQ_CODE_INT8) {                                                \
        if (a.cache.head_dim == 64) return fn<64, RRQ_CODE_INT8>(a, bf16, grid, block, stream);   \
        if (a.cache.head_dim == 128) return fn<128, RRQ_CODE_INT8>(a, bf16, grid, block, stream); \
        return fn<256, RRQ_CODE_INT8>(a, bf16, grid, block, stream);                         \
    }                                                                                        \
    if (a.cache.head_dim == 64) return fn<64, RRQ_CODE_FP8>(a, bf16, grid, block, stream);   \
    if (a.cache.head_dim == 128) return fn<128, RRQ_CODE_FP8>(a, bf16, grid, block, stream); \
    return fn<256, RRQ_CODE_FP8>(a, bf16, grid, block, stream);

hipError_t launch_cache_write(const CacheWrite &a, bool bf16, hipStream_t stream)
{
    RRQ_CACHE_DISPATCH(write_dim)
}

hipError_t launch_cache_read(const CacheRead &a, bool bf16, hipStream_t stream)
{
    RRQ_CACHE_DISPATCH(read_dim)
}

}  // namespace rrq_detail
