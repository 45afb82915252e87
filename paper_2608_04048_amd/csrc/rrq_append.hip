// Queries and keys rotated to their positions, keys and values quantised into the
// cache (rrq_draft.h: rrq_cache_append): one launch for what stands between the
// fused projection and attention.
//
// The first workgroups own one page of one kv head and its keys or its values, as
// in rrq_cache_write; the others rotate the queries of a few tokens. A unit of
// work is 8 channels of a row that are rotated among themselves: 8 in a run, or
// two runs of 4 half a rotation apart; channels past the rotated ones are units
// that are copied.
//
// Angles are position times frequency in 64 bits, as positions of long contexts
// take binary32 past the turn itself: cosine and sine by reduction to pi / 4 and
// Taylor's series (error below 4e-16), 64-bit operations being as fast here as 32-bit
// ones. A workgroup computes a token's once: of the queries for all heads, of the
// keys for its own.
//
// Memory bounds long calls: 8192 tokens of 40 query and 8 kv heads of 128 in binary32, 419
// MB, 83 us (5.0 TB/s). The last tokens of 24 sequences 5.6 us and 16 trees of 20 to 40
// drafts 9.3: a launch, and offsets, page and rows one after another.
#include "rrq_append_rows.h"
#include "rrq_cache_device.h"
#include "rrq_draft_launch.h"

namespace rrq_detail {
namespace {

// Cosine and sine. The angle less a multiple of pi / 2, which is held in two
// parts; then the series up to z^16 and z^15.
__device__ __forceinline__ void turn(double angle, double &c, double &s)
{
    constexpr double kHi = 1.57079632679489655800, kLo = 6.12323399573676603587e-17;
    const double q = __builtin_rint(angle * 0.63661977236758134308);
    double z = __builtin_fma(-q, kHi, angle);
    z = __builtin_fma(-q, kLo, z);
    const int n = (int)(q - 4.0 * __builtin_floor(q * 0.25));
    const double w = z * z;
    double p = -1.0 / 1307674368000.0;
    p = __builtin_fma(p, w, 1.0 / 6227020800.0);
    p = __builtin_fma(p, w, -1.0 / 39916800.0);
    p = __builtin_fma(p, w, 1.0 / 362880.0);
    p = __builtin_fma(p, w, -1.0 / 5040.0);
    p = __builtin_fma(p, w, 1.0 / 120.0);
    p = __builtin_fma(p, w, -1.0 / 6.0);
    const double sz = __builtin_fma(p * w, z, z);
    double r = 1.0 / 20922789888000.0;
    r = __builtin_fma(r, w, -1.0 / 87178291200.0);
    r = __builtin_fma(r, w, 1.0 / 479001600.0);
    r = __builtin_fma(r, w, -1.0 / 3628800.0);
    r = __builtin_fma(r, w, 1.0 / 40320.0);
    r = __builtin_fma(r, w, -1.0 / 720.0);
    r = __builtin_fma(r, w, 1.0 / 24.0);
    r = __builtin_fma(r, w, -0.5);
    const double cz = __builtin_fma(r, w, 1.0);
    c = n & 1 ? sz : cz;
    s = n & 1 ? cz : sz;
    if (n == 1 || n == 2) c = -c;
    if (n >= 2) s = -s;
}

// Where unit u's channels stand: runs of 4 from `a` and `b` on.
struct Unit {
    int a, b;
    bool rotated;
};
__device__ __forceinline__ Unit unit_of(const CacheAppend &a, int u)
{
    Unit r;
    r.rotated = 8 * u < a.rot;
    const bool half = r.rotated && !a.interleaved;
    r.a = half ? 4 * u : 8 * u;
    r.b = r.a + (half ? a.rot / 2 : 4);
    return r;
}

// The unit's values turned by its four pairs' cosines and sines.
__device__ __forceinline__ void rotate(const CacheAppend &a, f32x4 &x, f32x4 &y, const f32x4 &c,
                                       const f32x4 &s)
{
    if (a.interleaved) {
        const f32x4 u = x, v = y;
        x = f32x4{u[0] * c[0] - u[1] * s[0], u[1] * c[0] + u[0] * s[0],
                  u[2] * c[1] - u[3] * s[1], u[3] * c[1] + u[2] * s[1]};
        y = f32x4{v[0] * c[2] - v[1] * s[2], v[1] * c[2] + v[0] * s[2],
                  v[2] * c[3] - v[3] * s[3], v[3] * c[3] + v[2] * s[3]};
    } else {
        const f32x4 u = x;
        x = u * c - y * s;
        y = y * c + u * s;
    }
}

__device__ __forceinline__ float turned(const CacheAppend &a, double angle, float &s)
{
    double c64, s64;
    turn(angle, c64, s64);
    s = (float)(s64 * a.amplitude);
    return (float)(c64 * a.amplitude);
}

// The keys of a page of one kv head: a thread holds one unit of four tokens.
constexpr int kKeyTok = 4;
template <int D, int CODE, bool BF16>
__device__ __forceinline__ void append_keys(const CacheAppend &a, const PageSlot &p, int position0,
                                            int head, float *lds)
{
    constexpr int TPT = D / 8;
    const int t = threadIdx.x, P = a.cache.page_size;
    const int tokens = blockDim.x / TPT;
    const int slot0 = t / TPT;
    const Unit u = unit_of(a, t % TPT);
    const int64_t block = p.page * a.cache.n_kv_heads + head;
    uint8_t *codes = a.cache.k_codes + block * P * D;
    float *scale = a.cache.k_scales + block;
    f32x4 x[kKeyTok], y[kKeyTok];
    double f[4];
    int pos[kKeyTok];
#pragma unroll
    for (int i = 0; i < kKeyTok; ++i) {
        const int64_t row = p.row0 + p.near(slot0 + i * tokens);
        const int64_t at = row * a.k_token + head * a.k_head;
        x[i] = load4<BF16>(a.K, at + u.a);
        y[i] = load4<BF16>(a.K, at + u.b);
        pos[i] = a.positions ? a.positions[row] : position0 + p.near(slot0 + i * tokens);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = u.rotated ? a.frequencies[4 * (t % TPT) + e] : 0.0;
    const float stored = p.lo > 0 ? *scale : 0.0f;
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < kKeyTok; ++i) {
        const int slot = slot0 + i * tokens;
        // (most passes of a single token's page hold nothing new)
        if (!__any(slot >= p.lo && slot < p.hi)) continue;
        if (u.rotated) {
            f32x4 c, s;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float se;
                c[e] = turned(a, (double)pos[i] * f[e], se);
                s[e] = se;
            }
            rotate(a, x[i], y[i], c, s);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fmaxf(fabsf(x[i][e]), fabsf(y[i][e])));
    }
    amax = block_max(amax, lds);
    float inv, ratio;
    const float s = block_scale<CODE>(amax, stored, inv, ratio);
#pragma unroll
    for (int i = 0; i < kKeyTok; ++i) {
        const int slot = slot0 + i * tokens;
        uint32_t *ca = reinterpret_cast<uint32_t *>(codes + slot * D + u.a);
        uint32_t *cb = reinterpret_cast<uint32_t *>(codes + slot * D + u.b);
        if (slot >= p.lo && slot < p.hi) {
            *ca = encode4<CODE>(x[i] * inv);
            *cb = encode4<CODE>(y[i] * inv);
        } else if (slot < p.lo && ratio >= 0.0f) {
            *ca = encode4<CODE>(codes_f32<CODE>(*ca) * ratio);
            *cb = encode4<CODE>(codes_f32<CODE>(*cb) * ratio);
        }
    }
    if (t == 0) *scale = s;     // after the barrier of block_max: every thread has read it
}

template <bool BF16>
__device__ __forceinline__ void store4(void *base, int64_t at, const f32x4 &x)
{
    if (BF16)
        *reinterpret_cast<u32x2v *>(static_cast<uint16_t *>(base) + at) =
            u32x2v{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    else
        *reinterpret_cast<f32x4 *>(static_cast<float *>(base) + at) = x;
}

// Queries of group g of kQueryTok tokens. table: cosines and sines, [token][2][rot / 2].
constexpr int kQueryRows = 4;       // rows (token, head) a thread has in flight
template <int D, bool BF16>
__device__ __forceinline__ void rotate_queries(const CacheAppend &a, int64_t token0, float *table)
{
    const int pairs = a.rot / 2, t = threadIdx.x;
    const int64_t first = clamp_row(a.batch, 0), end = clamp_row(a.batch, (int)a.batch.n_seqs);
    const GroupRows g = group_rows(token0, a.query_tokens, first, end, a.n_heads);
    const int n = g.tokens;
    // a wave's lanes share a token at a time, so that one finds its sequence
    const int wave = t >> 6, waves = blockDim.x >> 6, lane = t & 63;
    for (int k = wave; k < n; k += waves) {
        const int64_t token = token0 + k;
        if (token < first) continue;
        int pos;
        if (a.positions) {
            pos = a.positions[token];
        } else {
            const int s = find_sequence(a.batch, (int)token, 1, 0, 0);
            pos = a.batch.lengths[s] - (clamp_row(a.batch, s + 1) - (int)token);
        }
        for (int i = lane; i < pairs; i += 64) {
            float s;
            table[k * a.rot + i] = turned(a, (double)pos * a.frequencies[i], s);
            table[k * a.rot + pairs + i] = s;
        }
    }
    __syncthreads();
    constexpr int TPT = D / 8;
    const Unit u = unit_of(a, t % TPT);
    const int step = blockDim.x / TPT, rows = g.end;
    for (int r0 = g.begin + t / TPT; r0 < rows; r0 += step * kQueryRows) {
        f32x4 x[kQueryRows], y[kQueryRows];
        int k[kQueryRows];
        int64_t out[kQueryRows];
#pragma unroll
        for (int i = 0; i < kQueryRows; ++i) {
            const int row = r0 + i * step < rows ? r0 + i * step : r0;
            k[i] = (int)((uint32_t)row / (uint32_t)a.n_heads);
            const int64_t at = (token0 + k[i]) * a.q_token + (row - k[i] * a.n_heads) * a.q_head;
            out[i] = (token0 * a.n_heads + row) * D;
            x[i] = load4<BF16>(a.Q, at + u.a);
            y[i] = load4<BF16>(a.Q, at + u.b);
        }
#pragma unroll
        for (int i = 0; i < kQueryRows; ++i) {
            if (r0 + i * step >= rows) break;
            if (u.rotated) {
                const float *c = table + k[i] * a.rot + 4 * (t % TPT);
                rotate(a, x[i], y[i], *reinterpret_cast<const f32x4 *>(c),
                       *reinterpret_cast<const f32x4 *>(c + pairs));
            }
            store4<BF16>(a.Q_out, out[i] + u.a, x[i]);
            store4<BF16>(a.Q_out, out[i] + u.b, y[i]);
        }
    }
}

template <int D, int CODE, bool BF16>
__global__ __launch_bounds__(1024) void cache_append_kernel(CacheAppend a)
{
    __shared__ float lds[16];
    extern __shared__ __attribute__((aligned(16))) float table[];
    if (blockIdx.x >= a.page_slots) {
        const int64_t unit = (int64_t)(blockIdx.x - a.page_slots) * gridDim.y + blockIdx.y;
        for (int64_t g = unit; g < a.query_groups; g += a.query_blocks) {
            rotate_queries<D, BF16>(a, g * a.query_tokens, table);
            __syncthreads();
        }
        return;
    }
    const int head = blockIdx.y >> 1;
    PageSlot p;
    int position0;
    if (!find_page(a.cache, a.batch, blockIdx.x, p, &position0)) return;
    if (p.page < 0 || p.page >= a.cache.n_pages) return;
    if (blockIdx.y & 1)
        write_values<D, CODE, BF16>(a, p, head, lds);
    else
        append_keys<D, CODE, BF16>(a, p, position0, head, lds);
}

template <int D, int CODE>
hipError_t append_code(const CacheAppend &a, bool bf16, dim3 grid, unsigned threads,
                       hipStream_t stream)
{
    const unsigned lds = (unsigned)(a.query_tokens * a.rot * 4);
    if (bf16)
        cache_append_kernel<D, CODE, true><<<grid, threads, lds, stream>>>(a);
    else
        cache_append_kernel<D, CODE, false><<<grid, threads, lds, stream>>>(a);
    return hipGetLastError();
}

template <int D>
hipError_t append_dim(const CacheAppend &a, bool bf16, dim3 grid, unsigned threads,
                      hipStream_t stream)
{
    return a.cache.code_type == RRQ_CODE_INT8
               ? append_code<D, RRQ_CODE_INT8>(a, bf16, grid, threads, stream)
               : append_code<D, RRQ_CODE_FP8>(a, bf16, grid, threads, stream);
}

}  // namespace

hipError_t launch_cache_append(CacheAppend a, bool bf16, hipStream_t stream)
{
    const unsigned threads = block_threads(a.cache);
    const unsigned y = 2 * a.cache.n_kv_heads;
    a.page_slots = (uint32_t)cache_page_slots(a.batch, a.cache.page_size);
    // tokens a workgroup takes: one where tokens are few, else about two rounds of
    // kQueryRows rows a thread
    const int64_t units = (int64_t)a.n_heads * a.cache.head_dim / 8;
    int64_t n = a.batch.n_tokens < 4 * kServeCus ? 1 : 2 * kQueryRows * threads / units;
    a.query_tokens = (int32_t)(n < 1 ? 1 : (n > 8 ? 8 : n));
    a.query_groups = (a.batch.n_tokens + a.query_tokens - 1) / a.query_tokens;
    // (a bound on the grid: workgroups go on to further groups)
    const int64_t want = a.query_groups < 65536 ? a.query_groups : 65536;
    const unsigned more = (unsigned)((want + y - 1) / y);
    a.query_blocks = (int64_t)more * y;
    const dim3 grid(a.page_slots + more, y);
    if (a.cache.head_dim == 64) return append_dim<64>(a, bf16, grid, threads, stream);
    if (a.cache.head_dim == 128) return append_dim<128>(a, bf16, grid, threads, stream);
    return append_dim<256>(a, bf16, grid, threads, stream);
}

}  // namespace rrq_detail
