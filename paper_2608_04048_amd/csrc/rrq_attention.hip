// Attention over the 8-bit cache (rrq_serve.h: rrq_cache_attention).
//
// One workgroup takes a tile of 16 rows (token, query head of the kv head's
// group) and a range of key positions; its four waves take 64-key tiles of
// the range in turn, each with its own running maximum, sum and output, and
// are joined at the end. A row tile whose range is split over several
// workgroups is joined by a second kernel.
//
// Both products run on the matrix cores in binary16 with binary32 sums, with
// the keys as rows: S^T = K Q^T and O^T = V^T P^T, so that the layout of the
// first's result (a lane holds 4 consecutive rows of a column) is the second's
// operand without any exchange between lanes. That fixes which key stands in
// which matrix row: in a tile of 64 keys lane group g (16 lanes) owns keys 16 g
// .. 16 g + 15, and row m of the i-th product takes key 16 (m / 4) + 4 i + m % 4.
// A run of 16 keys never spans pages, so a lane group has one key scale and one
// value scale a tile; the scales stay out of the operands (codes are exact in
// binary16): the key scale multiplies the product, the value scale the weight.
#include "rrq_serve_device.h"
#include "rrq_serve_launch.h"

namespace rrq_detail {
namespace {

constexpr int kTileKeys = 64;
// Positions are ints; tiles may reach past the last one.
constexpr int64_t kMaxPositions = (int64_t(1) << 31) - 4096;
// A split takes at least this many keys: below it a workgroup's fixed work
// (its query tile, the join) outweighs its share.
constexpr int kMinSplitKeys = 512;
// Weights are scaled by 2^14 before rounding to binary16, whose normal range
// then reaches 2^-28 below the largest weight.
constexpr float kWeightScale = 0x1p14f;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum over the four lane groups.
__device__ __forceinline__ float group_max(float a)
{
    a = fmaxf(a, __shfl_xor(a, 16));
    return fmaxf(a, __shfl_xor(a, 32));
}
__device__ __forceinline__ float group_sum(float a)
{
    a += __shfl_xor(a, 16);
    return a + __shfl_xor(a, 32);
}

// The rows and key range of a workgroup.
struct RowTile {
    int64_t seq, row0;      // first row of the tile within the sequence
    int64_t o0, n_rows;     // first dense row and rows (tokens x ratio) of the sequence
    int64_t len, start;     // sequence length, position of its first token here
};

__device__ __forceinline__ bool find_rows(const Attend &a, int64_t u, RowTile &r)
{
    const int64_t s = find_sequence(a.batch, u, a.ratio, kAttendRows, 1);
    r.seq = s;
    r.o0 = clamp_row(a.batch, s);
    const int64_t n = clamp_row(a.batch, s + 1) - r.o0;
    r.row0 = (u - (r.o0 * a.ratio / kAttendRows + s)) * kAttendRows;
    r.n_rows = n * a.ratio;
    if (n <= 0 || r.row0 < 0 || r.row0 >= r.n_rows) return false;    // < 0: before the first sequence
    const int64_t len = a.batch.lengths[s];
    r.start = len - n;
    int64_t cap = a.batch.max_pages * a.cache.page_size;
    if (cap > kMaxPositions) cap = kMaxPositions;
    r.len = len < 0 ? 0 : (len > cap ? cap : len);
    return true;
}

// Keys row token i sees: [lo, hi).
__device__ __forceinline__ void row_keys(const Attend &a, const RowTile &r, int64_t i, int &lo,
                                         int &hi)
{
    const int64_t pos = r.start + i;
    int64_t h = a.causal && pos + 1 < r.len ? pos + 1 : r.len;
    int64_t l = a.window > 0 && pos + 1 > a.window ? pos + 1 - a.window : 0;
    if (h < 0) h = 0;
    if (l > h) l = h;
    lo = (int)l;
    hi = (int)h;
}

template <int D, int CODE>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void attend_kernel(Attend a)
{
    constexpr int KL = D / 64;      // 16-byte key loads a lane and key row
    constexpr int ND = D / 16;      // 16-channel tiles of the output
    __shared__ float lds_o[4][16][D + 4];
    __shared__ float lds_ml[4][16][2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, g = lane >> 4;
    const int kvh = blockIdx.y, split = blockIdx.z;
    RowTile r;
    if (!find_rows(a, blockIdx.x, r)) return;

    // this lane's row
    const int64_t row = r.row0 + col;
    const bool live = row < r.n_rows;
    const int64_t token = (live ? row : r.n_rows - 1) / a.ratio;
    const int head = kvh * a.ratio + (int)((live ? row : r.n_rows - 1) % a.ratio);
    int lo, hi;
    row_keys(a, r, token, lo, hi);
    // keys any / every row of the tile sees: tokens ascend with rows
    int lo_any, hi_any, lo_all, hi_all;
    {
        const int64_t first = r.row0 / a.ratio;
        const int64_t last_row = r.row0 + kAttendRows < r.n_rows ? r.row0 + kAttendRows : r.n_rows;
        row_keys(a, r, first, lo_any, hi_all);
        row_keys(a, r, (last_row - 1) / a.ratio, lo_all, hi_any);
    }
    // this workgroup's range, in whole tiles
    const int t0 = lo_any / kTileKeys;
    const int tiles = hi_any > lo_any ? (hi_any + kTileKeys - 1) / kTileKeys - t0 : 0;
    int per = (tiles + a.n_splits - 1) / a.n_splits;
    if (per < kMinSplitKeys / kTileKeys) per = kMinSplitKeys / kTileKeys;
    const int tb = t0 + split * per;
    const int te = tb + per < t0 + tiles ? tb + per : t0 + tiles;

    const int P = a.cache.page_size, H = a.cache.n_kv_heads;
    const int32_t *table = a.batch.page_table + r.seq * a.batch.table_stride;

    // Queries: lane (col, g) holds channels 64 j + 16 g .. + 15 of its row,
    // scaled by a power of two so that the row's largest lies in [2^13, 2^14)
    // and rounded to binary16. qf undoes that and applies scale log2(e).
    f16x8 q[KL][2];
    float qf;
    {
        float x[KL][16];
        float amax = 0.0f;
        const int64_t at = (r.o0 + token) * a.q_token + head * a.q_head + 16 * g;
#pragma unroll
        for (int j = 0; j < KL; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                f32x4 y;
                if (a.q_bf16) {
                    const u32x2v w = *reinterpret_cast<const u32x2v *>(
                        static_cast<const uint16_t *>(a.Q) + at + 64 * j + 4 * v);
                    y = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u),
                              __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xFFFF0000u)};
                } else {
                    y = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(a.Q) + at +
                                                         64 * j + 4 * v);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[j][4 * v + e] = y[e];
                    amax = fmaxf(amax, fabsf(y[e]));
                }
            }
        amax = group_max(amax);
        int e = (int)(__float_as_uint(amax) >> 23) - 127;
        e = e < -100 ? -100 : (e > 120 ? 120 : e);
        const float up = __uint_as_float((uint32_t)(13 - e + 127) << 23);
        qf = __uint_as_float((uint32_t)(e - 13 + 127) << 23) * (a.scale * kLog2e);
#pragma unroll
        for (int j = 0; j < KL; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i) q[j][h][i] = (_Float16)(x[j][8 * h + i] * up);
    }

    float m = -kInf, l = 0.0f, vref = 0.0f;
    f32x4 o[ND];
#pragma unroll
    for (int n = 0; n < ND; ++n) o[n] = f32x4{0, 0, 0, 0};

    for (int tile = tb + wave; tile < te; tile += 4) {
        const int key0 = tile * kTileKeys;
        // page of the run this lane loads keys of (rows col: run col / 4) and
        // of the run it owns (g)
        const int krun = key0 + 16 * (col >> 2), orun = key0 + 16 * g;
        int64_t kpage = -1, opage = -1;
        if (krun < hi_any && krun + 16 > lo_any) kpage = table[krun / P];
        if (orun < hi_any && orun + 16 > lo_any) opage = table[orun / P];
        const bool there = opage >= 0 && opage < a.cache.n_pages;
        if (kpage < 0 || kpage >= a.cache.n_pages) kpage = 0;
        const int64_t ob = (there ? opage : 0) * H + kvh;
        const float ks = there ? a.cache.k_scales[ob] : 0.0f;
        const float vs = there ? a.cache.v_scales[ob] : 0.0f;
        const uint8_t *kc = a.cache.k_codes + (kpage * H + kvh) * P * D +
                            (krun % P + (col & 3)) * D + 16 * g;
        const uint8_t *vc = a.cache.v_codes + ob * P * D + (int64_t)col * P + orun % P;
        u32x4v kw[4][KL], vw[ND];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < KL; ++j)
                kw[i][j] = *reinterpret_cast<const u32x4v *>(kc + 4 * i * D + 64 * j);
#pragma unroll
        for (int n = 0; n < ND; ++n)
            vw[n] = *reinterpret_cast<const u32x4v *>(vc + 16 * n * P);

        // a lane's 16 keys: orun + 4 i + c
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 acc = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < KL; ++j) {
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    codes_f16<CODE>(kw[i][j][0], kw[i][j][1]), q[j][0], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    codes_f16<CODE>(kw[i][j][2], kw[i][j][3]), q[j][1], acc, 0, 0, 0);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) s[i][c] = acc[c] * (ks * qf);
        }
        // Keys a row does not see. The codes there may be left over from
        // another use of the page (not numbers, even), so scores are replaced
        // and value codes of keys that no row sees are cleared.
        if (key0 < lo_all || key0 + kTileKeys > hi_all || !__all(there)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int key = orun + 4 * i + c;
                    if (key < lo || key >= hi || !there) s[i][c] = -kInf;
                }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t keep = 0;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int key = orun + 4 * w + c;
                    if (key >= lo_any && key < hi_any && there) keep |= 255u << (8 * c);
                }
#pragma unroll
                for (int n = 0; n < ND; ++n) vw[n][w] &= keep;
            }
        }
        float tmax = -kInf;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) tmax = fmaxf(tmax, s[i][c]);
        const float mn = fmaxf(m, group_max(tmax));
        const float ms = mn == -kInf ? 0.0f : mn;
        float alpha = exp2_fast(m - ms);
        m = mn;
        // the value scales' reference: the largest so far, same in every lane
        const float vn = fmaxf(vref, group_max(vs));
        const float vr = vn > 0.0f ? 1.0f / vn : 0.0f;
        const float wf = vs * vr * kWeightScale;
        l *= alpha;
        f16x8 p[2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float e = exp2_fast(s[i][c] - ms);
                l += e;
                p[i >> 1][4 * (i & 1) + c] = (_Float16)(e * wf);
            }
        alpha *= vref * vr;
        vref = vn;
#pragma unroll
        for (int n = 0; n < ND; ++n) {
            o[n] *= alpha;
            o[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16<CODE>(vw[n][0], vw[n][1]),
                                                          p[0], o[n], 0, 0, 0);
            o[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16<CODE>(vw[n][2], vw[n][3]),
                                                          p[1], o[n], 0, 0, 0);
        }
    }

    // Join the waves: lane (col, g) holds channels 16 n + 4 g + c of row col.
    l = group_sum(l);
    const float of = vref * (1.0f / kWeightScale);
    if (g == 0) {
        lds_ml[wave][col][0] = m;
        lds_ml[wave][col][1] = l;
    }
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) lds_o[wave][col][16 * n + 4 * g + c] = o[n][c] * of;
    __syncthreads();
    // 16 threads a row, 4 channels each in turn
    const int orow = threadIdx.x >> 4, oc = (threadIdx.x & 15) * 4;
    if (r.row0 + orow >= r.n_rows) return;
    float f[4], mm = -kInf, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, lds_ml[w][orow][0]);
    const float ms = mm == -kInf ? 0.0f : mm;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        f[w] = exp2_fast(lds_ml[w][orow][0] - ms);
        ll += f[w] * lds_ml[w][orow][1];
    }
    const int64_t otok = r.o0 + (r.row0 + orow) / a.ratio;
    const int64_t at = otok * a.n_heads + kvh * a.ratio + (r.row0 + orow) % a.ratio;
    const int64_t part = (int64_t)split * a.batch.n_tokens * a.n_heads + at;
    if (a.n_splits > 1 && oc == 0) {
        a.part_ml[2 * part] = mm;
        a.part_ml[2 * part + 1] = ll;
    }
    const float norm = ll == 0.0f ? 0.0f : 1.0f / ll;
    for (int d = oc; d < D; d += 64) {
        f32x4 y = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int c = 0; c < 4; ++c) y[c] += f[w] * lds_o[w][orow][d + c];
        if (a.n_splits > 1) {
            if (te > tb) *reinterpret_cast<f32x4 *>(a.part_o + part * D + d) = y;
            continue;
        }
        y *= norm;
        if (a.out_bf16)
            *reinterpret_cast<u32x2v *>(static_cast<uint16_t *>(a.out) + at * D + d) =
                u32x2v{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])};
        else
            *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + at * D + d) = y;
    }
}

// Joins the key ranges of a row: one wave a (token, head), 64 channels a
// pass. A range without a visible key has sum 0 and is left out (its output
// was not written).
template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(Attend a)
{
    const int lane = threadIdx.x & 63;
    const int64_t rows = a.batch.n_tokens * a.n_heads;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= rows) return;
    const int64_t token = at / a.n_heads;
    if (token < clamp_row(a.batch, 0) || token >= clamp_row(a.batch, a.batch.n_seqs)) return;
    float m = -kInf;
    for (int s = 0; s < a.n_splits; ++s) m = fmaxf(m, a.part_ml[2 * (s * rows + at)]);
    const float ms = m == -kInf ? 0.0f : m;
    float l = 0.0f, y[D / 64] = {};
    for (int s = 0; s < a.n_splits; ++s) {
        const int64_t part = s * rows + at;
        const float pl = a.part_ml[2 * part + 1];
        if (pl == 0.0f) continue;
        const float f = exp2_fast(a.part_ml[2 * part] - ms);
        l += f * pl;
#pragma unroll
        for (int d = 0; d < D / 64; ++d) y[d] += f * a.part_o[part * D + 64 * d + lane];
    }
    const float norm = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int d = 0; d < D / 64; ++d) {
        const float v = y[d] * norm;
        if (a.out_bf16)
            static_cast<uint16_t *>(a.out)[at * D + 64 * d + lane] = (uint16_t)bf16_bits(v);
        else
            static_cast<float *>(a.out)[at * D + 64 * d + lane] = v;
    }
}

template <int D>
hipError_t launch_dim(const Attend &a, hipStream_t stream)
{
    const dim3 grid((unsigned)attend_row_tiles(a.batch, a.ratio), a.cache.n_kv_heads, a.n_splits);
    if (a.cache.code_type == RRQ_CODE_INT8)
        attend_kernel<D, RRQ_CODE_INT8><<<grid, 256, 0, stream>>>(a);
    else
        attend_kernel<D, RRQ_CODE_FP8><<<grid, 256, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_splits == 1) return e;
    const int64_t rows = a.batch.n_tokens * a.n_heads;
    attend_join_kernel<D><<<(unsigned)((rows + 3) / 4), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

int attend_splits(const rrq_cache &c, const rrq_batch &b, int n_heads)
{
    const int64_t units = attend_row_tiles(b, n_heads / c.n_kv_heads) * c.n_kv_heads;
    const int64_t most = (b.max_pages * c.page_size + kMinSplitKeys - 1) / kMinSplitKeys;
    int64_t n = kServeCus * 4 / units;
    n = n > most ? most : n;
    return n < 1 ? 1 : (n > 64 ? 64 : (int)n);
}

hipError_t launch_attend(const Attend &a, hipStream_t stream)
{
    if (a.cache.head_dim == 64) return launch_dim<64>(a, stream);
    if (a.cache.head_dim == 128) return launch_dim<128>(a, stream);
    return launch_dim<256>(a, stream);
}

}  // namespace rrq_detail
