// Attention over the 8-bit cache for many query rows a sequence (prompt
// chunks): tiles of 128 rows, four waves of 32, that share each 64-key tile
// through LDS.
//
// With many rows the products bound the kernel, not the cache's bytes, so the
// codes are turned to binary16 once a workgroup, on their way into LDS, and
// every wave reads its operands from there. As in the few-row form the keys
// are the matrix rows (S^T = K Q^T, O^T = V^T P^T): a lane's 16 results of a
// 32 x 32 product are keys 8 (r / 4) + 4 (lane / 32) + r % 4 of one query row,
// and become the second product's operand as they are, because the values'
// 16-key runs are laid out in LDS in that order.
//
// Scales: a run of 16 keys lies in one page, so its key scale and value scale
// are wave-uniform. A weight carries its value scale through the exponent,
//   w = exp2(s c + lv - m),  c = key scale x query factor, lv = log2(vs / vref),
// with m the largest s c + lv: weights are relative to the row's largest
// contribution, whatever the scales of other pages. The softmax's sum gets the
// scale back once a run: l += (vref / vs) sum w. vref is a scale of the range
// at hand that keeps the exponents small.
//
// Measured. 8 kv heads of 128, int8: 4096 rows of 40 query heads on 16384
// positions, 1.20 TFLOP in 1.31 to 1.37 ms, 880 to 919 TFLOP/s where a large
// binary16 product of the library makes 1133; the matrix cores are busy 40% of
// the cycles. A wave waits for its LDS operands and the softmax between its two
// products; two workgroups a compute unit (LDS and registers hold no more)
// overlap. 4 kv heads of 256, e4m3: five chunks of 174 to 900 tokens, window 1024,
// 44 GFLOP in 105 us (420 TFLOP/s): 340 row tiles on 256 compute units, and 32-key
// tiles, as LDS holds two workgroups' 64-key tiles of such heads no more (one a
// compute unit: 156 us). Registers are full there: 6 (int8) and 3 (e4m3) vector
// registers spill, and 37 scalar ones with heads of 64.
//
// The running maximum m moves only when a tile's exceeds it by 8 (weights
// then grow to 2^8 at most): most tiles skip the output's rescaling.
#include "rrq_attention.h"

namespace rrq_detail {
namespace {

// Weights carry a factor of 2^6: with the slack's 2^8 they reach 2^14 in
// binary16, and its normal range ends at 2^-20 of a row's largest weight. Weights
// of two parts need that range: no slack, 2^14.
constexpr float slack(int parts) { return parts > 1 ? 0.0f : 8.0f; }

// Passes a NaN on, unlike fmaxf, which needs its operands quieted first.
__device__ __forceinline__ float maximum(float a, float b)
{
    return __builtin_elementwise_maximum(a, b);
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

// The larger of a lane's value and that of the lane 32 away.
__device__ __forceinline__ float other_half_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Lane i's value in every lane.
__device__ __forceinline__ float lane_value(float x, int i)
{
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i));
}

// A key row in LDS: the first halves of its 16-channel pieces, then the second
// halves (so that a wave's 16-byte writes fall in different banks). First
// channel of the 16-byte slot.
template <int D>
__device__ __forceinline__ int channel_of(int slot)
{
    constexpr int KP = D / 16;
    return slot < KP ? 16 * slot : 16 * (slot - KP) + 8;
}

// KEYS: keys of a tile, 32 or 64; PARTS: of an operand (rrq_attention.h), two of
// which take the registers of a whole wave a SIMD.
template <int D, int CODE, int KEYS, int PARTS>
__global__ __launch_bounds__(256, PARTS > 1 ? 1 : 2) void attend_rows_kernel(Attend a)
{
    // LDS bytes of a row. 16 more than a multiple of 128, so that 8 rows span all
    // banks (values of 32-key tiles: 80, an odd number of 16s, which does as well).
    constexpr int KROW = D * 2 + 16, VROW = KEYS * 2 + 16;
    constexpr int KB = KEYS * KROW, VB = D * VROW;
    constexpr int BUF = KB + VB + 64;       // and the scales of its runs
    constexpr int R = kRowsTile;
    constexpr float kSlack = slack(PARTS);
    constexpr int KT = KEYS * D / 16 / 256;    // 16-code pieces a thread stages
    constexpr int ND = D / 32, NK = D / 16, NH = KEYS / 32, RUNS = KEYS / 16;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * BUF];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, hb = lane >> 5;
    const int H = a.cache.n_kv_heads, P = a.cache.page_size;
    // heads are the fastest index: workgroups go to the 8 XCDs in turn, so a
    // head's workgroups share an L2 (at 8 heads); the last rows, which see the
    // most keys, come first
    const int kvh = blockIdx.x % H;
    RowTile r;
    if (!find_rows<R>(a, gridDim.x / H - 1 - blockIdx.x / H, r)) return;

    const int row = r.row0 + 32 * wave + col;
    const bool live = row < r.n_rows;
    const RowPlace place = place_of(a, live ? row : r.n_rows - 1);
    const int64_t token = place.token;
    const int head = kvh * a.ratio + place.member;
    int lo, hi, lo_any, hi_any, lo_all, hi_all;
    row_keys(a, r, place.token, lo, hi);
    tile_keys<R>(a, r, lo_any, hi_any, lo_all, hi_all);
    int tb, te;
    const bool alone = split_tiles<R>(a, lo_any, hi_any, blockIdx.y, tb, te);
    if (alone && blockIdx.y > 0) return;
    if (!alone && te <= tb) {
        empty_range<R>(a, r, kvh, blockIdx.y);
        return;
    }
    tb *= kTileKeys / KEYS;                 // to tiles of KEYS
    te *= kTileKeys / KEYS;
    const int32_t *table = a.batch.page_table + r.seq * a.batch.table_stride;

    // queries: lane (col, hb) holds 8 channels of its row a product, in the
    // order in which key rows stand in LDS
    f16x8 q[PARTS][NK];
    float qf;
    {
        float x[NK][8];
        float amax = 0.0f;
        const int64_t at = (r.o0 + token) * a.q_token + head * a.q_head;
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            load_query<8>(a, at + channel_of<D>(2 * j + hb), x[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[j][e]));
        }
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        float up;
        query_factors(a, amax, up, qf);
#pragma unroll
        for (int j = 0; j < NK; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = x[j][e] * up;
                q[0][j][e] = (_Float16)y;
                if (PARTS > 1) q[PARTS - 1][j][e] = (_Float16)(y - (float)q[0][j][e]);
            }
    }

    // Staging. Keys: thread t takes 16-code piece t % KP of key rows t / KP +
    // KSTEP i; a wave's rows lie in one run, so their page is wave-uniform.
    // Values: run t % RUNS of channel t / RUNS + VSTEP i. Lane % RUNS is the run
    // whose page and scales a lane looks up.
    constexpr int KP = D / 16, KSTEP = 256 / KP, VSTEP = 256 / RUNS;
    const int shift = __builtin_ctz(P);
    const int64_t head_bytes = (int64_t)P * D;
    // With heads of 256 the registers are full (an output of 128, queries of 64
    // of 256): there addresses are formed anew from an opaque thread number
    // instead of kept.
    auto thread = [] {
        int t = threadIdx.x;
        if (D == 256) asm volatile("" : "+v"(t));
        return t;
    };
    u32x4v kw[KT], vw[KT];
    int page;                           // of the tile after the one in registers
    float ksr, vsr;                     // of the tile in registers: its scales
    bool absent;                        // and whether the lane's run is absent
    // Loads without a branch: tiles past the last are the last again (staged,
    // never used), a run past the keys has the last key's page, an absent page
    // is read as page 0.
    auto find_page = [&](int tile) {
        const int vrun = thread() % RUNS;
        const int key = (tile < te ? tile : te - 1) * KEYS + 16 * vrun;
        page = table[(key < hi_any ? key : hi_any - 1) >> shift];
    };
    auto load_tile = [&](int tile) {
        const int t = thread(), krow = t / KP, vrun = t % RUNS;
        const int key0 = (tile < te ? tile : te - 1) * KEYS, run = key0 + 16 * vrun;
        absent = run >= hi_any || run + 16 <= lo_any ||
                 (uint32_t)page >= (uint64_t)a.cache.n_pages;
        const int safe = absent ? 0 : page;
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            const int row0 = KSTEP * i + 64 / KP * wave;        // wave's first row
            const int64_t p = __builtin_amdgcn_readlane(safe, row0 >> 4);
            const uint8_t *src = a.cache.k_codes + (p * H + kvh) * head_bytes;
            kw[i] = *reinterpret_cast<const u32x4v *>(
                src + (uint32_t)(((key0 + krow + KSTEP * i) & (P - 1)) * D + 16 * (t % KP)));
        }
        const int64_t block = (int64_t)safe * H + kvh;
        const uint8_t *src = a.cache.v_codes + block * head_bytes +
                             (uint32_t)((t / RUNS) * P + ((key0 + 16 * vrun) & (P - 1)));
#pragma unroll
        for (int i = 0; i < KT; ++i)
            vw[i] = *reinterpret_cast<const u32x4v *>(src + VSTEP * i * P);
        ksr = a.cache.k_scales[block];
        vsr = a.cache.v_scales[block];
    };
    // Values of keys that no row sees may be left over from another use of the
    // page (not numbers, even): cleared.
    auto clear_unseen = [&](int tile) {
        const int vrun = thread() % RUNS;
        const int run = (tile < te ? tile : te - 1) * KEYS + 16 * vrun;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t keep = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int key = run + 4 * w + c;
                if (key >= lo_any && key < hi_any && !absent) keep |= 255u << (8 * c);
            }
#pragma unroll
            for (int i = 0; i < KT; ++i) vw[i][w] &= keep;
        }
    };
    auto store_tile = [&](uint8_t *buf) {
        const int t = thread(), krow = t / KP, vrun = t % RUNS;
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            uint8_t *at = buf + (krow + KSTEP * i) * KROW + 16 * (t % KP);
            *reinterpret_cast<f16x8 *>(at) = codes_f16<CODE>(kw[i][0], kw[i][1]);
            *reinterpret_cast<f16x8 *>(at + D) = codes_f16<CODE>(kw[i][2], kw[i][3]);
        }
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            uint8_t *at = buf + KB + (t / RUNS + VSTEP * i) * VROW + 32 * vrun;
            *reinterpret_cast<f16x8 *>(at) = codes_f16<CODE>(vw[i][0], vw[i][2]);
            *reinterpret_cast<f16x8 *>(at + 16) = codes_f16<CODE>(vw[i][1], vw[i][3]);
        }
        // a value scale below 0 marks an absent run
        if (t < RUNS)
            *reinterpret_cast<f32x2 *>(buf + KB + VB + 8 * t) =
                f32x2{absent ? 0.0f : ksr, absent ? -1.0f : vsr};
    };
    // tiles whose keys not every row sees
    auto at_edge = [&](int tile) {
        return tile * KEYS < lo_all || tile * KEYS + KEYS > hi_all;
    };

    // LDS accesses done; global loads stay in flight.
    auto barrier = [&] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };

    float m = -kInf, l = 0.0f, vref = 0.0f;
    f32x16 o[ND];
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[n][e] = 0.0f;

    if (tb < te) {
        find_page(tb);
        load_tile(tb);
        find_page(tb + 1);
        clear_unseen(tb);
        store_tile(lds + (tb & 1) * BUF);
        load_tile(tb + 1);
        find_page(tb + 2);
        barrier();
    }
    // A wave without rows (the tile's last ones) only stages.
    const bool busy = r.row0 + 32 * wave < r.n_rows;
    for (int tile = tb; tile < te && !busy; ++tile) {
        if (at_edge(tile + 1) || __any(absent)) clear_unseen(tile + 1);
        store_tile(lds + ((tile + 1) & 1) * BUF);
        load_tile(tile + 2);
        find_page(tile + 3);
        barrier();
    }
    for (int tile = tb; tile < te && busy; ++tile) {
        const uint8_t *buf = lds + (tile & 1) * BUF;
        if (at_edge(tile + 1) || __any(absent)) clear_unseen(tile + 1);
        // scales of run lane % RUNS, and the tile's absent runs
        const f32x2 scales = *reinterpret_cast<const f32x2 *>(buf + KB + VB + 8 * (lane % RUNS));
        const float kst = scales[0], vst = scales[1];
        const uint32_t gone = (uint32_t)__ballot(vst < 0.0f) & ((1u << RUNS) - 1);

        f32x16 s[NH];
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[h][e] = 0.0f;
        int place = thread();
        const uint8_t *krows = buf + (place & 31) * KROW + ((place >> 5) & 1) * 16;
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            // (operands read ahead by 4 products at most where registers are full)
            if (D == 256 && j > 0 && j % 4 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int h = 0; h < NH; ++h) {
                const f16x8 k =
                    *reinterpret_cast<const f16x8 *>(krows + 32 * h * KROW + 32 * j);
#pragma unroll
                for (int t = 0; t < PARTS; ++t)
                    s[h] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[t][j], s[h], 0, 0, 0);
            }
        }
        store_tile(lds + ((tile + 1) & 1) * BUF);
        load_tile(tile + 2);
        find_page(tile + 3);

        if (at_edge(tile) || gone) {
            // -inf stands for a key that the row does not see: its weight is
            // exp2(-inf) = 0
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = tile * KEYS + 32 * h + 8 * (e >> 2) + 4 * hb + (e & 3);
                    if (key < lo || key >= hi || ((gone >> (2 * h + (e >> 3))) & 1))
                        s[h][e] = -kInf;
                }
        }
        float vmax = lane_value(vst, 0);
#pragma unroll
        for (int i = 1; i < RUNS; ++i) vmax = maximum(vmax, lane_value(vst, i));
        if (vmax > vref * kReferAgain) {
            refer(vmax, vref, m, l);
            vref = vmax;
        }
        // vref / vs of the lane's run, and its log2
        const float backs = scale_back(vst, vref);
        const float lbacks = __builtin_amdgcn_logf(backs);
        // c: factor of a run's products. 0 (a block of zeros) becomes the least
        // number, which leaves -inf as it is.
        float tmax = -kInf, c[RUNS];
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
            c[i] = lane_value(kst, i) * qf;
            if (c[i] == 0.0f) c[i] = 0x1p-126f;
            float x = s[i >> 1][8 * (i & 1)];
#pragma unroll
            for (int e = 1; e < 8; ++e) x = maximum(x, s[i >> 1][8 * (i & 1) + e]);
            tmax = maximum(tmax, __builtin_fmaf(x, c[i], -lane_value(lbacks, i)));
        }
        tmax = other_half_max(tmax);
        if (__any(tmax > m + kSlack)) {
            const float mn = fmaxf(m, tmax);
            const float alpha = mn == -kInf ? 0.0f : exp2_fast(m - mn);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int n = 0; n < ND; ++n) o[n] *= alpha;
        }
        const float ms = (m == -kInf ? 0.0f : m) - (14.0f - kSlack);    // the weights' factor
        f16x8 p[PARTS][RUNS];
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
            const float sub = ms + lane_value(lbacks, i);
            // summed before they are rounded: binary16 loses the weights of a
            // run of small values, which still has its full share of the sum
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = exp2_fast(
                    __builtin_fmaf(s[i >> 1][8 * (i & 1) + e], c[i], -sub));
                p[0][i][e] = (_Float16)w;
                if (PARTS > 1) p[PARTS - 1][i][e] = (_Float16)(w - (float)p[0][i][e]);
                sum += w;
            }
            l += sum * lane_value(backs, i);
        }
        place = thread();
        const uint8_t *vrows = buf + KB + (place & 31) * VROW + ((place >> 5) & 1) * 16;
#pragma unroll
        for (int i = 0; i < RUNS; ++i)
#pragma unroll
            for (int n = 0; n < ND; ++n) {
                const f16x8 v =
                    *reinterpret_cast<const f16x8 *>(vrows + 32 * n * VROW + 32 * i);
#pragma unroll
                for (int t = 0; t < PARTS; ++t)
                    o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[t][i], o[n], 0, 0, 0);
            }
        barrier();
    }

    // l and o carry the weights' factor, l in kSumUnit
    l += __shfl_xor(l, 32);
    if (!live) return;
    const int64_t at = (r.o0 + token) * a.n_heads + head;
    const float norm = mean_factor(vref, l);
    if (alone && a.n_splits > 1 && hb == 0) a.part_ml[2 * at + 1] = kAlone;
    if (!alone) {
        const int64_t part = (int64_t)blockIdx.y * a.batch.n_tokens * a.n_heads + at;
        if (hb == 0) {
            a.part_ml[2 * part] = m;
            a.part_ml[2 * part + 1] = l;
        }
        float *dst = a.part_o + part * D + 4 * hb;
#pragma unroll
        for (int n = 0; n < ND; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4 *>(dst + 32 * n + 8 * g) =
                    f32x4{o[n][4 * g], o[n][4 * g + 1], o[n][4 * g + 2], o[n][4 * g + 3]} *
                    kSumUnit * norm;
        return;
    }
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 y = f32x4{o[n][4 * g], o[n][4 * g + 1], o[n][4 * g + 2],
                                  o[n][4 * g + 3]} * kSumUnit * norm;
            const int64_t d = at * D + 32 * n + 8 * g + 4 * hb;
            if (a.out_bf16)
                *reinterpret_cast<u32x2v *>(static_cast<uint16_t *>(a.out) + d) =
                    u32x2v{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])};
            else
                *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + d) = y;
        }
}

template <int D, int CODE>
hipError_t rows_code(const Attend &a, hipStream_t stream)
{
    const dim3 grid((unsigned)(attend_row_tiles(a.batch, a.ratio, kRowsTile) *
                               a.cache.n_kv_heads), a.n_splits);
    constexpr int KEYS = D == 256 ? 32 : 64;
    if (a.out_bf16)
        attend_rows_kernel<D, CODE, KEYS, 1><<<grid, 256, 0, stream>>>(a);
    else
        attend_rows_kernel<D, CODE, KEYS, 2><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <int D>
hipError_t rows_dim(const Attend &a, hipStream_t stream)
{
    return a.cache.code_type == RRQ_CODE_INT8 ? rows_code<D, RRQ_CODE_INT8>(a, stream)
                                              : rows_code<D, RRQ_CODE_FP8>(a, stream);
}

}  // namespace

hipError_t launch_attend_rows(const Attend &a, hipStream_t stream)
{
    if (a.cache.head_dim == 64) return rows_dim<64>(a, stream);
    if (a.cache.head_dim == 128) return rows_dim<128>(a, stream);
    return rows_dim<256>(a, stream);
}

}  // namespace rrq_detail
