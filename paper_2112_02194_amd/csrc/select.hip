// The best k of every row of scores after the rules, and the log of the sum of the exponentials (als_select).
//
// A candidate is one whole number: the score as ordered bits above, the complement of the item id below, so that a larger
// number is a better score, or an equal one with a smaller id.  A part of a row is walked a tile at a time: every thread keeps
// the running maximum and sum of its elements' exponentials, and elements at least as good as the bar are appended to a buffer in
// LDS.  The bar is a candidate that at least k of the part's reach: on the first tile the smallest of the four wavefronts'
// ceil(k / 4)-th best lanes, later the k-th best of the buffer, found whenever that is full enough and then cut back to k.
// The buffer has room for a whole tile beside what is kept, so no order of the scores and no number of equal ones overflows it.
#include <algorithm>
#include <cmath>

#include "score_rules.h"

namespace als {

constexpr int SELECT_KEEP = 1024;                // the buffer is cut back to k before a tile when it holds more
constexpr int SELECT_CAP = SELECT_KEEP + TILE;   // candidates in LDS
typedef unsigned long long Cand;

__device__ __forceinline__ uint32_t ordered_bits(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);  // -0 becomes 0: equal scores
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ Cand candidate(float v, int64_t item) { return (Cand)ordered_bits(v) << 32 | (uint32_t)~(uint32_t)item; }
constexpr uint32_t ORDERED_LOWEST = 0x007fffffu;  // ordered_bits(-inf): never a candidate

// The j-th largest of the wavefront's 64 values, 1 <= j <= 64.
__device__ __forceinline__ uint32_t wave_nth(uint32_t v, int j) {
    unsigned long long in = ~0ull;
    uint32_t result = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const unsigned long long ones = __ballot((v >> bit) & 1u) & in;
        const int c = __popcll(ones);
        if (c >= j) {
            in = ones;
            result |= 1u << bit;
        } else {
            j -= c;
            in &= ~ones;
        }
    }
    return result;
}

struct SelectShared {
    Cand buf[SELECT_CAP];
    uint32_t hist[256];
    uint32_t wave_bar[TILE_THREADS / 64];
    float wave_m[TILE_THREADS / 64], wave_s[TILE_THREADS / 64];
    Cand keep[ALS_TOPK_MAX_K];
    int count, kept, digit, rest;
};

// The k best of buf[0, count) to the front of buf (count > k) by counting the candidates' digits from the top; they are all
// different.  Returns the k-th best.  All threads call it; it ends with a barrier.
__device__ Cand cut_back(SelectShared &sh, int count, int k, int tid) {
    Cand prefix = 0, mask = 0;
    int want = k;
    for (int shift = 56; shift >= 0; shift -= 8) {
        sh.hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < count; i += TILE_THREADS)
            if ((sh.buf[i] & mask) == prefix) atomicAdd(&sh.hist[(sh.buf[i] >> shift) & 255], 1u);
        __syncthreads();
        int above = 0;  // candidates with a larger digit than tid
        for (int d = 255; d > tid; --d) above += (int)sh.hist[d];
        if (above < want && above + (int)sh.hist[tid] >= want) {
            sh.digit = tid;
            sh.rest = want - above;
        }
        __syncthreads();
        prefix |= (Cand)sh.digit << shift;
        mask |= (Cand)255 << shift;
        want = sh.rest;
        __syncthreads();
    }
    if (tid == 0) sh.kept = 0;
    __syncthreads();
    for (int i = tid; i < count; i += TILE_THREADS)
        if (sh.buf[i] >= prefix) sh.keep[atomicAdd(&sh.kept, 1)] = sh.buf[i];
    __syncthreads();
    if (tid < k) sh.buf[tid] = sh.keep[tid];
    if (tid == 0) sh.count = k;
    __syncthreads();
    return prefix;
}

// Running maximum and sum of exponentials, in units of exp2(scale * x).
struct ExpSum {
    float m = -INFINITY, s = 0.f;
    __device__ void add(float om, float os, float scale) {
        const float top = fmaxf(m, om);
        if (top == -INFINITY) {  // nothing yet, but for a NaN
            s += os;
            return;
        }
        s = (m == top ? s : s * exp2f((m - top) * scale)) + (om == top ? os : os * exp2f((om - top) * scale));
        m = top;
    }
};

// Ends a row: the best k of buf[0, count), count <= 64 or cut back to k, in order.
__device__ void write_row(SelectShared &sh, int k, int64_t row, int32_t *ids, float *scores, int tid) {
    const int count = sh.count;
    if (tid < k && tid >= count) {
        ids[row * k + tid] = -1;
        scores[row * k + tid] = -INFINITY;
    }
    if (tid < count) {
        const Cand mine = sh.buf[tid];
        int rank = 0;
        for (int i = 0; i < count; ++i) rank += sh.buf[i] > mine;
        if (rank < k) {
            ids[row * k + rank] = (int32_t)~(uint32_t)mine;
            scores[row * k + rank] = from_ordered((uint32_t)(mine >> 32));
        }
    }
}
__device__ __forceinline__ float log_sum(float m, float s, float temperature) {
    if (s != s || m == -INFINITY || m == INFINITY) return s != s ? s : m;
    return m / temperature + logf(s);
}

// Workgroup w: part w % parts (tiles_per_part tiles) of row w / parts.  With one part a row it writes the answer, otherwise the
// part's k best (0: none) and its exponential sum.
template <bool BF16>
__global__ __launch_bounds__(TILE_THREADS) void select_kernel(const void *__restrict__ X, int64_t ld, int64_t rows, int64_t cols, int k,
                                                              int parts, int64_t tiles_per_part, float temperature, float scale,
                                                              RuleArgs rules, Cand *__restrict__ part_cand, float2 *__restrict__ part_sum,
                                                              int32_t *__restrict__ ids, float *__restrict__ scores, float *__restrict__ lse) {
    extern __shared__ __align__(16) uint32_t words[];
    __shared__ SelectShared sh;
    uint32_t *count = words, *place = words + (rules.history.indptr ? TILE : 0);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t tiles = (cols + TILE - 1) / TILE;
    for (int64_t w = blockIdx.x; w < rows * parts; w += gridDim.x) {
        const int64_t row = w / parts;
        const int part = (int)(w % parts);
        const int64_t t0 = part * tiles_per_part, t1 = std::min<int64_t>(tiles, t0 + tiles_per_part);
        const RowRules mine(rules, row);
        ExpSum sum;
        Cand bar = 0;
        if (tid == 0) sh.count = 0;
        __syncthreads();
        for (int64_t t = t0; t < t1; ++t) {
            const int64_t first = t * TILE;
            float x[TILE_EPT / 4][4];
#pragma unroll
            for (int j = 0; j < TILE_EPT / 4; ++j) {
                const int64_t at = first + tile_item(j, tid);
                const int valid = (int)std::max<int64_t>(0, std::min<int64_t>(4, cols - at));
                load4<BF16>(X, row * ld + at, valid, x[j]);
            }
            tile_lists(rules, mine, first, count, place, tid);
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < TILE_EPT / 4; ++j) {
                const int item = tile_item(j, tid);
                const int valid = (int)std::max<int64_t>(0, std::min<int64_t>(4, cols - first - item));
                apply_rules(rules, mine, first, item, valid, count, place, x[j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (e >= valid) x[j][e] = -INFINITY;
                    top = fmaxf(top, x[j][e]);
                }
            }
            float part_s = 0.f;
            const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int j = 0; j < TILE_EPT / 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) part_s += x[j][e] == from ? 1.f : exp2f((x[j][e] - from) * scale);
            sum.add(top, part_s, scale);

            if (bar == 0) {  // the part's first tile
                const uint32_t nth = wave_nth(ordered_bits(top), (k + 3) / 4);
                if (lane == 0) sh.wave_bar[wave] = nth;
                __syncthreads();
                uint32_t least = sh.wave_bar[0];
                for (int i = 1; i < TILE_THREADS / 64; ++i) least = min(least, sh.wave_bar[i]);
                bar = (Cand)(least > ORDERED_LOWEST ? least : ORDERED_LOWEST + 1) << 32;
            }
#pragma unroll
            for (int j = 0; j < TILE_EPT / 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Cand c = candidate(x[j][e], first + tile_item(j, tid) + e);
                    if (x[j][e] > -INFINITY && c >= bar) sh.buf[atomicAdd(&sh.count, 1)] = c;
                }
            __syncthreads();
            const int have = sh.count;
            __syncthreads();
            if (have > SELECT_KEEP) bar = cut_back(sh, have, k, tid);
        }
        const int have = sh.count;
        __syncthreads();
        if (have > k) cut_back(sh, have, k, tid);

        for (int m = 1; m < 64; m <<= 1) sum.add(__shfl_xor(sum.m, m), __shfl_xor(sum.s, m), scale);
        if (lane == 0) {
            sh.wave_m[wave] = sum.m;
            sh.wave_s[wave] = sum.s;
        }
        __syncthreads();
        if (tid == 0) {
            ExpSum all;
            for (int i = 0; i < TILE_THREADS / 64; ++i) all.add(sh.wave_m[i], sh.wave_s[i], scale);
            if (parts > 1) part_sum[w] = make_float2(all.m, all.s);
            else if (lse) lse[row] = log_sum(all.m, all.s, temperature);
        }
        if (parts > 1) {
            if (tid < k) part_cand[w * k + tid] = tid < sh.count ? sh.buf[tid] : 0;
        } else {
            write_row(sh, k, row, ids, scores, tid);
        }
        __syncthreads();
    }
}

// The parts of a row together, one workgroup per row.
__global__ __launch_bounds__(TILE_THREADS) void select_merge_kernel(int64_t rows, int k, int parts, float temperature, float scale,
                                                                    const Cand *__restrict__ part_cand, const float2 *__restrict__ part_sum,
                                                                    int32_t *__restrict__ ids, float *__restrict__ scores, float *__restrict__ lse) {
    __shared__ SelectShared sh;
    const int tid = threadIdx.x;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        Cand bar = 1;  // 0 stands for none
        if (tid == 0) sh.count = 0;
        __syncthreads();
        const int64_t total = (int64_t)parts * k;
        for (int64_t i0 = 0; i0 < total; i0 += TILE) {
            for (int i = tid; i < TILE && i0 + i < total; i += TILE_THREADS) {
                const Cand c = part_cand[row * total + i0 + i];
                if (c >= bar) sh.buf[atomicAdd(&sh.count, 1)] = c;
            }
            __syncthreads();
            const int have = sh.count;
            __syncthreads();
            if (have > SELECT_KEEP || (have > k && i0 + TILE >= total)) bar = cut_back(sh, have, k, tid);
        }
        write_row(sh, k, row, ids, scores, tid);
        if (tid == 0 && lse) {
            ExpSum all;
            for (int i = 0; i < parts; ++i) all.add(part_sum[row * parts + i].x, part_sum[row * parts + i].y, scale);
            lse[row] = log_sum(all.m, all.s, temperature);
        }
        __syncthreads();
    }
}

als_status launch_select(als_ctx *ctx, const als_matrix *X, const als_rules *rules, float temperature, int k, int32_t *ids,
                         float *scores, float *lse, hipStream_t s) {
    const RuleArgs a = rule_args(rules);
    const int64_t tiles = (X->cols + TILE - 1) / TILE;
    // enough workgroups to fill the card
    int64_t parts = std::max<int64_t>(1, std::min<int64_t>(tiles, (int64_t)ctx->num_cu * 2 / X->rows));
    const int64_t per = std::max<int64_t>(1, (tiles + parts - 1) / parts);
    parts = std::max<int64_t>(1, (tiles + per - 1) / per);
    const float scale = 1.44269504f / temperature;
    Cand *cand = nullptr;
    float2 *sums = nullptr;
    if (parts > 1) {
        const size_t cand_bytes = ((size_t)X->rows * parts * k * sizeof(Cand) + 255) / 256 * 256;
        als_status st = ensure(ctx, ctx->select_partials, cand_bytes + (size_t)X->rows * parts * sizeof(float2));
        if (st != ALS_OK) return st;
        cand = (Cand *)ctx->select_partials.p;
        sums = (float2 *)((char *)ctx->select_partials.p + cand_bytes);
    }
    const dim3 grid((unsigned)std::min<int64_t>(X->rows * parts, 1 << 22)), block(TILE_THREADS);
    const size_t lds = (size_t)rule_words(a) * 4;
    const void *f = X->dtype == ALS_BF16 ? (const void *)select_kernel<true> : (const void *)select_kernel<false>;
    ALS_HIP(ctx, hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * TILE * 4));
    if (X->dtype == ALS_BF16)
        hipLaunchKernelGGL((select_kernel<true>), grid, block, lds, s, X->data, X->ld, X->rows, X->cols, k, (int)parts, per, temperature,
                           scale, a, cand, sums, ids, scores, lse);
    else
        hipLaunchKernelGGL((select_kernel<false>), grid, block, lds, s, X->data, X->ld, X->rows, X->cols, k, (int)parts, per, temperature,
                           scale, a, cand, sums, ids, scores, lse);
    if (parts > 1)
        hipLaunchKernelGGL(select_merge_kernel, dim3((unsigned)std::min<int64_t>(X->rows, 1 << 22)), block, 0, s, X->rows, k, (int)parts,
                           temperature, scale, (const Cand *)cand, (const float2 *)sums, ids, scores, lse);
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
