// The best k of every row of scores after the rules, and the log of the sum of the exponentials (als_select).
//
// A candidate is one whole number: the score as ordered bits above, the complement of the item id below, so that a larger
// number is a better score, or an equal one with a smaller id.
//
// select kernel  a part of a row (several parts where there are few rows), a tile at a time, one read of the scores.  Every
//                thread keeps the running maximum and sum of its elements' exponentials.  Scores above the bar are appended
//                to a buffer in LDS.  The bar is a score that at least k of the part reach: on the first tile just below the
//                smallest of the four wavefronts' ceil(k / 4)-th best lanes, later the k-th best of the buffer, found whenever
//                that is full enough and then cut back to k.  Items come in ascending order, so a later score that equals the
//                bar's loses against the k that are there.  A tile with more candidates than there is room for (an ascending
//                row) goes in a quarter or half at a time with the buffer cut back between: nothing overflows, whatever the
//                order or the number of equal scores.
// merge kernel   one workgroup per row: the parts' candidates, and their sums in a fixed order.
#include <algorithm>
#include <cmath>

#include "score_rules.h"

namespace als {

typedef unsigned long long Cand;
constexpr int SELECT_KEEP = 1024;  // the buffer is cut back to k when it holds more than this after a tile
constexpr int SELECT_CAP = 3072;   // room: what is kept and the largest piece of a tile, 2048
constexpr int PART_SLOTS = 128;    // candidates that a part hands on at most
constexpr int MERGE_THREADS = 1024;
static_assert(SELECT_KEEP + TILE_THREADS * 8 <= SELECT_CAP && ALS_TOPK_MAX_K <= 64 && 4 * ALS_TOPK_MAX_K <= TILE_THREADS, "");

__device__ __forceinline__ uint32_t ordered_bits(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);  // -0 becomes 0: equal scores
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ Cand candidate(float v, uint32_t item) { return (Cand)ordered_bits(v) << 32 | ~item; }
constexpr uint32_t ORDERED_LOWEST = 0x007fffffu, ORDERED_ZERO = 0x80000000u;  // of -inf, which is never a candidate, and of 0
// Scores equal to `o` are above the first, those equal to it are not above the second (`o` may be below -inf's).
__device__ __forceinline__ float bar_below(uint32_t o) { return from_ordered(max(o == ORDERED_ZERO ? o - 1 : o, ORDERED_LOWEST + 1) - 1); }
__device__ __forceinline__ float bar_at(Cand c) { return from_ordered(max((uint32_t)(c >> 32), ORDERED_LOWEST)); }

// One value from lanes of the wavefront by lane moves (v_add_f32_dpp and the like): rows of 16 lanes first, then across them.
// F is associative and commutative; the result is in lane 63.
template <class T, class F> __device__ __forceinline__ T wave_scan(T x, T none, F &&f) {
    auto step = [&](auto ctrl, auto rows) {
        const int moved = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x), ctrl(), rows(), 0xf, false);
        x = f(x, __builtin_bit_cast(T, moved));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});  // from 1, 2, 4, 8 lanes below in the row
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});  // the row's end to the next row: rows 1 and 3
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});  // lane 31 to rows 2 and 3
    return x;  // of the lanes up to this one
}
template <class T, class F> __device__ __forceinline__ T wave_all(T x, T none, F &&f) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_scan(x, none, f)), 63));
}

// A value that at least j of the wavefront's 64 reach, 1 <= j <= 64: the j-th largest without its last six bits (the lanes'
// numbers take their place, so that no two values are equal and a rank has one owner).
__device__ __forceinline__ uint32_t wave_nth(uint32_t v, int j) {
    v = (v & ~63u) | (63u - (threadIdx.x & 63));
    int before = 0;
#pragma unroll
    for (int i = 0; i < 64; ++i) before += (uint32_t)__builtin_amdgcn_readlane((int)v, i) > v;
    return (uint32_t)__builtin_amdgcn_readlane((int)v, __ffsll((long long)__ballot(before == j - 1)) - 1) & ~63u;
}

template <int CAP> struct Buffer {
    Cand cand[CAP], keep[ALS_TOPK_MAX_K];
    uint32_t hist[256], wave_sum[4];
    int kept, digit, rest, exact;

    // The k best of cand[0, count) to its front (count > k), by counting digits from the top; candidates are all different.
    // Returns a number that exactly k candidates reach.  All NT threads call it; it ends with a barrier.
    template <int NT> __device__ Cand cut_back(int count, int k, int tid) {
        Cand prefix = 0, mask = 0;
        int want = k;
        if (tid == 0) kept = 0;
        for (int shift = 56; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int i = tid; i < count; i += NT)
                if ((cand[i] & mask) == prefix) atomicAdd(&hist[(cand[i] >> shift) & 255], 1u);
            __syncthreads();
            uint32_t mine = 0, upto = 0;  // candidates with digit 255 - tid, and with that or a larger one
            if (tid < 256) {
                mine = upto = hist[255 - tid];
                for (int m = 1; m < 64; m <<= 1) {
                    const uint32_t o = __shfl_up(upto, m);
                    if ((tid & 63) >= m) upto += o;
                }
                if ((tid & 63) == 63) wave_sum[tid >> 6] = upto;
            }
            __syncthreads();
            if (tid < 256) {
                for (int i = 0; i < tid >> 6; ++i) upto += wave_sum[i];
                if ((int)upto >= want && (int)(upto - mine) < want) {
                    digit = 255 - tid;
                    rest = want - (int)(upto - mine);
                    exact = (int)upto == want;
                }
            }
            __syncthreads();
            prefix |= (Cand)digit << shift;
            mask |= (Cand)255 << shift;
            want = rest;
            if (exact) break;
        }
        for (int i = tid; i < count; i += NT)
            if (cand[i] >= prefix) keep[atomicAdd(&kept, 1)] = cand[i];
        __syncthreads();
        if (tid < k) cand[tid] = keep[tid];
        __syncthreads();
        return prefix;
    }
    // The best k of cand[0, count), count <= the workgroup's threads, in order, as the row's answer.
    __device__ void write_row(int count, int k, int64_t row, int32_t *ids, float *scores, int tid) const {
        if (tid < k && tid >= count) {
            ids[row * k + tid] = -1;
            scores[row * k + tid] = -INFINITY;
        }
        if (tid < count) {
            const Cand mine = cand[tid];
            int rank = 0;
            int i = 0;
            for (; i + 8 <= count; i += 8) {
#pragma unroll
                for (int u = 0; u < 8; ++u) rank += cand[i + u] > mine;
            }
            for (; i < count; ++i) rank += cand[i] > mine;
            if (rank < k) {
                ids[row * k + rank] = (int32_t)~(uint32_t)mine;
                scores[row * k + rank] = from_ordered((uint32_t)(mine >> 32));
            }
        }
    }
};

// Sum of exp(x / temperature) over some x, relative to the largest of them, m (-inf: none).  With c = m * scale as it was rounded
// (scale = log2(e) / temperature) the sum is s 2^c: an element costs one multiply-add and one exponential, and the rounding
// of c does no harm, since the same c is added in the end.  Where that product is out of range (scores near the type's
// limits, infinities) the sum is s exp(m / temperature), its terms are 2^((x - m) scale), 1 for x = m.
struct ExpSum {
    float m = -INFINITY, s = 0.f;
    static __device__ __forceinline__ bool plain(float m, float scale) { return fabsf(m * scale) < 1e30f; }
    // what a sum relative to m is multiplied by to be relative to top >= m
    static __device__ __forceinline__ float factor(float m, float top, float scale) {
        return m == top ? 1.f : __builtin_amdgcn_exp2f(plain(m, scale) && plain(top, scale) ? m * scale - top * scale : (m - top) * scale);
    }
    __device__ __forceinline__ void add(float om, float os, float scale) {
        const float top = fmaxf(m, om);
        s = s * factor(m, top, scale) + os * factor(om, top, scale);
        m = top;
    }
    __device__ __forceinline__ void over_lanes(float scale) {
        const float top = wave_all(m, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
        s = wave_all(s * factor(m, top, scale), 0.f, [](float a, float b) { return a + b; });
        m = top;
    }
    __device__ __forceinline__ float log(float temperature, float scale) const {
        if (s != s || m == -INFINITY || m == INFINITY) return s != s ? s : m;
        return plain(m, scale) ? (m * scale + log2f(s)) * 0.693147181f : m / temperature + logf(s);
    }
};

struct PartSum {
    float m, s;
    uint32_t best, unused;  // the best candidate's score, ordered; 0: none
};

// Workgroup (x, y): part x (tiles_per_part tiles) of row y.  With one part a row it writes the answer, otherwise the part's
// candidates, 0 in the slots that are left, and its exponential sum.
template <bool BF16, bool RULES>
__global__ __launch_bounds__(TILE_THREADS, RULES ? 4 : 6) void select_kernel(const char *__restrict__ X, int64_t row_bytes, int64_t first_row, uint32_t cols, int k,
                                                                 uint32_t tiles_per_part, float temperature, float scale, RuleArgs rules,
                                                                 Cand *__restrict__ part_cand, PartSum *__restrict__ part_sum,
                                                                 int32_t *__restrict__ ids, float *__restrict__ scores, float *__restrict__ lse) {
    typedef TileRow<BF16> Row;
    constexpr int PER = Row::PER, PIECES = Row::PIECES, WAVES = TILE_THREADS / 64;
    extern __shared__ __align__(16) uint32_t words[];
    __shared__ Buffer<SELECT_CAP> buf;
    __shared__ uint32_t wave_bar[WAVES];
    __shared__ float wave_m[WAVES], wave_s[WAVES];
    __shared__ int added[3];  // candidates of a tile, by turns: the last one is cleared while this one is read
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, parts = gridDim.x;
    const uint32_t begin = blockIdx.x * tiles_per_part * TILE;
    const uint32_t end = min(cols, (blockIdx.x + 1) * tiles_per_part * TILE);  // items of the part
    const int64_t row = first_row + blockIdx.y;
    const char *scores_row = X + row * row_bytes;
    Row in;
    if (begin < end) in.load(scores_row, begin, cols, tid);
    RowRules<Row> mine;
    if constexpr (RULES) mine.begin(rules, row, words, tid);
    ExpSum sum;
    float bar = -INFINITY;
    int have = 0, turn = 0;
    const int most = parts > 1 ? PART_SLOTS : TILE_THREADS;  // candidates at the end
    if (tid < 3) added[tid] = 0;
    __syncthreads();
    for (uint32_t first = begin; first < end; first += TILE) {
        float x[PIECES][PER];
        in.floats(x);
        const bool last = first + TILE >= end;
        if (!last) in.load(scores_row, first + TILE, cols, tid);
        if constexpr (RULES) mine.apply(rules, first, cols, tid, x);
        if (first + TILE > cols) {
            const uint32_t left = cols - first;
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    if (Row::item(j, tid) + e >= left) x[j][e] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < PIECES; ++j)
#pragma unroll
            for (int e = 0; e < PER; ++e) top = fmaxf(top, x[j][e]);
        const float m = fmaxf(sum.m, top);
        float part[2] = {0.f, 0.f};
        if (__any(!ExpSum::plain(m, scale) && m != -INFINITY)) {
            const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int e = 0; e < PER; ++e) part[0] += x[j][e] == from ? 1.f : __builtin_amdgcn_exp2f((x[j][e] - from) * scale);
        } else {
            const float c = m == -INFINITY ? 0.f : m * scale;
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int e = 0; e < PER; ++e) part[e & 1] += __builtin_amdgcn_exp2f(fmaf(x[j][e], scale, -c));
        }
        sum.s = sum.s * ExpSum::factor(sum.m, m, scale) + (part[0] + part[1]);
        sum.m = m;

        if (first == begin) {
            const uint32_t nth = wave_nth(ordered_bits(top), (k + WAVES - 1) / WAVES);
            if (lane == 0) wave_bar[wave] = nth;
            __syncthreads();
            uint32_t least = wave_bar[0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) least = min(least, wave_bar[i]);
            bar = bar_below(least);
        }
        // The scores above the bar into the buffer: all pieces at once, or, if they do not fit, one after the other.
        for (int j0 = 0, j1 = PIECES; j0 < PIECES;) {
            if (__any(top > bar)) {
                int mine_above = 0;
#pragma unroll
                for (int j = 0; j < PIECES; ++j)
#pragma unroll
                    for (int e = 0; e < PER; ++e) mine_above += j >= j0 && j < j1 && x[j][e] > bar;
                const int upto = wave_scan(mine_above, 0, [](int a, int b) { return a + b; });
                int at = 0;
                if (lane == 63) at = atomicAdd(&added[turn], upto);
                at = have + __builtin_amdgcn_readlane(at, 63) + upto - mine_above;
#pragma unroll
                for (int j = 0; j < PIECES; ++j)
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (j >= j0 && j < j1 && x[j][e] > bar) {
                            float v = x[j][e];
                            uint32_t from = first;
                            asm volatile("" : "+v"(v), "+s"(from));  // nothing is prepared for those that do not come here
                            if (at < SELECT_CAP) buf.cand[at] = candidate(v, from + Row::item(j, tid) + e);
                            ++at;
                        }
            }
            __syncthreads();
            int count = have + added[turn];
            if (tid == 0) added[turn == 0 ? 2 : turn - 1] = 0;
            turn = turn == 2 ? 0 : turn + 1;
            if (count > SELECT_CAP) {
                j1 = 1;
                continue;
            }
            j0 = j1;
            j1 = j0 + 1;
            if (count > (last && j0 == PIECES ? most : SELECT_KEEP)) {
                bar = bar_at(buf.template cut_back<TILE_THREADS>(count, k, tid));
                count = k;
            }
            have = count;
        }
    }
    sum.over_lanes(scale);
    if (lane == 0) {
        wave_m[wave] = sum.m;
        wave_s[wave] = sum.s;
    }
    __syncthreads();
    ExpSum all;
    {
        float top = wave_m[0], total = 0.f;
#pragma unroll
        for (int i = 1; i < WAVES; ++i) top = fmaxf(top, wave_m[i]);
#pragma unroll
        for (int i = 0; i < WAVES; ++i) total += wave_s[i] * ExpSum::factor(wave_m[i], top, scale);
        all.m = top;
        all.s = total;
    }
    if (parts > 1) {
        const int64_t w = row * parts + blockIdx.x;
        if (tid < PART_SLOTS) part_cand[w * PART_SLOTS + tid] = tid < have ? buf.cand[tid] : 0;
        if (tid == 0) part_sum[w] = PartSum{all.m, all.s, have ? ordered_bits(all.m) : 0, 0};
    } else {
        buf.write_row(have, k, row, ids, scores, tid);
        if (tid == 0 && lse) lse[row] = all.log(temperature, scale);
    }
}

// The parts of a row together, one workgroup per row.  A score that at least k candidates reach rules almost all of them out
// unread where there are many parts: the k-th best of the parts' best.  Where there are few they are all read once.
constexpr int MERGE_FEW = 64;  // parts; they give a thread MERGE_FEW * PART_SLOTS / MERGE_THREADS = 8 slots
__global__ __launch_bounds__(MERGE_THREADS) void select_merge_kernel(int64_t rows, int k, int parts, float temperature, float scale, const Cand *__restrict__ part_cand,
                                                                     const PartSum *__restrict__ part_sum, int32_t *__restrict__ ids,
                                                                     float *__restrict__ scores, float *__restrict__ lse) {
    constexpr int WAVES = MERGE_THREADS / 64, CAP = 2 * MERGE_THREADS, SLOTS = MERGE_FEW * PART_SLOTS / MERGE_THREADS;
    __shared__ Buffer<CAP> buf;
    __shared__ uint32_t wave_bar[WAVES];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int total = parts * PART_SLOTS;
        const Cand *cand = part_cand + row * total;
        const PartSum *part = part_sum + row * parts;
        if (tid == 0) count = 0;
        auto put = [&](Cand c, Cand bar) {
            if (c >= bar) {
                const int at = atomicAdd(&count, 1);
                if (at < CAP) buf.cand[at] = c;
            }
        };
        Cand bar;
        ExpSum all;
        if (parts <= MERGE_FEW) {
            Cand c[SLOTS];
            uint32_t best = 0;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                c[i] = i * MERGE_THREADS + tid < total ? cand[i * MERGE_THREADS + tid] : 0;
                best = max(best, (uint32_t)(c[i] >> 32));
            }
            if (wave == 0 && lane < parts) all.add(part[lane].m, part[lane].s, scale);
            const uint32_t nth = wave_nth(best, (k + WAVES - 1) / WAVES);
            if (lane == 0) wave_bar[wave] = nth;
            __syncthreads();
            uint32_t least = wave_bar[0];  // at least k candidates reach it, if there are as many
            for (int i = 1; i < WAVES; ++i) least = min(least, wave_bar[i]);
            bar = max((Cand)least << 32, (Cand)1);
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) put(c[i], bar);
        } else {
            // every wavefront for itself: the k-th best of the lanes' best, each of a few parts
            uint32_t best = 0;
            for (int i = lane; i < parts; i += 64) {
                const PartSum p = part[i];
                best = max(best, p.best);
                if (wave == 0) all.add(p.m, p.s, scale);
            }
            bar = max((Cand)wave_nth(best, k) << 32, (Cand)1);
            __syncthreads();
            int taken = 0;  // parts that reach the bar so far: the wavefronts take turns
            for (int i0 = 0; i0 < parts; i0 += 64) {
                unsigned long long who = __ballot(i0 + lane < parts && part[min(i0 + lane, parts - 1)].best >= (uint32_t)(bar >> 32));
                while (who) {
                    const int p = i0 + __ffsll((long long)who) - 1;
                    who &= who - 1;
                    if (taken++ % WAVES != wave) continue;
                    const Cand c0 = cand[p * PART_SLOTS + lane], c1 = cand[p * PART_SLOTS + 64 + lane];
                    put(c0, bar);
                    put(c1, bar);
                }
            }
        }
        __syncthreads();
        int have = count;
        if (have > CAP) {  // more than there is room for (equal scores): 1024 at a time
            have = 0;
            for (int i0 = 0; i0 < total; i0 += MERGE_THREADS) {
                __syncthreads();
                if (tid == 0) count = have;
                __syncthreads();
                if (i0 + tid < total) put(cand[i0 + tid], bar);
                __syncthreads();
                have = count;
                if (have > MERGE_THREADS) {
                    bar = buf.cut_back<MERGE_THREADS>(have, k, tid);
                    have = k;
                }
            }
        }
        __syncthreads();
        if (have > 256) {
            buf.cut_back<MERGE_THREADS>(have, k, tid);
            have = k;
        }
        buf.write_row(have, k, row, ids, scores, tid);
        if (wave == 0 && lse) {
            all.over_lanes(scale);
            if (lane == 0) lse[row] = all.log(temperature, scale);
        }
        __syncthreads();
    }
}

als_status launch_select(als_ctx *ctx, const als_matrix *X, const als_rules *rules, float temperature, int k, int32_t *ids,
                         float *scores, float *lse, hipStream_t s) {
    const RuleArgs a = rule_args(rules);
    const int64_t tiles = (X->cols + TILE - 1) / TILE;
    const bool bf = X->dtype == ALS_BF16, any = a.history.indptr || a.entries.indptr || a.bias || a.allowed;
    // parts of a row: as many workgroups as the card holds at a time, four or six per compute unit
    int64_t parts = std::max<int64_t>(1, std::min<int64_t>(tiles, ((int64_t)ctx->num_cu * (any ? 4 : 6) + X->rows - 1) / X->rows));
    const int64_t per = std::max<int64_t>(1, (tiles + parts - 1) / parts);
    parts = std::max<int64_t>(1, (tiles + per - 1) / per);
    const float scale = 1.44269504f / temperature;
    Cand *cand = nullptr;
    PartSum *sums = nullptr;
    if (parts > 1) {
        const size_t cand_bytes = (size_t)X->rows * parts * PART_SLOTS * sizeof(Cand);
        als_status st = ensure(ctx, ctx->select_partials, cand_bytes + (size_t)X->rows * parts * sizeof(PartSum));
        if (st != ALS_OK) return st;
        cand = (Cand *)ctx->select_partials.p;
        sums = (PartSum *)((char *)ctx->select_partials.p + cand_bytes);
    }
    auto go = [&](auto bf, auto with_rules) {
        for (int64_t row = 0; row < X->rows; row += 65535)  // a grid's second dimension
            hipLaunchKernelGGL((select_kernel<bf(), with_rules()>), dim3((unsigned)parts, (unsigned)std::min<int64_t>(X->rows - row, 65535)),
                           dim3(TILE_THREADS), rule_bytes(a), s, (const char *)X->data, X->ld * (bf() ? 2 : 4), row, (uint32_t)X->cols, k, (uint32_t)per, temperature, scale, a, cand, sums, ids,
                           scores, lse);
    };
    if (bf && any) go(std::true_type{}, std::true_type{});
    else if (bf) go(std::true_type{}, std::false_type{});
    else if (any) go(std::false_type{}, std::true_type{});
    else go(std::false_type{}, std::false_type{});
    if (parts > 1)
        hipLaunchKernelGGL(select_merge_kernel, dim3((unsigned)std::min<int64_t>(X->rows, 1 << 22)), dim3(MERGE_THREADS), 0, s, X->rows, k,
                           (int)parts, temperature, scale, (const Cand *)cand, (const PartSum *)sums, ids, scores, lse);
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
