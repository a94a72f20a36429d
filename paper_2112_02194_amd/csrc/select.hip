// The best k of every row of scores after the rules, and the log of the sum of the exponentials (als_select).
//
// A candidate is one whole number: the score as ordered bits above, the complement of the item id below, so that a larger
// number is a better score, or an equal one with a smaller id.
//
// select kernel  a part of a row (several parts where there are few rows), a tile at a time, one read of the scores.  Every
//                thread keeps the running maximum and sum of its elements' exponentials.  Scores above the bar are appended
//                to a buffer in LDS.  The bar is a score that at least k of the part reach: on the first tile just below what the
//                wavefronts' best lanes reach (WaveRanks), later the k-th best of the buffer, found whenever
//                that is full enough and then cut back to k.  Items come in ascending order, so a later score that equals the
//                bar's loses against the k that are there.  A tile with more candidates than there is room for (an ascending
//                row) goes in a step at a time with the buffer cut back between: nothing overflows, whatever the order or
//                the number of equal scores.
//                Memory bound up to the vector units' share: 512 x 1M bf16 202 us with k = 1 (5.1 TB/s, a copy's rate), 230 with
//                k = 50 (candidates found and cut back), 265 with every row's history (words cleared and counted a tile; the
//                vector units at work about 70 % of the time).  Short calls are chains of steps: 1 x 1M 9 us, 64 x 30000 with
//                all rules 11.
// merge kernel   one workgroup per row: the parts' candidates, and their sums in a fixed order.  A chain of loads and barriers:
//                10 us for the 245 parts of 1 x 1M, 12 for 512 rows.  As the last part's work in the select kernel (a count in
//                device memory, fences) it cost more than the launch: 21 us became 23, 293 became 352.
#include <algorithm>
#include <cmath>

#include "score_rules.h"

namespace als {

typedef unsigned long long Cand;
constexpr int PART_SLOTS = 128;  // the buffer is cut back to k when it holds more after a tile; what a part hands on at most
static_assert(ALS_TOPK_MAX_K <= PART_SLOTS && PART_SLOTS <= 256, "k fits in a part's slots, and one slot a thread is handed on");
// A tile that does not fit goes in STEPS steps; the buffer has room for what is kept and one of them.
template <int NT> constexpr int select_steps() { return NT == 1024 ? 8 : 4; }
template <int NT> constexpr int select_room() { return PART_SLOTS + NT * TILE_EPT / select_steps<NT>(); }

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

// Values that at least j of the wavefront's 64 reach, 1 <= j <= 64: the j-th largest without its last six bits (the lanes'
// numbers take their place, so that no two values are equal and a rank has one owner).
struct WaveRanks {
    uint32_t v;
    int before = 0;
    __device__ __forceinline__ explicit WaveRanks(uint32_t value) : v((value & ~63u) | (63u - (threadIdx.x & 63))) {
#pragma unroll
        for (int i = 0; i < 64; ++i) before += (uint32_t)__builtin_amdgcn_readlane((int)v, i) > v;
    }
    __device__ __forceinline__ uint32_t nth(int j) const {
        return (uint32_t)__builtin_amdgcn_readlane((int)v, __ffsll((long long)__ballot(before == j - 1)) - 1) & ~63u;
    }
};

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
// of c does no harm, since the same c is added in the end.  That holds while it is small: the largest element's own term is
// 2^(m * scale - c), at most 2^(1/32) up to |c| = 2^20 but beyond fp32's range from 2^31 on.  Above, the sum is
// s exp(m / temperature), its terms are 2^((x - m) scale), 1 for x = m.  No product is joined with a sum that uses c into one
// operation: c has to be the same number everywhere.
struct ExpSum {
    float m = -INFINITY, s = 0.f;
    static __device__ __forceinline__ bool plain(float m, float scale) { return fabsf(m * scale) < 0x1p20f; }
    // what a sum relative to m is multiplied by to be relative to top >= m
    static __device__ __forceinline__ float factor(float m, float top, float scale) {
#pragma clang fp contract(off)
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
    // The largest score's part is m / temperature, with one rounding: c has that of scale too, which a score of 5 at a temperature
    // of 0.01 shows in the fifth decimal of a log-probability (1.3e-4 by c ln 2, 0.5e-4 so).
    __device__ __forceinline__ float log(float temperature, float scale) const {
#pragma clang fp contract(off)
        if (s != s || m == -INFINITY || m == INFINITY) return s != s ? s : m;
        const float c = m * scale, more = fmaf(m, scale, -c);  // the sum is s 2^c, or (s 2^-more) 2^(m scale)
        return m / temperature + (plain(m, scale) ? logf(s) - more * 0.693147181f : logf(s));
    }
};

struct PartSum {
    float m, s;
    uint32_t best, unused;  // the best candidate's score, ordered; 0: none
};

// Wavefronts per SIMD that the registers are bounded for: as many as spill no more than two.  A workgroup of 256 threads has one on
// each SIMD.
constexpr int SELECT_MAX_WAVES = 6;
constexpr int select_waves(bool bf16, RuleSet rules, int threads) {
    return threads == 1024 ? 4 : rules == RULES_ALL ? (bf16 ? 5 : 4) : rules == RULES_HISTORY && !bf16 ? 5 : SELECT_MAX_WAVES;
}
// Rounds of workgroups that the parts of all rows may take, and the parts that there can be: the context holds room for as many from
// its creation on (13 MB), so that no call allocates and a recorded one keeps its address.
constexpr int SELECT_MAX_ROUNDS = 8;
static int64_t select_max_parts(const als_ctx *ctx) { return (int64_t)ctx->num_cu * SELECT_MAX_WAVES * SELECT_MAX_ROUNDS; }

// Workgroup (x, y): part x (tiles_per_part tiles) of row y.  With one part a row it writes the answer, otherwise the part's
// candidates, 0 in the slots that are left, and its exponential sum.
template <bool BF16, RuleSet RULES, int NT>
__global__ __launch_bounds__(NT, select_waves(BF16, RULES, NT)) void select_kernel(const char *__restrict__ X, int64_t row_bytes,
                                                                                   int64_t first_row, uint32_t cols, int k,
                                                                                   uint32_t tiles_per_part, float temperature, float scale,
                                                                                   RuleArgs rules, Cand *__restrict__ part_cand,
                                                                                   PartSum *__restrict__ part_sum, int32_t *__restrict__ ids,
                                                                                   float *__restrict__ scores, float *__restrict__ lse) {
    typedef TileRow<BF16, NT> Row;
    constexpr int PER = Row::PER, PIECES = Row::PIECES, WAVES = NT / 64, TILE = Row::TILE;
    constexpr int STEPS = select_steps<NT>(), EACH = TILE_EPT / STEPS, CAP = select_room<NT>();
    extern __shared__ __align__(16) uint32_t words[];
    __shared__ Buffer<CAP> buf;
    __shared__ uint32_t wave_bar[WAVES], wave_kth[WAVES];
    __shared__ float wave_m[WAVES], wave_s[WAVES];
    __shared__ int added[3];  // candidates of a tile, by turns: the last one is cleared while this one is read
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, parts = gridDim.x;
    const uint32_t begin = blockIdx.x * tiles_per_part * TILE;
    const uint32_t end = min(cols, (blockIdx.x + 1) * tiles_per_part * TILE);  // items of the part
    const int64_t row = first_row + blockIdx.y;
    const char *scores_row = X + row * row_bytes;
    Row in;
    if (begin < end) in.load(scores_row, begin, cols, tid);
    RowRules<Row, RULES> mine;
    if constexpr (RULES != RULES_NONE) mine.begin(rules, row, begin, words, tid);
    ExpSum sum;
    float bar = -INFINITY;
    int have = 0, turn = 0;
    if (tid < 3) added[tid] = 0;
    __syncthreads();
    for (uint32_t first = begin; first < end; first += TILE) {
        float x[PIECES][PER];
        in.floats(x);
        if (first + TILE < end) in.load(scores_row, first + TILE, cols, tid);
        if constexpr (RULES != RULES_NONE) mine.apply(rules, first, cols, tid, x);
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
            // at least k reach the smallest of the wavefronts' ceil(k / WAVES)-th, and any wavefront's k-th: the latter counts
            // where some wavefronts have nothing (short rows, sets that allow a stretch of items)
            const WaveRanks ranks(ordered_bits(top));
            const uint32_t nth = ranks.nth((k + WAVES - 1) / WAVES), kth = ranks.nth(k);
            if (lane == 0) {
                wave_bar[wave] = nth;
                wave_kth[wave] = kth;
            }
            __syncthreads();
            uint32_t least = wave_bar[0], most_kth = wave_kth[0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) {
                least = min(least, wave_bar[i]);
                most_kth = max(most_kth, wave_kth[i]);
            }
            least = max(least, most_kth);
            bar = bar_below(least);
        }
        // The scores above the bar into the buffer: all at once, or, if they do not fit, step by step.
        for (int q0 = 0, q1 = STEPS; q0 < STEPS;) {
            if (__any(top > bar)) {
                float step_bar[STEPS];
#pragma unroll
                for (int q = 0; q < STEPS; ++q) step_bar[q] = q >= q0 && q < q1 ? bar : INFINITY;
                int above = 0;
#pragma unroll
                for (int i = 0; i < TILE_EPT; ++i) above += __popcll(__ballot(x[i / PER][i % PER] > step_bar[i / EACH]));
                int at = 0;
                if (lane == 0) at = atomicAdd(&added[turn], above);
                at = have + __builtin_amdgcn_readfirstlane(at);
#pragma unroll
                for (int i = 0; i < TILE_EPT; ++i) {
                    const unsigned long long who = __ballot(x[i / PER][i % PER] > step_bar[i / EACH]);
                    if (who) {
                        float v = x[i / PER][i % PER];
                        uint32_t from = first;
                        asm volatile("" : "+v"(v), "+s"(from));  // nothing is prepared for those that do not come here
                        const int place = at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                        if (v > step_bar[i / EACH] && place < CAP) buf.cand[place] = candidate(v, from + Row::item(i / PER, tid) + i % PER);
                        at += __popcll(who);
                    }
                }
            }
            __syncthreads();
            int count = have + __builtin_amdgcn_readfirstlane(added[turn]);
            if (tid == 0) added[turn == 0 ? 2 : turn - 1] = 0;
            turn = turn == 2 ? 0 : turn + 1;
            if (count > CAP) {
                q1 = 1;
                continue;
            }
            q0 = q1;
            q1 = q0 + 1;
            if (count > PART_SLOTS) {
                const Cand nth = buf.template cut_back<NT>(count, k, tid);
                count = k;
                // the tile's other steps may hold an equal score with a smaller id, later tiles may not
                bar = q0 == STEPS ? bar_at(nth) : bar_below((uint32_t)(nth >> 32));
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
constexpr int MERGE_SLOTS = 8;  // per thread, where all are read
template <int MERGE_THREADS> constexpr int merge_few() { return MERGE_SLOTS * MERGE_THREADS / PART_SLOTS; }  // parts of which all are read
template <int MERGE_THREADS>
__global__ __launch_bounds__(MERGE_THREADS) void select_merge_kernel(int64_t rows, int k, int parts, float temperature, float scale, const Cand *__restrict__ part_cand,
                                                                     const PartSum *__restrict__ part_sum, int32_t *__restrict__ ids,
                                                                     float *__restrict__ scores, float *__restrict__ lse) {
    constexpr int WAVES = MERGE_THREADS / 64, CAP = 2048, SLOTS = MERGE_SLOTS, LIST = 1024;
    static_assert(2 * MERGE_THREADS <= CAP, "");
    __shared__ Buffer<CAP> buf;
    __shared__ uint32_t wave_bar[WAVES];
    __shared__ int count, listed, list[LIST];
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
        if (parts <= merge_few<MERGE_THREADS>()) {
            Cand c[SLOTS];
            uint32_t best = 0;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                c[i] = i * MERGE_THREADS + tid < total ? cand[i * MERGE_THREADS + tid] : 0;
                best = max(best, (uint32_t)(c[i] >> 32));
            }
            if (wave == 0 && lane < parts) all.add(part[lane].m, part[lane].s, scale);
            const uint32_t nth = WaveRanks(best).nth((k + WAVES - 1) / WAVES);
            if (lane == 0) wave_bar[wave] = nth;
            __syncthreads();
            uint32_t least = wave_bar[0];  // at least k candidates reach it, if there are as many
            for (int i = 1; i < WAVES; ++i) least = min(least, wave_bar[i]);
            bar = max((Cand)least << 32, (Cand)1);
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) put(c[i], bar);
        } else {
            // the bar from the parts' best, dealt out to the wavefronts evenly, then the parts that reach it
            if (tid == 0) listed = 0;
            uint32_t best = 0;
            for (int p = lane * WAVES + wave; p < parts; p += MERGE_THREADS) best = max(best, part[p].best);
            const uint32_t nth = WaveRanks(best).nth((k + WAVES - 1) / WAVES);
            if (lane == 0) wave_bar[wave] = nth;
            __syncthreads();
            uint32_t least = wave_bar[0];
            for (int i = 1; i < WAVES; ++i) least = min(least, wave_bar[i]);
            bar = max((Cand)least << 32, (Cand)1);
            for (int p = tid; p < parts; p += MERGE_THREADS) {
                const PartSum v = part[p];
                if (v.best >= least) {
                    const int at = atomicAdd(&listed, 1);
                    if (at < LIST) list[at] = p;
                }
            }
            if (wave == 0)
                for (int p = lane; p < parts; p += 64) all.add(part[p].m, part[p].s, scale);
            __syncthreads();
            const bool fits = listed <= LIST;
            const int slots = (fits ? listed : parts) * PART_SLOTS;
            for (int i0 = tid; i0 < slots; i0 += MERGE_SLOTS * MERGE_THREADS) {
                Cand c[MERGE_SLOTS];
#pragma unroll
                for (int u = 0; u < MERGE_SLOTS; ++u) {
                    const int i = min(i0 + u * MERGE_THREADS, slots - 1);
                    c[u] = cand[(fits ? list[i / PART_SLOTS] : i / PART_SLOTS) * PART_SLOTS + i % PART_SLOTS];
                }
#pragma unroll
                for (int u = 0; u < MERGE_SLOTS; ++u)
                    if (i0 + u * MERGE_THREADS < slots) put(c[u], bar);
            }
        }
        __syncthreads();
        int have = count;
        if (have > CAP) {  // more than there is room for (equal scores): a few at a time
            have = 0;
            for (int i0 = 0; i0 < total; i0 += MERGE_THREADS) {
                __syncthreads();
                if (tid == 0) count = have;
                __syncthreads();
                if (i0 + tid < total) put(cand[i0 + tid], bar);
                __syncthreads();
                have = count;
                if (have > CAP - MERGE_THREADS) {
                    bar = buf.template cut_back<MERGE_THREADS>(have, k, tid);
                    have = k;
                }
            }
        }
        __syncthreads();
        if (have > 256) {
            buf.template cut_back<MERGE_THREADS>(have, k, tid);
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

template <bool BF16, RuleSet RULES, int NT>
static als_status select_launch(als_ctx *ctx, const als_matrix *X, const RuleArgs &a, int64_t parts, int64_t tiles_per_part, float temperature,
                                int k, int32_t *ids, float *scores, float *lse, hipStream_t s) {
    constexpr int TILE = NT * TILE_EPT;
    const float scale = 1.44269504f / temperature;
    Cand *cand = nullptr;
    PartSum *sums = nullptr;
    if (parts > 1) {
        cand = (Cand *)ctx->select_partials.p;
        sums = (PartSum *)(cand + select_max_parts(ctx) * PART_SLOTS);
    }
    if (NT == 1024) {  // two lists' words are 128 KB
        static const hipError_t attr = hipFuncSetAttribute((const void *)select_kernel<BF16, RULES, NT>,
                                                           hipFuncAttributeMaxDynamicSharedMemorySize, 2 * TILE * 4);  // once per process
        ALS_HIP(ctx, attr);
    }
    for (int64_t row = 0; row < X->rows; row += 65535)  // a grid's second dimension
        hipLaunchKernelGGL((select_kernel<BF16, RULES, NT>), dim3((unsigned)parts, (unsigned)std::min<int64_t>(X->rows - row, 65535)), dim3(NT),
                           rule_bytes(a, TILE), s, (const char *)X->data, X->ld * (BF16 ? 2 : 4), row, (uint32_t)X->cols, k,
                           (uint32_t)tiles_per_part, temperature, scale, a, cand, sums, ids, scores, lse);
    if (parts > 1) {
        auto merge = [&](auto threads) {
            hipLaunchKernelGGL((select_merge_kernel<threads()>), dim3((unsigned)std::min<int64_t>(X->rows, 1 << 20)), dim3(threads()), 0, s,
                               X->rows, k, (int)parts, temperature, scale, (const Cand *)cand, (const PartSum *)sums, ids, scores, lse);
        };
        if (parts <= merge_few<256>()) merge(std::integral_constant<int, 256>{});
        else merge(std::integral_constant<int, 1024>{});
    }
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

als_status select_setup(als_ctx *ctx) {
    return ensure(ctx, ctx->select_partials, (size_t)select_max_parts(ctx) * (PART_SLOTS * sizeof(Cand) + sizeof(PartSum)));
}

als_status launch_select(als_ctx *ctx, const als_matrix *X, const als_rules *rules, float temperature, int k, int32_t *ids,
                         float *scores, float *lse, hipStream_t s) {
    const RuleArgs a = rule_args(rules);
    const RuleSet set = rule_set(a);
    const bool bf = X->dtype == ALS_BF16, all = set == RULES_ALL;
    constexpr int TILE = 256 * TILE_EPT;
    const int64_t tiles = (X->cols + TILE - 1) / TILE;
    // Parts of a row.  The card holds `slots` workgroups at a time (select_waves of them per compute unit; LDS for a buffer and
    // the lists' words); a row's parts are chosen so that the rounds of workgroups are full: with r rounds a workgroup
    // walks ceil(tiles / parts) tiles, and beginning and ending a part costs about as much as four more.
    const int64_t lds_bytes = (int64_t)rule_bytes(a, TILE) + (int64_t)sizeof(Buffer<select_room<256>()>) + 256;
    const int64_t slots = ctx->num_cu * std::min<int64_t>(select_waves(bf, set, 256), 160 * 1024 / lds_bytes);
    int64_t per = tiles, least = INT64_MAX;
    for (int64_t r = 1; r <= SELECT_MAX_ROUNDS; ++r) {
        const int64_t p = std::max<int64_t>(1, std::min<int64_t>(tiles, slots * r / X->rows)), each = std::max<int64_t>(1, (tiles + p - 1) / p);
        const int64_t cost = (X->rows * ((tiles + each - 1) / each) + slots - 1) / slots * (each + 4);
        if (cost < least) {
            least = cost;
            per = each;
        }
    }
    const int64_t parts = std::max<int64_t>(1, (tiles + per - 1) / std::max<int64_t>(1, per));
    // One workgroup of 1024 threads per row where a row is short and the rows do not fill the card: no parts to merge.  With parts /
    // so, in us, k = 50: 1 x 16000 17 / 14, 64 x 30000 17 / 15, 256 x 128000 42 / 34, with lists, biases and sets 64 x 16000 21 / 18,
    // 256 x 128000 74 / 61; but 64 x 128000 26 / 30, 64 x 30000 with all rules 21 / 23, 2048 x 16000 42 / 83.  The curve is laid through
    // these; between a quarter of the card and all of it nothing was measured.
    const int64_t wide_tiles = (X->cols + 4 * TILE - 1) / (4 * TILE);
    const double fill = (double)X->rows / ctx->num_cu;
    const bool wide = parts > 1 && fill <= 1 && (double)wide_tiles <= (all ? 1 : 2) + (all ? 7 : 6) * fill * fill;
    auto typed = [&](auto b, auto r) {
        if (wide) return select_launch<b(), r(), 1024>(ctx, X, a, 1, wide_tiles, temperature, k, ids, scores, lse, s);
        return select_launch<b(), r(), 256>(ctx, X, a, parts, per, temperature, k, ids, scores, lse, s);
    };
    auto with = [&](auto r) { return bf ? typed(std::true_type{}, r) : typed(std::false_type{}, r); };
    if (all) return with(std::integral_constant<RuleSet, RULES_ALL>{});
    if (set == RULES_HISTORY) return with(std::integral_constant<RuleSet, RULES_HISTORY>{});
    return with(std::integral_constant<RuleSet, RULES_NONE>{});
}

}  // namespace als
