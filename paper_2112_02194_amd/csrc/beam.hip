// Beam search: the best continuations of groups of beams (als_beam), and what goes with the beams in their new order (als_reorder).
//
// beam kernel     one workgroup per group: candidates of all beams (up to 4096, sixteen a thread) in registers, a bar that at
//                 least `beams` of them reach (the wavefronts' best lanes), those above it to LDS, cut back by digits where they
//                 are many, and ranked by counting.  A chain of loads and barriers: 4 us for 8 beams of 8, 9 for 128 groups of 32
//                 beams of 32 (33 KB a group: memory has no part in it)
// reorder kernel  a workgroup takes a slice of columns of all rows of a group (of several groups where rows are short): it reads the
//                 slice of every parent, then writes.  So a group's rows may change places within the buffer; rows that
//                 stay are neither read nor written there.  Memory bound: 4096 rows of 126 KB 174 us, 5.9 TB/s (a parent that several
//                 beams have is read once from memory); 7.7 us for 8 rows, the odd ends of rows one after the other
#include <algorithm>
#include <cmath>
#include <iterator>
#include <type_traits>

#include "candidates.h"

namespace als {

constexpr int BEAM_THREADS = 256, BEAM_MOST = ALS_TOPK_MAX_K * ALS_TOPK_MAX_K;

struct BeamArgs {
    const int32_t *ids;
    const float *scores, *lse, *totals;
    const int32_t *last, *lengths;
    const float *factors;
    int32_t beams, k, n_factors, end;
    float temperature;
};

// SLOTS candidates a thread: a group has at most 256 SLOTS.
template <int SLOTS>
__global__ __launch_bounds__(BEAM_THREADS) void beam_kernel(BeamArgs a, int64_t groups, int32_t *__restrict__ parents, int32_t *__restrict__ items,
                                                          float *__restrict__ totals, int32_t *__restrict__ lengths) {
    constexpr int WAVES = BEAM_THREADS / 64, CAP = SLOTS * BEAM_THREADS;
    static_assert(CAP <= BEAM_MOST, "");
    __shared__ Buffer<CAP> buf;
    __shared__ float all_totals[CAP];
    __shared__ int32_t beam_length[ALS_TOPK_MAX_K], beam_ended[ALS_TOPK_MAX_K];
    __shared__ uint32_t wave_bar[WAVES];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.beams * a.k;
    for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
        const int64_t first = group * a.beams;
        // what all candidates are made of, under way together
        int at[SLOTS], beam[SLOTS], id[SLOTS], last[SLOTS], length[SLOTS];
        float score[SLOTS], lse[SLOTS], before[SLOTS];
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            at[i] = i * BEAM_THREADS + tid;
            const int inside = min(at[i], n - 1);
            beam[i] = (int)((uint32_t)inside / (uint32_t)a.k);
            const int64_t row = first + beam[i];
            id[i] = a.ids[first * a.k + inside];
            score[i] = a.scores[first * a.k + inside];
            lse[i] = a.lse ? a.lse[row] : 0.f;
            before[i] = a.totals ? a.totals[row] : beam[i] == 0 ? 0.f : -INFINITY;
            last[i] = a.last ? a.last[row] : 0;
            length[i] = a.lengths ? a.lengths[row] : 0;
        }
        if (tid == 0) count = 0;
        Cand c[SLOTS];
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
#pragma clang fp contract(off)
            const bool ended = a.last && last[i] == a.end, leading = at[i] == beam[i] * a.k;
            length[i] += !ended;
            const float live = before[i] + (score[i] / a.temperature - lse[i]);
            const float total = ended ? (leading ? before[i] : -INFINITY) : id[i] >= 0 ? live : -INFINITY;
            float key = total;
            if (a.factors) key = total * a.factors[min(max(length[i], 0), a.n_factors - 1)];
            // the total as well as the key: a negative factor makes +inf of a total of -inf
            c[i] = at[i] < n && total > -INFINITY && key > -INFINITY ? candidate(key, (uint32_t)at[i]) : 0;
            all_totals[at[i]] = total;
            if (at[i] < n && leading) {
                beam_length[beam[i]] = length[i];
                beam_ended[beam[i]] = ended;
            }
            best = max(best, (uint32_t)(c[i] >> 32));
        }
        const uint32_t nth = WaveRanks(best).nth((a.beams + WAVES - 1) / WAVES);
        if (lane == 0) wave_bar[wave] = nth;
        __syncthreads();
        uint32_t least = wave_bar[0];  // at least `beams` candidates reach it, if there are as many
#pragma unroll
        for (int i = 1; i < WAVES; ++i) least = min(least, wave_bar[i]);
        const Cand bar = max((Cand)least << 32, (Cand)1);
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
            if (c[i] >= bar) buf.cand[atomicAdd(&count, 1)] = c[i];
        __syncthreads();
        int have = count;
        if (have > BEAM_THREADS) {
            buf.template cut_back<BEAM_THREADS>(have, a.beams, tid);
            have = a.beams;
        }
        if (tid < have) {
            const Cand mine = buf.cand[tid];
            int rank = 0, i = 0;
            for (; i + 8 <= have; i += 8) {
#pragma unroll
                for (int u = 0; u < 8; ++u) rank += buf.cand[i + u] > mine;
            }
            for (; i < have; ++i) rank += buf.cand[i] > mine;
            if (rank < a.beams) {
                const int place = (int)~(uint32_t)mine, from = (int)((uint32_t)place / (uint32_t)a.k);
                parents[first + rank] = (int32_t)(first + from);
                items[first + rank] = beam_ended[from] ? a.end : a.ids[first * a.k + place];
                totals[first + rank] = all_totals[place];
                if (lengths) lengths[first + rank] = beam_length[from];
            }
        }
        if (tid >= have && tid < a.beams) {
            parents[first + tid] = -1;
            items[first + tid] = -1;
            totals[first + tid] = -INFINITY;
            if (lengths) lengths[first + tid] = 0;
        }
        __syncthreads();
    }
}

als_status launch_beam(als_ctx *ctx, const als_beams *in, int32_t *parents, int32_t *items, float *totals, int32_t *lengths, hipStream_t s) {
    const BeamArgs a{in->ids, in->scores, in->lse, in->totals, in->last, in->lengths, in->factors, in->beams, in->k, in->n_factors, in->end, in->temperature};
    auto go = [&](auto slots) {
        hipLaunchKernelGGL((beam_kernel<slots()>), dim3((unsigned)std::min<int64_t>(in->groups, 1 << 20)), dim3(BEAM_THREADS), 0, s, a, in->groups,
                           parents, items, totals, lengths);
    };
    // as few slots as the group's candidates take: a slot is work and registers for every thread
    const int n = in->beams * in->k;
    if (n <= BEAM_THREADS) go(std::integral_constant<int, 1>{});
    else if (n <= 4 * BEAM_THREADS) go(std::integral_constant<int, 4>{});
    else go(std::integral_constant<int, 16>{});
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

// ---------------------------------------------------------------------------------------------- reorder

constexpr int REORDER_THREADS = 256, REORDER_EACH = 8, REORDER_PIECES = REORDER_THREADS * REORDER_EACH;  // of 16 bytes
constexpr int REORDER_STATES = 32;  // of a launch: they are its arguments
static_assert(REORDER_PIECES >= 16 * ALS_TOPK_MAX_K, "a slice of a group's rows is at least 256 bytes wide");

struct ReorderState {
    const char *x;
    char *y;
    int64_t ldx, ldy, bytes;  // of a row
    uint32_t slices;          // of a row
    int32_t width;            // pieces of a slice: 2^width
    int32_t groups;           // of a slice
    int32_t es;
};
struct ReorderStates {
    uint32_t slices;
    int n;
    uint32_t first[REORDER_STATES];  // numbers of the states' first slices in the launch
    ReorderState t[REORDER_STATES];
};

__global__ __launch_bounds__(REORDER_THREADS) void reorder_kernel(ReorderStates all, const int32_t *__restrict__ parents, int64_t rows, int beams) {
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    typedef Words Any __attribute__((aligned(2)));
    for (uint32_t slice = blockIdx.x; slice < all.slices; slice += gridDim.x) {
        // the state that has the slice: the arguments come in one go, where a search would wait for each
        int j = -1;
#pragma unroll
        for (int i = 0; i < REORDER_STATES; ++i) j += all.first[i] <= slice;
        const ReorderState &t = all.t[j];
        const uint32_t at = slice - all.first[j], some = at / t.slices;
        const int64_t first = (int64_t)some * t.groups * beams, end = min(rows, first + (int64_t)t.groups * beams);
        const int64_t column = ((int64_t)(at - some * t.slices) << t.width) * 16;
        const bool in_place = t.x == t.y;
        Words v[REORDER_EACH];
        int left[REORDER_EACH];  // bytes of the piece that are written
        int32_t from[REORDER_EACH];
        // all parents, then all pieces: each of the two waits for memory once
#pragma unroll
        for (int i = 0; i < REORDER_EACH; ++i) {
            const int piece = i * REORDER_THREADS + threadIdx.x;
            from[i] = parents[min(first + (piece >> t.width), rows - 1)];
        }
#pragma unroll
        for (int i = 0; i < REORDER_EACH; ++i) {
            const int piece = i * REORDER_THREADS + threadIdx.x;
            const int64_t row = first + (piece >> t.width), byte = column + (int64_t)(piece & ((1 << t.width) - 1)) * 16;
            const int32_t group = (int32_t)(row - (uint32_t)row % (uint32_t)beams);
            left[i] = row < end && byte < t.bytes && !(in_place && from[i] == row) ? (int)min(t.bytes - byte, (int64_t)16) : 0;
            const bool there = from[i] >= group && from[i] - group < beams && left[i] > 0;
            v[i] = Words{0, 0, 0, 0};
            if (t.bytes >= 16) {  // otherwise no row has a whole piece
                const bool whole = there && left[i] == 16;
                const Words w = *(const Any *)(t.x + (whole ? (int64_t)from[i] * t.ldx + byte : 0));
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] = whole ? w[e] : 0;
            }
            if (there && left[i] < 16) {  // elements of 2 or 4 bytes up to the row's end
                const char *p = t.x + (int64_t)from[i] * t.ldx + byte;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (4 * e < left[i]) {
                        if (t.es == 4) v[i][e] = ((const uint32_t *)p)[e];
                        else v[i][e] = ((const uint16_t *)p)[2 * e] | (4 * e + 2 < left[i] ? (uint32_t)((const uint16_t *)p)[2 * e + 1] << 16 : 0u);
                    }
            }
        }
        if (in_place) {
            // every value is there before any row is written
#pragma unroll
            for (int i = 0; i < REORDER_EACH; ++i) asm volatile("" : "+v"(v[i]));
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < REORDER_EACH; ++i) {
            const int piece = i * REORDER_THREADS + threadIdx.x;
            char *p = t.y + (first + (piece >> t.width)) * t.ldy + column + (int64_t)(piece & ((1 << t.width) - 1)) * 16;
            if (left[i] == 16) {
                *(Any *)p = v[i];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (4 * e < left[i]) {
                        if (t.es == 4) {
                            ((uint32_t *)p)[e] = v[i][e];
                        } else {
                            ((uint16_t *)p)[2 * e] = (uint16_t)v[i][e];
                            if (4 * e + 2 < left[i]) ((uint16_t *)p)[2 * e + 1] = (uint16_t)(v[i][e] >> 16);
                        }
                    }
            }
        }
    }
}

als_status launch_reorder(als_ctx *ctx, const int32_t *parents, int64_t groups, int beams, const als_matrix *X, const als_matrix *Y, int n,
                          hipStream_t s) {
    const int64_t rows = groups * beams;
    for (int j = 0; j < n;) {
        ReorderStates all{};
        std::fill(std::begin(all.first), std::end(all.first), ~0u);
        for (; j < n && all.n < REORDER_STATES; ++j) {
            const als_matrix &x = X[j], &y = Y ? Y[j] : X[j];
            if (x.cols == 0) continue;
            ReorderState &t = all.t[all.n++];
            t.es = x.dtype == ALS_BF16 ? 2 : 4;
            t.x = (const char *)x.data;
            t.y = (char *)y.data;
            t.ldx = x.ld * t.es;
            t.ldy = y.ld * t.es;
            t.bytes = x.cols * t.es;
            const int64_t pieces = (t.bytes + 15) / 16;
            while (((int64_t)1 << t.width) < pieces && (2 << t.width) * beams <= REORDER_PIECES) ++t.width;
            const int64_t slices = (pieces + (1 << t.width) - 1) >> t.width;
            t.groups = std::max(1, REORDER_PIECES / (beams << t.width));
            const int64_t every = (groups + t.groups - 1) / t.groups;
            if (slices > (1 << 30) / every) return fail(ctx, ALS_ESHAPE, "als_reorder: X has too many elements");
            t.slices = (uint32_t)slices;
            all.first[all.n - 1] = all.slices;
            all.slices += (uint32_t)(every * slices);
        }
        if (all.n)
            hipLaunchKernelGGL(reorder_kernel, dim3(std::min<uint32_t>(all.slices, 1u << 22)), dim3(REORDER_THREADS), 0, s, all, parents, rows, beams);
    }
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
