// Beam search: the best continuations of groups of beams (als_beam), and what goes with the beams in their new order (als_reorder).
//
// beam kernel     one workgroup per group: candidates of all beams (up to 4096, sixteen a thread) in registers, a bar that at
//                 least `beams` of them reach (the wavefronts' best lanes), those above it to LDS, cut back by digits where they
//                 are many, and ranked by counting
// reorder kernel  a workgroup takes a slice of columns of all rows of a group (of several groups where rows are short): it reads the
//                 slice of every parent, then writes.  So a group's rows may change places within the buffer; rows that
//                 stay are neither read nor written there
#include <algorithm>
#include <cmath>

#include "candidates.h"

namespace als {

constexpr int BEAM_THREADS = 256, BEAM_SLOTS = ALS_TOPK_MAX_K * ALS_TOPK_MAX_K / BEAM_THREADS;

struct BeamArgs {
    const int32_t *ids;
    const float *scores, *lse, *totals;
    const int32_t *last, *lengths;
    const float *factors;
    int32_t beams, k, n_factors, end;
    float temperature;
};

// Candidate `place` of beam `beam` of the group whose first row is `first`.
__device__ __forceinline__ float beam_total(const BeamArgs &a, int64_t first, int beam, int place, bool &ended, int &length, int &item) {
#pragma clang fp contract(off)
    const int64_t row = first + beam;
    ended = a.last && a.last[row] == a.end;
    length = (a.lengths ? a.lengths[row] : 0) + (ended ? 0 : 1);
    const float before = a.totals ? a.totals[row] : beam == 0 ? 0.f : -INFINITY;
    if (ended) {
        item = a.end;
        return place == 0 ? before : -INFINITY;
    }
    item = a.ids[row * a.k + place];
    if (item < 0) return -INFINITY;
    const float s = a.scores[row * a.k + place] / a.temperature;
    return before + (s - (a.lse ? a.lse[row] : 0.f));
}

__global__ __launch_bounds__(BEAM_THREADS) void beam_kernel(BeamArgs a, int64_t groups, int32_t *__restrict__ parents, int32_t *__restrict__ items,
                                                          float *__restrict__ totals, int32_t *__restrict__ lengths) {
    constexpr int WAVES = BEAM_THREADS / 64;
    __shared__ Buffer<ALS_TOPK_MAX_K * ALS_TOPK_MAX_K> buf;
    __shared__ uint32_t wave_bar[WAVES];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.beams * a.k;
    for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
        const int64_t first = group * a.beams;
        Cand c[BEAM_SLOTS];
        uint32_t best = 0;
        if (tid == 0) count = 0;
#pragma unroll
        for (int i = 0; i < BEAM_SLOTS; ++i) {
            const int at = i * BEAM_THREADS + tid;
            c[i] = 0;
            if (at < n) {
                bool ended;
                int length, item;
                const int beam = at / a.k;
                float key = beam_total(a, first, beam, at - beam * a.k, ended, length, item);
                if (a.factors) key *= a.factors[min(max(length, 0), a.n_factors - 1)];
                if (key > -INFINITY) c[i] = candidate(key, (uint32_t)at);
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
        for (int i = 0; i < BEAM_SLOTS; ++i)
            if (c[i] >= bar) buf.cand[atomicAdd(&count, 1)] = c[i];
        __syncthreads();
        int have = count;
        if (have > BEAM_THREADS) {
            buf.template cut_back<BEAM_THREADS>(have, a.beams, tid);
            have = a.beams;
        }
        if (tid < have) {
            const Cand mine = buf.cand[tid];
            int rank = 0;
            for (int i = 0; i < have; ++i) rank += buf.cand[i] > mine;
            if (rank < a.beams) {
                bool ended;
                int length, item;
                const int at = (int)~(uint32_t)mine, beam = at / a.k;
                const float total = beam_total(a, first, beam, at - beam * a.k, ended, length, item);
                parents[first + rank] = (int32_t)(first + beam);
                items[first + rank] = item;
                totals[first + rank] = total;
                if (lengths) lengths[first + rank] = length;
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
    hipLaunchKernelGGL(beam_kernel, dim3((unsigned)std::min<int64_t>(in->groups, 1 << 20)), dim3(BEAM_THREADS), 0, s, a, in->groups, parents, items,
                       totals, lengths);
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
    int64_t first;            // number of the state's first slice in the launch
    int64_t slices;           // of a row
    int32_t width;            // pieces of a slice: 2^width
    int32_t groups;           // of a slice
    int32_t es;
};
struct ReorderStates {
    ReorderState t[REORDER_STATES];
    int64_t slices;
    int n;
};

__global__ __launch_bounds__(REORDER_THREADS) void reorder_kernel(ReorderStates all, const int32_t *__restrict__ parents, int64_t rows, int beams) {
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    typedef Words Any __attribute__((aligned(2)));
    int j = 0;
    for (int64_t slice = blockIdx.x; slice < all.slices; slice += gridDim.x) {
        while (j + 1 < all.n && slice >= all.t[j + 1].first) ++j;
        const ReorderState &t = all.t[j];
        const int64_t at = slice - t.first, some = at / t.slices;
        const int64_t first = some * t.groups * beams, end = min(rows, first + (int64_t)t.groups * beams);
        const int64_t column = ((at - some * t.slices) << t.width) * 16;
        const bool in_place = t.x == t.y;
        Words v[REORDER_EACH];
        int64_t to[REORDER_EACH];
        int left[REORDER_EACH];  // bytes of the piece
#pragma unroll
        for (int i = 0; i < REORDER_EACH; ++i) {
            const int piece = i * REORDER_THREADS + threadIdx.x;
            const int64_t row = first + (piece >> t.width), byte = column + (int64_t)(piece & ((1 << t.width) - 1)) * 16;
            left[i] = 0;
            to[i] = row * t.ldy + byte;
            v[i] = Words{0, 0, 0, 0};
            if (row < end && byte < t.bytes) {
                const int from = parents[row], group = (int)row - (int)((uint32_t)row % (uint32_t)beams);
                if (!in_place || from != (int)row) {
                    left[i] = (int)min(t.bytes - byte, (int64_t)16);
                    if (from >= group && from - group < beams) {
                        const char *p = t.x + (int64_t)from * t.ldx + byte;
                        if (left[i] == 16) {
                            v[i] = *(const Any *)p;
                        } else {  // elements of 2 or 4 bytes up to the row's end
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (4 * e < left[i]) {
                                    if (t.es == 4) v[i][e] = ((const uint32_t *)p)[e];
                                    else v[i][e] = ((const uint16_t *)p)[2 * e] | (4 * e + 2 < left[i] ? (uint32_t)((const uint16_t *)p)[2 * e + 1] << 16 : 0u);
                                }
                        }
                    }
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
            char *p = t.y + to[i];
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
            t.slices = (pieces + (1 << t.width) - 1) >> t.width;
            t.groups = std::max(1, REORDER_PIECES / (beams << t.width));
            t.first = all.slices;
            all.slices += (groups + t.groups - 1) / t.groups * t.slices;
        }
        if (all.n)
            hipLaunchKernelGGL(reorder_kernel, dim3((unsigned)std::min<int64_t>(all.slices, 1 << 22)), dim3(REORDER_THREADS), 0, s, all, parents, rows, beams);
    }
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
