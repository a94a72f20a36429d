// Candidates of a selection: what als_select keeps of a row of scores, and als_beam of a group of beams.
//
// A candidate is one whole number: the score as ordered bits above, the complement of the item id (of the place) below, so that a
// larger number is a better score, or an equal one with a smaller id.
#pragma once

#include "als_internal.h"

namespace als {

typedef unsigned long long Cand;

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

}  // namespace als
