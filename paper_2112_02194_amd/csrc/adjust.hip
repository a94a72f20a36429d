// Scores changed by rules (als_adjust): penalties for items a row has had before, biases, sets of allowed items.
// One read and one write of the matrix; memory bound: 256 rows of 1M fp32 with their histories 407 us, 5.0 TB/s, a copy's rate.
// A workgroup per tile: nothing is carried from tile to tile, and the lists of a row, read again for each of its tiles, come from
// the L2.
#include <algorithm>

#include "score_rules.h"

namespace als {

constexpr int ADJUST_THREADS = 256, ADJUST_TILE = ADJUST_THREADS * TILE_EPT;

// Workgroup (x, y) works on tile y of row x: the rows of one tile share its biases and a shared set of allowed items.
template <bool BF_IN, bool BF_OUT>
__global__ __launch_bounds__(ADJUST_THREADS) void adjust_kernel(const void *X, int64_t ldx, void *Y, int64_t ldy, int64_t rows,
                                                              uint32_t cols, RuleArgs rules) {
    typedef TileRow<BF_IN, ADJUST_THREADS> Row;
    constexpr uint32_t TILE = Row::TILE;
    extern __shared__ __align__(16) uint32_t words[];
    const int tid = threadIdx.x;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x)
        for (uint32_t first = blockIdx.y * TILE; first < cols; first += gridDim.y * TILE) {
        Row in;
        in.load((const char *)X + row * ldx * (BF_IN ? 2 : 4), first, cols, tid);
        RowRules<Row, RULES_ALL> mine;
        mine.begin(rules, row, first, words, tid);
        float x[Row::PIECES][Row::PER];
        in.floats(x);
        mine.apply(rules, first, cols, tid, x);
        char *out = (char *)Y + (row * ldy + first) * (BF_OUT ? 2 : 4);
        const uint32_t left = cols - first;
#pragma unroll
        for (int j = 0; j < Row::PIECES; ++j)
#pragma unroll
            for (int q = 0; q < Row::PER; q += 4) {
                const uint32_t at = Row::item(j, tid) + q;
                typedef __bf16 Half __attribute__((ext_vector_type(4)));
                typedef Half AnyHalf __attribute__((aligned(2)));
                typedef float Full __attribute__((ext_vector_type(4)));
                typedef Full AnyFull __attribute__((aligned(4)));
                const Full v = {x[j][q], x[j][q + 1], x[j][q + 2], x[j][q + 3]};
                if (at + 4 <= left) {
                    if constexpr (BF_OUT) *(AnyHalf *)(out + at * 2) = __builtin_convertvector(v, Half);
                    else *(AnyFull *)(out + at * 4) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (at + e < left) {
                            if constexpr (BF_OUT) ((__bf16 *)out)[at + e] = (__bf16)v[e];
                            else ((float *)out)[at + e] = v[e];
                        }
                }
            }
        __syncthreads();  // the next tile's lists take the same words
    }
}

als_status launch_adjust(als_ctx *ctx, const als_matrix *X, const als_rules *rules, const als_matrix *Y, hipStream_t s) {
    const RuleArgs a = rule_args(rules);
    const dim3 grid((unsigned)std::min<int64_t>(X->rows, 1 << 16), (unsigned)std::min<int64_t>((X->cols + ADJUST_TILE - 1) / ADJUST_TILE, 1 << 15));
    const dim3 block(ADJUST_THREADS);
    const bool bi = X->dtype == ALS_BF16, bo = Y->dtype == ALS_BF16;
    auto go = [&](auto in, auto out) {
        hipLaunchKernelGGL((adjust_kernel<in(), out()>), grid, block, rule_bytes(a, ADJUST_TILE), s, X->data, X->ld, Y->data, Y->ld, X->rows,
                           (uint32_t)X->cols, a);
    };
    if (bi && bo) go(std::true_type{}, std::true_type{});
    else if (bi) go(std::true_type{}, std::false_type{});
    else if (bo) go(std::false_type{}, std::true_type{});
    else go(std::false_type{}, std::false_type{});
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
