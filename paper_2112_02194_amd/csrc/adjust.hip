// Scores changed by rules (als_adjust): penalties for items a row has had before, biases, sets of allowed items.
// One read and one write of the matrix; memory bound.
#include <algorithm>

#include "score_rules.h"

namespace als {

// Workgroup w works on tile w / rows of row w % rows: the rows of one tile share its biases and a shared set of allowed items.
template <bool BF_IN, bool BF_OUT>
__global__ __launch_bounds__(TILE_THREADS) void adjust_kernel(const void *X, int64_t ldx, void *Y, int64_t ldy, int64_t rows,
                                                              int64_t cols, int64_t work, RuleArgs rules) {
    extern __shared__ __align__(16) uint32_t words[];
    uint32_t *count = words, *place = words + (rules.history.indptr ? TILE : 0);
    const int tid = threadIdx.x;
    for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const int64_t row = w % rows, first = w / rows * TILE;
        const RowRules mine(rules, row);
        float x[TILE_EPT / 4][4];
#pragma unroll
        for (int j = 0; j < TILE_EPT / 4; ++j) {
            const int64_t at = first + tile_item(j, tid);
            const int valid = (int)std::max<int64_t>(0, std::min<int64_t>(4, cols - at));
            load4<BF_IN>(X, row * ldx + at, valid, x[j]);
        }
        tile_lists(rules, mine, first, count, place, tid);
#pragma unroll
        for (int j = 0; j < TILE_EPT / 4; ++j) {
            const int item = tile_item(j, tid);
            const int64_t at = first + item;
            const int valid = (int)std::max<int64_t>(0, std::min<int64_t>(4, cols - at));
            apply_rules(rules, mine, first, item, valid, count, place, x[j]);
            store4<BF_OUT>(Y, row * ldy + at, valid, x[j]);
        }
    }
}

als_status launch_adjust(als_ctx *ctx, const als_matrix *X, const als_rules *rules, const als_matrix *Y, hipStream_t s) {
    const RuleArgs a = rule_args(rules);
    const int64_t work = (X->cols + TILE - 1) / TILE * X->rows;
    const dim3 grid((unsigned)std::min<int64_t>(work, 1 << 22)), block(TILE_THREADS);
    const size_t lds = (size_t)rule_words(a) * 4;
    const bool bi = X->dtype == ALS_BF16, bo = Y->dtype == ALS_BF16;
#define ADJUST(I, O) \
    hipLaunchKernelGGL((adjust_kernel<I, O>), grid, block, lds, s, X->data, X->ld, Y->data, Y->ld, X->rows, X->cols, work, a)
    if (bi && bo) ADJUST(true, true);
    else if (bi) ADJUST(true, false);
    else if (bo) ADJUST(false, true);
    else ADJUST(false, false);
#undef ADJUST
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
