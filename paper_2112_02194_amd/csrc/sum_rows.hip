// Sums of a table's rows over the rows of a CSR matrix (als_sum_rows).
#include <algorithm>
#include <type_traits>

#include "entry_rows.h"

namespace als {

constexpr int SUM_THREADS = 256;

template <int D, bool BF>
__global__ __launch_bounds__(SUM_THREADS) void sum_rows_kernel(Lists y, const float *values, RowsOf E, RowsOf X) {
    constexpr int N = BF ? 8 : 4, L = D / N;
    const int lane = threadIdx.x % L;
    for (int64_t u = (blockIdx.x * (int64_t)SUM_THREADS + threadIdx.x) / L; u < y.rows; u += (int64_t)gridDim.x * SUM_THREADS / L) {
        int64_t b, e;
        row_range(y.indptr, u, y.nnz, b, e);
        float sum[N] = {};
        for (int64_t p = b; p < e; ++p) {
            const int64_t i = y.ids[p];
            if (i < 0 || i >= y.cols) continue;
            const float w = values ? values[p] : 1.f;
            float x[N];
            load_piece<BF, N>(E.p + i * E.ld, lane, x);
#pragma unroll
            for (int c = 0; c < N; ++c) sum[c] = fmaf(w, x[c], sum[c]);
        }
        store_piece(X, u, lane, sum);
    }
}

als_status launch_sum_rows(als_ctx *ctx, const als_csr *Y, const als_table *E, const als_table *X, hipStream_t s) {
    auto go = [&](auto d, auto bf) {
        const int64_t lanes = d() / (bf() ? 8 : 4);
        const unsigned grid = (unsigned)std::min<int64_t>((Y->rows * lanes + SUM_THREADS - 1) / SUM_THREADS, 1 << 22);
        hipLaunchKernelGGL((sum_rows_kernel<d(), bf()>), dim3(grid), dim3(SUM_THREADS), 0, s, lists_of(Y), Y->values, rows_of(E), rows_of(X));
    };
    auto typed = [&](auto d) { E->dtype == ALS_BF16 ? go(d, std::true_type{}) : go(d, std::false_type{}); };
    switch (E->d) {
        case 16: typed(std::integral_constant<int, 16>{}); break;
        case 32: typed(std::integral_constant<int, 32>{}); break;
        case 64: typed(std::integral_constant<int, 64>{}); break;
        default: typed(std::integral_constant<int, 128>{}); break;
    }
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
