// Scores of queries against a table in 4 bits an entry (als_scores): S[q][i] = sum_g scale(i, g) sum_{j in g} Q[q][j] code(i, j).
#include <algorithm>

#include "als_internal.h"

namespace als {

// One thread per item and query: codes widened, products and sums in fp32, a group's sum times its scale.
template <bool BF_Q, bool BF_S, int D>
__global__ __launch_bounds__(256) void scores_kernel(const void *__restrict__ Q, int64_t ldq, int64_t nq,
                                                     const uint32_t *__restrict__ codes, const uint16_t *__restrict__ scales,
                                                     int group, int64_t n, void *__restrict__ S, int64_t lds) {
    __shared__ float q[D];
    const int64_t stretches = (n + 255) / 256;
    for (int64_t w = blockIdx.x; w < stretches * nq; w += gridDim.x) {
        const int64_t row = w % nq, item = w / nq * 256 + threadIdx.x;
        __syncthreads();
        if (threadIdx.x < D) q[threadIdx.x] = load_elem<BF_Q>(Q, row * ldq + threadIdx.x);
        __syncthreads();
        if (item >= n) continue;
        float sum = 0.f;
        for (int g = 0; g < D / group; ++g) {
            float part = 0.f;
            for (int j = 0; j < group / 8; ++j) {
                const int32_t word = (int32_t)codes[item * (D / 8) + g * (group / 8) + j];
#pragma unroll
                for (int e = 0; e < 8; ++e) part = fmaf(q[g * group + 8 * j + e], (float)(word << (28 - 4 * e) >> 28), part);
            }
            sum = fmaf(part, bf16_to_f32(scales[item * (D / group) + g]), sum);
        }
        store_elem<BF_S>(S, row * lds + item, sum);
    }
}

als_status launch_scores(als_ctx *ctx, const als_table *Q, const als_qtable *T, const als_matrix *S, hipStream_t s) {
    const int64_t work = (T->rows + 255) / 256 * Q->rows;
    const dim3 grid((unsigned)std::min<int64_t>(work, 1 << 20));
    auto go = [&](auto bq, auto bs, auto d) {
        hipLaunchKernelGGL((scores_kernel<bq(), bs(), d()>), grid, dim3(256), 0, s, Q->data, Q->ld, Q->rows, (const uint32_t *)T->codes,
                           (const uint16_t *)T->scales, T->group, T->rows, S->data, S->ld);
    };
    auto typed = [&](auto bq, auto bs) {
        switch (Q->d) {
            case 16: return go(bq, bs, std::integral_constant<int, 16>{});
            case 32: return go(bq, bs, std::integral_constant<int, 32>{});
            case 64: return go(bq, bs, std::integral_constant<int, 64>{});
            default: return go(bq, bs, std::integral_constant<int, 128>{});
        }
    };
    const bool bq = Q->dtype == ALS_BF16, bs = S->dtype == ALS_BF16;
    if (bq && bs) typed(std::true_type{}, std::true_type{});
    else if (bq) typed(std::true_type{}, std::false_type{});
    else if (bs) typed(std::false_type{}, std::true_type{});
    else typed(std::false_type{}, std::false_type{});
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
