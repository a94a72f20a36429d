// Tables in 4 bits an entry with one bf16 scale per group of entries (als_quantize, als_dequantize).
// A lane owns eight consecutive entries (four bytes of codes); the lanes of a group share its largest magnitude by shuffles.
// One read and one write of everything; memory bound.
#include <algorithm>

#include "als_internal.h"

namespace als {

template <bool BF16, int D>
__global__ __launch_bounds__(256) void quantize_kernel(const void *__restrict__ X, int64_t ld, int64_t pieces, int group_lanes,
                                                       uint32_t *__restrict__ codes, uint16_t *__restrict__ scales) {
    // pieces is a multiple of the lanes of a group, and so is the stride: the lanes of a group go round together
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t off = i / (D / 8) * ld + i % (D / 8) * 8;
        float x[2][4];
        load_vec<4, BF16>(X, off, x[0]);
        load_vec<4, BF16>(X, off + 4, x[1]);
        // the largest magnitude as bits: they order like the values, with infinity and NaN above all others
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e / 4][e % 4]) & 0x7fffffffu);
        for (int m = 1; m < group_lanes; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
        const uint16_t sb = f32_to_bf16_rne(__uint_as_float(top) / 7.f);
        const float s = bf16_to_f32(sb);
        const bool usable = s > 0.f && s < INFINITY;
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float c = fminf(fmaxf(rintf(x[e / 4][e % 4] / s), -7.f), 7.f);
            word |= ((uint32_t)(int)(usable ? c : 0.f) & 15u) << (4 * e);
        }
        codes[i] = word;
        if (threadIdx.x % group_lanes == 0) scales[i / group_lanes] = sb;
    }
}

template <bool BF16, int D>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint32_t *__restrict__ codes, const uint16_t *__restrict__ scales,
                                                         int64_t pieces, int group_lanes, void *__restrict__ X, int64_t ld) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t off = i / (D / 8) * ld + i % (D / 8) * 8;
        const int32_t word = (int32_t)codes[i];
        const float s = bf16_to_f32(scales[i / group_lanes]);
#pragma unroll
        for (int e = 0; e < 8; ++e) store_elem<BF16>(X, off + e, (float)(word << (28 - 4 * e) >> 28) * s);
    }
}

static dim3 quantize_grid(const als_ctx *ctx, int64_t pieces) {
    return dim3((unsigned)std::min<int64_t>((pieces + 255) / 256, (int64_t)ctx->num_cu * 64));
}

als_status launch_quantize(als_ctx *ctx, const als_table *X, const als_qtable *T, hipStream_t s) {
    const int64_t pieces = X->rows * (X->d / 8);
    auto go = [&](auto bf, auto d) {
        hipLaunchKernelGGL((quantize_kernel<bf(), d()>), quantize_grid(ctx, pieces), dim3(256), 0, s, X->data, X->ld, pieces,
                           T->group / 8, (uint32_t *)T->codes, (uint16_t *)T->scales);
    };
    auto typed = [&](auto bf) {
        switch (X->d) {
            case 16: return go(bf, std::integral_constant<int, 16>{});
            case 32: return go(bf, std::integral_constant<int, 32>{});
            case 64: return go(bf, std::integral_constant<int, 64>{});
            default: return go(bf, std::integral_constant<int, 128>{});
        }
    };
    if (X->dtype == ALS_BF16) typed(std::true_type{});
    else typed(std::false_type{});
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

als_status launch_dequantize(als_ctx *ctx, const als_qtable *T, const als_table *X, hipStream_t s) {
    const int64_t pieces = X->rows * (X->d / 8);
    auto go = [&](auto bf, auto d) {
        hipLaunchKernelGGL((dequantize_kernel<bf(), d()>), quantize_grid(ctx, pieces), dim3(256), 0, s, (const uint32_t *)T->codes,
                           (const uint16_t *)T->scales, pieces, T->group / 8, X->data, X->ld);
    };
    auto typed = [&](auto bf) {
        switch (X->d) {
            case 16: return go(bf, std::integral_constant<int, 16>{});
            case 32: return go(bf, std::integral_constant<int, 32>{});
            case 64: return go(bf, std::integral_constant<int, 64>{});
            default: return go(bf, std::integral_constant<int, 128>{});
        }
    };
    if (X->dtype == ALS_BF16) typed(std::true_type{});
    else typed(std::false_type{});
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
