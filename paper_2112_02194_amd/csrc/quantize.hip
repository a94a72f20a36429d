// Tables in 4 bits an entry with one bf16 scale per group of entries (als_quantize, als_dequantize).
//
// One read and one write of everything.  A lane owns 16 bytes of the table, four or eight consecutive entries, so that a wavefront
// moves 1 KB in one piece; the lanes of a group share its largest magnitude by lane moves.  Reading back is bound by memory (10M x 128
// to fp32 1.32 ms, 4.4 TB/s, to bf16 0.62 ms, 5.3 TB/s), quantizing by the vector units: 35 instructions an entry of
// fp32, 26 of bf16, at work 96 and 85 % of the time (10M x 128 fp32 1.26 ms, 4.6 TB/s; 1M x 64 bf16 54 us, 3.0 TB/s, where memory would
// need 33).
#include <algorithm>

#include "row_piece.h"

namespace als {

// Entries of a lane, and 16-byte pieces of a row.
template <bool BF16> constexpr int PER = BF16 ? 8 : 4;
template <bool BF16, int D> constexpr int PIECES = D / PER<BF16>;
constexpr int ROUNDS = 4;  // pieces of a thread under way

// A code is x / s rounded to the nearest whole number, halves to even, of the quotient as IEEE division gives it.  That division takes
// a dozen instructions; x * (1 / s) is within four units in the last place of it (|quotient| < 8, so within 4e-6), which settles
// every quotient that is not so near to a half.  The few others are divided, and all where s is so small that 1 / s may overflow.
// A table of 10M x 128 fp32 entries, quantized and read back: 2.60 ms, 4.5 TB/s (with a division each and four-byte stores: 2.88).
__device__ __forceinline__ float quotient(float x, float s, float inverse, bool exact) {
    const float q = x * inverse, off = q - rintf(q);
    return exact || !(fabsf(fabsf(off) - 0.5f) > 1e-5f) ? x / s : q;
}

template <bool BF16, int D>
__global__ __launch_bounds__(256) void quantize_kernel(const void *__restrict__ X, int64_t ld, int64_t pieces, int group_lanes,
                                                       uint8_t *__restrict__ codes, uint16_t *__restrict__ scales) {
    constexpr int N = PER<BF16>;
    // the lanes of a group go round together: both `pieces` and the stride are multiples of their number
    for (int64_t i0 = (int64_t)blockIdx.x * (256 * ROUNDS) + threadIdx.x; i0 < pieces; i0 += (int64_t)gridDim.x * (256 * ROUNDS)) {
        float x[ROUNDS][N];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = std::min<int64_t>(i0 + 256 * r, pieces - 1), off = i / PIECES<BF16, D> * ld + i % PIECES<BF16, D> * N;
            if constexpr (BF16) piece_floats<true>(piece_load<true>(X, off), x[r]);
            else load_vec<4, false>(X, off, x[r]);
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = i0 + 256 * r;
            // the largest magnitude as bits: they order like the values, with infinity and NaN above all others
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(x[r][e]) & 0x7fffffffu);
            for (int m = 1; m < group_lanes; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
            const uint16_t sb = f32_to_bf16_rne(__uint_as_float(top) / 7.f);
            const float s = bf16_to_f32(sb);
            const bool usable = s > 0.f && s < INFINITY, exact = !(s >= 1.2e-38f);
            const float inverse = 1.f / s;
            uint32_t word = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float c = fminf(fmaxf(rintf(quotient(x[r][e], s, inverse, exact)), -7.f), 7.f);
                word |= ((uint32_t)(int)(usable ? c : 0.f) & 15u) << (4 * e);
            }
            if (i < pieces) {
                if constexpr (BF16) ((uint32_t *)codes)[i] = word;
                else ((uint16_t *)codes)[i] = (uint16_t)word;
                if (threadIdx.x % group_lanes == 0) scales[i / group_lanes] = sb;
            }
        }
    }
}

template <bool BF16, int D>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t *__restrict__ codes, const uint16_t *__restrict__ scales,
                                                         int64_t pieces, int group_lanes, void *__restrict__ X, int64_t ld) {
    constexpr int N = PER<BF16>;
    for (int64_t i0 = (int64_t)blockIdx.x * (256 * ROUNDS) + threadIdx.x; i0 < pieces; i0 += (int64_t)gridDim.x * (256 * ROUNDS)) {
        int32_t word[ROUNDS];
        float s[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = std::min<int64_t>(i0 + 256 * r, pieces - 1);
            word[r] = BF16 ? ((const int32_t *)codes)[i] : (int32_t)((const uint16_t *)codes)[i];
            s[r] = bf16_to_f32(scales[i / group_lanes]);
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = i0 + 256 * r, off = i / PIECES<BF16, D> * ld + i % PIECES<BF16, D> * N;
            typedef float Values __attribute__((ext_vector_type(N)));
            typedef __bf16 Halves __attribute__((ext_vector_type(N)));
            Values v;
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = (float)(word[r] << (28 - 4 * e) >> 28) * s[r];
            if (i < pieces) {
                if constexpr (BF16) *(Halves *)((uint16_t *)X + off) = __builtin_convertvector(v, Halves);
                else *(Values *)((float *)X + off) = v;
            }
        }
    }
}

static dim3 quantize_grid(const als_ctx *ctx, int64_t pieces) {
    return dim3((unsigned)std::min<int64_t>((pieces + 256 * ROUNDS - 1) / (256 * ROUNDS), (int64_t)ctx->num_cu * 64));
}

als_status launch_quantize(als_ctx *ctx, const als_table *X, const als_qtable *T, hipStream_t s) {
    auto go = [&](auto bf, auto d) {
        const int64_t pieces = X->rows * PIECES<bf(), d()>;
        hipLaunchKernelGGL((quantize_kernel<bf(), d()>), quantize_grid(ctx, pieces), dim3(256), 0, s, X->data, X->ld, pieces,
                           T->group / PER<bf()>, (uint8_t *)T->codes, (uint16_t *)T->scales);
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
    auto go = [&](auto bf, auto d) {
        const int64_t pieces = X->rows * PIECES<bf(), d()>;
        hipLaunchKernelGGL((dequantize_kernel<bf(), d()>), quantize_grid(ctx, pieces), dim3(256), 0, s, (const uint8_t *)T->codes,
                           (const uint16_t *)T->scales, pieces, T->group / PER<bf()>, X->data, X->ld);
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
