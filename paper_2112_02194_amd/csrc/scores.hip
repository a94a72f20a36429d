// Scores of queries against a table in 4 bits an entry (als_scores): S[q][i] = sum_g scale(i, g) sum_{j in g} Q[q][j] code(i, j).
//
// Codes become fp16 numbers, exactly, two at a time: a code plus 8 put into the low bits of 1024's mantissa is the number
// 1024 + code + 8, from which a packed subtraction takes 1032; nibbles four bits further up come out times 16 and take a
// packed multiply-add instead.  About nine vector instructions for eight codes.  Both kernels form the group's sum first and
// multiply it by the group's scale once.
//
// few queries    (one or two) the vector units: 32 codes of an item per lane, products with the query's fp32 entries by
//                mixed-precision multiply-adds, sums over the lanes of an item by lane moves.
// more           the matrix cores, 32 queries x 32 items x 16 entries an instruction.  Query rows become two fp16 parts,
//                hi + lo, after a shift by a power of two that brings their largest entry to 2^13 .. 2^14: 22 bits and more of
//                every entry within 2^-16 of the largest, an absolute error of 2^-39 of the largest below (bf16 queries need
//                no lo: their 8 bits fit one part down to 2^-31 of the largest).  A wavefront keeps 32 queries' operands in
//                registers and walks item tiles, so that the codes are the only thing read.
#include <algorithm>

#include "row_piece.h"

namespace als {

typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The eight codes of a word as fp16 numbers: element e of the word is c[e % 4][e / 4].
__device__ __forceinline__ void unpack8(uint32_t w, halfx2 (&c)[4]) {
    w ^= 0x88888888u;  // two's complement to code + 8
    const halfx2 k1 = {(_Float16)1032.f, (_Float16)1032.f}, k2 = {(_Float16)0.0625f, (_Float16)0.0625f}, k3 = {(_Float16)72.f, (_Float16)72.f};
    const uint32_t v = w >> 8;
    c[0] = __builtin_bit_cast(halfx2, (w & 0x000f000fu) | 0x64006400u) - k1;
    c[1] = __builtin_bit_cast(halfx2, (w & 0x00f000f0u) | 0x64006400u) * k2 - k3;
    c[2] = __builtin_bit_cast(halfx2, (v & 0x000f000fu) | 0x64006400u) - k1;
    c[3] = __builtin_bit_cast(halfx2, (v & 0x00f000f0u) | 0x64006400u) * k2 - k3;
}

// ------------------------------------------------------------------------------------------------ few queries
template <bool BF_Q, bool BF_S, int D, int G, int NQ>
__global__ __launch_bounds__(256, 4) void scores_few_kernel(const void *__restrict__ Q, int64_t ldq, const uint8_t *__restrict__ codes,
                                                            const uint16_t *__restrict__ scales, int64_t n, void *__restrict__ S,
                                                            int64_t lds) {
    constexpr int CPL = D < 32 ? D : 32, LPI = D / CPL, IPS = 64 / LPI, U = 4;  // codes per lane, lanes per item, items per step, steps
    constexpr int W = CPL / 8, NG = CPL > G ? CPL / G : 1, WPG = W / NG;         // words and groups per lane, words per group
    const int lane = threadIdx.x & 63, chunk = lane % LPI;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), waves = (int64_t)gridDim.x * 4;
    float q[NQ][CPL];
#pragma unroll
    for (int r = 0; r < NQ; ++r)
#pragma unroll
        for (int p = 0; p < W; ++p) {
            float x[8];
            piece_floats<BF_Q>(piece_load<BF_Q>(Q, r * ldq + chunk * CPL + 8 * p), x);
#pragma unroll
            for (int e = 0; e < 8; ++e) q[r][8 * p + e] = x[e];
        }
    for (int64_t i0 = wave * (IPS * U); i0 < n; i0 += waves * (IPS * U)) {
        uint32_t w[U][W];
        float s[U][NG];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t item = std::min<int64_t>(i0 + u * IPS + lane / LPI, n - 1);
            const uint8_t *at = codes + item * (D / 2) + chunk * (CPL / 2);
            if constexpr (W == 4) {
                const u32x4 t = *(const u32x4 *)at;
#pragma unroll
                for (int p = 0; p < 4; ++p) w[u][p] = t[p];
            } else {
                const u32x2 t = *(const u32x2 *)at;
#pragma unroll
                for (int p = 0; p < 2; ++p) w[u][p] = t[p];
            }
            const uint16_t *sc = scales + item * (D / G) + chunk * CPL / G;
            if constexpr (NG == 2) {
                const uint32_t t = *(const uint32_t *)sc;
                s[u][0] = __uint_as_float(t << 16);
                s[u][1] = __uint_as_float(t & 0xffff0000u);
            } else {
                s[u][0] = bf16_to_f32(*sc);
            }
        }
        float sum[NQ][U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int r = 0; r < NQ; ++r) sum[r][u] = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float part[NQ];
#pragma unroll
                for (int r = 0; r < NQ; ++r) part[r] = 0.f;
#pragma unroll
                for (int p = g * WPG; p < (g + 1) * WPG; ++p) {
                    halfx2 c[4];
                    unpack8(w[u][p], c);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int r = 0; r < NQ; ++r) part[r] = fmaf((float)c[e % 4][e / 4], q[r][8 * p + e], part[r]);
                }
#pragma unroll
                for (int r = 0; r < NQ; ++r) sum[r][u] = fmaf(part[r], s[u][g], sum[r][u]);
            }
#pragma unroll
            for (int r = 0; r < NQ; ++r)
                if constexpr (LPI > 1) sum[r][u] = group_reduce<LPI>(sum[r][u], [](float a, float b) { return a + b; });
        }
        // every lane of an item holds its sum: lane `chunk` of it stores the item's of step `chunk` (+ LPI, ...)
#pragma unroll
        for (int t = 0; t < U / LPI; ++t) {
            const int64_t item = i0 + (t * LPI + chunk) * IPS + lane / LPI;
#pragma unroll
            for (int r = 0; r < NQ; ++r) {
                float v = sum[r][t * LPI];
#pragma unroll
                for (int c = 1; c < LPI; ++c) v = chunk == c ? sum[r][t * LPI + c] : v;
                if (item < n) store_elem<BF_S>(S, r * lds + item, v);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ matrix cores
// A wavefront's 32 queries (A operand: query = lane % 32) and 32 items a tile (B operand: item = lane % 32).  In step s of group
// part t (32 entries, or 16 for groups of 16) half h = lane / 32 of the wavefront holds eight entries of the group; which ones
// only has to be the same on both sides: one word of codes.
template <int D, int G> struct ScoreSteps {
    static constexpr int PART = G == 16 ? 16 : 32, PARTS = D / PART, STEPS = PART / 16;  // steps per part
    static __device__ __forceinline__ int word(int t, int s, int h) { return t * (PART / 8) + h * STEPS + s; }  // of the row's D / 8
};

template <bool BF_Q, bool BF_S, int D, int G>
__global__ __launch_bounds__(256, 2) void scores_tile_kernel(const void *__restrict__ Q, int64_t ldq, int64_t nq,
                                                             const uint32_t *__restrict__ codes, const uint16_t *__restrict__ scales,
                                                             int64_t n, void *__restrict__ S, int64_t lds, int64_t qgroups,
                                                             int64_t tiles_per_wave, int64_t units) {
    typedef ScoreSteps<D, G> T;
    constexpr int NP = BF_Q ? 1 : 2, NS = D / G;  // parts of a query entry, scales of an item
    const int lane = threadIdx.x & 63, a = lane & 31, h = lane >> 5;
    // Consecutive workgroups go to different XCDs: wavefronts that read the same items for other queries are kept on one.
    const int64_t per_xcd = ((units + 7) / 8 + 3) / 4 * 4;
    const int64_t in_xcd = (int64_t)(blockIdx.x >> 3) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t unit = (blockIdx.x & 7) * per_xcd + in_xcd;
    if (in_xcd >= per_xcd || unit >= units) return;
    const int64_t q0 = unit % qgroups * 32, first = unit / qgroups * tiles_per_wave;
    const int64_t tiles = (n + 31) / 32, last = std::min(tiles, first + tiles_per_wave);

    // the queries as operands, shifted so that the largest finite entry of a row lies in [2^13, 2^14)
    halfx8 A[T::PARTS][T::STEPS][NP];
    int shift;
    {
        float x[T::PARTS][T::STEPS][8];
        uint32_t top = 0;
#pragma unroll
        for (int t = 0; t < T::PARTS; ++t)
#pragma unroll
            for (int s = 0; s < T::STEPS; ++s) {
                Piece<BF_Q> p = piece_zero<BF_Q>();
                if (q0 + a < nq) p = piece_load<BF_Q>(Q, (q0 + a) * ldq + 8 * T::word(t, s, h));
                piece_floats<BF_Q>(p, x[t][s]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t m = __float_as_uint(x[t][s][e]) & 0x7fffffffu;
                    top = max(top, m < 0x7f800000u ? m : 0u);
                }
            }
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        shift = top ? 14 - __builtin_amdgcn_frexp_expf(__uint_as_float(top)) : 0;
#pragma unroll
        for (int t = 0; t < T::PARTS; ++t)
#pragma unroll
            for (int s = 0; s < T::STEPS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = 2 * (e % 4) + e / 4;  // the order in which unpack8 leaves a word's codes
                    const float v = ldexpf(x[t][s][e], shift);
                    const _Float16 hi = (_Float16)v;
                    A[t][s][0][at] = hi;
                    if constexpr (NP == 2) {
                        const float rest = v - (float)hi;  // NaN where v is not finite
                        A[t][s][1][at] = rest == rest ? (_Float16)rest : (_Float16)0.f;
                    }
                }
    }
    // 2^-shift of the rows that this lane's results belong to: result v is <query 8 (v / 4) + 4 h + v % 4, item a>
    auto shift_of = [&](int v) { return __shfl(shift, 8 * (v >> 2) + 4 * h + (v & 3)); };
    float back[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) back[v] = ldexpf(1.f, -shift_of(v));
    const bool q_wide = __any(shift > 60 || shift < -60);

    uint32_t w[T::PARTS][T::STEPS];
    float sc[NS];
    auto fetch = [&](int64_t tile) {
        const int64_t item = std::min<int64_t>(tile * 32 + a, n - 1);
#pragma unroll
        for (int t = 0; t < T::PARTS; ++t) {
            const uint32_t *at = codes + item * (D / 8) + T::word(t, 0, h);
            if constexpr (T::STEPS == 2) {
                const u32x2 v = *(const u32x2 *)at;
                w[t][0] = v[0];
                w[t][1] = v[1];
            } else {
                w[t][0] = *at;
            }
        }
        const uint16_t *ps = scales + item * NS;
        if constexpr (NS == 1) {
            sc[0] = bf16_to_f32(*ps);
        } else {
            uint32_t raw[NS / 2];
            __builtin_memcpy(raw, __builtin_assume_aligned(ps, NS < 8 ? 2 * NS : 16), 2 * NS);
#pragma unroll
            for (int g = 0; g < NS; ++g) sc[g] = __uint_as_float(g & 1 ? raw[g / 2] & 0xffff0000u : raw[g / 2] << 16);
        }
    };

    fetch(first);
    for (int64_t tile = first; tile < last; ++tile) {
        float total[16];
#pragma unroll
        for (int v = 0; v < 16; ++v) total[v] = 0.f;
        uint32_t cw[T::PARTS][T::STEPS];
        float cs[NS];
#pragma unroll
        for (int t = 0; t < T::PARTS; ++t)
#pragma unroll
            for (int s = 0; s < T::STEPS; ++s) cw[t][s] = w[t][s];
#pragma unroll
        for (int g = 0; g < NS; ++g) cs[g] = sc[g];
        if (tile + 1 < last) fetch(tile + 1);
        // Sums of shifted queries times a scale stay in fp32's range while neither factor is beyond 2^60 or below 2^-60.
        // Elsewhere the scales of an item are shifted too, and the results back in one step.
        int k = 0;
        bool wide = q_wide;
        {
            uint32_t top = 0;
#pragma unroll
            for (int g = 0; g < NS; ++g) {
                const uint32_t m = __float_as_uint(cs[g]) & 0x7fffffffu;
                top = max(top, m < 0x7f800000u ? m : 0u);
            }
            wide = __any(wide || (top && (top > 0x5d800000u || top < 0x21800000u)));
            if (wide) {
                k = top ? __builtin_amdgcn_frexp_expf(__uint_as_float(top)) : 0;
#pragma unroll
                for (int g = 0; g < NS; ++g) cs[g] = ldexpf(cs[g], -k);
            }
        }
#pragma unroll
        for (int t = 0; t < T::PARTS; ++t) {
            floatx16 acc;
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
            for (int s = 0; s < T::STEPS; ++s) {
                halfx2 c[4];
                unpack8(cw[t][s], c);
                const u32x4 bits = {__builtin_bit_cast(uint32_t, c[0]), __builtin_bit_cast(uint32_t, c[1]),
                                    __builtin_bit_cast(uint32_t, c[2]), __builtin_bit_cast(uint32_t, c[3])};
                const halfx8 B = __builtin_bit_cast(halfx8, bits);
#pragma unroll
                for (int p = 0; p < NP; ++p) acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(A[t][s][p], B, acc, 0, 0, 0);
            }
            const float scale = cs[t * T::PART / G];
#pragma unroll
            for (int v = 0; v < 16; ++v) total[v] = fmaf(acc[v], scale, total[v]);
        }
        if (wide) {
#pragma unroll
            for (int v = 0; v < 16; ++v) total[v] = ldexpf(total[v], k - shift_of(v));
        } else {
#pragma unroll
            for (int v = 0; v < 16; ++v) total[v] *= back[v];
        }
        const int64_t item = tile * 32 + a;
        if (q0 + 32 <= nq && tile * 32 + 32 <= n) {
            if constexpr (BF_S) {
                // neighbouring lanes swap so that each stores two items of one row: the even one row v, the odd one row v + 1
                const uint32_t pick = lane & 1 ? 0x07060302u : 0x01000504u;
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                typedef float floatx2 __attribute__((ext_vector_type(2)));
                typedef uint32_t u32_any __attribute__((aligned(2)));
#pragma unroll
                for (int v = 0; v < 16; v += 2) {
                    const floatx2 f = {total[v], total[v + 1]};
                    const uint32_t own = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
                    const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)own, 0xB1, 0xf, 0xf, true);
                    const uint32_t pair = __builtin_amdgcn_perm(own, other, pick);
                    const int64_t row = q0 + 8 * (v >> 2) + 4 * h + (v & 3) + (lane & 1);
                    *(u32_any *)((uint16_t *)S + row * lds + (item & ~(int64_t)1)) = pair;
                }
            } else {
#pragma unroll
                for (int v = 0; v < 16; ++v) ((float *)S)[(q0 + 8 * (v >> 2) + 4 * h + (v & 3)) * lds + item] = total[v];
            }
        } else if (item < n) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int64_t row = q0 + 8 * (v >> 2) + 4 * h + (v & 3);
                if (row < nq) store_elem<BF_S>(S, row * lds + item, total[v]);
            }
        }
    }
}

constexpr int SCORES_FEW = 2;  // queries up to which the vector units work

template <bool BF_Q, bool BF_S, int D, int G>
static void scores_typed(const als_ctx *ctx, const als_table *Q, const als_qtable *T, const als_matrix *S, hipStream_t s) {
    const int64_t n = T->rows, nq = Q->rows;
    if (nq <= SCORES_FEW) {
        constexpr int ITEMS = 4 * 4 * 64 / (D / (D < 32 ? D : 32));  // of a workgroup's round
        const dim3 grid((unsigned)std::min<int64_t>((n + ITEMS - 1) / ITEMS, (int64_t)ctx->num_cu * 8));
        auto go = [&](auto count) {
            hipLaunchKernelGGL((scores_few_kernel<BF_Q, BF_S, D, G, count()>), grid, dim3(256), 0, s, Q->data, Q->ld,
                               (const uint8_t *)T->codes, (const uint16_t *)T->scales, n, S->data, S->ld);
        };
        if (nq == 1) go(std::integral_constant<int, 1>{});
        else go(std::integral_constant<int, 2>{});
        return;
    }
    const int64_t qgroups = (nq + 31) / 32, tiles = (n + 31) / 32;
    const int64_t per = std::max<int64_t>(1, std::min<int64_t>(64, tiles * qgroups / ((int64_t)ctx->num_cu * 16)));
    const int64_t units = (tiles + per - 1) / per * qgroups, per_xcd = ((units + 7) / 8 + 3) / 4 * 4;
    hipLaunchKernelGGL((scores_tile_kernel<BF_Q, BF_S, D, G>), dim3((unsigned)(per_xcd / 4 * 8)), dim3(256), 0, s, Q->data, Q->ld, nq,
                       (const uint32_t *)T->codes, (const uint16_t *)T->scales, n, S->data, S->ld, qgroups, per, units);
}

template <bool BF_Q, bool BF_S>
static void scores_sized(const als_ctx *ctx, const als_table *Q, const als_qtable *T, const als_matrix *S, hipStream_t s) {
    switch (T->d * 256 + T->group) {
        case 16 * 256 + 16: return scores_typed<BF_Q, BF_S, 16, 16>(ctx, Q, T, S, s);
        case 32 * 256 + 16: return scores_typed<BF_Q, BF_S, 32, 16>(ctx, Q, T, S, s);
        case 32 * 256 + 32: return scores_typed<BF_Q, BF_S, 32, 32>(ctx, Q, T, S, s);
        case 64 * 256 + 16: return scores_typed<BF_Q, BF_S, 64, 16>(ctx, Q, T, S, s);
        case 64 * 256 + 32: return scores_typed<BF_Q, BF_S, 64, 32>(ctx, Q, T, S, s);
        case 64 * 256 + 64: return scores_typed<BF_Q, BF_S, 64, 64>(ctx, Q, T, S, s);
        case 128 * 256 + 16: return scores_typed<BF_Q, BF_S, 128, 16>(ctx, Q, T, S, s);
        case 128 * 256 + 32: return scores_typed<BF_Q, BF_S, 128, 32>(ctx, Q, T, S, s);
        case 128 * 256 + 64: return scores_typed<BF_Q, BF_S, 128, 64>(ctx, Q, T, S, s);
        default: return scores_typed<BF_Q, BF_S, 128, 128>(ctx, Q, T, S, s);
    }
}

als_status launch_scores(als_ctx *ctx, const als_table *Q, const als_qtable *T, const als_matrix *S, hipStream_t s) {
    const bool bq = Q->dtype == ALS_BF16, bs = S->dtype == ALS_BF16;
    if (bq && bs) scores_sized<true, true>(ctx, Q, T, S, s);
    else if (bq) scores_sized<true, false>(ctx, Q, T, S, s);
    else if (bs) scores_sized<false, true>(ctx, Q, T, S, s);
    else scores_sized<false, false>(ctx, Q, T, S, s);
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
