// The norm over many tensors, and all of them scaled where it is above a bound (als_clip).
//
// norm kernel   workgroups take tiles of 4096 elements in turn; squares and their sums in fp64: no fp32 element over- or underflows
//               there, and at two operations an element the sums stay below the memory's time
// scale kernel  every workgroup adds the workgroups' sums in the same order, so all have the same bits of the norm, and takes its
//               tiles from the end: the last ones read are those that the cache may still hold
#include <algorithm>
#include <type_traits>
#include <vector>

#include "als_internal.h"

namespace als {

constexpr int CLIP_THREADS = 256, CLIP_EPT = 16, CLIP_TILE = CLIP_THREADS * CLIP_EPT;
constexpr int CLIP_TENSORS = 48;    // of a launch: they are its arguments
constexpr int CLIP_PARTIALS = 8192;  // workgroups' sums of a call

struct ClipTensor {
    const char *x;
    char *y;
    int64_t cols, ldx, ldy;  // of a row, in elements; one row where they lie one after the other
    int64_t row_tiles, first;  // tiles of a row; number of the first one in the launch
    int64_t bf16;
};
struct ClipTensors {
    ClipTensor t[CLIP_TENSORS];
    int64_t tiles;
    int n;
};

// Sixteen elements of a tile, as 16-byte pieces; those behind the row's end are zeros.
template <bool BF16> struct ClipTile {
    static constexpr int PER = BF16 ? 8 : 4, PIECES = CLIP_EPT / PER;
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    typedef Words Any __attribute__((aligned(2)));
    Words raw[PIECES];
    static __device__ __forceinline__ int item(int j, int tid) { return (j * CLIP_THREADS + tid) * PER; }
    __device__ __forceinline__ void load(const char *tile, int64_t left, int tid) {
        constexpr int ES = BF16 ? 2 : 4;
        if (left >= CLIP_TILE) {
#pragma unroll
            for (int j = 0; j < PIECES; ++j) raw[j] = *(const Any *)(tile + item(j, tid) * ES);
        } else {
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                const int at = item(j, tid);
                raw[j] = Words{0, 0, 0, 0};
                if (at + PER <= left) {
                    raw[j] = *(const Any *)(tile + at * ES);
                } else {
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (at + e < left) {
                            if constexpr (BF16) raw[j][e / 2] |= (uint32_t)((const uint16_t *)tile)[at + e] << (e & 1) * 16;
                            else raw[j][e] = ((const uint32_t *)tile)[at + e];
                        }
                }
            }
        }
    }
    __device__ __forceinline__ float value(int j, int e) const {
        return !BF16 ? __uint_as_float(raw[j][e]) : __uint_as_float(e & 1 ? raw[j][e / 2] & 0xffff0000u : raw[j][e / 2] << 16);
    }
    // times c; a factor near or below the normal range of fp32 has no bits to spare there: products in fp64
    __device__ __forceinline__ void store(char *tile, int64_t left, int tid, double wide) const {
        typedef __bf16 Half __attribute__((ext_vector_type(8)));
        typedef Half AnyHalf __attribute__((aligned(2)));
        typedef float Full __attribute__((ext_vector_type(4)));
        typedef Full AnyFull __attribute__((aligned(4)));
        const float c = (float)wide;
        const bool small = wide < 0x1p-100;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int at = item(j, tid);
            float v[PER];
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = c == 1.f ? value(j, e) : value(j, e) * c;
            if (small) {
#pragma unroll
                for (int e = 0; e < PER; ++e) v[e] = (float)(value(j, e) * wide);
            }
            if (at + PER <= left) {
                if constexpr (BF16) {
                    typedef float Eight __attribute__((ext_vector_type(8)));
                    const Eight w = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
                    *(AnyHalf *)(tile + at * 2) = __builtin_convertvector(w, Half);
                } else {
                    *(AnyFull *)(tile + at * 4) = Full{v[0], v[1], v[2], v[3]};
                }
            } else {
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    if (at + e < left) {
                        if constexpr (BF16) ((__bf16 *)tile)[at + e] = (__bf16)v[e];
                        else ((float *)tile)[at + e] = v[e];
                    }
            }
        }
    }
};

__device__ __forceinline__ double workgroup_sum(double s, double *lds) {
    for (int m = 32; m > 0; m >>= 1) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
    for (int i = 0; i < CLIP_THREADS / 64; ++i) s += lds[i];
    return s;
}

// Tensor j of the launch that has the tile, from the one that had the workgroup's last.
template <bool BACK> __device__ __forceinline__ void find_tensor(const ClipTensors &all, int64_t tile, int &j) {
    if (BACK) while (tile < all.t[j].first) --j;
    else while (j + 1 < all.n && tile >= all.t[j + 1].first) ++j;
}

__global__ __launch_bounds__(CLIP_THREADS) void clip_norm_kernel(ClipTensors all, double *__restrict__ partials) {
    __shared__ double lds[CLIP_THREADS / 64];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    int j = 0;
    for (int64_t tile = blockIdx.x; tile < all.tiles; tile += gridDim.x) {
        find_tensor<false>(all, tile, j);
        const ClipTensor &t = all.t[j];
        const int64_t at = tile - t.first, row = at / t.row_tiles, col = (at - row * t.row_tiles) * CLIP_TILE;
        auto add = [&](auto bf) {
            ClipTile<bf()> in;
            in.load(t.x + (row * t.ldx + col) * (bf() ? 2 : 4), t.cols - col, threadIdx.x);
#pragma unroll
            for (int i = 0; i < CLIP_EPT; ++i) {
                const double v = in.value(i / in.PER, i % in.PER);
                s[i & 3] = fma(v, v, s[i & 3]);
            }
        };
        if (t.bf16) add(std::true_type{});
        else add(std::false_type{});
    }
    const double sum = workgroup_sum((s[0] + s[1]) + (s[2] + s[3]), lds);
    if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

__global__ __launch_bounds__(CLIP_THREADS) void clip_scale_kernel(ClipTensors all, const double *__restrict__ partials, int n_partials,
                                                                double bound, double *norm) {
    __shared__ double lds[CLIP_THREADS / 64];
    double s = 0.0;
    for (int i = threadIdx.x; i < n_partials; i += CLIP_THREADS) s += partials[i];
    const double total = sqrt(workgroup_sum(s, lds));
    const double c = total > bound && total < (double)INFINITY ? bound / total : 1.0;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = total;
    int j = all.n - 1;
    for (int64_t tile = all.tiles - 1 - blockIdx.x; tile >= 0; tile -= gridDim.x) {
        find_tensor<true>(all, tile, j);
        const ClipTensor &t = all.t[j];
        if (c == 1.0 && t.y == t.x) continue;
        const int64_t at = tile - t.first, row = at / t.row_tiles, col = (at - row * t.row_tiles) * CLIP_TILE;
        auto scale = [&](auto bf) {
            ClipTile<bf()> in;
            in.load(t.x + (row * t.ldx + col) * (bf() ? 2 : 4), t.cols - col, threadIdx.x);
            in.store(t.y + (row * t.ldy + col) * (bf() ? 2 : 4), t.cols - col, threadIdx.x, c);
        };
        if (t.bf16) scale(std::true_type{});
        else scale(std::false_type{});
    }
}

als_status clip_setup(als_ctx *ctx) { return ensure(ctx, ctx->clip_partials, CLIP_PARTIALS * sizeof(double)); }

als_status launch_clip(als_ctx *ctx, const als_matrix *X, const als_matrix *Y, int n, double bound, double *norm, hipStream_t s) {
    double *partials = (double *)ctx->clip_partials.p;
    // the tensors that have elements, CLIP_TENSORS a launch
    auto next = [&](int &j, ClipTensors &all) {
        all.n = 0;
        all.tiles = 0;
        for (; j < n && all.n < CLIP_TENSORS; ++j) {
            const als_matrix &x = X[j], &y = Y ? Y[j] : X[j];
            if (x.rows == 0 || x.cols == 0) continue;
            const bool flat = x.rows == 1 || (x.ld == x.cols && y.ld == y.cols);
            ClipTensor &t = all.t[all.n++];
            t.x = (const char *)x.data;
            t.y = (char *)y.data;
            t.cols = flat ? x.rows * x.cols : x.cols;
            t.ldx = x.ld;
            t.ldy = y.ld;
            t.row_tiles = (t.cols + CLIP_TILE - 1) / CLIP_TILE;
            t.first = all.tiles;
            t.bf16 = x.dtype == ALS_BF16;
            all.tiles += t.row_tiles * (flat ? 1 : x.rows);
        }
        return all.n > 0;
    };
    ClipTensors all{};
    const int launches = std::max(1, (n + CLIP_TENSORS - 1) / CLIP_TENSORS);
    const int64_t most = std::min<int64_t>(ctx->num_cu * 8, CLIP_PARTIALS / launches);
    static_assert(CLIP_PARTIALS >= ALS_CLIP_MAX / CLIP_TENSORS + 1, "a sum for every launch");
    int used = 0;
    for (int j = 0; next(j, all);) {
        const int64_t grid = std::min(all.tiles, most);
        hipLaunchKernelGGL(clip_norm_kernel, dim3((unsigned)grid), dim3(CLIP_THREADS), 0, s, all, partials + used);
        used += (int)grid;
    }
    int j = 0;
    bool more = next(j, all);
    do {
        hipLaunchKernelGGL(clip_scale_kernel, dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(all.tiles, ctx->num_cu * 8))), dim3(CLIP_THREADS), 0, s, all,
                           (const double *)partials, used, bound, norm);
        norm = nullptr;
        more = more && next(j, all);
    } while (more);
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
