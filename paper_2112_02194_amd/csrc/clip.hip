// The norm over many tensors, and all of them scaled where it is above a bound (als_clip).
//
// norm kernel   workgroups take tiles of 4096 elements in turn; squares and their sums in fp64: no fp32 element over- or underflows
//               there, and at two operations an element the sums stay below the memory's time
//               (1e9 fp32 elements 0.67 ms, 6.0 TB/s)
// scale kernel  every workgroup adds the workgroups' sums in the same order, so all have the same bits of the norm, and takes its
//               tiles from the end: the last ones read are those that the cache may still hold (1.52 ms, 5.3 TB/s; in place and below the
//               bound nothing is read or written)
// Rows with gaps share a tile where they are short (5M x 64 fp32, 128 apart: 0.74 ms, a tile a row 16.2).  Small calls are the host's:
// 60 tensors of 2M elements in all 6 + 8 us here, 47 with the marshalling of 120 tensors.
#include <algorithm>
#include <iterator>
#include <type_traits>

#include "als_internal.h"

namespace als {

constexpr int CLIP_THREADS = 256, CLIP_EPT = 16, CLIP_TILE = CLIP_THREADS * CLIP_EPT;
constexpr int CLIP_PARTIALS = 8192;  // workgroups' sums of a call

// The tensors of a launch are its arguments (4 KB).  Those whose elements lie one after the other take less room there: 60 of
// them are one launch instead of two.
struct FlatTensor {
    static constexpr int MOST = 112;
    const char *x;
    char *y;
    int64_t n_and_type;  // elements * 2, + 1: bf16
    __device__ __forceinline__ bool bf16() const { return n_and_type & 1; }
    // the tensor's tile `at`
    template <class Tile> __device__ __forceinline__ void load(Tile &in, uint32_t at) const {
        const int64_t from = (int64_t)at * CLIP_TILE;
        in.load(x + from * Tile::ES, (n_and_type >> 1) - from);
    }
    template <class Tile> __device__ __forceinline__ void store(const Tile &in, uint32_t at, double c) const {
        const int64_t from = (int64_t)at * CLIP_TILE;
        in.store(y + from * Tile::ES, (n_and_type >> 1) - from, c);
    }
};
// A tile is a part of a row, or of several rows where they are short: 2^width pieces of 16 bytes of each.
struct RowTensor {
    static constexpr int MOST = 64;
    const char *x;
    char *y;
    int64_t rows, cols, ldx, ldy;  // in elements
    uint32_t row_tiles;
    uint16_t width, type;
    __device__ __forceinline__ bool bf16() const { return type; }
    // piece q of tile `at`: its place, and the elements that the row has from there
    template <int PER> __device__ __forceinline__ void piece(uint32_t at, int q, int64_t &row, int64_t &col, int64_t &left) const {
        constexpr int LOG = PER == 4 ? 10 : 9;  // pieces of a tile
        row = ((int64_t)(at / row_tiles) << (LOG - width)) + (q >> width);
        col = (int64_t)(at % row_tiles) * CLIP_TILE + (q & ((1 << width) - 1)) * PER;
        left = row < rows ? cols - col : 0;
    }
    template <class Tile> __device__ __forceinline__ void load(Tile &in, uint32_t at) const {
#pragma unroll
        for (int j = 0; j < Tile::PIECES; ++j) {
            int64_t row, col, left;
            piece<Tile::PER>(at, j * CLIP_THREADS + threadIdx.x, row, col, left);
            in.load_piece(j, x + (row * ldx + col) * Tile::ES, left);
        }
    }
    template <class Tile> __device__ __forceinline__ void store(const Tile &in, uint32_t at, double c) const {
#pragma unroll
        for (int j = 0; j < Tile::PIECES; ++j) {
            int64_t row, col, left;
            piece<Tile::PER>(at, j * CLIP_THREADS + threadIdx.x, row, col, left);
            in.store_piece(j, y + (row * ldy + col) * Tile::ES, left, c);
        }
    }
};
template <class T> struct ClipTensors {
    uint32_t tiles;
    int n;
    uint32_t first[T::MOST];  // numbers of the tensors' first tiles in the launch; ~0 behind the last
    T t[T::MOST];
};
static_assert(sizeof(ClipTensors<FlatTensor>) <= 4000 && sizeof(ClipTensors<RowTensor>) <= 4000, "a launch's arguments");

// Sixteen elements of a tile, as 16-byte pieces; those behind a row's end are zeros.
template <bool BF16> struct ClipTile {
    static constexpr int ES = BF16 ? 2 : 4, PER = 16 / ES, PIECES = CLIP_EPT / PER;
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    typedef Words Any __attribute__((aligned(2)));
    Words raw[PIECES];
    static __device__ __forceinline__ int item(int j) { return (j * CLIP_THREADS + threadIdx.x) * PER; }
    // left: elements from p on
    __device__ __forceinline__ void load_piece(int j, const char *p, int64_t left) {
        raw[j] = Words{0, 0, 0, 0};
        if (left >= PER) {
            raw[j] = *(const Any *)p;
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (e < left) {
                    if constexpr (BF16) raw[j][e / 2] |= (uint32_t)((const uint16_t *)p)[e] << (e & 1) * 16;
                    else raw[j][e] = ((const uint32_t *)p)[e];
                }
        }
    }
    __device__ __forceinline__ void load(const char *tile, int64_t left) {
        if (left >= CLIP_TILE) {
#pragma unroll
            for (int j = 0; j < PIECES; ++j) raw[j] = *(const Any *)(tile + item(j) * ES);
        } else {
#pragma unroll
            for (int j = 0; j < PIECES; ++j) load_piece(j, tile + item(j) * ES, left - item(j));
        }
    }
    __device__ __forceinline__ float value(int j, int e) const {
        return !BF16 ? __uint_as_float(raw[j][e]) : __uint_as_float(e & 1 ? raw[j][e / 2] & 0xffff0000u : raw[j][e / 2] << 16);
    }
    // times c; a factor near or below the normal range of fp32 has no bits to spare there: products in fp64
    __device__ __forceinline__ void store_piece(int j, char *p, int64_t left, double wide) const {
        typedef __bf16 Half __attribute__((ext_vector_type(8)));
        typedef Half AnyHalf __attribute__((aligned(2)));
        typedef float Full __attribute__((ext_vector_type(4)));
        typedef Full AnyFull __attribute__((aligned(4)));
        const float c = (float)wide;
        float v[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = c == 1.f ? value(j, e) : value(j, e) * c;
        if (wide < 0x1p-100) {
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = (float)(value(j, e) * wide);
        }
        if (left >= PER) {
            if constexpr (BF16) {
                typedef float Eight __attribute__((ext_vector_type(8)));
                const Eight w = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
                *(AnyHalf *)p = __builtin_convertvector(w, Half);
            } else {
                *(AnyFull *)p = Full{v[0], v[1], v[2], v[3]};
            }
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (e < left) {
                    if constexpr (BF16) ((__bf16 *)p)[e] = (__bf16)v[e];
                    else ((float *)p)[e] = v[e];
                }
        }
    }
    __device__ __forceinline__ void store(char *tile, int64_t left, double c) const {
#pragma unroll
        for (int j = 0; j < PIECES; ++j) store_piece(j, tile + item(j) * ES, left - item(j), c);
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

// The tensor of the launch that has the tile: the arguments come in one go, where a search would wait for each.
template <class T> __device__ __forceinline__ int find_tensor(const ClipTensors<T> &all, uint32_t tile) {
    int before = 0;
#pragma unroll
    for (int i = 0; i < T::MOST; ++i) before += all.first[i] <= tile;
    return before - 1;
}

template <class T> __global__ __launch_bounds__(CLIP_THREADS) void clip_norm_kernel(ClipTensors<T> all, double *__restrict__ partials) {
    __shared__ double lds[CLIP_THREADS / 64];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    int j = blockIdx.x < all.tiles ? find_tensor(all, blockIdx.x) : 0;
    for (uint32_t tile = blockIdx.x; tile < all.tiles; tile += gridDim.x) {
        while (j + 1 < all.n && tile >= all.first[j + 1]) ++j;
        const T &t = all.t[j];
        auto add = [&](auto bf) {
            ClipTile<bf()> in;
            t.load(in, tile - all.first[j]);
#pragma unroll
            for (int i = 0; i < CLIP_EPT; ++i) {
                const double v = in.value(i / in.PER, i % in.PER);
                s[i & 3] = fma(v, v, s[i & 3]);
            }
        };
        if (t.bf16()) add(std::true_type{});
        else add(std::false_type{});
    }
    const double sum = workgroup_sum((s[0] + s[1]) + (s[2] + s[3]), lds);
    if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

template <class T>
__global__ __launch_bounds__(CLIP_THREADS) void clip_scale_kernel(ClipTensors<T> all, const double *__restrict__ partials, int n_partials,
                                                                double bound, double *norm) {
    __shared__ double lds[CLIP_THREADS / 64];
    double s = 0.0;
    for (int i = threadIdx.x; i < n_partials; i += CLIP_THREADS) s += partials[i];
    const double total = sqrt(workgroup_sum(s, lds));
    const double c = total > bound && total < (double)INFINITY ? bound / total : 1.0;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = total;
    int j = blockIdx.x < all.tiles ? find_tensor(all, all.tiles - 1 - blockIdx.x) : 0;
    for (int64_t tile = (int64_t)all.tiles - 1 - blockIdx.x; tile >= 0; tile -= gridDim.x) {
        while ((uint32_t)tile < all.first[j]) --j;
        const T &t = all.t[j];
        if (c == 1.0 && t.y == t.x) continue;
        auto scale = [&](auto bf) {
            ClipTile<bf()> in;
            t.load(in, (uint32_t)tile - all.first[j]);
            t.store(in, (uint32_t)tile - all.first[j], c);
        };
        if (t.bf16()) scale(std::true_type{});
        else scale(std::false_type{});
    }
}

als_status clip_setup(als_ctx *ctx) { return ensure(ctx, ctx->clip_partials, CLIP_PARTIALS * sizeof(double)); }

als_status launch_clip(als_ctx *ctx, const als_matrix *X, const als_matrix *Y, int n, double bound, double *norm, hipStream_t s) {
    double *partials = (double *)ctx->clip_partials.p;
    bool too_large = false;  // a tensor of 2^31 tiles: 35 TB
    auto is_flat = [&](int j) { return X[j].rows <= 1 || (X[j].ld == X[j].cols && (!Y || Y[j].ld == Y[j].cols)); };
    // the next tensors of a kind that have elements, as many as a launch takes
    auto next = [&](int &j, auto &all) {
        constexpr bool flat = std::is_same_v<std::decay_t<decltype(all.t[0])>, FlatTensor>;
        all.n = 0;
        all.tiles = 0;
        std::fill(std::begin(all.first), std::end(all.first), ~0u);
        for (; j < n && all.n < (int)std::size(all.t); ++j) {
            const als_matrix &x = X[j], &y = Y ? Y[j] : X[j];
            if (x.rows == 0 || x.cols == 0 || is_flat(j) != flat) continue;
            const int64_t cols = flat ? x.rows * x.cols : x.cols, each = (cols + CLIP_TILE - 1) / CLIP_TILE;
            const int per = x.dtype == ALS_BF16 ? 8 : 4;
            int width = 0;  // of rows with gaps: 2^width pieces of a tile are one row's
            while ((int64_t)per << width < std::min<int64_t>(cols, CLIP_TILE)) ++width;
            const int64_t rows = CLIP_TILE / per >> width, tiles = flat ? each : each * ((x.rows + rows - 1) / rows);
            if (tiles > INT32_MAX - all.tiles) {
                if (all.n == 0) too_large = true;
                break;
            }
            auto &t = all.t[all.n];
            all.first[all.n++] = all.tiles;
            all.tiles += (uint32_t)tiles;
            t.x = (const char *)x.data;
            t.y = (char *)y.data;
            if constexpr (flat) {
                t.n_and_type = cols * 2 + (x.dtype == ALS_BF16);
            } else {
                t.rows = x.rows;
                t.cols = cols;
                t.ldx = x.ld;
                t.ldy = y.ld;
                t.row_tiles = (uint32_t)each;
                t.width = (uint16_t)width;
                t.type = x.dtype == ALS_BF16;
            }
        }
        return all.n > 0;
    };
    ClipTensors<FlatTensor> flat{};
    ClipTensors<RowTensor> rows{};
    int launches = 0;
    for (int j = 0; next(j, flat);) ++launches;
    for (int j = 0; next(j, rows);) ++launches;
    if (too_large || launches > CLIP_PARTIALS) return fail(ctx, ALS_ESHAPE, "als_clip: X has too many elements");
    launches = std::max(launches, 1);
    const int64_t most = std::min<int64_t>(ctx->num_cu * 8, CLIP_PARTIALS / launches);
    static_assert(CLIP_PARTIALS >= ALS_CLIP_MAX / FlatTensor::MOST + ALS_CLIP_MAX / RowTensor::MOST + 2, "a sum for every launch of ordinary tensors");
    int used = 0;
    auto norms = [&](auto &all) {
        for (int j = 0; next(j, all);) {
            const int64_t grid = std::min<int64_t>(all.tiles, most);
            hipLaunchKernelGGL((clip_norm_kernel<std::decay_t<decltype(all.t[0])>>), dim3((unsigned)grid), dim3(CLIP_THREADS), 0, s, all, partials + used);
            used += (int)grid;
        }
    };
    norms(flat);
    norms(rows);
    auto scales = [&](auto &all, bool always) {
        for (int j = 0; next(j, all) || always; always = false) {
            hipLaunchKernelGGL((clip_scale_kernel<std::decay_t<decltype(all.t[0])>>), dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(all.tiles, ctx->num_cu * 8))),
                               dim3(CLIP_THREADS), 0, s, all, (const double *)partials, used, bound, norm);
            norm = nullptr;
        }
    };
    scales(flat, true);  // the norm is written by the first launch, also where there is nothing
    scales(rows, false);
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
