// Pieces of table rows as the kernels over ordered entries read and write them: N consecutive columns a lane, fp32 in registers.
#pragma once

#include <type_traits>

#include "als_internal.h"

namespace als {

// A table as a kernel sees it: rows `ld` bytes apart.
struct RowsOf {
    char *p;  // null: not given
    int64_t ld;
    int bf16;
};
inline RowsOf rows_of(const als_table *t) {
    return t ? RowsOf{(char *)t->data, t->ld * (t->dtype == ALS_BF16 ? 2 : 4), t->dtype == ALS_BF16} : RowsOf{nullptr, 0, 0};
}

template <bool BF16, int N> __device__ __forceinline__ void load_piece(const char *row, int lane, float (&x)[N]) {
    static_assert(N == 4 || N == 8, "16 bytes of one of the types");
    if constexpr (!BF16) {
#pragma unroll
        for (int j = 0; j < N / 4; ++j) {
            const float4 v = *(const float4 *)(row + (lane * N + 4 * j) * 4);
            x[4 * j] = v.x; x[4 * j + 1] = v.y; x[4 * j + 2] = v.z; x[4 * j + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < N / 4; ++j) {
            const uint2 v = *(const uint2 *)(row + (lane * N + 4 * j) * 2);
            x[4 * j] = __uint_as_float(v.x << 16);
            x[4 * j + 1] = __uint_as_float(v.x & 0xffff0000u);
            x[4 * j + 2] = __uint_as_float(v.y << 16);
            x[4 * j + 3] = __uint_as_float(v.y & 0xffff0000u);
        }
    }
}
template <bool BF16, int N> __device__ __forceinline__ void store_piece(char *row, int lane, const float (&x)[N]) {
    typedef float Full __attribute__((ext_vector_type(4)));
    typedef __bf16 Half __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
        const Full v = {x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
        if constexpr (BF16) *(Half *)(row + (lane * N + 4 * j) * 2) = __builtin_convertvector(v, Half);
        else *(Full *)(row + (lane * N + 4 * j) * 4) = v;
    }
}
// The same where only the call knows the type: pieces that are read or written once a row.
template <int N> __device__ __forceinline__ void load_piece(const RowsOf &t, int64_t row, int lane, float (&x)[N]) {
    if (t.bf16) load_piece<true, N>(t.p + row * t.ld, lane, x);
    else load_piece<false, N>(t.p + row * t.ld, lane, x);
}
template <int N> __device__ __forceinline__ void store_piece(const RowsOf &t, int64_t row, int lane, const float (&x)[N]) {
    if (t.bf16) store_piece<true, N>(t.p + row * t.ld, lane, x);
    else store_piece<false, N>(t.p + row * t.ld, lane, x);
}

// The same pieces as they lie in memory: 16 bytes, or four columns.
typedef uint32_t Words __attribute__((ext_vector_type(4)));
typedef uint32_t HalfWords __attribute__((ext_vector_type(2)));
template <bool BF16> using Part = std::conditional_t<BF16, HalfWords, Words>;
template <bool BF16, int N, class W> __device__ __forceinline__ void widen(const W &w, float (&x)[N]) {
    static_assert(sizeof(W) == N * (BF16 ? 2 : 4), "");
#pragma unroll
    for (int c = 0; c < N; ++c) x[c] = !BF16 ? __uint_as_float(w[c]) : __uint_as_float(c & 1 ? w[c / 2] & 0xffff0000u : w[c / 2] << 16);
}

// Row `id` of a table, or the row that stands for entries without an item where it is negative.  The address is computed for every
// lane and then chosen: of a choice with work on one side the compiler makes a branch of some lanes.
__device__ __forceinline__ const char *item_row(const RowsOf &t, int id, const char *none) {
    uint64_t at = (uint64_t)t.p + (uint32_t)id * (uint64_t)t.ld;
    asm("" : "+v"(at));
    return id < 0 ? none : (const char *)at;
}

// s = 1 / (1 + exp(-g)) and 1 - s, each to its own size: with e = exp(-g) they are 1 / (1 + e) and e / (1 + e).  e is kept within
// 2^126, where s is 2^-126; a NaN stays one.
__device__ __forceinline__ void gate(float g, float &keep, float &take) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504f * __builtin_elementwise_maximum(g, -87.3365448f));
    keep = __builtin_amdgcn_rcpf(1.f + e);
    take = e * keep;
}

// The share of a state that a map keeps, held so that its bits are those that count: below 7/8 as it is, above it as what is missing to 1,
// with a minus sign.  Near 1 half a step is 2^-25; that, once an entry, is 1e-3 of a state that 65000 entries with the same gate have
// made, where what is given away (1 - s, and t + v - t v of two) has all its bits.  All of it kept is -0, and 0 nothing.
constexpr float KEEPS_ALL = -0.f;
__device__ __forceinline__ float share_of(float keep, float take) { return take < 0.125f ? -take : keep; }
// `s` where the sign of `q` is set, 0 elsewhere
__device__ __forceinline__ float where_negative(float q, float s) { return __int_as_float(__float_as_int(s) & __float_as_int(q) >> 31); }
// the state s after a map with share q and what it adds; what an infinite state gives away is a number, so that it stays
__device__ __forceinline__ float after_map(float q, float s, float b) {
    const float number = __builtin_amdgcn_fmed3f(s, -__FLT_MAX__, __FLT_MAX__);
    return fmaf(q, __float_as_int(q) < 0 ? number : s, b) + where_negative(q, s);
}
// The share of two maps after each other: p q of kept ones; -(t + v - t v) of t and v given away, q (1 - t) of one of each.  What is
// given away stays below 1/2, else 1 + k, which is exact, is what is kept.
__device__ __forceinline__ float share_of_both(float p, float q) {
    const float zp = where_negative(q, p), zq = where_negative(p, q);
    float k = fmaf(p, q, zp) + zq;
    k = __uint_as_float(__float_as_uint(k) | (__float_as_uint(zp) & 0x80000000u));  // -0 and -0 stay -0
    return k < -0.5f ? k + 1.f : k;
}
// One of two values that both are there.
__device__ __forceinline__ float chosen(bool first, float a, float b) {
    asm("" : "+v"(a), "+v"(b));
    return first ? a : b;
}

// Entries of row u, whatever indptr holds.
__device__ __forceinline__ void row_range(const int64_t *indptr, int64_t u, int64_t nnz, int64_t &b, int64_t &e) {
    b = indptr[u];
    e = indptr[u + 1];
    if (b < 0) b = 0;
    if (e > nnz) e = nnz;
    if (e < b) e = b;
}

// Lists over a table: entry p takes row ids[p], or its own where ids is null.
struct Lists {
    const int64_t *indptr;
    const int32_t *ids;
    int64_t rows, nnz, cols;
};
inline Lists lists_of(const als_csr *y) { return Lists{y->indptr, y->indices, y->rows, y->nnz, y->cols}; }

}  // namespace als
