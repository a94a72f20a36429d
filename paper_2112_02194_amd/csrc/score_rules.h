// Rules on scores (als_rules) as als_adjust and als_select evaluate them, a tile of one row at a time.
//
// A workgroup of 256 threads works on TILE consecutive items of one row.  Lists (history, entries) hold a row's items in any
// order, so nothing says which of them lie in the tile: the workgroup walks the whole list once per tile and counts, in LDS,
// how often every item of the tile occurs (history) and where it is stored last (entries).  Integer atomics: the result does
// not depend on their order.  An element then reads its two words.
#pragma once

#include "als_internal.h"

namespace als {

constexpr int TILE = 4096, TILE_THREADS = 256, TILE_EPT = TILE / TILE_THREADS;  // items per tile, threads, items per thread

struct RowList {
    const int64_t *indptr;  // null: no such list
    const int32_t *indices;
    const float *values;
    int64_t nnz;
};
struct RuleArgs {
    RowList history, entries;
    const float *bias;
    const uint32_t *allowed;
    int64_t allowed_ld;
    const float *penalties;
    float repetition, presence, frequency;
};

inline RuleArgs rule_args(const als_rules *r) {
    RuleArgs a{};
    a.repetition = 1.f;
    if (!r) return a;
    auto list = [](const als_csr *y) {
        return y && y->nnz > 0 ? RowList{y->indptr, y->indices, y->values, y->nnz} : RowList{};
    };
    a.history = list(r->history);
    a.entries = list(r->entries);
    a.bias = r->bias;
    a.allowed = r->allowed;
    a.allowed_ld = r->allowed_ld;
    a.penalties = r->penalties;
    a.repetition = r->repetition;
    a.presence = r->presence;
    a.frequency = r->frequency;
    return a;
}
// LDS words that the lists need
inline int rule_words(const RuleArgs &a) { return (a.history.indptr ? TILE : 0) + (a.entries.indptr ? TILE : 0); }

// Four consecutive elements; rows need not be aligned beyond their elements.
template <bool BF16> __device__ __forceinline__ void load4(const void *base, int64_t off, int valid, float (&x)[4]) {
    if (valid >= 4) {
        if constexpr (BF16) {
            typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));
            const u16x4 t = *(const u16x4 *)((const uint16_t *)base + off);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = bf16_to_f32(t[e]);
        } else {
            typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
            const f32x4 t = *(const f32x4 *)((const float *)base + off);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = t[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = e < valid ? load_elem<BF16>(base, off + e) : 0.f;
    }
}
template <bool BF16> __device__ __forceinline__ void store4(void *base, int64_t off, int valid, const float (&x)[4]) {
    if (valid >= 4) {
        if constexpr (BF16) {
            typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));
            u16x4 t;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = f32_to_bf16_rne(x[e]);
            *(u16x4 *)((uint16_t *)base + off) = t;
        } else {
            typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
            *(f32x4 *)((float *)base + off) = f32x4{x[0], x[1], x[2], x[3]};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < valid) store_elem<BF16>(base, off + e, x[e]);
    }
}

// Item of element e of piece j of a thread, relative to its tile
__device__ __forceinline__ int tile_item(int j, int tid) { return (j * TILE_THREADS + tid) * 4; }

// The rules of one row.
struct RowRules {
    int64_t h0, h1, e0, e1;  // the row's parts of the lists; empty without a list
    float r, p, f;
    const uint32_t *allowed;
    __device__ RowRules(const RuleArgs &a, int64_t row) {
        auto part = [row](const RowList &l, int64_t &b, int64_t &e) {
            b = e = 0;
            if (l.indptr) {
                b = l.indptr[row];
                e = l.indptr[row + 1];
                if (b < 0) b = 0;
                if (e > l.nnz) e = l.nnz;
            }
        };
        part(a.history, h0, h1);
        part(a.entries, e0, e1);
        r = a.repetition; p = a.presence; f = a.frequency;
        if (a.penalties) {
            r = a.penalties[3 * row];
            p = a.penalties[3 * row + 1];
            f = a.penalties[3 * row + 2];
        }
        allowed = a.allowed ? a.allowed + row * a.allowed_ld : nullptr;
    }
    __device__ bool listed() const { return h0 < h1 || e0 < e1; }
};

// Counts and places of the tile's items: `count` and `place` hold TILE words each (place: 0, or 1 + the entry's index in its row).
// All threads of the workgroup call it; it ends with a barrier.
__device__ __forceinline__ void tile_lists(const RuleArgs &a, const RowRules &row, int64_t first, uint32_t *count, uint32_t *place, int tid) {
    const bool h = row.h0 < row.h1, e = row.e0 < row.e1;
    if (!h && !e) return;
    __syncthreads();  // the last tile's words have been read
    for (int i = tid * 4; i < TILE; i += TILE_THREADS * 4) {
        if (h) *(uint4 *)(count + i) = make_uint4(0, 0, 0, 0);
        if (e) *(uint4 *)(place + i) = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    if (h)
        for (int64_t i = row.h0 + tid; i < row.h1; i += TILE_THREADS) {
            const int64_t at = (int64_t)a.history.indices[i] - first;
            if (at >= 0 && at < TILE) atomicAdd(count + at, 1u);
        }
    if (e)
        for (int64_t i = row.e0 + tid; i < row.e1; i += TILE_THREADS) {
            const int64_t at = (int64_t)a.entries.indices[i] - first;
            if (at >= 0 && at < TILE) atomicMax(place + at, (uint32_t)(i - row.e0) + 1u);
        }
    __syncthreads();
}

// x changed by the rules; `at`: items relative to the tile, a multiple of 4.  Every operation rounds by itself, as it is defined.
__device__ __forceinline__ void apply_rules(const RuleArgs &a, const RowRules &row, int64_t first, int at, int valid,
                                            const uint32_t *count, const uint32_t *place, float (&x)[4]) {
#pragma clang fp contract(off)
    if (row.h0 < row.h1) {
        const uint4 c4 = *(const uint4 *)(count + at);
        const uint32_t c[4] = {c4.x, c4.y, c4.z, c4.w};
        if (c4.x | c4.y | c4.z | c4.w) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c[e]) {
                    const float v = x[e] > 0.f ? x[e] / row.r : x[e] * row.r;
                    const float t = row.f * (float)c[e];
                    x[e] = (v - t) - row.p;
                }
        }
    }
    if (a.bias) {
        float b[4];
        load4<false>(a.bias, first + at, valid, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = x[e] + b[e];
    }
    if (row.e0 < row.e1) {
        const uint4 p4 = *(const uint4 *)(place + at);
        const uint32_t p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (p[e]) x[e] = x[e] + (a.entries.values ? a.entries.values[row.e0 + p[e] - 1] : 1.f);
    }
    if (row.allowed && valid > 0) {
        const uint32_t bits = row.allowed[(first + at) >> 5] >> (at & 31);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!((bits >> e) & 1u)) x[e] = -INFINITY;
    }
}

}  // namespace als
