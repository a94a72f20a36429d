// Rules on scores (als_rules) as als_adjust and als_select evaluate them, a tile of one row at a time.
//
// A workgroup works on a tile of consecutive items of one row, sixteen per thread, a thread on pieces of 16 bytes of scores.  Lists
// (history, entries) hold a row's items in any order, so nothing says which of them lie in the tile.  A word per item in LDS counts how
// often it occurs (history) or tells where it is stored last (entries); integer atomics, so the order does not matter.
//   short lists (up to LIST_REGS per lane): every wavefront holds the row's whole list in registers and enters the items that
//                its own elements cover, so that a tile needs no barrier, and none of this where the list has no item in it
//   long lists   the workgroup walks the list together, once per tile: the list times the row's tiles (als_select of 64 x 128000 with
//                250, 257 and 4000 ids a row: 28, 30 and 34 us)
#pragma once

#include <algorithm>

#include "als_internal.h"

namespace als {

constexpr int TILE_EPT = 16;  // items of a tile per thread
constexpr int LIST_REGS = 4;

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
// LDS bytes that the lists need for a tile
inline size_t rule_bytes(const RuleArgs &a, int tile) { return ((a.history.indptr ? tile : 0) + (a.entries.indptr ? tile : 0)) * sizeof(uint32_t); }

// A value that all lanes read and no kernel of the call writes, through the scalar cache.
template <class T> __device__ __forceinline__ T uniform_load(const T *p) {
    return *(const __attribute__((address_space(4))) T *)(uintptr_t)p;
}

// One value from lanes of the wavefront by lane moves (v_add_f32_dpp and the like): rows of 16 lanes first, then across them.
// F is associative and commutative; the result is in lane 63.
template <class T, class F> __device__ __forceinline__ T wave_scan(T x, T none, F &&f) {
    auto step = [&](auto ctrl, auto rows) {
        const int moved = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x), ctrl(), rows(), 0xf, false);
        x = f(x, __builtin_bit_cast(T, moved));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});  // from 1, 2, 4, 8 lanes below in the row
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});  // the row's end to the next row: rows 1 and 3
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});  // lane 31 to rows 2 and 3
    return x;  // of the lanes up to this one
}
template <class T, class F> __device__ __forceinline__ T wave_all(T x, T none, F &&f) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_scan(x, none, f)), 63));
}

// A thread's elements of a tile: PIECES times PER consecutive ones, 16 bytes.  Rows need not be aligned beyond their elements.
template <bool BF16, int NT> struct TileRow {
    static constexpr int THREADS = NT, TILE = NT * TILE_EPT;
    static constexpr int PER = BF16 ? 8 : 4, PIECES = TILE_EPT / PER;
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    Words raw[PIECES];
    static __device__ __forceinline__ int item(int j, int tid) { return (j * NT + tid) * PER; }  // relative to the tile
    // wavefront that has item `at` of the tile
    static __device__ __forceinline__ int owner(int at) { return (at / (64 * PER)) % (NT / 64); }

    // `row`: the row's scores; items from cols on are not read
    __device__ __forceinline__ void load(const char *row, uint32_t first, uint32_t cols, int tid) {
        typedef uint32_t Any __attribute__((ext_vector_type(4), aligned(2)));
        constexpr uint32_t ES = BF16 ? 2 : 4;
        const char *tile = row + (uint64_t)first * ES;
        if (first + TILE <= cols) {
#pragma unroll
            for (int j = 0; j < PIECES; ++j) raw[j] = *(const Any *)(tile + (uint32_t)item(j, tid) * ES);
        } else {
            // the row's last tile: what is read beyond its end is the last element again
            const uint32_t left = cols - first;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                const uint32_t at = item(j, tid);
                if (at + PER <= left) {
                    raw[j] = *(const Any *)(tile + at * ES);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (BF16) {
                            const uint16_t *t = (const uint16_t *)tile;
                            raw[j][e] = t[min(at + 2 * e, left - 1)] | (uint32_t)t[min(at + 2 * e + 1, left - 1)] << 16;
                        } else {
                            raw[j][e] = ((const uint32_t *)tile)[min(at + e, left - 1)];
                        }
                    }
                }
            }
        }
    }
    __device__ __forceinline__ void floats(float (&x)[PIECES][PER]) const {
#pragma unroll
        for (int j = 0; j < PIECES; ++j)
#pragma unroll
            for (int e = 0; e < PER; ++e)
                x[j][e] = !BF16 ? __uint_as_float(raw[j][e]) : __uint_as_float(e & 1 ? raw[j][e / 2] & 0xffff0000u : raw[j][e / 2] << 16);
    }
};

// One of a row's lists over the tiles that a workgroup works on.
template <class Row, bool PLACES> struct TileList {
    const int32_t *ids;
    int64_t begins = 0;  // the row's part of the list; none without a list
    int count = 0;
    uint32_t next = ~0u;    // short lists: the least item of the list that no tile has had yet
    int32_t id[LIST_REGS];  // short lists: entry 64 r + lane, -1 beyond
    uint32_t *words;        // a tile's words in LDS

    __device__ __forceinline__ bool in_regs() const { return count <= 64 * LIST_REGS; }
    __device__ __forceinline__ void find_next(uint32_t from) {
        uint32_t least = ~0u;  // ids below 0 are beyond all items as unsigned numbers
#pragma unroll
        for (int r = 0; r < LIST_REGS; ++r) least = min(least, (uint32_t)id[r] >= from ? (uint32_t)id[r] : ~0u);
        next = wave_all(least, ~0u, [](uint32_t a, uint32_t b) { return min(a, b); });
    }
    __device__ __forceinline__ void begin(const RowList &l, int64_t row, uint32_t first, uint32_t *lds, int tid) {
        words = lds;
        begins = count = 0;
        if (l.indptr) {
            int64_t b = uniform_load(l.indptr + row), e = uniform_load(l.indptr + row + 1);
            if (b < 0) b = 0;
            if (e > l.nnz) e = l.nnz;
            if (e > b) {
                begins = b;
                count = (int)std::min<int64_t>(e - b, INT32_MAX - 8 * Row::THREADS);
            }
        }
        ids = l.indices + begins;
        if (count == 0 || !in_regs()) return;
#pragma unroll
        for (int r = 0; r < LIST_REGS; ++r) id[r] = 64 * r + (tid & 63) < count ? ids[64 * r + (tid & 63)] : -1;
        // the words of the wavefront's own elements
#pragma unroll
        for (int j = 0; j < Row::PIECES; ++j)
#pragma unroll
            for (int c = 0; c < Row::PER; c += 4) *(uint4 *)(words + Row::item(j, tid) + c) = make_uint4(0, 0, 0, 0);
        find_next(first);
    }
    // Enters the tile's items; true where the wavefront's words may be other than 0.  Long lists: all threads come here, with barriers.
    __device__ __forceinline__ bool enter(uint32_t first, int tid) {
        if (in_regs()) {
            if (next - first >= Row::TILE) return false;
#pragma unroll
            for (int r = 0; r < LIST_REGS; ++r) {
                const uint32_t at = (uint32_t)id[r] - first;
                if (at < Row::TILE && Row::owner((int)at) == tid >> 6) {
                    if constexpr (PLACES) atomicMax(words + at, (uint32_t)(64 * r + (tid & 63)) + 1u);
                    else atomicAdd(words + at, 1u);
                }
            }
            return true;
        }
        __syncthreads();  // the last tile's words have been read
        for (int i = tid * 4; i < Row::TILE; i += Row::THREADS * 4) *(uint4 *)(words + i) = make_uint4(0, 0, 0, 0);
        __syncthreads();
#pragma unroll 1
        for (int i0 = tid; i0 < count; i0 += 8 * Row::THREADS) {  // eight loads under way
            uint32_t at[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) at[u] = (uint32_t)ids[min(i0 + u * Row::THREADS, count - 1)] - first;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = i0 + u * Row::THREADS;
                if (at[u] < Row::TILE && i < count) {
                    if constexpr (PLACES) atomicMax(words + at[u], (uint32_t)i + 1u);
                    else atomicAdd(words + at[u], 1u);
                }
            }
        }
        __syncthreads();
        return true;
    }
    // The words are read: those that were entered become 0 again.
    __device__ __forceinline__ void leave(uint32_t first, int tid) {
        if (!in_regs()) return;
#pragma unroll
        for (int r = 0; r < LIST_REGS; ++r) {
            const uint32_t at = (uint32_t)id[r] - first;
            if (at < Row::TILE && Row::owner((int)at) == tid >> 6) words[at] = 0;
        }
        find_next(first + Row::TILE);
    }
};

// Which rules a kernel has the code for: what a call has not given costs registers and a look per tile.
// Rules that als_select's kernels are built for: registers of rules that are not there cost wavefronts.  512 x 1M bf16 with
// history: 301 us by the kernel for all rules, 276 by its own.  als_adjust, which memory bounds with either, has one kernel.
enum RuleSet { RULES_NONE, RULES_HISTORY, RULES_ALL };
inline RuleSet rule_set(const RuleArgs &a) {
    return a.entries.indptr || a.bias || a.allowed ? RULES_ALL : a.history.indptr ? RULES_HISTORY : RULES_NONE;
}

// The rules of one row over the tiles that a workgroup works on.
template <class Row, RuleSet SET> struct RowRules {
    TileList<Row, false> history;
    TileList<Row, true> entries;
    float r, p, f;
    const uint32_t *allowed;
    // `first`: the first item that the workgroup works on
    __device__ __forceinline__ void begin(const RuleArgs &a, int64_t row, uint32_t first, uint32_t *lds, int tid) {
        history.begin(a.history, row, first, lds, tid);
        if constexpr (SET == RULES_ALL) entries.begin(a.entries, row, first, lds + (a.history.indptr ? Row::TILE : 0), tid);
        r = a.repetition; p = a.presence; f = a.frequency;
        if (a.penalties) {
            r = uniform_load(a.penalties + 3 * row);
            p = uniform_load(a.penalties + 3 * row + 1);
            f = uniform_load(a.penalties + 3 * row + 2);
        }
        if constexpr (SET == RULES_ALL) allowed = a.allowed ? a.allowed + row * a.allowed_ld : nullptr;
    }
    // x changed by the rules.  All threads of the workgroup come here.  Every operation rounds by itself, as it is defined.
    __device__ __forceinline__ void apply(const RuleArgs &a, uint32_t first, uint32_t cols, int tid, float (&x)[Row::PIECES][Row::PER]) {
#pragma clang fp contract(off)
        const bool had = history.enter(first, tid);
        bool added = false;
        if constexpr (SET == RULES_ALL) added = entries.enter(first, tid);
        if (had) {
#pragma unroll
            for (int j = 0; j < Row::PIECES; ++j)
#pragma unroll
                for (int q = 0; q < Row::PER; q += 4) {
                    const uint4 c4 = *(const uint4 *)(history.words + Row::item(j, tid) + q);
                    const uint32_t c[4] = {c4.x, c4.y, c4.z, c4.w};
                    if (c4.x | c4.y | c4.z | c4.w) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (c[e]) {
                                float &v = x[j][q + e];
                                const float t = v > 0.f ? v / r : v * r, u = f * (float)c[e];
                                v = (t - u) - p;
                            }
                    }
                }
            history.leave(first, tid);
        }
        if constexpr (SET != RULES_ALL) return;
        const uint32_t left = cols - first;
        __builtin_amdgcn_sched_barrier(0);  // one rule after the other: their loads together take more registers than there are
        if (a.bias) {
            const float *bias = a.bias + first;
#pragma unroll
            for (int j = 0; j < Row::PIECES; ++j)
#pragma unroll
                for (int q = 0; q < Row::PER; q += 4) {
                    const uint32_t at = Row::item(j, tid) + q;
                    if (at + 4 <= left) {
                        typedef float Any __attribute__((ext_vector_type(4), aligned(4)));
                        const Any b4 = *(const Any *)(bias + at);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[j][q + e] = x[j][q + e] + b4[e];
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[j][q + e] = x[j][q + e] + bias[min(at + e, left - 1)];
                    }
                }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (added) {
            const float *values = a.entries.values ? a.entries.values + entries.begins - 1 : nullptr;
#pragma unroll
            for (int j = 0; j < Row::PIECES; ++j)
#pragma unroll
                for (int q = 0; q < Row::PER; q += 4) {
                    const uint4 p4 = *(const uint4 *)(entries.words + Row::item(j, tid) + q);
                    const uint32_t place[4] = {p4.x, p4.y, p4.z, p4.w};
                    if (p4.x | p4.y | p4.z | p4.w) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (place[e]) x[j][q + e] = x[j][q + e] + (values ? values[place[e]] : 1.f);
                    }
                }
            entries.leave(first, tid);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (allowed) {
            const uint32_t *bits = allowed + (first >> 5);
#pragma unroll
            for (int j = 0; j < Row::PIECES; ++j) {
                const uint32_t at = Row::item(j, tid);
                const uint32_t word = (at < left ? bits[at >> 5] : 0u) >> (at & 31);
#pragma unroll
                for (int e = 0; e < Row::PER; ++e)
                    if (!((word >> e) & 1u)) x[j][e] = -INFINITY;
            }
        }
    }
};

}  // namespace als
