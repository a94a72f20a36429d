// Linear recurrences along the rows of a CSR matrix, entries taken together however rows lie among them.
//
// Every entry is a map s -> k s + b of a row's state, in each column by itself; maps compose to maps (k2 k1, k2 b1 + b2), so a row can
// be cut anywhere and its parts joined.  What a lane walks one entry after the other are products; 1 - k goes along, and where a state
// crosses a group's or a piece's border k near 1 is held as what is missing to it (share_of), so that the rounding of a gate near 1
// counts for some entries, not once for every entry of the row (sums of 1 - k: one multiply-add an entry, recur_rows 469 -> 484 us; shares
// for every entry by itself: 603).  The entries are cut into chunks of the same length, one per wavefront, so that the work is
// even whatever the rows' lengths are; groups of lanes hold the d columns of one entry, 16 bytes of the tables each.
//
//   last states, sums       a group walks a stretch of the chunk's entries from a state of zero, a row after the other, the next entries
//   (last_states)           under way; where a row began before the stretch, its map is kept too.  The stretches are joined once.
//   all states, gradients   a tile at a time: each group composes the maps of K entries, the groups' maps are joined (log2 steps across the
//   (entries)               wavefront), and with the state that comes in each group walks its entries again from registers.
//
// Rows of at most `longest` entries belong whole to the chunk that they begin in.  A longer row is cut at the chunks' borders, and its
// pieces' maps go to the workspace (one size from als_create on):
//   last states, sums       join_kernel composes the pieces of each long row
//   all states, gradients   pieces_kernel makes the pieces' maps first, join_kernel the state at each border, from which the walk goes on.
//                           The tables are read twice for entries of long rows; a row's maps cannot wait for the rows before, and what
//                           the card holds of the entries at a time (128 MB of registers) is a tenth of a large call's.
// Memory bounds all of it for large calls (figures at the operators).  A wavefront is its own workgroup: nothing waits for others.
// Chunks: 495, 482, 489, 562 us with 8192, 16384, 32768, 65536 of them for the last states of 300000 rows (d = 128, bf16), 1435, 1363, 1365,
// 1442 for all states.  Rows of up to 1, 2, 4, 8 chunks uncut 489, 497, 524, 575: a long row at the end keeps one wavefront busy and the
// others wait.  Where all states are wanted, and entries of cut rows are read twice, it is the same: 1365, 1380, 1416, 1483, and gradients
// of a page of 2000 rows of 20 (d = 64) 42.6 and 50 with 1 and 2.
//
// Both walks, along a row and from its end, are this one: index i counts in the direction of the walk.  Branches and loops around values
// are the wavefront's, never some lanes' (those have stores alone), and no vector register is spilled: the compiler was seen to place a
// copy of a live address at the end of such a branch, before the other lanes are back.  So what a choice takes is computed for
// every lane first; test_walk_registers.py looks at what was built.
#pragma once

#include <algorithm>
#include <type_traits>

#include "entry_rows.h"

namespace als {

constexpr int WALK_STAGE = 128;         // entries whose ids and marks are in LDS at a time
constexpr int LAST_STAGE = 512;         // the same where only last states are wanted: the groups' maps are joined once a stage
constexpr int WALK_MAX_CHUNKS = 32768;  // 2 KB of workspace each
// A row's pieces among so few chunks are composed by every wavefront that needs them, without a launch of their own: the states of a row of
// 300 entries 16.5 us instead of 20.3 (d = 64), of 1000 17.8 and 21.0; from 2000 on, beyond it, the same.  With 192 instead of 48, 21 us for
// 2000 entries and 38 for 6000: a wavefront composes a hundred pieces.
constexpr int FEW_CHUNKS = 48;

// Chunks, and what is kept of each for rows that cross its border: maps (k, b) of `d` columns.
//   across  of the part of a long row up to the border that the walk leaves the chunk by
//   close   of the part that ends within the chunk; or, where states are needed, the state that comes in (b)
//   rows    the long row whose pieces join_kernel composes on behalf of this chunk
struct JoinedRow {
    int32_t row, pieces;  // none: 0 pieces
};
struct Chunks {
    int64_t size, count, longest;
    float *across, *close;  // [count][2][d]
    JoinedRow *rows;          // [count]
};

template <int STAGE> struct Marks {
    int32_t id[STAGE], start[STAGE], end[STAGE];  // item, or -1; row that begins, ends there in the walk, or -1
};

// A value that all lanes of the wavefront have.
__device__ __forceinline__ int64_t wave_uniform(int64_t v) {
    return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) | (int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32;
}
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
    return (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)v, lane) | (int64_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32;
}

// The lists as a wavefront walks them.  indptr is clamped wherever it is read, so that no index leaves the buffers.
struct RowFinder {
    Lists y;
    int64_t first, end;  // entries that belong to rows
    __device__ __forceinline__ int64_t at(int64_t u) const { return min(max(y.indptr[u], (int64_t)0), y.nnz); }
    __device__ __forceinline__ explicit RowFinder(const Lists &lists) : y(lists) {
        first = wave_uniform(at(0));
        end = max(first, wave_uniform(at(y.rows)));
    }
    // The last rows that begin at or before p and q: 64 places at a time, both searches' loads under way together.
    __device__ void rows_of(int64_t p, int64_t q, int64_t &up, int64_t &uq) const {
        int64_t lo[2] = {0, 0}, hi[2] = {y.rows, y.rows};
        while (hi[0] - lo[0] > 1 || hi[1] - lo[1] > 1) {
            int64_t step[2], b[2], u[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                step[i] = (hi[i] - lo[i] + 63) / 64;
                u[i] = lo[i] + (threadIdx.x & 63) * step[i];
                b[i] = at(min(u[i], y.rows));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const unsigned long long below = __ballot((u[i] < hi[i]) & (b[i] <= (i ? q : p)));
                const int k = below ? 63 - __builtin_clzll(below) : 0;
                lo[i] += k * step[i];
                hi[i] = min(hi[i], lo[i] + step[i]);
            }
        }
        up = lo[0];
        uq = lo[1];
    }
    __device__ __forceinline__ int64_t row_of(int64_t p) const {
        int64_t u, same;
        rows_of(p, p, u, same);
        return u;
    }
    struct Row {
        int64_t u, b, e;
    };
};

// What a chunk has of rows: entries [low, high), and the long rows that cross its borders.
struct ChunkRows {
    int64_t low, high;           // borders of the chunk among the rows' entries
    bool split_low, split_high;  // a long row crosses that border
    RowFinder::Row at_low, at_high;  // the rows at the chunk's first entry and behind its last
    // the border at x: behind a short row that lies across it
    static __device__ __forceinline__ int64_t border(const RowFinder &f, int64_t x, int64_t longest, const RowFinder::Row &r, bool &split) {
        split = false;
        if (x <= f.first) return f.first;
        if (x >= f.end) return f.end;
        if (r.b >= x || r.e <= x) return x;
        if (r.e - r.b <= longest) return min(r.e, f.end);
        split = true;
        return x;
    }
    __device__ __forceinline__ ChunkRows(const RowFinder &f, const Chunks &c, int64_t chunk) {
        const int64_t x = chunk * c.size, last = max(f.end - 1, f.first);
        f.rows_of(min(max(x, f.first), last), min(max(x + c.size, f.first), last), at_low.u, at_high.u);
        const int64_t bl = f.at(at_low.u), el = f.at(at_low.u + 1), bh = f.at(at_high.u), eh = f.at(at_high.u + 1);
        at_low.b = wave_uniform(bl);
        at_low.e = wave_uniform(el);
        at_high.b = wave_uniform(bh);
        at_high.e = wave_uniform(eh);
        low = border(f, x, c.longest, at_low, split_low);
        high = border(f, x + c.size, c.longest, at_high, split_high);
    }
    __device__ __forceinline__ bool through() const { return split_low && split_high && at_low.u == at_high.u; }  // one row all over
    // where the search for the rows of a walk from `from` on (down from it) begins
    __device__ __forceinline__ int64_t row_from(int64_t from) const { return from >= at_low.e ? at_low.u + 1 : at_low.u; }
};

// Ids and marks of entries i = 0 .. n-1 of the walk from `from` on (down from from - 1 where BACK).  `row`: where the search for rows
// begins, moved along.  Workgroups are single wavefronts.
template <bool BACK, int STAGE> __device__ void stage_entries(const RowFinder &f, Marks<STAGE> &m, int64_t from, int n, int64_t &row) {
    const int lane = threadIdx.x;
    __syncthreads();
#pragma unroll 2
    for (int i = lane; i < STAGE; i += 64) {
        const int64_t p = BACK ? from - 1 - min(i, n - 1) : from + min(i, n - 1);  // behind the last one: the last one again
        const int id = f.y.ids ? f.y.ids[p] : (int)p;
        m.id[i] = (i < n) & (id < f.y.cols) ? id : -1;
        m.start[i] = m.end[i] = -1;
    }
    __syncthreads();
    const int64_t t0 = BACK ? from - n : from, t1 = BACK ? from : from + n;
    for (int64_t base = row;;) {
        const int64_t u = BACK ? base - lane : base + lane;
        const bool some = u >= 0 && u < f.y.rows;
        const int64_t inside = min(max(u, (int64_t)0), f.y.rows - 1), bu = f.at(inside), eu = f.at(inside + 1);
        const int64_t b = some ? bu : BACK ? t0 : t1, e = some ? eu : b;
        const bool active = some & (b < e) & (b < t1) & (e > t0);
        if (active) {
            if (b >= t0) (BACK ? m.end : m.start)[BACK ? t1 - 1 - b : b - t0] = (int)u;
            if (e <= t1) (BACK ? m.start : m.end)[BACK ? t1 - e : e - 1 - t0] = (int)u;
        }
        const unsigned long long who = __ballot(active);
        if (who) row = BACK ? base - (63 - __builtin_clzll(who)) : base + (63 - __builtin_clzll(who));
        const int64_t far = lane_value(BACK ? b : e, 63);  // where the row behind these begins
        if (BACK) {
            if (base < 64 || far <= t0) break;
            base = who ? base - 64 : min(base - 64, f.row_of(far - 1));
        } else {
            if (base + 64 >= f.y.rows || far >= t1) break;
            base = who ? base + 64 : max(base + 64, f.row_of(far));
        }
    }
    __syncthreads();
}

// The state behind a map that keeps the share k.
template <class Op> __device__ __forceinline__ float after(float k, float s, float b) { return Op::ONES ? s + b : after_map(k, s, b); }

// A wavefront's walk.  Op:
//   N, K, L           columns a lane, entries a group of lanes takes in a tile, lanes of a group
//   BACK, ONES        from the rows' ends; k is 1 everywhere (sums: last_states alone)
//   STEP              entries a group takes at a time where only last states or maps are wanted
//   EARLY             what rows begin with is loaded along with their entries, into registers
//   Raw               what is loaded of one entry
//   load(raw, p, id)  of entry p; id -1: it has no item, and what is loaded in the item's place leaves the state as it is
//   load_map(raw, p, id)   what its map takes of that
//   map(raw, k, t, b) its map: what it keeps, 1 - k to bits of its own, what it adds
//   begin(row, s)     a row's first state
//   KEEP: output(p, valid, s)   after an entry whose map was kept in registers
//   otherwise: entry(raw, has an item, p, valid, ending, ends, i, s)   moves s on by itself; ends[i]: the row that ends there
//   finish(row, mine, s)   a row's last state, where `mine`
template <class Op> struct Walk {
    static constexpr int N = Op::N, K = Op::K, L = Op::L, GROUPS = 64 / L, TILE = GROUPS * K, STEP = Op::STEP, LAST_TILE = GROUPS * STEP;
    static_assert(WALK_STAGE % TILE == 0 && LAST_STAGE % LAST_TILE == 0, "a stage is whole tiles");
    const Op &op;
    const RowFinder &rows;
    int lane, group;
    float s[N];  // the state that comes into the tile, the same in all groups
    __device__ __forceinline__ Walk(const Op &o, const RowFinder &r) : op(o), rows(r), lane(threadIdx.x % L), group(threadIdx.x / L) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = 0.f;
    }

    // The groups' maps (k, 1 - k as t, b) joined: the state that comes into every group, and s behind the tile.
    // seen: the group's entries hold a row's start, so that nothing of what comes in reaches its end.
    __device__ __forceinline__ void join(float (&k)[N], float (&t)[N], float (&b)[N], bool seen, float (&in)[N]) {
#pragma unroll
        for (int step = 1; step < GROUPS; step *= 2) {
            const unsigned long long starts = __ballot(seen);
            const bool take = group >= step && !seen;
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const float bo = __shfl_up(b[c], step * L);
                if (!Op::ONES) {
                    const float ko = __shfl_up(k[c], step * L), to = __shfl_up(t[c], step * L);
                    b[c] = take ? fmaf(k[c], bo, b[c]) : b[c];
                    t[c] = take ? fmaf(k[c], to, t[c]) : t[c];
                    k[c] = take ? k[c] * ko : k[c];
                } else {
                    b[c] = take ? b[c] + bo : b[c];
                }
            }
            if (group >= step) seen = seen || (starts >> (threadIdx.x - step * L) & 1);
        }
        // the state behind each group; it comes into the next one, the last group's into the next tile
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const float behind = chosen(seen, b[c], after<Op>(share_of(k[c], t[c]), s[c], b[c]));
            const float prior = __shfl_up(behind, L);
            in[c] = group == 0 ? s[c] : prior;
            s[c] = __shfl(behind, (GROUPS - 1) * L + lane);
        }
    }

    // Entries [from, from + n) (down from from - 1 where BACK) with all their rows; s is the state that comes in.
    // row: where the search for their rows begins.
    __device__ void entries(Marks<WALK_STAGE> &m, int64_t from, int64_t n, int64_t row) {
        for (int64_t done = 0; done < n; done += WALK_STAGE) {
            const int64_t here = Op::BACK ? from - done : from + done;
            const int many = (int)min(n - done, (int64_t)WALK_STAGE);
            stage_entries<Op::BACK, WALK_STAGE>(rows, m, here, many, row);
            for (int tile = 0; tile < many; tile += TILE) {
                const int i0 = tile + group * K;
                typename Op::Raw raw[K];
                float early[Op::EARLY ? K : 1][N];
                int starts = 0, ends = 0;  // a bit per entry: a row starts, ends there
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    const int id = m.id[i0 + j];
                    starts |= (m.start[i0 + j] >= 0) << j;
                    ends |= (m.end[i0 + j] >= 0) << j;
                    if constexpr (Op::EARLY) {  // what a row begins with, under way with the rest
                        if (__any(starts >> j & 1)) op.begin(max(m.start[i0 + j], 0), lane, early[j]);
                    }
                    // entries behind the last one: any that is there
                    op.load(raw[j], Op::BACK ? here - 1 - min(i0 + j, many - 1) : here + min(i0 + j, many - 1), id, lane);
                }
                // No branch that some lanes take but for stores: a value is chosen, what is read for it is somewhere that can be read.
                float k[N], t[N], b[N], keep[Op::KEEP ? K : 1][N], add[Op::KEEP ? K : 1][N];
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    float kj[N], tj[N], bj[N];
                    op.map(raw[j], kj, tj, bj);
                    const bool starting = starts >> j & 1;
                    if (j == 0) {
#pragma unroll
                        for (int c = 0; c < N; ++c) b[c] = 0.f;
                    }
                    if (__any(starting)) {
                        float first[N];
                        if constexpr (!Op::EARLY) op.begin(max(m.start[i0 + j], 0), lane, first);
#pragma unroll
                        for (int c = 0; c < N; ++c) b[c] = starting ? (Op::EARLY ? early[j][c] : first[c]) : b[c];
                    }
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        b[c] = fmaf(kj[c], b[c], bj[c]);
                        t[c] = j ? fmaf(tj[c], k[c], t[c]) : tj[c];
                        k[c] = j ? k[c] * kj[c] : kj[c];
                        if constexpr (Op::KEEP) {
                            keep[j][c] = kj[c];
                            add[j][c] = bj[c];
                        }
                    }
                }
                float h[N];
                join(k, t, b, starts != 0, h);
                int64_t p0 = Op::BACK ? here - 1 - i0 : here + i0;
                asm("" : "+v"(p0));  // known here: addresses of all K outputs carried along the loop take 32 registers
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    const bool starting = starts >> j & 1, ending = ends >> j & 1;
                    if (__any(starting)) {
                        float first[N];
                        if constexpr (!Op::EARLY) op.begin(max(m.start[i0 + j], 0), lane, first);
#pragma unroll
                        for (int c = 0; c < N; ++c) h[c] = starting ? (Op::EARLY ? early[j][c] : first[c]) : h[c];
                    }
                    const int64_t p = Op::BACK ? p0 - j : p0 + j;
                    if constexpr (Op::KEEP) {
#pragma unroll
                        for (int c = 0; c < N; ++c) h[c] = fmaf(keep[j][c], h[c], add[j][c]);
                        op.output(p, i0 + j < many, lane, h);
                    } else {
                        op.entry(raw[j], m.id[i0 + j] >= 0, p, i0 + j < many, ending, m.end, i0 + j, lane, h);
                    }
                    if (__any(ending)) op.finish(max(m.end[i0 + j], 0), ending, lane, h);
                }
            }
        }
    }

    // The same where only rows' last states are wanted: every group walks a stretch of a stage's entries from a state of zero, and
    // the stretches' maps are joined once.  A row that ends in a stretch but began before it waits for that.
    __device__ void last_states(Marks<LAST_STAGE> &m, int64_t from, int64_t n, int64_t row) {
        for (int64_t done = 0; done < n; done += LAST_STAGE) {
            const int64_t here = from + done;
            const int many = (int)min(n - done, (int64_t)LAST_STAGE);
            stage_entries<false, LAST_STAGE>(rows, m, here, many, row);
            const int stretch = (many + LAST_TILE - 1) / LAST_TILE * STEP, first = group * stretch;
            float k[N], t[N], b[N], head_k[N], head_b[N];
            int head = -1;
            bool seen = false;
#pragma unroll
            for (int c = 0; c < N; ++c) {
                k[c] = 1.f;
                head_k[c] = KEEPS_ALL;
                t[c] = b[c] = head_b[c] = 0.f;
            }
            typename Op::Raw raw[2][STEP];
            auto load = [&](auto which, int at) {
#pragma unroll
                for (int j = 0; j < STEP; ++j) {
                    const int i = min(first + at + j, LAST_STAGE - 1);
                    op.load(raw[which()][j], here + min(i, many - 1), m.id[i], lane);
                }
            };
            auto walk = [&](auto which, int at) {
                const bool open = __any(!seen);
#pragma unroll
                for (int j = 0; j < STEP; ++j) {
                    const int i = min(first + at + j, LAST_STAGE - 1);
                    const int start = m.start[i], end = m.end[i];
                    float kj[N], tj[N], bj[N];
                    op.map(raw[which()][j], kj, tj, bj);
                    if (__any(start >= 0)) {
                        float s0[N];
                        op.begin(max(start, 0), lane, s0);
#pragma unroll
                        for (int c = 0; c < N; ++c) b[c] = start >= 0 ? s0[c] : b[c];
                        seen = seen || start >= 0;
                    }
#pragma unroll
                    for (int c = 0; c < N; ++c) b[c] = Op::ONES ? b[c] + bj[c] : fmaf(kj[c], b[c], bj[c]);
                    if (!Op::ONES && open) {
#pragma unroll
                        for (int c = 0; c < N; ++c) {
                            t[c] = fmaf(tj[c], k[c], t[c]);
                            k[c] *= kj[c];
                        }
                    }
                    if (__any(end >= 0)) {
                        if (__any(end >= 0 && !seen)) {
                            const bool wait = end >= 0 && !seen;
#pragma unroll
                            for (int c = 0; c < N; ++c) {
                                head_k[c] = wait ? share_of(k[c], t[c]) : head_k[c];
                                head_b[c] = wait ? b[c] : head_b[c];
                            }
                            head = wait ? end : head;
                        }
                        op.finish(max(end, 0), end >= 0 && seen, lane, b);
                    }
                }
            };
            constexpr std::integral_constant<int, 0> even{};
            constexpr std::integral_constant<int, 1> odd{};
            load(even, 0);
            for (int at = 0; at < stretch; at += 2 * STEP) {
                if (at + STEP < stretch) load(odd, at + STEP);
                walk(even, at);
                if (at + STEP < stretch) {
                    if (at + 2 * STEP < stretch) load(even, at + 2 * STEP);
                    walk(odd, at + STEP);
                }
            }
            float in[N];
            join(k, t, b, seen, in);
            if (__any(head >= 0)) {
#pragma unroll
                for (int c = 0; c < N; ++c) head_b[c] = after<Op>(head_k[c], in[c], head_b[c]);
                op.finish(max(head, 0), head >= 0, lane, head_b);
            }
        }
    }

    // The map of entries [from, from + n) of one row (down from from - 1 where BACK), of the row's first state and them where
    // `row` >= 0; to `out` [2][d].  Every group takes a stretch.
    __device__ void piece(int64_t from, int64_t n, int64_t row, float *out) {
        const int64_t stretch = (n + LAST_TILE - 1) / LAST_TILE * STEP, first = group * stretch;
        float k[N], b[N];           // of all entries so far: the share that is kept, what is added
        float rk[N], rt[N], rb[N];  // of the last up to 32, as products
#pragma unroll
        for (int c = 0; c < N; ++c) {
            k[c] = KEEPS_ALL;
            rk[c] = 1.f;
            b[c] = rt[c] = rb[c] = 0.f;
        }
        if (row >= 0) {  // the first group's stretch begins with the row
            float s0[N];
            op.begin(row, lane, s0);
#pragma unroll
            for (int c = 0; c < N; ++c) {
                b[c] = group == 0 ? s0[c] : 0.f;
                k[c] = group == 0 ? 0.f : KEEPS_ALL;
            }
        }
        int id[STEP];
        typename Op::Raw raw[STEP];
        auto find = [&](int64_t at) {
#pragma unroll
            for (int j = 0; j < STEP; ++j) {
                const int64_t i = first + at + j, inside = min(i, n - 1), p = Op::BACK ? from - 1 - inside : from + inside;
                id[j] = rows.y.ids ? rows.y.ids[p] : (int)p;
                if (i >= n || id[j] >= rows.y.cols) id[j] = -1;
            }
        };
        find(0);
        for (int64_t at = 0; at < stretch; at += STEP) {
#pragma unroll
            for (int j = 0; j < STEP; ++j) {
                const int64_t inside = min(first + at + j, n - 1);
                op.load_map(raw[j], Op::BACK ? from - 1 - inside : from + inside, id[j], lane);
            }
            if (at + STEP < stretch) find(at + STEP);
#pragma unroll
            for (int j = 0; j < STEP; ++j) {
                float kj[N], tj[N], bj[N];
                op.map(raw[j], kj, tj, bj);
                if (Op::BACK) {  // gradients of entries without an item count, those behind the end do not
                    const bool on = first + at + j < n;
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        bj[c] = on ? bj[c] : 0.f;
                        kj[c] = on ? kj[c] : 1.f;
                        tj[c] = on ? tj[c] : 0.f;
                    }
                }
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    rb[c] = Op::ONES ? rb[c] + bj[c] : fmaf(kj[c], rb[c], bj[c]);
                    if (!Op::ONES) rt[c] = fmaf(tj[c], rk[c], rt[c]);
                    if (!Op::ONES) rk[c] *= kj[c];
                }
            }
            if (at + STEP < stretch && (at / STEP + 1) % (32 / STEP) != 0) continue;
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const float q = share_of(rk[c], rt[c]);
                b[c] = after<Op>(q, b[c], rb[c]);
                if (!Op::ONES) k[c] = share_of_both(k[c], q);
                rk[c] = 1.f;
                rt[c] = rb[c] = 0.f;
            }
        }
#pragma unroll
        for (int step = 1; step < GROUPS; step *= 2) {
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const float bo = __shfl_up(b[c], step * L), ko = __shfl_up(k[c], step * L);
                const bool take = group >= step;
                b[c] = chosen(take, after<Op>(k[c], bo, b[c]), b[c]);
                if (!Op::ONES) k[c] = chosen(take, share_of_both(ko, k[c]), k[c]);
            }
        }
        if (group == GROUPS - 1) {
#pragma unroll
            for (int c = 0; c < N; ++c) {
                out[lane * N + c] = k[c];
                out[N * L + lane * N + c] = b[c];
            }
        }
    }
};

// The rows without entries, 64 looked at and GROUPS written at a time; workgroup `at` of `of`.
template <class Op> __device__ void empty_rows(const Op &op, const RowFinder &f, int64_t at, int64_t of) {
    constexpr int GROUPS = 64 / Op::L;
    const int lane = threadIdx.x % Op::L, group = threadIdx.x / Op::L;
    for (int64_t u0 = at * 64; u0 < f.y.rows; u0 += of * 64) {
        const int64_t u = min(u0 + threadIdx.x, f.y.rows - 1);
        const unsigned long long none = __ballot(u0 + threadIdx.x < f.y.rows && f.at(u) >= f.at(u + 1));
        if (none == 0) continue;
#pragma unroll 4
        for (int i = group; i < 64; i += GROUPS) {
            const bool mine = none >> i & 1;
            const int64_t row = mine ? u0 + i : u0;
            float s[Op::N];
            op.begin(row, lane, s);
            op.finish(row, mine, lane, s);
        }
    }
}

// The long row that join_kernel composes on behalf of a chunk (uniform in the wavefront).
__device__ __forceinline__ void leave_long_row(const Chunks &c, int64_t chunk, bool some, const RowFinder::Row &r) {
    if (threadIdx.x == 0) {
        const int64_t first = r.b / c.size, last = min((r.e - 1) / c.size, c.count - 1);
        c.rows[chunk] = JoinedRow{(int32_t)r.u, some ? (int32_t)max(last - first, (int64_t)0) : 0};
    }
}

// Last states: every chunk's short rows, and the maps of its long rows' pieces.
template <class Op> __global__ __launch_bounds__(64, Op::WAVES) void walk_last_kernel(Op op, Lists y, Chunks c) {
    constexpr int D = Op::N * Op::L;
    __shared__ __align__(16) Marks<LAST_STAGE> m;
    const RowFinder f(y);
    const int64_t chunk = blockIdx.x;
    if (chunk >= c.count) return empty_rows(op, f, chunk - c.count, gridDim.x - c.count);
    const ChunkRows r(f, c, chunk);
    leave_long_row(c, chunk, r.split_low && !r.through(), r.at_low);
    int64_t low = r.low, high = r.high;
    if (r.split_low && low < high) {
        const int64_t e = min(r.at_low.e, high);
        Walk<Op>(op, f).piece(low, e - low, -1, (r.through() ? c.across : c.close) + chunk * 2 * D);
        low = e;
    }
    if (r.split_high && low < high) {
        const int64_t b = max(r.at_high.b, low);
        Walk<Op>(op, f).piece(b, high - b, r.at_high.u, c.across + chunk * 2 * D);
        high = b;
    }
    if (low < high) Walk<Op>(op, f).last_states(m, low, high - low, r.row_from(low));
}

// A long row's pieces one after the other, on behalf of the chunk that the walk along the row begins in (CARRY: the state at every
// border it crosses goes to the chunk behind it) or ends in (otherwise: the row's last state).
template <class Op, bool CARRY> struct Pieces {
    static constexpr int N = Op::N, D = N * Op::L, AHEAD = 4;
    const Chunks &c;
    int64_t chunk;
    int count, lane;
    float k[N], s[N];
    // piece i of the walk is kept with chunk at(i); without CARRY the chunk itself has the closing one
    __device__ __forceinline__ int64_t at(int i) const {
        return min(max(CARRY ? (Op::BACK ? chunk - i : chunk + i) : chunk - count + i, (int64_t)0), c.count - 1);
    }
    // pieces begin .. end - 1, which may be other ones in every lane: the loop is the wavefront's.  MAP: the share k too
    template <bool STORE, bool MAP> __device__ __forceinline__ void walk(int begin, int end) {
        for (int i0 = begin; __any(i0 < end); i0 += AHEAD) {
            float kp[AHEAD][N], bp[AHEAD][N];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const float *map = c.across + at(min(i0 + a, end - 1)) * 2 * D + lane * N;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    kp[a][j] = map[j];
                    bp[a][j] = map[D + j];
                }
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const bool on = i0 + a < end, first = i0 + a == 0;  // the first piece has the row's own first state in it
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float behind = after<Op>(kp[a][j], s[j], bp[a][j]), now = first ? bp[a][j] : behind;
                    s[j] = on ? now : s[j];
                    if (MAP && !Op::ONES) k[j] = chosen(on, share_of_both(k[j], kp[a][j]), k[j]);
                }
                if (STORE && on) {
                    float *to = c.close + (at(i0 + a + 1) * 2 + 1) * D + lane * N;
#pragma unroll
                    for (int j = 0; j < N; ++j) to[j] = s[j];
                }
            }
        }
    }
    __device__ __forceinline__ void finish(const Op &op, int row, bool mine) {
        const float *map = c.close + chunk * 2 * D + lane * N;
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] = after<Op>(map[j], s[j], map[D + j]);
        op.finish(row, mine, lane, s);
    }
};

// All entries' outputs; rows that come in begin with the state that join_kernel left, or, where chunks are few, with what the
// wavefront composes of the row's pieces itself: that saves a launch.
template <class Op> __global__ __launch_bounds__(64, Op::WAVES) void walk_all_kernel(Op op, Lists y, Chunks c) {
    constexpr int D = Op::N * Op::L;
    __shared__ __align__(16) Marks<WALK_STAGE> m;
    const RowFinder f(y);
    const int64_t chunk = blockIdx.x;
    if (chunk >= c.count) return empty_rows(op, f, chunk - c.count, gridDim.x - c.count);
    const ChunkRows r(f, c, chunk);
    if (r.low >= r.high) return;
    Walk<Op> walk(op, f);
    if (Op::BACK ? r.split_high : r.split_low) {
        if (c.count <= FEW_CHUNKS) {
            const int64_t from = Op::BACK ? min((r.at_high.e - 1) / c.size, c.count - 1) : r.at_low.b / c.size;
            const int pieces = (int)(Op::BACK ? from - chunk : chunk - from);
            Pieces<Op, true> p{c, from, pieces, walk.lane, {}, {}};
            p.template walk<false, false>(0, pieces);
#pragma unroll
            for (int j = 0; j < Op::N; ++j) walk.s[j] = p.s[j];
        } else {
#pragma unroll
            for (int j = 0; j < Op::N; ++j) walk.s[j] = c.close[(chunk * 2 + 1) * D + walk.lane * Op::N + j];
        }
    }
    walk.entries(m, Op::BACK ? r.high : r.low, r.high - r.low, Op::BACK ? r.at_high.u : r.row_from(r.low));
}

// The map of the part of a long row that leads to the border where the walk leaves the chunk.
template <class Op> __global__ __launch_bounds__(64, Op::WAVES) void pieces_kernel(Op op, Lists y, Chunks c) {
    constexpr int D = Op::N * Op::L;
    const RowFinder f(y);
    const int64_t chunk = c.count - 1 - blockIdx.x;  // the walk begins with the chunks that were read last: the cache may hold them
    const ChunkRows r(f, c, chunk);
    const RowFinder::Row row = Op::BACK ? r.at_low : r.at_high;
    const bool out = Op::BACK ? r.split_low : r.split_high;
    leave_long_row(c, chunk, out && !r.through(), row);
    if (!out || r.low >= r.high) return;
    const int64_t low = max(r.low, row.b), high = min(r.high, row.e);
    Walk<Op>(op, f).piece(Op::BACK ? high : low, high - low, r.through() ? -1 : row.u, c.across + chunk * 2 * D);
}

// A workgroup looks at 64 chunks (16 rows of 1024 pieces of d = 128: 21 us).  Rows of a few pieces: a group of lanes each.  Others: their
// pieces are dealt out in stretches to all groups, whose maps are joined through LDS; the columns are dealt out to the workgroups of a
// second dimension.  JOIN_FEW: 8, 24, 72 are within a percent of each other where rows are of all lengths (gradients of 100000 rows 570,
// 569, 576 us) or all long; rows of 3000 entries 487, 486, 475.
constexpr int JOIN_THREADS = 512, JOIN_CHUNKS = 64, JOIN_FEW = 24;
template <class Op> constexpr int join_lanes() { return Op::L < 8 ? Op::L : 8; }
template <class Op, bool CARRY> __global__ __launch_bounds__(JOIN_THREADS) void join_kernel(Op op, Chunks c) {
    constexpr int N = Op::N, LANES = join_lanes<Op>(), GROUPS = JOIN_THREADS / LANES;
    __shared__ float maps[GROUPS][2][LANES * N];
    __shared__ int few_at[JOIN_CHUNKS];
    const int64_t chunk0 = (int64_t)blockIdx.x * JOIN_CHUNKS, look = chunk0 + (threadIdx.x & 63);
    const JoinedRow entry = c.rows[min(look, c.count - 1)];
    const int pieces = look < c.count ? entry.pieces : 0;
    if (blockIdx.y == 0) {
        const unsigned long long few = __ballot((pieces > 0) & (pieces <= JOIN_FEW));
        const int many = __popcll(few), lane = threadIdx.x % Op::L;
        // the places of the bits, the same from every wavefront
        if (few >> (threadIdx.x & 63) & 1) few_at[__popcll(few & ((1ull << (threadIdx.x & 63)) - 1))] = threadIdx.x & 63;
        __syncthreads();
        for (int n0 = 0; n0 < many; n0 += JOIN_THREADS / Op::L) {
            const int n = n0 + threadIdx.x / Op::L;  // the row that this group of lanes takes
            const bool mine = n < many;
            const int64_t chunk = chunk0 + few_at[min(n, many - 1)];
            const JoinedRow r = c.rows[chunk];
            Pieces<Op, CARRY> p{c, chunk, r.pieces, lane, {}, {}};
            p.template walk<CARRY, false>(0, mine ? r.pieces : 0);
            if (!CARRY) p.finish(op, r.row, mine);
        }
    }
    const int in_group = threadIdx.x % LANES, group = threadIdx.x / LANES;
    for (unsigned long long rest = __ballot(pieces > JOIN_FEW); rest; rest &= rest - 1) {
        const int64_t chunk = chunk0 + __ffsll((long long)rest) - 1;
        const JoinedRow r = c.rows[chunk];
        const int each = (r.pieces + GROUPS - 1) / GROUPS, begin = min(group * each, r.pieces), end = min(begin + each, r.pieces);
        const int groups = (r.pieces + each - 1) / each;
        Pieces<Op, CARRY> p{c, chunk, r.pieces, (int)blockIdx.y * LANES + in_group, {}, {}};
#pragma unroll
        for (int j = 0; j < N; ++j) p.k[j] = KEEPS_ALL;
        p.template walk<false, true>(begin, end);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            maps[group][0][in_group * N + j] = p.k[j];
            maps[group][1][in_group * N + j] = p.s[j];
        }
        __syncthreads();
        const int upto = CARRY ? min(group, groups) : groups;
        for (int g = 0; __any(g < upto); ++g)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float bg = maps[g][1][in_group * N + j], behind = after<Op>(maps[g][0][in_group * N + j], p.s[j], bg);
                const float now = g ? behind : bg;
                p.s[j] = g < upto ? now : p.s[j];
            }
        if (CARRY) p.template walk<true, false>(begin, end);
        else p.finish(op, r.row, group == 0);
        __syncthreads();
    }
}

// Chunks of the call's entries, and the longest rows that are not cut: a chunk, 4 tiles at least.  For small calls as many as the
// card holds wavefronts, of a tile at least; then of 64 entries, so that a chunk's search for its rows does not weigh; then as many as
// there is room for.
inline Chunks chunks_of(const als_ctx *ctx, int64_t nnz, int tile) {
    Chunks c{};
    const int64_t resident = (int64_t)ctx->num_cu * 12;
    const int64_t wanted = std::max((nnz + WALK_MAX_CHUNKS - 1) / WALK_MAX_CHUNKS, std::min<int64_t>(64, (nnz + resident - 1) / resident));
    c.size = std::max<int64_t>(1, (wanted + tile - 1) / tile) * tile;
    c.count = (nnz + c.size - 1) / c.size;
    c.longest = std::max<int64_t>(c.size, 4 * tile);
    c.across = (float *)ctx->walk_maps.p;
    c.close = c.across + (int64_t)WALK_MAX_CHUNKS * 2 * 128;
    c.rows = (JoinedRow *)(c.close + (int64_t)WALK_MAX_CHUNKS * 2 * 128);
    return c;
}
// behind the chunks': rows for entries without an item, 512 bytes each: zeros, gates in fp32, gates in bf16
constexpr size_t WALK_NONE = (size_t)WALK_MAX_CHUNKS * (4 * 128 * sizeof(float) + sizeof(JoinedRow)), WALK_BYTES = WALK_NONE + 3 * 512;
inline const char *none_row(const als_ctx *ctx, bool gates, bool bf16) { return (const char *)ctx->walk_maps.p + WALK_NONE + (!gates ? 0 : bf16 ? 1024 : 512); }
// Workgroups that look for empty rows, at most: 1M empty rows take 52, 48, 45 us with 1024, 4096, 16384 of them, 30M 1437, 1507, 1514.
constexpr int EMPTY_GROUPS = 4096;
template <class Op> dim3 join_grid(const Chunks &c) { return dim3((unsigned)((c.count + JOIN_CHUNKS - 1) / JOIN_CHUNKS), Op::L / join_lanes<Op>()); }
inline unsigned walk_grid(const Chunks &c, int64_t rows) { return (unsigned)(c.count + std::min<int64_t>((rows + 63) / 64, EMPTY_GROUPS)); }

template <class Op> void launch_last(const als_ctx *ctx, const Op &op, const als_csr *Y, hipStream_t s) {
    const Chunks c = chunks_of(ctx, Y->nnz, Walk<Op>::LAST_TILE);
    const Lists y = lists_of(Y);
    hipLaunchKernelGGL((walk_last_kernel<Op>), dim3(walk_grid(c, Y->rows)), dim3(64), 0, s, op, y, c);
    if (Y->nnz > c.longest) hipLaunchKernelGGL((join_kernel<Op, false>), join_grid<Op>(c), dim3(JOIN_THREADS), 0, s, op, c);
}

// F(bool) for a value that only the call knows
template <class F> auto pick(bool v, F &&f) { return v ? f(std::true_type{}) : f(std::false_type{}); }
template <class F> auto pick_d(int d, F &&f) {
    switch (d) {
        case 16: return f(std::integral_constant<int, 16>{});
        case 32: return f(std::integral_constant<int, 32>{});
        case 64: return f(std::integral_constant<int, 64>{});
        default: return f(std::integral_constant<int, 128>{});
    }
}

}  // namespace als
