// Linear recurrences along the rows of a CSR matrix, entries taken together however rows lie among them.
//
// Every entry is a map s -> k s + b of a row's state (a column each); a row begins with a state of its own.  The entries are cut into
// chunks of the same length, one per wavefront, so that the work is even whatever the rows' lengths are.  A wavefront
// walks its chunk a tile at a time: a group of lanes holds the d columns of one entry, each group takes the next K entries.  The
// group joins its entries' maps, the groups' maps are joined across the wavefront (log2 steps), and with the state that comes in each
// group walks its entries again from registers, where outputs are made.  One read of the tables.
//
// Rows of at most `longest` entries belong whole to the chunk that they begin in.  A longer row is cut at the chunks' borders; its
// pieces' maps go to the workspace:
//   last states and sums   the same launch leaves the pieces, join_kernel composes those of each long row
//   all states, gradients  pieces_kernel makes the pieces' maps first (the tables are read twice for entries of long rows),
//                          carry_kernel the state at each border, then the walk begins with it
// Both walks, along a row and from its end, are this one: index i counts in the direction of the walk.
#pragma once

#include <algorithm>
#include <type_traits>

#include "entry_rows.h"

namespace als {

constexpr int WALK_STAGE = 128;       // entries whose ids and marks are in LDS at a time
constexpr int WALK_MAX_CHUNKS = 16384;

// Chunks, and what is kept of each for rows that cross its border: maps (k, b) of `d` columns.
//   across  of the part of a long row up to the border that the walk leaves the chunk by
//   close   of the part that ends within the chunk; or, where states are needed, the state that comes in (b)
struct Chunks {
    int64_t size, count, longest;
    float *across, *close;  // [count][2][d]
};

struct Marks {
    int32_t id[WALK_STAGE], start[WALK_STAGE], end[WALK_STAGE];  // item, or -1; row that begins, ends there in the walk, or -1
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
    // The last row that begins at or before p: 64 places at a time.
    __device__ int64_t row_of(int64_t p) const {
        int64_t lo = 0, hi = y.rows;
        while (hi - lo > 1) {
            const int64_t step = (hi - lo + 63) / 64, u = lo + (threadIdx.x & 63) * step;
            const unsigned long long below = __ballot(u < hi && at(u) <= p);
            const int k = below ? 63 - __builtin_clzll(below) : 0;
            lo += k * step;
            hi = min(hi, lo + step);
        }
        return lo;
    }
    struct Row {
        int64_t u, b, e;
    };
    __device__ __forceinline__ Row row_at(int64_t p) const {
        const int64_t u = row_of(p);
        return Row{u, wave_uniform(at(u)), wave_uniform(at(u + 1))};
    }
};

// What a chunk has of rows: entries [begin, end) of the walk without long rows' pieces, and the pieces.
struct ChunkRows {
    int64_t low, high;       // borders of the chunk among the rows' entries
    bool split_low, split_high;  // a long row crosses that border
    RowFinder::Row at_low, at_high;
    // the border at x: behind a short row that lies across it
    static __device__ __forceinline__ int64_t border(const RowFinder &f, int64_t x, int64_t longest, bool &split, RowFinder::Row &r) {
        split = false;
        r = RowFinder::Row{-1, 0, 0};
        if (x <= f.first) return f.first;
        if (x >= f.end) return f.end;
        r = f.row_at(x);
        if (r.b >= x || r.e <= x) return x;
        if (r.e - r.b <= longest) return min(r.e, f.end);
        split = true;
        return x;
    }
    __device__ __forceinline__ ChunkRows(const RowFinder &f, const Chunks &c, int64_t chunk) {
        low = border(f, chunk * c.size, c.longest, split_low, at_low);
        high = border(f, (chunk + 1) * c.size, c.longest, split_high, at_high);
    }
};

// Ids and marks of entries i = 0 .. n-1 of the walk from `from` on (down from from - 1 where BACK).  `row`: where the search for rows
// begins, moved along.  Workgroups are single wavefronts.
template <bool BACK> __device__ void stage_entries(const RowFinder &f, Marks &m, int64_t from, int n, int64_t &row) {
    const int lane = threadIdx.x;
    __syncthreads();
#pragma unroll
    for (int i = lane; i < WALK_STAGE; i += 64) {
        int id = -1;
        if (i < n) {
            const int64_t p = BACK ? from - 1 - i : from + i;
            id = f.y.ids ? f.y.ids[p] : (int)p;
            if (id >= f.y.cols) id = -1;
        }
        m.id[i] = id;
        m.start[i] = m.end[i] = -1;
    }
    __syncthreads();
    const int64_t t0 = BACK ? from - n : from, t1 = BACK ? from : from + n;
    for (int64_t base = row;;) {
        const int64_t u = BACK ? base - lane : base + lane;
        const bool some = u >= 0 && u < f.y.rows;
        const int64_t b = some ? f.at(u) : BACK ? t0 : t1, e = some ? f.at(u + 1) : b;
        const bool active = some && b < e && b < t1 && e > t0;
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

// A wavefront's walk.  Op:
//   N, K, L           columns a lane, entries a group of lanes takes in a tile, lanes of a group
//   BACK, ONES        from the rows' ends; k is 1 everywhere (sums)
//   Raw               what is loaded of one entry
//   load(raw, p, id)  of entry p (id >= 0, or any row of the tables where the entry has no item)
//   map(raw, some, k, b)   its map; the identity where it has no item (`some` false)
//   begin(row, s)     a row's first state
//   KEEP: output(p, valid, s)   after an entry whose map was kept in registers
//   otherwise: entry(raw, some, p, valid, ending, ends, i, s)   moves s on by itself; ends[i]: the row that ends there
//   finish(row, mine, s)   a row's last state, where `mine`
template <class Op> struct Walk {
    static constexpr int N = Op::N, K = Op::K, L = Op::L, GROUPS = 64 / L, TILE = GROUPS * K;
    static_assert(WALK_STAGE % TILE == 0, "");
    const Op &op;
    const RowFinder &rows;
    int lane, group;
    float s[N];  // the state that comes into the tile, the same in all groups
    __device__ __forceinline__ Walk(const Op &o, const RowFinder &r) : op(o), rows(r), lane(threadIdx.x % L), group(threadIdx.x / L) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = 0.f;
    }

    // The groups' maps joined: s_in for every group, and the tile's map as a whole in the last group's lanes (k, b, seen).
    // seen: the group's entries hold a row's start, so that nothing of what comes in reaches its end.
    __device__ __forceinline__ void join(float (&k)[N], float (&b)[N], bool &seen, float (&in)[N]) {
#pragma unroll
        for (int step = 1; step < GROUPS; step *= 2) {
            const unsigned long long starts = __ballot(seen);
            const bool take = group >= step && !seen;
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const float bo = __shfl_up(b[c], step * L);
                if (!Op::ONES) {
                    const float ko = __shfl_up(k[c], step * L);
                    b[c] = take ? fmaf(k[c], bo, b[c]) : b[c];
                    k[c] = take ? k[c] * ko : k[c];
                } else {
                    b[c] = take ? b[c] + bo : b[c];
                }
            }
            if (group >= step) seen = seen || (starts >> (threadIdx.x - step * L) & 1);
        }
        const unsigned long long starts = __ballot(seen);
        const bool before = group > 0 && (starts >> (threadIdx.x - L) & 1);
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const float bo = __shfl_up(b[c], L), ko = Op::ONES ? 1.f : __shfl_up(k[c], L);
            in[c] = group == 0 ? s[c] : before ? bo : Op::ONES ? s[c] + bo : fmaf(ko, s[c], bo);
        }
    }

    // Entries [from, from + n) (down from from - 1 where BACK) with all their rows; s is the state that comes in.
    __device__ void entries(Marks &m, int64_t from, int64_t n) {
        if (n <= 0) return;
        int64_t row = rows.row_of(Op::BACK ? from - 1 : from);
        for (int64_t done = 0; done < n; done += WALK_STAGE) {
            const int64_t here = Op::BACK ? from - done : from + done;
            const int many = (int)min(n - done, (int64_t)WALK_STAGE);
            stage_entries<Op::BACK>(rows, m, here, many, row);
            for (int tile = 0; tile < many; tile += TILE) {
                const int i0 = tile + group * K;
                typename Op::Raw raw[K];
                int some = 0, starts = 0, ends = 0;  // a bit per entry: has an item, a row starts, ends there
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    const int id = m.id[i0 + j];
                    some |= (id >= 0) << j;
                    starts |= (m.start[i0 + j] >= 0) << j;
                    ends |= (m.end[i0 + j] >= 0) << j;
                    // entries behind the last one: any that is there
                    op.load(raw[j], Op::BACK ? here - 1 - min(i0 + j, many - 1) : here + min(i0 + j, many - 1), max(id, 0), lane);
                }
                // No branch that some lanes take but for stores: a value is chosen, what is read for it is somewhere that can be read.
                float k[N], b[N], keep[Op::KEEP && !Op::ONES ? K : 1][N], add[Op::KEEP ? K : 1][N];
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    float kj[N], bj[N];
                    op.map(raw[j], some >> j & 1, kj, bj);
                    const bool starting = starts >> j & 1;
                    if (j == 0) {
#pragma unroll
                        for (int c = 0; c < N; ++c) b[c] = 0.f;
                    }
                    if (__any(starting)) {
                        float first[N];
                        op.begin(max(m.start[i0 + j], 0), lane, first);
#pragma unroll
                        for (int c = 0; c < N; ++c) b[c] = starting ? first[c] : b[c];
                    }
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        b[c] = Op::ONES ? b[c] + bj[c] : fmaf(kj[c], b[c], bj[c]);
                        k[c] = j ? k[c] * kj[c] : kj[c];
                        if constexpr (Op::KEEP && !Op::ONES) keep[j][c] = kj[c];
                        if constexpr (Op::KEEP) add[j][c] = bj[c];
                    }
                }
                bool seen = starts != 0;
                float h[N];
                join(k, b, seen, h);
                {
                    const bool all = __ballot(seen) >> 63;
                    const int from_lane = (GROUPS - 1) * L + lane;
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        const float bo = __shfl(b[c], from_lane), ko = Op::ONES ? 1.f : __shfl(k[c], from_lane);
                        s[c] = all ? bo : Op::ONES ? s[c] + bo : fmaf(ko, s[c], bo);
                    }
                }
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    const bool starting = starts >> j & 1, ending = ends >> j & 1;
                    if (__any(starting)) {
                        float first[N];
                        op.begin(max(m.start[i0 + j], 0), lane, first);
#pragma unroll
                        for (int c = 0; c < N; ++c) h[c] = starting ? first[c] : h[c];
                    }
                    const int64_t p = Op::BACK ? here - 1 - (i0 + j) : here + i0 + j;
                    if constexpr (Op::KEEP) {
#pragma unroll
                        for (int c = 0; c < N; ++c) h[c] = Op::ONES ? h[c] + add[j][c] : fmaf(keep[j][c], h[c], add[j][c]);
                        op.output(p, i0 + j < many, lane, h);
                    } else {
                        op.entry(raw[j], some >> j & 1, p, i0 + j < many, ending, m.end, i0 + j, lane, h);
                    }
                    if (__any(ending)) op.finish(max(m.end[i0 + j], 0), ending, lane, h);
                }
            }
        }
    }

    // The map of entries [from, from + n) of one row (down from from - 1 where BACK), of the row's first state and them where
    // `row` >= 0; to `out` [2][d].
    __device__ void piece(int64_t from, int64_t n, int64_t row, float *out) {
        float wk[N], wb[N];
#pragma unroll
        for (int c = 0; c < N; ++c) {
            wk[c] = 1.f;
            wb[c] = 0.f;
        }
        if (row >= 0) {
            op.begin(row, lane, wb);
#pragma unroll
            for (int c = 0; c < N; ++c) wk[c] = 0.f;
        }
        for (int64_t done = 0; done < n; done += TILE) {
            typename Op::Raw raw[K];
            bool some[K];
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const int64_t i = done + group * K + j, at = min(i, n - 1), p = Op::BACK ? from - 1 - at : from + at;
                int id = rows.y.ids ? rows.y.ids[p] : (int)p;
                some[j] = i < n && id >= 0 && id < rows.y.cols;
                if (!some[j]) id = 0;
                op.load_map(raw[j], p, id, lane);
            }
            float k[N], b[N];
#pragma unroll
            for (int j = 0; j < K; ++j) {
                float kj[N], bj[N];
                op.map(raw[j], some[j], kj, bj);
                if (Op::BACK && done + group * K + j >= n) {  // gradients of entries without an item count, those behind the end do not
#pragma unroll
                    for (int c = 0; c < N; ++c) bj[c] = 0.f;
                }
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    b[c] = j ? (Op::ONES ? b[c] + bj[c] : fmaf(kj[c], b[c], bj[c])) : bj[c];
                    k[c] = j ? k[c] * kj[c] : kj[c];
                }
            }
            // joined in pairs; the last group's lanes have the tile's map
#pragma unroll
            for (int step = 1; step < GROUPS; step *= 2) {
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    const float bo = __shfl_up(b[c], step * L), ko = __shfl_up(k[c], step * L);
                    if (group >= step) {
                        b[c] = fmaf(k[c], bo, b[c]);
                        k[c] *= ko;
                    }
                }
            }
            const int from_lane = (GROUPS - 1) * L + lane;
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const float bt = __shfl(b[c], from_lane), kt = __shfl(k[c], from_lane);
                wb[c] = fmaf(kt, wb[c], bt);
                wk[c] *= kt;
            }
        }
        if (group == 0) {
#pragma unroll
            for (int c = 0; c < N; ++c) {
                out[lane * N + c] = wk[c];
                out[N * L + lane * N + c] = wb[c];
            }
        }
    }
};

// The rows without entries, 64 at a time; workgroup `at` of `of`.
template <class Op> __device__ void empty_rows(const Op &op, const RowFinder &f, int64_t at, int64_t of) {
    const int lane = threadIdx.x;
    for (int64_t u0 = at * 64; u0 < f.y.rows; u0 += of * 64) {
        const int64_t u = u0 + lane;
        const bool none = u < f.y.rows && f.at(u) >= f.at(min(u + 1, f.y.rows));
        for (unsigned long long who = __ballot(none); who; who &= who - 1) {
            const int64_t row = u0 + __ffsll((long long)who) - 1;
            if (lane < Op::L) {
                float s[Op::N];
                op.begin(row, lane, s);
                op.finish(row, true, lane, s);
            }
        }
    }
}

// Last states: every chunk's short rows, and the maps of its long rows' pieces.
template <class Op> __global__ __launch_bounds__(64, Op::WAVES) void walk_last_kernel(Op op, Lists y, Chunks c) {
    constexpr int D = Op::N * Op::L;
    __shared__ __align__(16) Marks m;
    const RowFinder f(y);
    const int64_t chunk = blockIdx.x;
    if (chunk >= c.count) return empty_rows(op, f, chunk - c.count, gridDim.x - c.count);
    const ChunkRows r(f, c, chunk);
    int64_t low = r.low, high = r.high;
    if (low >= high) return;
    if (r.split_low) {
        const int64_t e = min(r.at_low.e, high);
        Walk<Op>(op, f).piece(low, e - low, -1, (e == r.at_low.e && !(r.split_high && r.at_high.u == r.at_low.u) ? c.close : c.across) + chunk * 2 * D);
        low = e;
    }
    if (r.split_high && low < high) {
        const int64_t b = max(r.at_high.b, low);
        Walk<Op>(op, f).piece(b, high - b, r.at_high.u, c.across + chunk * 2 * D);
        high = b;
    }
    Walk<Op>(op, f).entries(m, low, high - low);
}

// All entries' outputs; rows that come in begin with the state that carry_kernel left.
template <class Op> __global__ __launch_bounds__(64, Op::WAVES) void walk_all_kernel(Op op, Lists y, Chunks c) {
    constexpr int D = Op::N * Op::L;
    __shared__ __align__(16) Marks m;
    const RowFinder f(y);
    const int64_t chunk = blockIdx.x;
    if (chunk >= c.count) return empty_rows(op, f, chunk - c.count, gridDim.x - c.count);
    const ChunkRows r(f, c, chunk);
    Walk<Op> walk(op, f);
    if (Op::BACK ? r.split_high : r.split_low) {
#pragma unroll
        for (int j = 0; j < Op::N; ++j) walk.s[j] = c.close[(chunk * 2 + 1) * D + walk.lane * Op::N + j];
    }
    walk.entries(m, Op::BACK ? r.high : r.low, r.high - r.low);
}

// The map of the part of a long row that leads to the border where the walk leaves the chunk.
template <class Op> __global__ __launch_bounds__(64, Op::WAVES) void pieces_kernel(Op op, Lists y, Chunks c) {
    constexpr int D = Op::N * Op::L;
    const RowFinder f(y);
    const int64_t chunk = blockIdx.x;
    const ChunkRows r(f, c, chunk);
    if (!(Op::BACK ? r.split_low : r.split_high) || r.low >= r.high) return;
    const RowFinder::Row row = Op::BACK ? r.at_low : r.at_high;
    const int64_t low = max(r.low, row.b), high = min(r.high, row.e);
    const bool whole = Op::BACK ? row.e <= r.high : row.b >= r.low;
    Walk<Op>(op, f).piece(Op::BACK ? high : low, high - low, whole ? row.u : -1, c.across + chunk * 2 * D);
}

// A long row's pieces one after the other, by the wavefront of the chunk that the walk along the row begins in (CARRY: the state
// at every border it crosses goes to the chunk behind it) or ends in (otherwise: the row's last state).
template <class Op, bool CARRY> __global__ __launch_bounds__(64) void join_kernel(Op op, Lists y, Chunks c) {
    constexpr int D = Op::N * Op::L, AHEAD = 8;
    const RowFinder f(y);
    const int64_t chunk = blockIdx.x;
    const ChunkRows r(f, c, chunk);
    RowFinder::Row row;
    if (CARRY) {
        // begins here: it crosses the border that the walk leaves by, and not the other one
        if (!(Op::BACK ? r.split_low : r.split_high) || r.low >= r.high) return;
        row = Op::BACK ? r.at_low : r.at_high;
        if (Op::BACK ? r.split_high && r.at_high.u == row.u : r.split_low && r.at_low.u == row.u) return;
    } else {
        if (!r.split_low || (r.split_high && r.at_high.u == r.at_low.u)) return;
        row = r.at_low;
    }
    const int64_t first = row.b / c.size, last = (row.e - 1) / c.size, from = Op::BACK ? last : first;
    const int64_t pieces = min(last - first, c.count - 1);  // but for the closing one
    const int lane = threadIdx.x;
    if (lane >= Op::L) return;
    float s[Op::N];
#pragma unroll
    for (int j = 0; j < Op::N; ++j) s[j] = 0.f;
    for (int64_t i0 = 0; i0 < pieces; i0 += AHEAD) {
        float k[AHEAD][Op::N], b[AHEAD][Op::N];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int64_t i = min(i0 + a, pieces - 1), at = min(max(Op::BACK ? from - i : from + i, (int64_t)0), c.count - 1);
#pragma unroll
            for (int j = 0; j < Op::N; ++j) {
                k[a][j] = c.across[at * 2 * D + lane * Op::N + j];
                b[a][j] = c.across[(at * 2 + 1) * D + lane * Op::N + j];
            }
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int64_t i = i0 + a;
            if (i < pieces) {
#pragma unroll
                for (int j = 0; j < Op::N; ++j) s[j] = i ? fmaf(k[a][j], s[j], b[a][j]) : b[a][j];
                if (CARRY) {
                    const int64_t to = min(max(Op::BACK ? from - i - 1 : from + i + 1, (int64_t)0), c.count - 1);
#pragma unroll
                    for (int j = 0; j < Op::N; ++j) c.close[(to * 2 + 1) * D + lane * Op::N + j] = s[j];
                }
            }
        }
    }
    if (!CARRY) {
#pragma unroll
        for (int j = 0; j < Op::N; ++j) s[j] = fmaf(c.close[chunk * 2 * D + lane * Op::N + j], s[j], c.close[(chunk * 2 + 1) * D + lane * Op::N + j]);
        op.finish(row.u, true, lane, s);
    }
}

// Chunks of the call's entries: enough for every wavefront that the card holds to have some, of at least a few tiles.
inline Chunks chunks_of(const als_ctx *ctx, int64_t nnz, int d, int tile) {
    Chunks c{};
    const int64_t least = tile > 64 ? tile : 64;
    c.size = (nnz + WALK_MAX_CHUNKS - 1) / WALK_MAX_CHUNKS;
    c.size = std::max(least, (c.size + 63) / 64 * 64);
    c.count = (nnz + c.size - 1) / c.size;
    c.longest = c.size;
    c.across = (float *)ctx->walk_maps.p;
    c.close = c.across + (int64_t)WALK_MAX_CHUNKS * 2 * 128;
    return c;
}
constexpr size_t WALK_BYTES = (size_t)WALK_MAX_CHUNKS * 4 * 128 * sizeof(float);
constexpr int EMPTY_GROUPS = 1024;  // workgroups that look for empty rows, at most
inline unsigned walk_grid(const Chunks &c, int64_t rows) { return (unsigned)(c.count + std::min<int64_t>((rows + 63) / 64, EMPTY_GROUPS)); }

template <class Op> void launch_last(const als_ctx *ctx, const Op &op, const als_csr *Y, hipStream_t s) {
    const Chunks c = chunks_of(ctx, Y->nnz, Op::N * Op::L, Walk<Op>::TILE);
    const Lists y = lists_of(Y);
    hipLaunchKernelGGL((walk_last_kernel<Op>), dim3(walk_grid(c, Y->rows)), dim3(64), 0, s, op, y, c);
    if (Y->nnz > c.longest) hipLaunchKernelGGL((join_kernel<Op, false>), dim3((unsigned)c.count), dim3(64), 0, s, op, y, c);
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
