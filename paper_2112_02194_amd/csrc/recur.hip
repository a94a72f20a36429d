// The gated linear recurrence over the entries of CSR rows (als_recur), its gradients and its single step.  How rows and entries are
// dealt out stands in entry_walk.h; here are an entry's maps and outputs.
//
// Bytes that have to be moved, at the rates of a large copy (4.7 to 4.9 TB/s read and written), and what was measured:
//   last states  300000 rows, 6.0M entries, d = 128, tables of 1M rows in bf16 (popular items often)  484 us.  3.1 GB gathered, 2.8 of them
//                from behind the L2: 5.9 TB/s, about what reading alone reaches.  The vector units are at work for 84 % of the time (18
//                instructions an entry and column, of which the exponential and the reciprocal take four slots each)
//   all states   16 rows of 65537 entries, d = 128, fp32  527 us: pieces 217 (1.07 GB), their states 21, the walk 280 (1.61 GB)
//   gradients    100000 rows, 2.0M entries, d = 64, fp32  568 us: 0.27 GB in pieces 75, joined 14, the walk 471 (2.2 GB and what the cache
//                misses of the gathers); 16 x 65537 in bf16 with fp32 states  700 us: 175 (0.8 GB), 21, 490 (2.7 GB)
#include <algorithm>
#include <type_traits>

#include "entry_walk.h"

namespace als {

constexpr int RECUR_THREADS = 256;

// h = s h + (1 - s) x along a row (als_recur).  K entries a group and tile: 64 registers of maps, at 3 wavefronts per SIMD without spills
// (with last states alone, which keep none, 4; 8 columns a lane in bf16 take 3).
template <int D, bool BF, bool SBF, bool STATES> struct Forward {
    static constexpr int N = BF ? 8 : 4, K = 32 / N, L = D / N, WAVES = STATES || BF ? 3 : 4;
    static constexpr bool BACK = false, ONES = false, KEEP = true, EARLY = false;
    static constexpr int STEP = 4;
    RowsOf V, F, H0, states, last;
    const char *no_x, *no_g;
    struct Raw {
        Words x, g;
    };
    __device__ __forceinline__ void load(Raw &r, int64_t, int id, int lane) const {
        r.x = *(const Words *)(item_row(V, id, no_x) + lane * 16);
        r.g = *(const Words *)(item_row(F, id, no_g) + lane * 16);
    }
    __device__ __forceinline__ void load_map(Raw &r, int64_t p, int id, int lane) const { load(r, p, id, lane); }
    __device__ __forceinline__ void map(const Raw &r, float (&k)[N], float (&t)[N], float (&b)[N]) const {
        float x[N], g[N];
        widen<BF, N>(r.x, x);
        widen<BF, N>(r.g, g);
#pragma unroll
        for (int c = 0; c < N; ++c) {
            gate(g[c], k[c], t[c]);
            b[c] = t[c] * x[c];
        }
    }
    __device__ __forceinline__ void begin(int64_t row, int lane, float (&s)[N]) const {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = 0.f;
        if (H0.p) load_piece(H0, row, lane, s);
    }
    __device__ __forceinline__ void output(int64_t p, bool valid, int lane, const float (&s)[N]) const {
        if (valid) store_piece<SBF, N>(states.p + p * states.ld, lane, s);
    }
    __device__ __forceinline__ void finish(int64_t row, bool mine, int lane, const float (&s)[N]) const {
        if (last.p && mine) store_piece(last, row, lane, s);
    }
};

// g = d + a, a = s g from a row's end (als_recur_backward): a, what an entry gets from those behind it, is the state.  Gates are
// computed again in the second walk: what would be kept of them takes more registers than there are, and memory bounds the kernel.
// What rows begin with is loaded early: 100000 rows of 20, d = 16, 255 us and 263 without, d = 64 and more the same.
template <int D, bool BF, bool SBF> struct Backward {
    static constexpr int N = 4, K = 4, L = D / N, WAVES = 3;
    static constexpr bool BACK = true, ONES = false, KEEP = false, EARLY = true;
    static constexpr int STEP = 4;
    RowsOf V, F, H0, states, d_states, d_last, dV, dF, dH0;
    const char *no_x, *no_g;
    struct Raw {
        Part<BF> x, g;
        Part<SBF> d, h;
    };
    __device__ __forceinline__ void load_map(Raw &r, int64_t p, int id, int lane) const {
        r.g = *(const Part<BF> *)(item_row(F, id, no_g) + lane * sizeof(Part<BF>));
        r.d = Part<SBF>{};
        if (d_states.p) r.d = *(const Part<SBF> *)(d_states.p + p * d_states.ld + lane * sizeof(Part<SBF>));
    }
    __device__ __forceinline__ void load(Raw &r, int64_t p, int id, int lane) const {
        load_map(r, p, id, lane);
        r.x = *(const Part<BF> *)(item_row(V, id, no_x) + lane * sizeof(Part<BF>));
        r.h = *(const Part<SBF> *)(states.p + max(p - 1, (int64_t)0) * states.ld + lane * sizeof(Part<SBF>));
    }
    __device__ __forceinline__ void map(const Raw &r, float (&k)[N], float (&t)[N], float (&b)[N]) const {
        float g[N], d[N];
        widen<BF, N>(r.g, g);
        widen<SBF, N>(r.d, d);
#pragma unroll
        for (int c = 0; c < N; ++c) {
            gate(g[c], k[c], t[c]);
            b[c] = k[c] * d[c];
        }
    }
    __device__ __forceinline__ void begin(int64_t row, int lane, float (&s)[N]) const {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = 0.f;
        if (d_last.p) load_piece(d_last, row, lane, s);
    }
    __device__ __forceinline__ void entry(const Raw &r, bool some, int64_t p, bool valid, bool first, const int32_t *rows, int i, int lane,
                                          float (&s)[N]) const {
        float x[N], g[N], d[N], h[N], dv[N], df[N];
        widen<BF, N>(r.x, x);
        widen<BF, N>(r.g, g);
        widen<SBF, N>(r.d, d);
        widen<SBF, N>(r.h, h);
        if (__any(first)) {
            float before[N] = {};
            if (H0.p) load_piece(H0, max(rows[i], 0), lane, before);
#pragma unroll
            for (int c = 0; c < N; ++c) h[c] = first ? before[c] : h[c];
        }
#pragma unroll
        for (int c = 0; c < N; ++c) {
            float keep, take;
            gate(g[c], keep, take);
            const float all = d[c] + s[c];
            s[c] = keep * all;
            dv[c] = some ? take * all : 0.f;
            df[c] = some ? s[c] * take * (h[c] - x[c]) : 0.f;
        }
        if (valid) {
            store_piece<SBF, N>(dV.p + p * dV.ld, lane, dv);
            store_piece<SBF, N>(dF.p + p * dF.ld, lane, df);
        }
    }
    __device__ __forceinline__ void finish(int64_t row, bool mine, int lane, const float (&s)[N]) const {
        if (dH0.p && mine) store_piece(dH0, row, lane, s);
    }
};

// One entry per row, from a parent row: two loads after each other, 2.9 us for 512 rows.  X may be H where there are no parents: a row is read and written by the same lanes.
template <int D, bool BF>
__global__ __launch_bounds__(RECUR_THREADS) void recur_step_kernel(int64_t rows, const int32_t *items, const int32_t *parents, int64_t cols,
                                                                   int64_t from_rows, RowsOf V, RowsOf F, RowsOf H, RowsOf X) {
    constexpr int N = BF ? 8 : 4, L = D / N;
    const int lane = threadIdx.x % L;
    for (int64_t u = (blockIdx.x * (int64_t)RECUR_THREADS + threadIdx.x) / L; u < rows; u += (int64_t)gridDim.x * RECUR_THREADS / L) {
        const int64_t i = items[u], p = parents ? parents[u] : u;
        float h[N] = {}, x[N] = {}, g[N];
        const bool some = i >= 0 && i < cols;
        if (p >= 0 && p < from_rows) load_piece(H, p, lane, h);
        if (some) {
            load_piece<BF, N>(V.p + i * V.ld, lane, x);
            load_piece<BF, N>(F.p + i * F.ld, lane, g);
#pragma unroll
            for (int c = 0; c < N; ++c) {
                float keep, take;
                gate(g[c], keep, take);
                h[c] = after_map(share_of(keep, take), h[c], take * x[c]);
            }
        }
        store_piece(X, u, lane, h);
    }
}

static unsigned groups_grid(int64_t rows, int lanes) {
    return (unsigned)std::min<int64_t>((rows * lanes + RECUR_THREADS - 1) / RECUR_THREADS, 1 << 22);
}

als_status walk_setup(als_ctx *ctx) {
    als_status st = ensure(ctx, ctx->walk_maps, WALK_BYTES);
    if (st != ALS_OK) return st;
    uint32_t none[3][128];
    for (int i = 0; i < 128; ++i) {
        none[0][i] = 0;
        none[1][i] = 0x7f800000u;  // +inf: 1 / (1 + exp(-inf)) keeps all
        none[2][i] = 0x7f807f80u;
    }
    ALS_HIP(ctx, hipMemcpy((char *)ctx->walk_maps.p + WALK_NONE, none, sizeof(none), hipMemcpyHostToDevice));
    return ALS_OK;
}

template <class Op> static void launch_all(const als_ctx *ctx, const Op &op, const als_csr *Y, hipStream_t s) {
    const Chunks c = chunks_of(ctx, Y->nnz, Walk<Op>::TILE);
    const Lists y = lists_of(Y);
    if (Y->nnz > c.longest) {  // there may be rows that are cut
        hipLaunchKernelGGL((pieces_kernel<Op>), dim3((unsigned)c.count), dim3(64), 0, s, op, y, c);
        if (c.count > FEW_CHUNKS)
            hipLaunchKernelGGL((join_kernel<Op, true>), join_grid<Op>(c), dim3(JOIN_THREADS), 0, s, op, c);
    }
    hipLaunchKernelGGL((walk_all_kernel<Op>), dim3(walk_grid(c, Y->rows)), dim3(64), 0, s, op, y, c);
}

als_status launch_recur(als_ctx *ctx, const als_csr *Y, const als_table *V, const als_table *F, const als_table *H0,
                        const als_table *states, const als_table *last, hipStream_t s) {
    const RowsOf v = rows_of(V), f = rows_of(F), h0 = rows_of(H0), all = rows_of(states), end = rows_of(last);
    const char *no_x = none_row(ctx, false, false), *no_g = none_row(ctx, true, V->dtype == ALS_BF16);
    pick_d(V->d, [&](auto d) {
        pick(V->dtype == ALS_BF16, [&](auto bf) {
            if (states) {
                pick(states->dtype == ALS_BF16, [&](auto sbf) { launch_all(ctx, Forward<d(), bf(), sbf(), true>{v, f, h0, all, end, no_x, no_g}, Y, s); });
            } else {
                launch_last(ctx, Forward<d(), bf(), false, false>{v, f, h0, all, end, no_x, no_g}, Y, s);
            }
        });
    });
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

als_status launch_recur_backward(als_ctx *ctx, const als_csr *Y, const als_table *V, const als_table *F, const als_table *H0,
                                 const als_table *states, const als_table *d_states, const als_table *d_last, const als_table *dV,
                                 const als_table *dF, const als_table *dH0, hipStream_t s) {
    const char *no_x = none_row(ctx, false, false), *no_g = none_row(ctx, true, V->dtype == ALS_BF16);
    pick_d(V->d, [&](auto d) {
        pick(V->dtype == ALS_BF16, [&](auto bf) {
            pick(states->dtype == ALS_BF16, [&](auto sbf) {
                launch_all(ctx, Backward<d(), bf(), sbf()>{rows_of(V), rows_of(F), rows_of(H0), rows_of(states), rows_of(d_states), rows_of(d_last), rows_of(dV),
                                                           rows_of(dF), rows_of(dH0), no_x, no_g}, Y, s);
            });
        });
    });
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

als_status launch_recur_step(als_ctx *ctx, const int32_t *items, const int32_t *parents, const als_table *V, const als_table *F,
                             const als_table *H, const als_table *X, hipStream_t s) {
    pick_d(V->d, [&](auto d) {
        pick(V->dtype == ALS_BF16, [&](auto bf) {
            hipLaunchKernelGGL((recur_step_kernel<d(), bf()>), dim3(groups_grid(X->rows, d() / (bf() ? 8 : 4))), dim3(RECUR_THREADS), 0, s, X->rows,
                               items, parents, V->rows, H->rows, rows_of(V), rows_of(F), rows_of(H), rows_of(X));
        });
    });
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
