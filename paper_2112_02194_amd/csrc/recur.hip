// The gated linear recurrence over the entries of CSR rows (als_recur), its gradients and its single step.
// A group of lanes holds a row's d columns, 16 bytes of the tables each, and walks its entries.
#include <algorithm>
#include <type_traits>

#include "entry_rows.h"

namespace als {

constexpr int RECUR_THREADS = 256;

// F(bool) for a value that only the call knows
template <class F> static auto pick(bool v, F &&f) { return v ? f(std::true_type{}) : f(std::false_type{}); }
template <class F> static auto pick_d(int d, F &&f) {
    switch (d) {
        case 16: return f(std::integral_constant<int, 16>{});
        case 32: return f(std::integral_constant<int, 32>{});
        case 64: return f(std::integral_constant<int, 64>{});
        default: return f(std::integral_constant<int, 128>{});
    }
}

template <int D, bool BF, bool SBF>
__global__ __launch_bounds__(RECUR_THREADS) void recur_kernel(Lists y, RowsOf V, RowsOf F, RowsOf H0, RowsOf states, RowsOf last) {
    constexpr int N = BF ? 8 : 4, L = D / N;
    const int lane = threadIdx.x % L;
    for (int64_t u = (blockIdx.x * (int64_t)RECUR_THREADS + threadIdx.x) / L; u < y.rows; u += (int64_t)gridDim.x * RECUR_THREADS / L) {
        int64_t b, e;
        row_range(y.indptr, u, y.nnz, b, e);
        float h[N] = {};
        if (H0.p) load_piece(H0, u, lane, h);
        for (int64_t p = b; p < e; ++p) {
            const int64_t i = y.ids ? y.ids[p] : p;
            if (i >= 0 && i < y.cols) {
                float x[N], g[N];
                load_piece<BF, N>(V.p + i * V.ld, lane, x);
                load_piece<BF, N>(F.p + i * F.ld, lane, g);
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    float keep, take;
                    gate(g[c], keep, take);
                    h[c] = fmaf(keep, h[c], take * x[c]);
                }
            }
            if (states.p) store_piece<SBF, N>(states.p + p * states.ld, lane, h);
        }
        if (last.p) store_piece(last, u, lane, h);
    }
}

template <int D, bool BF, bool SBF>
__global__ __launch_bounds__(RECUR_THREADS) void recur_backward_kernel(Lists y, RowsOf V, RowsOf F, RowsOf H0, RowsOf states,
                                                                     RowsOf d_states, RowsOf d_last, RowsOf dV, RowsOf dF, RowsOf dH0) {
    constexpr int N = BF ? 8 : 4, L = D / N;
    const int lane = threadIdx.x % L;
    for (int64_t u = (blockIdx.x * (int64_t)RECUR_THREADS + threadIdx.x) / L; u < y.rows; u += (int64_t)gridDim.x * RECUR_THREADS / L) {
        int64_t b, e;
        row_range(y.indptr, u, y.nnz, b, e);
        float a[N] = {};  // s_{t+1} g_{t+1}
        if (d_last.p) load_piece(d_last, u, lane, a);
        for (int64_t p = e - 1; p >= b; --p) {
            if (d_states.p) {
                float d[N];
                load_piece<SBF, N>(d_states.p + p * d_states.ld, lane, d);
#pragma unroll
                for (int c = 0; c < N; ++c) a[c] += d[c];
            }
            const int64_t i = y.ids ? y.ids[p] : p;
            float dv[N] = {}, df[N] = {};
            if (i >= 0 && i < y.cols) {
                float x[N], g[N], h[N] = {};
                load_piece<BF, N>(V.p + i * V.ld, lane, x);
                load_piece<BF, N>(F.p + i * F.ld, lane, g);
                if (p > b) load_piece<SBF, N>(states.p + (p - 1) * states.ld, lane, h);
                else if (H0.p) load_piece(H0, u, lane, h);
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    float keep, take;
                    gate(g[c], keep, take);
                    dv[c] = take * a[c];
                    a[c] *= keep;
                    df[c] = a[c] * take * (h[c] - x[c]);
                }
            }
            store_piece<SBF, N>(dV.p + p * dV.ld, lane, dv);
            store_piece<SBF, N>(dF.p + p * dF.ld, lane, df);
        }
        if (dH0.p) store_piece(dH0, u, lane, a);
    }
}

// One entry per row, from a parent row.  X may be H where there are no parents: a row is read and written by the same lanes.
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
                h[c] = fmaf(keep, h[c], take * x[c]);
            }
        }
        store_piece(X, u, lane, h);
    }
}

static unsigned groups_grid(int64_t rows, int lanes) {
    return (unsigned)std::min<int64_t>((rows * lanes + RECUR_THREADS - 1) / RECUR_THREADS, 1 << 22);
}

als_status launch_recur(als_ctx *ctx, const als_csr *Y, const als_table *V, const als_table *F, const als_table *H0,
                        const als_table *states, const als_table *last, hipStream_t s) {
    pick_d(V->d, [&](auto d) {
        pick(V->dtype == ALS_BF16, [&](auto bf) {
            pick(states && states->dtype == ALS_BF16, [&](auto sbf) {
                hipLaunchKernelGGL((recur_kernel<d(), bf(), sbf()>), dim3(groups_grid(Y->rows, d() / (bf() ? 8 : 4))), dim3(RECUR_THREADS), 0, s,
                                   lists_of(Y), rows_of(V), rows_of(F), rows_of(H0), rows_of(states), rows_of(last));
            });
        });
    });
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

als_status launch_recur_backward(als_ctx *ctx, const als_csr *Y, const als_table *V, const als_table *F, const als_table *H0,
                                 const als_table *states, const als_table *d_states, const als_table *d_last, const als_table *dV,
                                 const als_table *dF, const als_table *dH0, hipStream_t s) {
    pick_d(V->d, [&](auto d) {
        pick(V->dtype == ALS_BF16, [&](auto bf) {
            pick(states->dtype == ALS_BF16, [&](auto sbf) {
                hipLaunchKernelGGL((recur_backward_kernel<d(), bf(), sbf()>), dim3(groups_grid(Y->rows, d() / (bf() ? 8 : 4))), dim3(RECUR_THREADS),
                                   0, s, lists_of(Y), rows_of(V), rows_of(F), rows_of(H0), rows_of(states), rows_of(d_states), rows_of(d_last),
                                   rows_of(dV), rows_of(dF), rows_of(dH0));
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
