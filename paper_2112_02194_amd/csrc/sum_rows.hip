// Sums of a table's rows over the rows of a CSR matrix (als_sum_rows): the walk of entry_walk.h with maps s -> s + y x.  A sum is fp32: a
// running one of up to 256 entries in a lane's stretch (32, and sums of these, where a row is cut), then of the lane groups, of a lane's
// up to 512 pieces and of 64 to 256 lanes.  So an entry is rounded some hundred times on its way into the sum of a long row, below 2000
// of 2^31 entries, where one running sum would round it once for every entry behind it.  Memory bound: the gradient of 1M items
// from 6.0M entries, d = 64, fp32  398 us for 1.82 GB, 4.6 TB/s in rows of 256 bytes anywhere; items with one entry and with 60000 are
// the same work.
#include "entry_walk.h"

namespace als {

template <int D, bool BF> struct SumRows {
    static constexpr int N = BF ? 8 : 4, STEP = 4, K = STEP, L = D / N, WAVES = 4;
    static constexpr bool BACK = false, ONES = true;
    RowsOf E, X;
    const float *values;
    const char *no_x;
    struct Raw {
        Words x;
        float w;
    };
    __device__ __forceinline__ void load(Raw &r, int64_t p, int id, int lane) const {
        r.x = *(const Words *)(item_row(E, id, no_x) + lane * 16);
        r.w = id < 0 || !values ? 1.f : values[p];
    }
    __device__ __forceinline__ void load_map(Raw &r, int64_t p, int id, int lane) const { load(r, p, id, lane); }
    __device__ __forceinline__ void map(const Raw &r, float (&k)[N], float (&t)[N], float (&b)[N]) const {
        widen<BF, N>(r.x, b);
#pragma unroll
        for (int c = 0; c < N; ++c) {
            k[c] = 1.f;
            t[c] = 0.f;
            b[c] *= r.w;
        }
    }
    __device__ __forceinline__ void begin(int64_t, int, float (&s)[N]) const {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = 0.f;
    }
    __device__ __forceinline__ void finish(int64_t row, bool mine, int lane, const float (&s)[N]) const {
        if (mine) store_piece(X, row, lane, s);
    }
};

als_status launch_sum_rows(als_ctx *ctx, const als_csr *Y, const als_table *E, const als_table *X, hipStream_t s) {
    pick_d(E->d, [&](auto d) {
        pick(E->dtype == ALS_BF16, [&](auto bf) { launch_last(ctx, SumRows<d(), bf()>{rows_of(E), rows_of(X), Y->values, none_row(ctx, false, false)}, Y, s); });
    });
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
