// Scores of queries against a table in 4 bits an entry (als_scores): S[q][i] = sum_g scale(i, g) sum_{j in g} Q[q][j] code(i, j).
//
// Both kernels form a group's sum of products first and multiply it by the group's scale once.
//
// few queries    (up to two to four) the vector units: 32 or 16 codes of an item per lane.  Codes are put into the upper halves of
//                signed bytes, 16 times their value, and converted to fp32 from there (11 instructions for eight); the queries are
//                held in fp32, a sixteenth of their value (rows with entries beyond 2^64 another 2^-64, and rows without any beyond
//                2^-16 their value, which their scores take back).  Sums over the lanes of an item by lane moves.
// more           the matrix cores, 32 queries x 32 items x 16 entries an instruction.  Query rows become two fp16 parts, hi + lo,
//                after a shift by a power of two that brings their largest entry to 2^14 .. 2^15: 22 bits and more of every entry within
//                2^-17 of the largest, 19 within 2^-20 (bf16 queries need no lo: their 8 bits fit one part down to 2^-31 of the
//                largest).  Where a group of 32 queries has a row with entries below that (not 0), they become bf16 numbers, three
//                of fp32 and one of bf16, which hold every bit down to 2^-100 of the largest: three products instead of two, six
//                more instructions to unpack eight codes, and guarded stores.  512 x 1M, d = 128, fp32 scores of fp32 queries: 655 us
//                with such a row in every group, 486 with none; bf16 of bf16 423 and 329; the bf16 parts and the common stores for
//                all 547, where the fp16 parts for all took 478.  Ordinary rows of d = 128 make it one group in a hundred.  A workgroup keeps 32 queries' operands in LDS, its
//                wavefronts walk item tiles with the next tile's codes under way.
#include <algorithm>

#include "row_piece.h"

namespace als {

typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The eight codes of a word as fp16 numbers, exactly (the well-known conversion of small integers through the mantissa of a large
// power of two): element e of the word is c[e % 4][e / 4].  A code plus 8 put into the low
// bits of 1024's mantissa is the number 1024 + code + 8, from which a packed subtraction takes 1032; nibbles four bits further
// up come out times 16 and take a packed multiply-add instead: nine instructions.  (w & mask) ^ bits is one of them: the exclusive
// or turns two's complement into code + 8 beside filling in the exponent.
__device__ __forceinline__ void unpack8(uint32_t w, halfx2 (&c)[4]) {
    const halfx2 k1 = {(_Float16)1032.f, (_Float16)1032.f}, k2 = {(_Float16)0.0625f, (_Float16)0.0625f}, k3 = {(_Float16)72.f, (_Float16)72.f};
    const uint32_t v = w >> 8;
    auto put = [](uint32_t x, uint32_t mask, uint32_t bits) {
        return __builtin_bit_cast(halfx2, (uint32_t)__builtin_amdgcn_bitop3_b32(x, mask, bits, 0x6a));
    };
    c[0] = put(w, 0x000f000fu, 0x64086408u) - k1;
    c[1] = put(w, 0x00f000f0u, 0x64806480u) * k2 - k3;
    c[2] = put(v, 0x000f000fu, 0x64086408u) - k1;
    c[3] = put(v, 0x00f000f0u, 0x64806480u) * k2 - k3;
}

// The eight codes of a word as bf16 numbers times 16, in the order of the entries: signed bytes that hold the codes in their upper halves,
// converted to fp32, whose upper halves are the bf16 numbers (five significant bits at most).
__device__ __forceinline__ bf16x8 unpack8_wide(uint32_t w) {
    const uint32_t even = w << 4 & 0xf0f0f0f0u, odd = w & 0xf0f0f0f0u;
    u32x4 c;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c[i] = __builtin_amdgcn_perm(__float_as_uint((float)(int8_t)(odd >> (8 * i))), __float_as_uint((float)(int8_t)(even >> (8 * i))), 0x07060302u);
    return __builtin_bit_cast(bf16x8, c);
}

// ------------------------------------------------------------------------------------------------ few queries
// What bounds it: the read of the codes (1 x 20M, d = 128, groups of 32: 298 us, 5.1 TB/s, as fast as a copy; 1 x 1M 15 to 17), with
// more queries the vector units.
template <bool BF_Q, bool BF_S, int D, int G, int NQ>
__global__ __launch_bounds__(256, NQ > 2 ? 3 : 4) void scores_few_kernel(const void *__restrict__ Q, int64_t ldq, const uint8_t *__restrict__ codes,
                                                            const uint16_t *__restrict__ scales, int64_t n, void *__restrict__ S,
                                                            int64_t lds) {
    // codes per lane, lanes per item, items per step, steps
    constexpr int CPL = D < 32 || NQ > 2 ? 16 : 32, LPI = D / CPL, IPS = 64 / LPI, U = LPI > 4 ? LPI : 4;
    constexpr int W = CPL / 8, NG = CPL > G ? CPL / G : 1, WPG = W / NG;  // words and groups per lane, words per group
    const int lane = threadIdx.x & 63, chunk = lane % LPI;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), waves = (int64_t)gridDim.x * 4;
    uint32_t next_w[U][W];
    uint32_t next_s[U];
    auto fetch = [&](int64_t i0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t item = std::min<int64_t>(i0 + u * IPS + lane / LPI, n - 1);
            const uint8_t *at = codes + item * (D / 2) + chunk * (CPL / 2);
            if constexpr (W == 4) {
                const u32x4 t = *(const u32x4 *)at;
#pragma unroll
                for (int p = 0; p < 4; ++p) next_w[u][p] = t[p];
            } else {
                const u32x2 t = *(const u32x2 *)at;
#pragma unroll
                for (int p = 0; p < 2; ++p) next_w[u][p] = t[p];
            }
            const uint16_t *sc = scales + item * (D / G) + chunk * CPL / G;
            next_s[u] = NG == 2 ? *(const uint32_t *)sc : *sc;
        }
    };
    int64_t i0 = wave * (IPS * U);
    if (i0 < n) fetch(i0);  // on its way while the queries are prepared
    float q[NQ][CPL], back[NQ];
#pragma unroll
    for (int r = 0; r < NQ; ++r)
#pragma unroll
        for (int p = 0; p < W; ++p) {
            float x[8];
            piece_floats<BF_Q>(piece_load<BF_Q>(Q, r * ldq + chunk * CPL + 8 * p), x);
#pragma unroll
            for (int e = 0; e < 8; ++e) q[r][8 * p + e] = x[e];
        }
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < CPL; ++e) top = fmaxf(top, fabsf(q[r][e]));
        // a group's sum of a query with large entries could pass fp32's range where its product with the scale does not; small entries
        // would leave it, and need no room above: their sums times the largest scale stay within it
        const bool far = __any(top > 0x1p64f), small = !__any(top > 0x1p-16f);
        back[r] = far ? 0x1p64f : small ? 0x1p-4f : 1.f;
        const float by = far ? 0x1p-68f : small ? 1.f : 0x1p-4f;
#pragma unroll
        for (int e = 0; e < CPL; ++e) q[r][e] *= by;
    }
    for (; i0 < n; i0 += waves * (IPS * U)) {
        uint32_t w[U][W];
        float s[U][NG];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int p = 0; p < W; ++p) w[u][p] = next_w[u][p];
            s[u][0] = __uint_as_float(next_s[u] << 16);
            if constexpr (NG == 2) s[u][1] = __uint_as_float(next_s[u] & 0xffff0000u);
        }
        if (i0 + waves * (IPS * U) < n) fetch(i0 + waves * (IPS * U));
        float sum[NQ][U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int r = 0; r < NQ; ++r) sum[r][u] = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float part[NQ];
#pragma unroll
                for (int r = 0; r < NQ; ++r) part[r] = 0.f;
#pragma unroll
                for (int p = g * WPG; p < (g + 1) * WPG; ++p) {
                    const uint32_t half[2] = {w[u][p] << 4 & 0xf0f0f0f0u, w[u][p] & 0xf0f0f0f0u};  // even and odd entries
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float c = (float)(int8_t)(half[e & 1] >> (8 * (e / 2)));
#pragma unroll
                        for (int r = 0; r < NQ; ++r) part[r] = fmaf(c, q[r][8 * p + e], part[r]);
                    }
                }
#pragma unroll
                for (int r = 0; r < NQ; ++r) sum[r][u] = fmaf(part[r], s[u][g], sum[r][u]);
            }
#pragma unroll
            for (int r = 0; r < NQ; ++r)
                if constexpr (LPI > 1) sum[r][u] = group_reduce<LPI>(sum[r][u], [](float a, float b) { return a + b; });
        }
        // every lane of an item holds its sum: lane `chunk` of it stores the item's of step `chunk` (+ LPI, ...)
#pragma unroll
        for (int t = 0; t < U / LPI; ++t) {
            const int64_t item = i0 + (t * LPI + chunk) * IPS + lane / LPI;
#pragma unroll
            for (int r = 0; r < NQ; ++r) {
                float v = sum[r][t * LPI];
#pragma unroll
                for (int c = 1; c < LPI; ++c) v = chunk == c ? sum[r][t * LPI + c] : v;
                if (item < n) store_elem<BF_S>(S, r * lds + item, v * back[r]);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ matrix cores
// What bounds it: the write of the scores (512 x 1M, d = 64, bf16: 216 us, 1.0 GB at 4.7 TB/s, all of it written once, the codes read
// from memory about twice for 16 groups of queries), for few items the launch and one chain of loads (64 x 30000: 6.5 us).
// An item's row is read by one lane in 16-byte loads: with loads of 8 bytes in the order of the products, which touch every line
// eight times, it took 248 us, 554 instead of 474 with d = 128 in fp32, 193 instead of 136 for 100 x 1M, groups of 16.  The two item
// tiles of a round follow one another, so that four wavefronts per SIMD have registers.
//
// A wavefront's 32 queries (A operand: query = lane % 32) and 32 items a tile (B operand: item = lane % 32).  In step s of group
// part t (32 entries, or 16 for groups of 16) half h = lane / 32 of the wavefront holds eight entries of the group; which ones
// only has to be the same on both sides: one word of codes.
template <int D, int G> struct ScoreSteps {
    static constexpr int PART = G == 16 ? 16 : 32, PARTS = D / PART, STEPS = PART / 16;  // steps per part
    static __device__ __forceinline__ int word(int t, int s, int h) { return t * (PART / 8) + h * STEPS + s; }  // of the row's D / 8
};

// How the results of a round, 32 queries x 64 items, are stored: a lane has items 2 a and 2 a + 1 of the round, so that it
// stores two neighbours and half a wavefront 128 or 256 bytes of a row.  Loads and stores of a wavefront are counted together
// and in order, and where a store may or may not have happened the compiler waits for all of them before it uses a load: on the
// way from round to round there is no branch around a store.  Rows beyond the last query have an empty buffer behind them and are
// dropped by the bounds check.
enum class StoreAs {
    BUFFER,  // fp32, or bf16 with rows that are 4-byte aligned
    PLAIN,   // bf16 rows of any alignment: unaligned words without a bounds check, for 32 whole queries
    GUARDED  // a branch around every element: the rest
};

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef const __attribute__((address_space(3))) u32x4 SharedParts;  // in LDS, also where a pointer to it is kept in a structure
typedef const __attribute__((address_space(3))) float SharedFloat;
typedef const __attribute__((address_space(3))) floatx4 SharedFloat4;

// What a wavefront has to know for its rounds.
struct TileWork {
    const uint32_t *codes;
    const uint16_t *scales;
    int64_t n;
    void *S;
    int64_t lds, q0, nq, first, last, step;
    StoreAs as;
};

// The rounds of a wavefront, with NP parts of a query entry in fp16, or (SPREAD) in bf16.  Two forms of the whole walk: a choice within a
// round costs the common one its last registers (512 x 1M, d = 128, fp32 queries, bf16 scores 382 us, so 412), and so does a second
// form with all ways to store.
template <bool BF_S, int D, int G, int NP, bool SPREAD> struct TileWalk : TileWork {
    typedef ScoreSteps<D, G> T;
    static constexpr int NS = D / G;  // scales of an item
    SharedParts *operand;             // the queries' parts
    SharedFloat *back;                // 2^-shift of every row
    int shift;                        // of row lane % 32
    bool q_wide;                      // some row's shift is far from 0
    int lane, a, h;
    uint32_t w[D / 8], raw[(NS + 1) / 2];
    __device__ __forceinline__ TileWalk(const TileWork &work, SharedParts *operand, SharedFloat *back)
        : TileWork(work), operand(operand), back(back), shift(0), q_wide(false), lane(threadIdx.x & 63), a(lane & 31), h(lane >> 5) {}

    // An item's row and scales are read by one lane, 16 bytes at a time: lane <a, h> has item 2 a + h of the round.  compute
    // exchanges them between the halves of the wavefront, as the products take them.
    __device__ __forceinline__ void fetch(int64_t span) {
        const int64_t item = std::min<int64_t>(span * 64 + 2 * a + h, n - 1);
        __builtin_memcpy(w, __builtin_assume_aligned(codes + item * (D / 8), D < 32 ? 8 : 16), D / 2);
        const uint16_t *ps = scales + item * NS;
        if constexpr (NS == 1) raw[0] = *ps;
        else __builtin_memcpy(raw, __builtin_assume_aligned(ps, NS < 8 ? 2 * NS : 16), 2 * NS);
    }

    // Waits for fetch's loads: at the end of a round the compiler knows how many stores came after them and lets those be.
    __device__ __forceinline__ void arrived() {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) asm volatile("" : "+v"(w[i]));
#pragma unroll
        for (int i = 0; i < (NS + 1) / 2; ++i) asm volatile("" : "+v"(raw[i]));
    }

    // the round's sums, and the next round's codes on their way
    __device__ __forceinline__ void compute(int64_t next, float (&total)[2][16]) {
        uint32_t cw[2][T::PARTS][T::STEPS];
        float cs[2][NS];
        uint32_t top[2] = {0, 0};
        // Sums of shifted queries times a scale stay in fp32's range while neither factor is beyond 2^60 or below 2^-60.
        // Elsewhere the scales of an item are shifted too, and the results back in one step.
        bool wide = q_wide;
#pragma unroll
        for (int t = 0; t < T::PARTS; ++t)
#pragma unroll
            for (int s = 0; s < T::STEPS; ++s) {
                // the upper half's first word against the lower half's second
                const auto both = __builtin_amdgcn_permlane32_swap(w[T::word(t, s, 0)], w[T::word(t, s, 1)], false, false);
                cw[0][t][s] = both[0];
                cw[1][t][s] = both[1];
            }
        uint32_t own[2][(NS + 1) / 2];
#pragma unroll
        for (int i = 0; i < (NS + 1) / 2; ++i) {
            const auto both = __builtin_amdgcn_permlane32_swap(raw[i], raw[i], false, false);
            own[0][i] = both[0];
            own[1][i] = both[1];
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int g = 0; g < NS; ++g) {
                const uint32_t bits = g & 1 ? own[c][g / 2] & 0xffff0000u : own[c][g / 2] << 16, m = bits & 0x7fffffffu;
                cs[c][g] = __uint_as_float(bits);
                top[c] = max(top[c], m < 0x7f800000u ? m : 0u);
            }
            wide = wide || (top[c] && (top[c] > 0x5d800000u || top[c] < 0x21800000u));
        }
        fetch(next);
        asm volatile("" ::: "memory");  // the operands are read from LDS in every round, not kept in registers
        int k[2] = {0, 0};
        wide = __any(wide);
        if (wide) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                k[c] = top[c] ? __builtin_amdgcn_frexp_expf(__uint_as_float(top[c])) : 0;
#pragma unroll
                for (int g = 0; g < NS; ++g) cs[c][g] = ldexpf(cs[c][g], -k[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int v = 0; v < 16; ++v) total[c][v] = 0.f;
#pragma unroll
            for (int t = 0; t < T::PARTS; ++t) {
                floatx16 acc;
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
                for (int s = 0; s < T::STEPS; ++s) {
                    if constexpr (SPREAD) {
                        const bf16x8 B = unpack8_wide(cw[c][t][s]);
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            const bf16x8 A = __builtin_bit_cast(bf16x8, operand[((t * T::STEPS + s) * NP + p) * 64 + lane]);
                            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, B, acc, 0, 0, 0);
                        }
                    } else {
                        halfx2 e[4];
                        unpack8(cw[c][t][s], e);
                        const u32x4 bits = {__builtin_bit_cast(uint32_t, e[0]), __builtin_bit_cast(uint32_t, e[1]),
                                            __builtin_bit_cast(uint32_t, e[2]), __builtin_bit_cast(uint32_t, e[3])};
                        const halfx8 B = __builtin_bit_cast(halfx8, bits);
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            const halfx8 A = __builtin_bit_cast(halfx8, operand[((t * T::STEPS + s) * NP + p) * 64 + lane]);
                            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(A, B, acc, 0, 0, 0);
                        }
                    }
                }
                const float scale = cs[c][t * T::PART / G];
#pragma unroll
                for (int v = 0; v < 16; ++v) total[c][v] = fmaf(acc[v], scale, total[c][v]);
            }
            asm volatile("" ::: "memory");
        }
        // result v is <query 8 (v / 4) + 4 h + v % 4, item 2 a + c>
        if (wide) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int r = __shfl(shift, 8 * (v >> 2) + 4 * h + (v & 3));
                total[0][v] = ldexpf(total[0][v], k[0] - r);
                total[1][v] = ldexpf(total[1][v], k[1] - r);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const floatx4 b4 = *(SharedFloat4 *)(back + 8 * j + 4 * h);
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    total[0][4 * j + v] *= b4[v];
                    total[1][4 * j + v] *= b4[v];
                }
            }
        }
    }

    __device__ __forceinline__ void run() {
        float total[2][16];
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        typedef float floatx2 __attribute__((ext_vector_type(2)));
        constexpr int ES = BF_S ? 2 : 4;
        const int rows = (int)std::min<int64_t>(32, nq - q0);
        int64_t span = first;
        const int64_t whole = std::min(last, n / 64);
        arrived();
        if (!SPREAD && as == StoreAs::BUFFER) {
            const uint32_t half = (uint32_t)(4 * lds * ES);  // bytes from a row to that of the upper half's lanes
            const uint32_t place = h * half + a * 2 * ES;
            for (; span < whole; span += step) {
                compute(std::min(span + step, last - 1), total);
                char *at = (char *)S + (q0 * lds + span * 64) * ES;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int row = 8 * (v >> 2) + (v & 3);  // and row + 4 in the upper half
                    // up to the end of the last of the two that exists
                    const uint32_t bytes = rows > row + 4 ? half + 64 * ES : rows > row ? 64 * ES : 0;
                    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(at, 0, (int)bytes, 0x00020000);
                    const floatx2 f = {total[0][v], total[1][v]};
                    if constexpr (BF_S) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2)), rsrc, (int)place, 0, 0);
                    else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f), rsrc, (int)place, 0, 0);
                    at += lds * (ES * ((v & 3) == 3 ? 5 : 1));
                }
                arrived();
            }
        } else if (!SPREAD && BF_S && as == StoreAs::PLAIN && rows == 32) {
            for (; span < whole; span += step) {
                compute(std::min(span + step, last - 1), total);
                char *at = (char *)S + ((q0 + 4 * h) * lds + span * 64 + 2 * a) * ES;
                asm volatile("" : "+v"(at));  // sixteen addresses are not kept from round to round
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    typedef uint32_t u32_any __attribute__((aligned(2)));
                    const floatx2 f = {total[0][v], total[1][v]};
                    *(u32_any *)at = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
                    at += lds * (ES * ((v & 3) == 3 ? 5 : 1));
                }
                arrived();
            }
        }
        for (; span < last; span += step) {
            compute(std::min(span + step, last - 1), total);
            const int64_t item = span * 64 + 2 * a;
            char *at = (char *)S + ((q0 + 4 * h) * lds + item) * ES;
            asm volatile("" : "+v"(at));
            const int left = rows - 4 * h;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                if (8 * (v >> 2) + (v & 3) < left) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        if (item + c < n) {
                            if constexpr (BF_S) ((__bf16 *)at)[c] = (__bf16)total[c][v];
                            else ((float *)at)[c] = total[c][v];
                        }
                }
                at += lds * (ES * ((v & 3) == 3 ? 5 : 1));
            }
        }
    }
};

template <bool BF_Q, bool BF_S, int D, int G>
__global__ __launch_bounds__(256, 4)
void scores_tile_kernel(const void *__restrict__ Q, int64_t ldq, int64_t nq, const uint32_t *__restrict__ codes,
                        const uint16_t *__restrict__ scales, int64_t n, void *__restrict__ S, int64_t lds, StoreAs as, unsigned qgroups,
                        unsigned stretch, unsigned rounds, unsigned units) {
    typedef ScoreSteps<D, G> T;
    constexpr int NP = BF_Q ? 1 : 2, NP_WIDE = BF_Q ? 1 : 3;  // parts of a query entry, in fp16 and in bf16
    const int lane = threadIdx.x & 63, a = lane & 31, h = lane >> 5;
    // Units of work, a workgroup's each: a block of `stretch` x `rounds` x 4 x 64 items is walked by `stretch` workgroups side by side
    // for one group of 32 queries, then for the next group.  So what is written at one time lies close together in few rows,
    // and a block's codes are read from the L2 by all but the first group (consecutive workgroups go to different XCDs, which
    // have an L2 each: every XCD has its own run of units).
    const unsigned per_xcd = (units + 7) / 8, unit = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per_xcd || unit >= units) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned block = unit / (qgroups * stretch), in_block = unit % (qgroups * stretch);
    const int64_t q0 = (int64_t)(in_block / stretch) * 32, spans = (n + 63) / 64;
    const int64_t step = 4 * (int64_t)stretch, begin = block * (step * rounds);
    const int64_t first = begin + 4 * (in_block % stretch) + wave, last = std::min(spans, begin + step * rounds);

    constexpr int NSTEP = D / 16, MINE = (NSTEP + 3) / 4;
    __shared__ u32x4 operand[NSTEP * NP_WIDE * 64 > NSTEP * NP * 64 ? NSTEP * NP_WIDE * 64 : NSTEP * NP * 64];
    __shared__ uint2 row_ends[4][32];
    __shared__ __align__(16) float back[32];  // 2^-shift of every row
    TileWalk<BF_S, D, G, NP, false> walk({codes, scales, n, S, lds, q0, nq, first, last, step, as}, (SharedParts *)operand, (SharedFloat *)back);
    if (first < last) walk.fetch(first);  // on its way while the queries are prepared

    // The queries as operands, in LDS for the four wavefronts (registers for them would halve the wavefronts), shifted so that
    // the largest finite entry of a row lies in [2^14, 2^15).  Each wavefront makes every fourth step's.
    int shift;
    bool spread;  // entries of one row too far apart for the fp16 parts
    {
        float x[MINE][8];
        // The largest finite magnitude and the smallest but 0 as bits, which order like the values: top is NONE + 2 * magnitude, where
        // infinities and NaN wrap around to less than NONE, low is 2 * magnitude - 1, where they and 0 come out above all others.
        constexpr uint32_t NONE = 0x01000000u;
        uint32_t top = NONE, low = ~0u;
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            const int i = 4 * j + wave;
            Piece<BF_Q> p = piece_zero<BF_Q>();
            if (i < NSTEP && q0 + a < nq) p = piece_load<BF_Q>(Q, (q0 + a) * ldq + 8 * T::word(i / T::STEPS, i % T::STEPS, h));
            piece_floats<BF_Q>(p, x[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t m = (__float_as_uint(x[j][e]) << 1) + NONE;
                top = max(top, m);
                low = min(low, m - (NONE + 1));
            }
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        low = min(low, (uint32_t)__shfl_xor((int)low, 32));
        if (h == 0) row_ends[wave][a] = make_uint2(top, low);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint2 ends = row_ends[i][a];
            top = max(top, ends.x);
            low = min(low, ends.y);
        }
        const float largest = __uint_as_float((top - NONE) >> 1);
        shift = top > NONE ? 15 - __builtin_amdgcn_frexp_expf(largest) : 0;
        const uint32_t least = 2 * __float_as_uint(ldexpf(largest, BF_Q ? -31 : -20));
        spread = __any(least > 0 && low < least - 1);
        if (threadIdx.x < 32) back[a] = ldexpf(1.f, -shift);
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            const int i = 4 * j + wave;
            if (i < NSTEP && spread) {
                uint32_t part[NP_WIDE][8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = ldexpf(x[j][e], shift - 4);  // the codes are times 16
#pragma unroll
                    for (int p = 0; p < NP_WIDE; ++p) {
                        const __bf16 b = (__bf16)v;
                        part[p][e] = __builtin_bit_cast(uint16_t, b);
                        const float rest = v - (float)b;  // NaN where v is not finite
                        v = rest == rest ? rest : 0.f;
                    }
                }
#pragma unroll
                for (int p = 0; p < NP_WIDE; ++p)
                    operand[(i * NP_WIDE + p) * 64 + lane] = u32x4{part[p][0] | part[p][1] << 16, part[p][2] | part[p][3] << 16,
                                                                   part[p][4] | part[p][5] << 16, part[p][6] | part[p][7] << 16};
            } else if (i < NSTEP) {
                halfx8 hi, lo;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = 2 * (e % 4) + e / 4;  // the order in which unpack8 leaves a word's codes
                    const float v = ldexpf(x[j][e], shift);
                    hi[at] = (_Float16)v;
                    const float rest = v - (float)hi[at];  // NaN where v is not finite
                    lo[at] = rest == rest ? (_Float16)rest : (_Float16)0.f;
                }
                operand[(i * NP) * 64 + lane] = __builtin_bit_cast(u32x4, hi);
                if constexpr (NP == 2) operand[(i * NP + 1) * 64 + lane] = __builtin_bit_cast(u32x4, lo);
            }
        }
        __syncthreads();
    }
    if (first >= last) return;
    const bool q_wide = __any(shift > 60 || shift < -60);
    if (spread) {
        TileWalk<BF_S, D, G, NP_WIDE, true> other(walk, walk.operand, walk.back);
        other.shift = shift;
        other.q_wide = q_wide;
        other.fetch(first);
        other.run();
        return;
    }
    walk.shift = shift;
    walk.q_wide = q_wide;
    walk.run();
}

// Queries up to which the vector units work; on them / on the matrix cores, in us: 3 and 4 x 1M, d = 128,
// fp32 28 / 31 and 35 / 31; 2 and 3 x 10M, d = 128, bf16 (one part of a query on the matrix cores) 168 / 178 and 227 / 180; 4 x 3M, d = 64,
// groups of 16 47 / 49; 4 x 1M, d = 16, bf16 8 / 14.
template <bool BF_Q, int D> constexpr int scores_few() { return D < 128 ? 4 : BF_Q ? 2 : 3; }

template <bool BF_Q, bool BF_S, int D, int G>
static void scores_typed(const als_ctx *ctx, const als_table *Q, const als_qtable *T, const als_matrix *S, hipStream_t s) {
    const int64_t n = T->rows, nq = Q->rows;
    if (nq <= scores_few<BF_Q, D>()) {
        auto go = [&](auto count) {
            constexpr int LPI = D / (D < 32 || count() > 2 ? 16 : 32), ITEMS = 4 * (64 / LPI) * (LPI > 4 ? LPI : 4);  // of a workgroup's round
            const dim3 grid((unsigned)std::min<int64_t>((n + ITEMS - 1) / ITEMS, (int64_t)ctx->num_cu * 8));
            hipLaunchKernelGGL((scores_few_kernel<BF_Q, BF_S, D, G, count()>), grid, dim3(256), 0, s, Q->data, Q->ld,
                               (const uint8_t *)T->codes, (const uint16_t *)T->scales, n, S->data, S->ld);
        };
        if (nq == 1) go(std::integral_constant<int, 1>{});
        else if (nq == 2) go(std::integral_constant<int, 2>{});
        else if constexpr (scores_few<BF_Q, D>() > 2) {
            if (nq == 3) go(std::integral_constant<int, 3>{});
            else if constexpr (scores_few<BF_Q, D>() > 3) go(std::integral_constant<int, 4>{});
        }
        return;
    }
    const int64_t qgroups = (nq + 31) / 32, spans = (n + 63) / 64;
    // Rounds per wavefront and workgroups side by side, where the table is long enough for 16 wavefronts per compute unit.  What
    // counts is how close together the writes under way are, most of all where the rows' pieces of a round do not end with a 128-byte
    // line, which two wavefronts then write a part of each.  2, 4, 6, 8 rounds of 16 workgroups: whole lines 293, 266, 252, 252 us (512
    // queries x 1M items, d = 64, bf16) and 514, 484, 474, 479 us (d = 128, fp32), shared lines (1 000 001 items) 262, 322, 368, 386 us
    // and 533, 645, 691, 717 us; 2 x 32 or 4 x 8 are no better.  Workgroups of one item stretch and all query groups at one time
    // took 1.6 times as long.
    const int64_t es = BF_S ? 2 : 4, most = S->ld * es % 128 == 0 && (uintptr_t)S->data % 128 == 0 ? 6 : 2;
    const int64_t rounds = std::max<int64_t>(1, std::min<int64_t>(most, spans * qgroups / ((int64_t)ctx->num_cu * 16)));
    const int64_t stretch = std::max<int64_t>(1, std::min<int64_t>(16, spans / (32 * rounds)));
    // a buffer's offsets have 32 bits: five rows must fit
    const bool near = S->ld < (int64_t)1 << 27, words = !BF_S || (S->ld % 2 == 0 && (uintptr_t)S->data % 4 == 0);
    const StoreAs as = !near ? StoreAs::GUARDED : words ? StoreAs::BUFFER : StoreAs::PLAIN;
    // units of work, as many groups of queries at a time as a grid holds
    const int64_t per_group = (spans + 4 * rounds * stretch - 1) / (4 * rounds * stretch) * stretch;
    const int64_t batch = std::max<int64_t>(1, ((int64_t)1 << 22) / per_group);
    for (int64_t g = 0; g < qgroups; g += batch) {
        const int64_t q0 = g * 32, groups = std::min(batch, qgroups - g), units = per_group * groups;
        hipLaunchKernelGGL((scores_tile_kernel<BF_Q, BF_S, D, G>), dim3((unsigned)((units + 7) / 8 * 8)), dim3(256), 0, s,
                           (const char *)Q->data + q0 * Q->ld * (BF_Q ? 2 : 4), Q->ld, std::min(nq - q0, groups * 32),
                           (const uint32_t *)T->codes, (const uint16_t *)T->scales, n, (char *)S->data + q0 * S->ld * (BF_S ? 2 : 4), S->ld, as,
                           (unsigned)groups, (unsigned)stretch, (unsigned)rounds, (unsigned)units);
    }
}

template <bool BF_Q, bool BF_S>
static void scores_sized(const als_ctx *ctx, const als_table *Q, const als_qtable *T, const als_matrix *S, hipStream_t s) {
    switch (T->d * 256 + T->group) {
        case 16 * 256 + 16: return scores_typed<BF_Q, BF_S, 16, 16>(ctx, Q, T, S, s);
        case 32 * 256 + 16: return scores_typed<BF_Q, BF_S, 32, 16>(ctx, Q, T, S, s);
        case 32 * 256 + 32: return scores_typed<BF_Q, BF_S, 32, 32>(ctx, Q, T, S, s);
        case 64 * 256 + 16: return scores_typed<BF_Q, BF_S, 64, 16>(ctx, Q, T, S, s);
        case 64 * 256 + 32: return scores_typed<BF_Q, BF_S, 64, 32>(ctx, Q, T, S, s);
        case 64 * 256 + 64: return scores_typed<BF_Q, BF_S, 64, 64>(ctx, Q, T, S, s);
        case 128 * 256 + 16: return scores_typed<BF_Q, BF_S, 128, 16>(ctx, Q, T, S, s);
        case 128 * 256 + 32: return scores_typed<BF_Q, BF_S, 128, 32>(ctx, Q, T, S, s);
        case 128 * 256 + 64: return scores_typed<BF_Q, BF_S, 128, 64>(ctx, Q, T, S, s);
        default: return scores_typed<BF_Q, BF_S, 128, 128>(ctx, Q, T, S, s);
    }
}

als_status launch_scores(als_ctx *ctx, const als_table *Q, const als_qtable *T, const als_matrix *S, hipStream_t s) {
    const bool bq = Q->dtype == ALS_BF16, bs = S->dtype == ALS_BF16;
    if (bq && bs) scores_sized<true, true>(ctx, Q, T, S, s);
    else if (bq) scores_sized<true, false>(ctx, Q, T, S, s);
    else if (bs) scores_sized<false, true>(ctx, Q, T, S, s);
    else scores_sized<false, false>(ctx, Q, T, S, s);
    ALS_HIP(ctx, hipGetLastError());
    return ALS_OK;
}

}  // namespace als
