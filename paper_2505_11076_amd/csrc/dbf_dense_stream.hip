// Products with ordinary weights, few rows: the weights stream past rows of x that stay in registers (include/dbf.h: dbf_dense_gemm, dbf_grouped_gemm; dbf_dense.h: the
// instructions).
#include "dbf_dense.h"

namespace {

typedef const __attribute__((address_space(1))) unsigned* Global;
typedef __attribute__((address_space(3))) unsigned* Shared;

// A workgroup has a share of all pieces of work, 16 outputs (gated: of both matrices) for 16 rows each, those of the same rows one behind the other.  Its wavefronts have SPAN
// steps of the long axis each: their part of the rows stays in registers, weights go from memory to LDS by C steps, three times that ahead of those that are multiplied, and
// their sums meet in LDS, where one wavefront, each in turn, adds them up in order.
// (Weights straight to registers, 16 lanes a row each: every 16 bytes were an access of their own to the first cache, and these took two thirds of the time.  Here eight
// lanes have 128 bytes of a row.  In LDS a row's piece p is at place p ^ (row % 8), so that 16 rows' pieces lie in all banks evenly.)
// Bound by memory: 13 rows through a head of 4096 x 128256 in 8 bits, 529 MB, 82 us = 6.4 TB/s, beside the 7.0 of a bare read, for 103 with weights straight to registers,
// 98 with loads that leave their lines in the caches and 97 with two places; the kernel for few rows 112.  Experts of few rows (147 MB, 28.5 us, 5.2 TB/s) wait besides at the
// start of each share, where rows have to be there before the first product.  (Scales of a byte are widened in the round of the loop that loads them, for which the compiler waits for all
// loads once a round; it does not show: with fp32 scales, which have no such wait, the head takes 82.5 for 82.7, the experts 28.4 for 28.7.)
constexpr int KW = 8;
template <int TYPE, bool FLOAT, bool GATED, bool EXACT, int SPAN, int C>
__global__ __launch_bounds__(64 * KW) void dbf_dense_stream_kernel(const DenseArgs a) {
    constexpr int ROWS = 16, N = GATED ? 2 : 1, PARTS = SPAN / C, LOADS = 2 * N * C + (TYPE == DBF_E4M3 ? N : 0), AHEAD = 3, PLACES = AHEAD + 1;
    static_assert((PARTS % PLACES == 0 || PLACES % PARTS == 0) && AHEAD * LOADS < 64, "parts go into the places in turn; the count of loads");
    // (objects of their own: the compiler then knows that a load into one is not read from another)
    constexpr int PLACE = KW * N * C * 2048;
    __shared__ __align__(16) uint8_t s0[PLACE], s1[PLACE], s2[PLACE], s3[PLACE];
    uint8_t* const places[PLACES] = {s0, s1, s2, s3};
    __shared__ dbf_f4 sums[2][KW][N][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, q = lane >> 4;
    const int n16 = (a.n_out + 15) / 16, tiles = a.starts ? tiles_of(a, ROWS) : (a.n_rows + ROWS - 1) / ROWS, kb = (a.k_bytes + STEP - 1) / STEP;
    const long long all = (long long)tiles * n16;
    auto step_of = [&](int part, int s) { return (part * KW + wave) * C + s; };   // a part of all wavefronts is one stretch of the rows
    // a compute die (workgroup modulo 8) has shares that follow each other
    const int share = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    long long item = all * share / gridDim.x;
    const long long end = all * (share + 1) / gridDim.x;
    // where a lane's pieces of the weights lie in a row; behind its end the last one (the rows have zeros there)
    int at[SPAN];
#pragma unroll
    for (int s = 0; s < SPAN; ++s) at[s] = min(step_of(s / C, s % C) * STEP + 16 * ((lane & 7) ^ (lane >> 3)), a.k_bytes - 16);
    const int read_at = wave * (N * C * 2048) + c * STEP + 16 * (q ^ (c & 7));
    int turn = 0;
    while (item < end) {
        const int t = (int)(item / n16), from_n = (int)(item - (long long)t * n16), to_n = (int)min((long long)n16, from_n + end - item);
        const Tile tile = tile_of(a, t, ROWS);
        const int last_n = to_n - 1;
        int scale[PLACES][N];   // of the weights; lane s has step s's
        // (behind the last of the rows' pieces of work one address for all lanes, so that no round has other loads under way than another)
        // What wait() counts on is that a part is LOADS loads at least and that parts set out one behind the other: nothing passes the two marks, and the build counts what is between them.
        auto fetch = [&](int place, int n, int part) {
            asm volatile("; loads of a part" ::: "memory");
            unsigned live = n <= last_n ? ~0u : 0u;
            asm("" : "+v"(live));   // (as a number: no branches beside the loads)
            n = min(n, last_n);
            uint8_t* to = places[place];
            if (TYPE == DBF_E4M3) {
                const long long of = tile.group * a.w_scale_group + (16 * n / DBF_SCALE_BLOCK) * a.w_scale_row + min(step_of(part, lane & (C - 1)), kb - 1);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    scale[place][i] = FLOAT ? static_cast<const int*>(i ? a.w_up_scale : a.w_scale)[of] : static_cast<const uint8_t*>(i ? a.w_up_scale : a.w_scale)[of];
            }
            const long long base = tile.group * a.w_group + 16LL * n * a.w_row;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const unsigned row = (unsigned)min(8 * half + (lane >> 3), a.n_out - 1 - 16 * n) * (unsigned)a.w_row;
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int s = 0; s < C; ++s)
                        __builtin_amdgcn_global_load_lds((Global)((i ? a.w_up : a.w) + base + ((row + at[part * C + s]) & live)), (Shared)(to + wave * (N * C * 2048) + (i * C + s) * 2048 + 1024 * half),
                                                         16, 0, 2);   // (2: read once, so it need not stay in the caches: 96 -> 81 us for 525 MB)
            }
            asm volatile("; end of a part's loads" ::: "memory");
        };
        // the loads before those of the last three parts have arrived; what was read from LDS is in registers
        auto wait = [&]() {
            __builtin_amdgcn_s_waitcnt(0x0070 | (AHEAD * LOADS & 15) | (AHEAD * LOADS >> 4) << 14);
            asm volatile("" ::: "memory");
        };
#pragma unroll
        for (int p = 0; p < AHEAD; ++p) fetch(p, from_n + p / PARTS, p % PARTS);
        // the rows
        const int row = tile.row + min(c, tile.rows - 1);
        int from = a.x_rows ? a.x_rows[row] : row;
        const bool known = (unsigned)from < (unsigned)a.n_x_rows;
        if (!known) from = 0;
        v8i x[SPAN];
        unsigned xs[PARTS];
#pragma unroll
        for (int s = 0; s < SPAN; ++s) {
            dbf_u4 v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int in_row = step_of(s / C, s % C) * STEP + 16 * q + 64 * h;
                v[h] = *reinterpret_cast<const dbf_u4*>(a.x + from * a.x_row + min(in_row, a.k_bytes - 16));
                if (in_row >= a.k_bytes) v[h] = (dbf_u4){0, 0, 0, 0};
            }
            x[s] = both(v[0], v[1]);
        }
        if constexpr (TYPE == DBF_E4M3) {
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {   // (C divides 4: a part's bytes are in one word)
                const int s = min(step_of(i, 0), kb - 1);
                xs[i] = *reinterpret_cast<const unsigned*>(a.x_scale + from * a.x_scale_row + (s & ~3)) >> (8 * (s & 3));
            }
            // A step behind the row's end, whose values are zeros, has the last block's scale where it is its part's first, else 1: what lies behind that block's byte may be 255, no
            // number, and so would be its products.
            if constexpr (C > 1) {
                static_assert(C == 2, "a part's second step is its last");
#pragma unroll
                for (int i = 0; i < PARTS; ++i) {
                    const bool there = step_of(i, 1) < kb;
                    xs[i] = (xs[i] & (there ? ~0u : 255u)) | (there ? 0u : 127u << 8);
                }
            }
        }
        dbf_f4 acc[N];
        auto products = [&](int place, int part) {
            const uint8_t* of = places[place];
            if constexpr (TYPE == DBF_E4M3) {
#pragma unroll
                for (int i = 0; i < N; ++i) asm volatile("" : "+v"(scale[place][i]));   // (not looked at before the wait)
            }
#pragma unroll
            for (int s = 0; s < C; ++s) {
                const int step = part * C + s, x_scale = TYPE == DBF_E4M3 ? xs[part] >> (8 * s) & 255 : 0;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const uint8_t* w_at = of + read_at + (i * C + s) * 2048;
                    const v8i w = both(*reinterpret_cast<const dbf_u4*>(w_at), *reinterpret_cast<const dbf_u4*>(of + (read_at ^ 64) + (i * C + s) * 2048));
                    const int w_scale = TYPE == DBF_E4M3 ? __builtin_amdgcn_readlane(scale[place][i], s) : 0;
                    if constexpr (EXACT) multiply_exactly<FLOAT>(acc[i], w, x[step], w_scale, x_scale);
                    else multiply<TYPE, FLOAT>(acc[i], w, x[step], w_scale, x_scale);
                }
            }
        };
        auto clear = [&]() {
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = (dbf_f4){0.f, 0.f, 0.f, 0.f};
        };
        auto join = [&](int n) {
#pragma unroll
            for (int i = 0; i < N; ++i) sums[turn & 1][wave][i][lane] = acc[i];
            __builtin_amdgcn_s_waitcnt(0xC07F);   // LDS only: the next weights stay under way
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (wave == turn % KW) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    acc[i] = sums[turn & 1][0][i][lane];
#pragma unroll
                    for (int k = 1; k < KW; ++k) acc[i] += sums[turn & 1][k][i][lane];
                }
                if constexpr (GATED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[0][e] = gate(acc[0][e], acc[1][e]);
                }
                if (!known) acc[0] = (dbf_f4){0.f, 0.f, 0.f, 0.f};
                if (c < tile.rows && 16 * n + 4 * q < a.n_out) store4(a, row, 16 * n + 4 * q, acc[0]);
            }
            ++turn;
        };
        constexpr int ITEMS = PARTS < PLACES ? PLACES / PARTS : 1;   // until the places come round
        for (int n = from_n; n < to_n; n += ITEMS) {
#pragma unroll
            for (int u = 0; u < ITEMS; ++u) {   // (without a way out between: registers whose loads are under way would be copied there)
                clear();
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    const int g = u * PARTS + part;
                    __builtin_amdgcn_s_waitcnt(0xC07F);   // (what was read from the place that the next loads take)
                    asm volatile("" ::: "memory");
                    fetch((g + AHEAD) % PLACES, n + u + (part + AHEAD) / PARTS, (part + AHEAD) % PARTS);
                    wait();
                    products(g % PLACES, part);
                }
                if (n + u < to_n) join(n + u);
            }
        }
        __builtin_amdgcn_s_waitcnt(0x0070);   // (the loads ahead, before other weights go there)
        asm volatile("" ::: "memory");
        item += to_n - from_n;
    }
}

template <int TYPE, bool FLOAT, bool GATED, bool EXACT, int SPAN, int C>
int launch(const DenseArgs& a, hipStream_t stream) {
    const long long most = ((a.n_rows + 15LL) / 16 + (a.starts ? std::min(a.n_groups, a.n_rows) : 0)) * ((a.n_out + 15) / 16);
    constexpr int LDS = KW * (GATED ? 2 : 1) * (4 * C * 2048 + 2048);
    const long long grid = std::min(256LL * std::min(163840 / LDS, 2), most);   // what the chip holds at once
    hipLaunchKernelGGL((dbf_dense_stream_kernel<TYPE, FLOAT, GATED, EXACT, SPAN, C>), dim3((unsigned)((grid + 7) / 8 * 8)), dim3(64 * KW), 0, stream, a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}
template <int TYPE, bool FLOAT, bool GATED, bool EXACT>
int launch(const DenseArgs& a, hipStream_t stream) {
    const int steps = (a.k_bytes + STEP - 1) / STEP;
    constexpr int C = GATED ? 1 : 2;
    if (steps <= 8) return launch<TYPE, FLOAT, GATED, EXACT, 1, 1>(a, stream);
    if (steps <= 16) return launch<TYPE, FLOAT, GATED, EXACT, 2, C>(a, stream);
    if (steps <= 32) return launch<TYPE, FLOAT, GATED, EXACT, 4, C>(a, stream);
    return launch<TYPE, FLOAT, GATED, EXACT, 8, C>(a, stream);
}
template <int TYPE, bool FLOAT, bool EXACT>
int launch(const DenseArgs& a, hipStream_t stream) {
    return a.w_up ? launch<TYPE, FLOAT, true, EXACT>(a, stream) : launch<TYPE, FLOAT, false, EXACT>(a, stream);
}

}  // namespace

bool dbf_dense_streams(int k_bytes) { return k_bytes % 16 == 0 && k_bytes <= KW * 8 * STEP; }

int dbf_dense_stream(const void* args, int type, bool float_scales, hipStream_t stream) {
    const DenseArgs& a = *static_cast<const DenseArgs*>(args);
    if (type == DBF_F16) return launch<DBF_F16, false, false>(a, stream);
    if (type == DBF_BF16) return launch<DBF_BF16, false, false>(a, stream);
    if (a.out_dtype == DBF_F32) return float_scales ? launch<DBF_E4M3, true, true>(a, stream) : launch<DBF_E4M3, false, true>(a, stream);
    return float_scales ? launch<DBF_E4M3, true, false>(a, stream) : launch<DBF_E4M3, false, false>(a, stream);
}
