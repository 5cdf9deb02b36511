// Products with ordinary weights, many rows: tiles of weights and rows in LDS (include/dbf.h: dbf_dense_gemm, dbf_grouped_gemm; dbf_dense.h: the instructions).
#include "dbf_dense.h"

#include <cmath>

namespace {

typedef const __attribute__((address_space(1))) unsigned* Global;
typedef __attribute__((address_space(3))) unsigned* Shared;

// A tile is BN rows of weights (gated: 16 of w, 16 of w_up, in turn) times BM rows of x, WN x WM wavefronts.  A step is 128 bytes of all rows; LDS holds two, of which a
// row is 128 bytes, its piece p at place p ^ (row % 8): the 64 pieces that a wavefront reads at once lie in all banks evenly.
// A wavefront has its weights of a step in registers and its rows of x in pairs of 16.  Before a step's last pair all have read what the step has in LDS: there they meet,
// the next step but one sets out for its place, and as each of the weights has done its last product the next step's comes from LDS into its registers: reads and loads are
// under way beside products at all times.
// Bound by the matrix cores and by what feeds them: 2047 rows through 2 x 11008 x 4096 in 8 bits (gated; 369 GFLOP, 140 us at a library's rate for 8192^3) in 171 to 182 us by passes in
// turn, under a profiler 196 in the median and 177 at least (the clock falls as it goes on): 1.9 to 2.2 PFLOP/s, the
// matrix cores busy for half the time.  Steps, timed when each was made: the first form, whose scales were loaded to registers, 246; scales through LDS 206; next weights in place 194; scales in
// the step's own buffer 181; loads given out beside the products of two steps and more 171.  Its 688 tiles are 2.7 rounds of 256 compute units.  fp32 scales cost four operations beside each matrix
// instruction: the same with them 208 us for 180, 16384 rows of 32 experts, 550 GFLOP, 365 to 391.  Four wavefronts of 128 x 128 with sums in the second half of the registers took 257 for the same, weights straight to
// registers did not fit.  A wavefront's sums are all of its 128 accumulators at two wavefronts a SIMD: hence 256 x 256 by eight.
template <int TYPE, bool FLOAT, bool GATED, bool EXACT, int BN, int BM, int WN, int WM, int EACH>
__global__ __launch_bounds__(64 * WN * WM) __attribute__((amdgpu_waves_per_eu(EACH, EACH))) void dbf_dense_tiles_kernel(const DenseArgs a, int n_tiles, int m_tiles) {
    constexpr int WAVES = WN * WM, NS = BN / WN / 16, MS = BM / WM / 16, OUTS = GATED ? BN / 2 : BN;
    constexpr int W_LOADS = BN / 8 / WAVES, X_LOADS = BM / 8 / WAVES;
    static_assert(W_LOADS * 8 * WAVES == BN && X_LOADS * 8 * WAVES == BM && MS % 2 == 0, "whole loads");
    static_assert((64 * WAVES) % BM == 0 && BM % 64 == 0, "a thread or more for each scale's word");
    constexpr int SCALES = (BN + BM) * STEP, ROOM = SCALES + (TYPE == DBF_E4M3 ? 4 * BM + 256 : 0);   // behind the rows x's scales, a word each: of four steps
    // (objects of their own: the compiler then knows that a load into one is not read from another)
    __shared__ __align__(16) uint8_t s0[ROOM], s1[ROOM];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, q = lane >> 4;
    const int wn = wave % WN, wm = wave / WN;
    // a compute die (workgroup modulo 8) has neighbouring tiles, up to 8 tiles of rows with the same weights
    if (a.starts) m_tiles = tiles_of(a, BM);
    const int total = n_tiles * m_tiles, die = blockIdx.x & 7, slot = blockIdx.x >> 3, per = total >> 3, extra = total & 7;
    if (slot >= per + (die < extra ? 1 : 0)) return;
    const int id = die * per + min(die, extra) + slot, band = id / (8 * n_tiles), in_band = id - band * 8 * n_tiles, high = min(8, m_tiles - 8 * band);
    const Tile tile = tile_of(a, 8 * band + in_band % high, BM);
    const int out0 = in_band / high * OUTS;
    const int steps = a.k_bytes / (2 * STEP) * 2, all_steps = (a.k_bytes + STEP - 1) / STEP, last = all_steps - 1;   // steps: in rounds of two; up to two are left

    // where a lane's pieces lie, in bytes: of the weights behind the tile's first row, of x behind the tile's first or, where rows are given, behind x's
    auto x_from = [&](int row) -> int {
        if (!a.x_rows) return row;
        const int from = a.x_rows[tile.row + row];
        return (unsigned)from < (unsigned)a.n_x_rows ? from : 0;
    };
    unsigned w_at[W_LOADS], x_at[X_LOADS];
    const int place = 16 * ((lane & 7) ^ (lane >> 3));
    const long long x0 = a.x_rows ? 0 : tile.row, w0 = tile.group * a.w_group + out0 * a.w_row;
#pragma unroll
    for (int i = 0; i < W_LOADS; ++i) {
        const int row = 8 * (WAVES * i + wave) + (lane >> 3), n = GATED ? row / 32 * 16 + row % 16 : row;
        w_at[i] = (unsigned)(min(n, a.n_out - 1 - out0) * (int)a.w_row + place);
    }
#pragma unroll
    for (int i = 0; i < X_LOADS; ++i) {
        const int row = min(8 * (WAVES * i + wave) + (lane >> 3), tile.rows - 1);
        x_at[i] = (unsigned)x_from(row) * (unsigned)a.x_row + place;
    }
    // (of the last step the pieces behind the rows' end are not read: the row's first of the step in their place, which zeros overwrite)
    const int behind = last * STEP + place < a.k_bytes ? 0 : place;
    constexpr int LOADS = W_LOADS + X_LOADS;
    auto fetch = [&](uint8_t* to, int step, int from_load, int to_load) {
        const int back = step == last ? behind : 0;
#pragma unroll
        for (int k = from_load; k < to_load; ++k) {
            if (k < W_LOADS) {
                const int row = 8 * (WAVES * k + wave);
                const uint8_t* from = (GATED && row / 16 % 2 ? a.w_up : a.w) + w0 + step * STEP;
                __builtin_amdgcn_global_load_lds((Global)(from + (w_at[k < W_LOADS ? k : 0] - back)), (Shared)(to + row * STEP), 16, 0, 0);
            } else {
                const int i = k - W_LOADS;
                const uint8_t* from = a.x + x0 * a.x_row + step * STEP;
                __builtin_amdgcn_global_load_lds((Global)(from + (x_at[i < 0 ? 0 : i] - back)), (Shared)(to + (BN + 8 * (WAVES * i + wave)) * STEP), 16, 0, 0);
            }
        }
    };
    // scales: those of the rows go through LDS, the words that have a step's bytes; the weights' are the wavefront's
    unsigned x_scale_at = 0;
    const uint8_t *w_scale = nullptr, *up_scale = nullptr;
    if constexpr (TYPE == DBF_E4M3) {
        x_scale_at = (unsigned)x_from(min((int)threadIdx.x % BM, tile.rows - 1)) * (unsigned)a.x_scale_row;
        const long long block = tile.group * a.w_scale_group + (min(out0 + (GATED ? 8 : 16) * NS * wn, a.n_out - 1) / DBF_SCALE_BLOCK) * a.w_scale_row;
        w_scale = static_cast<const uint8_t*>(a.w_scale) + block * (FLOAT ? 4 : 1);
        up_scale = static_cast<const uint8_t*>(a.w_up_scale) + block * (FLOAT ? 4 : 1);
    }
    // A word has the bytes of four steps and stays for the two of them that its place is used for: in the other two, and in wavefronts without rows of their own, all lanes load one word to
    // where nobody reads.  (Each lane's word is a cache line of its own: all words in every step were a quarter of what the second cache was asked for.  No branch: it would end the block of
    // instructions, and the compiler then moves products behind it, where the operands of all of them are alive at once.)
    auto fetch_x_scales = [&](uint8_t* to, int step) {
        if constexpr (TYPE == DBF_E4M3) {
            const bool needed = (step & 2) == 0 && wave < BM / 64;
            unsigned lanes = needed ? ~0u : 0u;
            asm("" : "+v"(lanes));
            __builtin_amdgcn_global_load_lds((Global)(a.x_scale + x0 * a.x_scale_row + (step & ~3) + (x_scale_at & lanes)), (Shared)(to + SCALES + 256 * (needed ? wave : BM / 64)), 4, 0, 0);
        }
    };
    int ws = 0, us = 0, ws_next = 0, us_next = 0;
    auto fetch_w_scales = [&](int step) {
        if constexpr (TYPE == DBF_E4M3) {
            ws_next = FLOAT ? reinterpret_cast<const int*>(w_scale)[step] : w_scale[step];
            if constexpr (GATED) us_next = FLOAT ? reinterpret_cast<const int*>(up_scale)[step] : up_scale[step];
        }
    };
    dbf_f4 acc[NS][MS];
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int j = 0; j < MS; ++j) acc[i][j] = (dbf_f4){0.f, 0.f, 0.f, 0.f};
    // pieces q and q + 4 of a row (row % 8 is c % 8)
    const int at0 = c * STEP + 16 * (q ^ (c & 7)), at1 = at0 ^ 64;
    auto read = [&](const uint8_t* from) -> v8i { return both(*reinterpret_cast<const dbf_u4*>(from + at0), *reinterpret_cast<const dbf_u4*>(from + at1)); };
    v8i w[NS], x[3];
    int xs[3];
    auto read_w = [&](const uint8_t* from, int i) { w[i] = read(from + 16 * (NS * wn + i) * STEP); };
    auto read_x = [&](const uint8_t* from, int s, int j, int to) {
        x[to] = read(from + (BN + 16 * (MS * wm + j)) * STEP);
        if constexpr (TYPE == DBF_E4M3) {
            int scale_at = 4 * (16 * MS * wm + c) + (s & 3);
            asm("" : "+v"(scale_at));   // (rows by the instruction's offset: not an address for each, kept for all steps)
            xs[to] = from[SCALES + scale_at + 64 * j];
        } else {
            xs[to] = 0;
        }
    };
    auto product = [&](int i, int j, int of) {
        dbf_f4& sum = acc[i][j];
        const int scale = GATED && i % 2 ? us : ws;
        if constexpr (EXACT) multiply_exactly<FLOAT>(sum, w[i], x[of], scale, xs[of]);
        else multiply<TYPE, FLOAT>(sum, w[i], x[of], scale, xs[of]);
    };
    auto meet = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt = 0, lgkmcnt = 0
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    static_assert(MS % 2 == 0 && MS >= 4, "rows of 16");
    constexpr int AT_ONCE = LOADS / 4, LATER = MS > 4 ? 3 : 2;   // of a step's loads: those beside the last products of the step before the last; sets of products that the others are beside
    static_assert(LATER <= MS - 2, "all loads are given out");
    // In rows of 16: a step's first is in place ODD of x, the next one in the other, and so on in turn; the last in place 2, so that the next step's first has the place of
    // the last but two.
    auto step = [&](uint8_t* now, uint8_t* next, int s, auto odd) {
        constexpr int ODD = decltype(odd)::value;
        const int after = min(s + 1, last);   // (behind the last step that one again, so that no round has other loads under way than another)
        fetch_w_scales(after);
#pragma unroll
        for (int j = 0; j + 2 < MS; ++j) {
            // the rest of the next step's loads, a few beside each of the first products: a wavefront waits where it gives more than are taken
            if (j < LATER) fetch(next, after, AT_ONCE + (LOADS - AT_ONCE) * j / LATER, AT_ONCE + (LOADS - AT_ONCE) * (j + 1) / LATER);
            read_x(now, s, j + 1, (j + 1) % 2 ^ ODD);
            if (j + 3 == MS) read_x(now, s, MS - 1, 2);
#pragma unroll
            for (int i = 0; i < NS; ++i) product(i, j, j % 2 ^ ODD);
            __builtin_amdgcn_sched_barrier(0);   // (else all reads go first, and their registers are too many)
        }
        meet();
        read_x(next, after, 0, 1 - ODD);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            product(i, MS - 2, ODD);
            product(i, MS - 1, 2);
            read_w(next, i);
            fetch(now, min(s + 2, last), AT_ONCE * i / NS, AT_ONCE * (i + 1) / NS);
            if (i == 0) fetch_x_scales(now, min(s + 2, last));
        }
        __builtin_amdgcn_sched_barrier(0);
        ws = ws_next;
        us = us_next;
    };
    fetch_w_scales(0);
    fetch(s0, 0, 0, LOADS);
    fetch_x_scales(s0, 0);
    if (steps) {
        meet();
        fetch(s1, 1, 0, AT_ONCE);
        fetch_x_scales(s1, 1);
        ws = ws_next;
        us = us_next;
        read_x(s0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < NS; ++i) read_w(s0, i);
        for (int s = 0; s < steps; s += 2) {
            step(s0, s1, s, std::integral_constant<int, 0>());
            step(s1, s0, s + 1, std::integral_constant<int, 1>());
        }
        fetch(s1, min(steps + 1, last), AT_ONCE, LOADS);
    } else {
        fetch(s1, min(1, last), 0, LOADS);
        fetch_x_scales(s1, min(1, last));
    }
    // What is left, which has set out already.  Behind the rows' end it becomes zeros, of both operands (a code there may be no number).
    auto left = [&](uint8_t* of, int s) {
        const int have_all = a.k_bytes - s * STEP;
        fetch_w_scales(s);
        meet();
        if (have_all < STEP) {
            for (int i = threadIdx.x; i < (BN + BM) * 8; i += 64 * WAVES) {
                const int row = i >> 3, have = have_all - 16 * ((i ^ row) & 7);
                if (have < 16) {
                    dbf_u4 v = *reinterpret_cast<dbf_u4*>(of + 16 * i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = have <= 4 * e ? 0u : have >= 4 * e + 4 ? v[e] : v[e] & (0xFFFFFFFFu >> (32 - 8 * (have - 4 * e)));
                    *reinterpret_cast<dbf_u4*>(of + 16 * i) = v;
                }
            }
            __syncthreads();
        }
        ws = ws_next;
        us = us_next;
#pragma unroll
        for (int i = 0; i < NS; ++i) read_w(of, i);
#pragma unroll
        for (int j = 0; j < MS; ++j) {
            read_x(of, s, j, 0);
#pragma unroll
            for (int i = 0; i < NS; ++i) product(i, j, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (steps < all_steps) left(s0, steps);
    if (steps + 1 < all_steps) left(s1, steps + 1);
    __builtin_amdgcn_s_waitcnt(0x0070);
    // outputs of rows 16 (MS wm + j) .. + 15: lane c's row, four columns for each i
    auto output = [&](int i, int j, bool known) -> dbf_f4 {
        dbf_f4 v = acc[i][j];
        if constexpr (GATED) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = gate(v[e], acc[i + 1][j][e]);
        }
        return known ? v : (dbf_f4){0.f, 0.f, 0.f, 0.f};
    };
    auto is_known = [&](int r) { return !a.x_rows || r >= tile.rows || (unsigned)a.x_rows[tile.row + r] < (unsigned)a.n_x_rows; };
    constexpr int COLS = GATED ? 8 * NS : 16 * NS;   // of a wavefront
    if (a.quads) {
#pragma unroll
        for (int j = 0; j < MS; ++j) {
            const int r = 16 * (MS * wm + j) + c, n0 = out0 + COLS * wn + 4 * q;
            const bool known = is_known(r);
            if (r >= tile.rows) continue;
#pragma unroll
            for (int i = 0; i < NS; i += GATED ? 2 : 1) {
                const int n = n0 + 16 * (GATED ? i / 2 : i);
                const dbf_f4 v = output(i, j, known);
                if (n < a.n_out) store4(a, tile.row + r, n, v);
            }
        }
        return;
    }
    // Where four outputs are no word that can be stored, each goes by itself: through LDS, so that a wavefront's 64 are neighbours and not four of sixteen rows (6126 rows of 60 experts,
    // 1000 x 2047 in bf16, 111 us for 117; with 128 values a row 26 for 36).
    __syncthreads();
    auto one_by_one = [&](auto type) {
        typedef decltype(type) T;
        constexpr int PITCH = COLS + 16 / sizeof(T);
        static_assert(16 * PITCH * sizeof(T) * WAVES <= SCALES, "a part of LDS for each wavefront");
        T* mine = reinterpret_cast<T*>(s0 + wave * (SCALES / WAVES / 16 * 16));
#pragma unroll
        for (int j = 0; j < MS; ++j) {
            const bool known = is_known(16 * (MS * wm + j) + c);
#pragma unroll
            for (int i = 0; i < NS; i += GATED ? 2 : 1) {
                const dbf_f4 v = output(i, j, known);
                T* to = mine + c * PITCH + 16 * (GATED ? i / 2 : i) + 4 * q;
#pragma unroll
                for (int e = 0; e < 4; ++e) to[e] = dbf_from_float<T>(v[e]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < COLS / 4; ++k) {
                const int at = 64 * k + lane, r = 16 * (MS * wm + j) + at / COLS, n = out0 + COLS * wn + at % COLS;
                const T v = mine[at / COLS * PITCH + at % COLS];
                if (r < tile.rows && n < a.n_out) static_cast<T*>(a.y)[(tile.row + r) * a.y_stride + n] = v;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (a.out_dtype == DBF_F16) one_by_one(_Float16());
    else if (a.out_dtype == DBF_BF16) one_by_one(dbf_bf16());
    else one_by_one(float());
}

template <int TYPE, bool FLOAT, bool GATED, bool EXACT, int BN, int BM, int WN, int WM, int EACH>
int launch(const DenseArgs& a, hipStream_t stream) {
    constexpr int OUTS = GATED ? BN / 2 : BN;
    const long long m_tiles = (a.n_rows + BM - 1LL) / BM + (a.starts ? std::min(a.n_groups, a.n_rows) : 0), n_tiles = (a.n_out + OUTS - 1) / OUTS;
    if (m_tiles * n_tiles > INT_MAX / 512) return DBF_EINVAL;
    hipLaunchKernelGGL((dbf_dense_tiles_kernel<TYPE, FLOAT, GATED, EXACT, BN, BM, WN, WM, EACH>), dim3((unsigned)(m_tiles * n_tiles)), dim3(64 * WN * WM), 0, stream, a, (int)n_tiles,
                       (int)m_tiles);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}
// What a launch costs, in us a step, by how many tiles it has: `full` where all places of the chip have one, `alone` for the first; from these times (us, rows by outputs, 4096 values in 8 bits):
//   256 x 256   64 x 4096 39    512 x 16384 49   1024 x 16384 60   2048 x 16384 118  2048 x 4096 51
//   128 x 128   64 x 4096 21    256 x 16384 32    512 x 16384 37   1024 x 16384 73   2048 x 16384 140   2048 x 4096 38
//   128 x 64    64 x 4096 16    256 x 16384 26    512 x 16384 49   512 x 4096 23     1024 x 4096 26     2048 x 4096 51
//   64 x 64     64 x 4096 14    256 x 16384 30    512 x 16384 66   512 x 4096 23     1024 x 4096 29     2048 x 4096 66
// Of a group's last tile half is taken to be empty (16384 rows of 32 experts, fp32 scales, gated, 366 us, with 128 x 128 455).
// They are 8 bits' with scales of a byte.  16 bits, fp32 scales and fp16 instructions cost more a step and go by the same, as the order of the four is much the same: 60 experts, 1000 x 2047 in bf16,
// 6126 rows 111 us by 128 x 64 for 109 by 128 x 128, 1800 rows 67 for 75.
double cost_of(const DenseArgs& a, int outs, int rows, int places, double alone, double full) {
    const double groups = a.starts ? std::min(a.n_groups, a.n_rows) : 1, each = a.n_rows / groups;
    const double m_tiles = groups * (a.starts ? std::max(1.0, each / rows + 0.5) : std::ceil(each / rows));
    const double tiles = m_tiles * ((a.n_out + outs - 1) / outs), rounds = std::floor(tiles / places), left = tiles / places - rounds;
    return rounds * full + (left > 0 ? alone + (full - alone) * left : 0);
}
template <int TYPE, bool FLOAT, bool GATED, bool EXACT>
int launch(const DenseArgs& a, hipStream_t stream) {
    constexpr int OF = GATED ? 2 : 1;
    const double large = EXACT ? 1e30 : cost_of(a, 256 / OF, 256, 256, 1.2, 1.85), square = cost_of(a, 128 / OF, 128, 512, 0.68, 1.15);
    const double low = cost_of(a, 128 / OF, 64, 768, 0.45, 1.13), small = cost_of(a, 64 / OF, 64, 1024, 0.43, 0.92);
    const double least = std::min({large, square, low, small});
    if constexpr (!EXACT)   // (in fp16 its operands have no registers)
        if (large <= least) return launch<TYPE, FLOAT, GATED, EXACT, 256, 256, 4, 2, 2>(a, stream);
    if (square <= least) return launch<TYPE, FLOAT, GATED, EXACT, 128, 128, 2, 2, EXACT ? 1 : 2>(a, stream);
    if (low <= least) return launch<TYPE, FLOAT, GATED, EXACT, 128, 64, 4, 1, 2>(a, stream);
    return launch<TYPE, FLOAT, GATED, EXACT, 64, 64, 2, 1, 2>(a, stream);
}
template <int TYPE, bool FLOAT, bool EXACT>
int launch(const DenseArgs& a, hipStream_t stream) {
    return a.w_up ? launch<TYPE, FLOAT, true, EXACT>(a, stream) : launch<TYPE, FLOAT, false, EXACT>(a, stream);
}

}  // namespace

int dbf_dense_tiles(const void* args, int type, bool float_scales, hipStream_t stream) {
    const DenseArgs& a = *static_cast<const DenseArgs*>(args);
    if (type == DBF_F16) return launch<DBF_F16, false, false>(a, stream);
    if (type == DBF_BF16) return launch<DBF_BF16, false, false>(a, stream);
    if (a.out_dtype == DBF_F32) return float_scales ? launch<DBF_E4M3, true, true>(a, stream) : launch<DBF_E4M3, false, true>(a, stream);
    return float_scales ? launch<DBF_E4M3, true, false>(a, stream) : launch<DBF_E4M3, false, false>(a, stream);
}
