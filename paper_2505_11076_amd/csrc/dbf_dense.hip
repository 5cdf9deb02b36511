// Products with ordinary weights, in 8 bits with a scale for each block of 128 or in 16 bits, of one matrix or of a matrix for each group of rows
// (include/dbf.h: dbf_dense_gemm, dbf_grouped_gemm).
//
// y^T = W x^T on the matrix cores: the weights are the operand of the result's rows, so that a lane has four neighbouring outputs of one row of y.  A step is 128 bytes of
// a row: in 8 bits one instruction over a block of 128 (exactly one scale of each operand, powers of two applied by the instruction; fp32 scales of weights on its
// result), in 16 bits two over 32 values each.  Of a step's eight 16-byte pieces lane group q = lane / 16 has pieces q and q + 4, of both operands: any order of k does.
#include "dbf_dense.h"

namespace {

// Few rows: a workgroup has 16 NS weights (gated: of each matrix) and 16 MS rows; its wavefronts have every KW-th four steps of them, and their sums meet in LDS.  Operands come
// straight from memory as the matrix cores take them: of four steps 512 bytes of a row, four steps' loads under way at a time.
// Bound by latencies: of a row through 4096 x 4096 in 8 bits (16.8 MB: 2.4 us at a bare read's rate) 5.6 us, where the rounding of 7 rows
// to 8 bits, a launch with next to nothing to do, takes 2.8;
// eight share the 32 steps of a workgroup's 16 weights, so that each waits for memory once.  Through LDS there is nothing to gain: no operand is used twice.
constexpr int GROUP = 4;   // steps
template <int TYPE, bool FLOAT, bool GATED, bool EXACT, int NS, int MS, int KW>
__global__ __launch_bounds__(64 * KW) void dbf_dense_few_kernel(const DenseArgs a) {
    constexpr int ROWS = 16 * MS, N = GATED ? 2 * NS : NS;   // N: sets of 16 weights
    __shared__ dbf_f4 sums[KW > 1 ? KW - 1 : 1][N * MS][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, q = lane >> 4;
    const int out0 = 16 * NS * blockIdx.x;
    for (int t = blockIdx.y;; t += gridDim.y) {
        const Tile tile = tile_of(a, t, ROWS);
        if (!tile.rows) return;
        const uint8_t *x[MS], *x_scale[MS], *w[N];
        const uint8_t* w_scale[N];
#pragma unroll
        for (int j = 0; j < MS; ++j) {
            const int row = tile.row + min(16 * j + c, tile.rows - 1);
            int from = a.x_rows ? a.x_rows[row] : row;
            if ((unsigned)from >= (unsigned)a.n_x_rows) from = 0;
            x[j] = a.x + from * a.x_row;
            x_scale[j] = a.x_scale + from * a.x_scale_row;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int n0 = out0 + 16 * (GATED ? i / 2 : i);
            const bool up = GATED && i % 2;
            w[i] = (up ? a.w_up : a.w) + tile.group * a.w_group + min(n0 + c, a.n_out - 1) * a.w_row;
            const long long block = tile.group * a.w_scale_group + (min(n0, a.n_out - 1) / DBF_SCALE_BLOCK) * a.w_scale_row;
            w_scale[i] = static_cast<const uint8_t*>(up ? a.w_up_scale : a.w_scale) + block * (FLOAT ? 4 : 1);
        }
        dbf_f4 acc[N][MS];
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < MS; ++j) acc[i][j] = (dbf_f4){0.f, 0.f, 0.f, 0.f};
        // (scales as they lie: bytes, or fp32 numbers' bits)
        auto products = [&](const v8i (&ws)[N], const v8i (&xs)[MS], const int (&scale_w)[N], const int (&scale_x)[MS]) {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < MS; ++j) {
                    if constexpr (EXACT) multiply_exactly<FLOAT>(acc[i][j], ws[i], xs[j], scale_w[i], scale_x[j]);
                    else multiply<TYPE, FLOAT>(acc[i][j], ws[i], xs[j], scale_w[i], scale_x[j]);
                }
        };
        auto weight_scale = [&](int i, int s) -> int {
            if constexpr (TYPE != DBF_E4M3) return 0;
            return FLOAT ? reinterpret_cast<const int*>(w_scale[i])[s] : w_scale[i][s];
        };
        const int steps = a.k_bytes / STEP;
        int s = GROUP * wave;
        for (; s + GROUP <= steps; s += GROUP * KW) {
            v8i ws[GROUP][N], xs[GROUP][MS];
            int scale_w[GROUP][N];
            unsigned word[MS];
#pragma unroll
            for (int g = 0; g < GROUP; ++g) {
                const int at = (s + g) * STEP + 16 * q;
#pragma unroll
                for (int i = 0; i < N; ++i) ws[g][i] = both(*reinterpret_cast<const dbf_u4*>(w[i] + at), *reinterpret_cast<const dbf_u4*>(w[i] + at + 64));
#pragma unroll
                for (int j = 0; j < MS; ++j) xs[g][j] = both(*reinterpret_cast<const dbf_u4*>(x[j] + at), *reinterpret_cast<const dbf_u4*>(x[j] + at + 64));
#pragma unroll
                for (int i = 0; i < N; ++i) scale_w[g][i] = weight_scale(i, s + g);
            }
            if constexpr (TYPE == DBF_E4M3) {
#pragma unroll
                for (int j = 0; j < MS; ++j) word[j] = *reinterpret_cast<const unsigned*>(x_scale[j] + s);
            }
#pragma unroll
            for (int g = 0; g < GROUP; ++g) {
                int scale_x[MS];
#pragma unroll
                for (int j = 0; j < MS; ++j) scale_x[j] = TYPE == DBF_E4M3 ? word[j] >> (8 * g) & 255 : 0;
                products(ws[g], xs[g], scale_w[g], scale_x);
            }
        }
        // what is left of the wavefront's last four steps
        for (int g = 0; g < GROUP && (s + g) * STEP < a.k_bytes; ++g) {
            const int at = (s + g) * STEP + 16 * q;
            v8i ws[N], xs[MS];
            int scale_w[N], scale_x[MS];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ws[i] = both(piece(w[i], at, a.k_bytes), piece(w[i], at + 64, a.k_bytes));
                scale_w[i] = weight_scale(i, s + g);
            }
#pragma unroll
            for (int j = 0; j < MS; ++j) {
                xs[j] = both(piece(x[j], at, a.k_bytes), piece(x[j], at + 64, a.k_bytes));
                scale_x[j] = TYPE == DBF_E4M3 ? x_scale[j][s + g] : 0;
            }
            products(ws, xs, scale_w, scale_x);
        }
        if (KW > 1) {
            if (wave) {
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int j = 0; j < MS; ++j) sums[wave - 1][i * MS + j][lane] = acc[i][j];
            }
            __syncthreads();
            if (!wave) {
#pragma unroll
                for (int k = 0; k < KW - 1; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int j = 0; j < MS; ++j) acc[i][j] += sums[k][i * MS + j][lane];
            }
        }
        if (!wave) {
#pragma unroll
            for (int j = 0; j < MS; ++j) {
                const int r = 16 * j + c, row = tile.row + r;
                if (r >= tile.rows) continue;
                const bool known = !a.x_rows || (unsigned)a.x_rows[row] < (unsigned)a.n_x_rows;
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    const int n = out0 + 16 * i + 4 * q;
                    dbf_f4 v = acc[GATED ? 2 * i : i][j];
                    if constexpr (GATED) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = gate(v[e], acc[2 * i + 1][j][e]);
                    }
                    if (!known) v = (dbf_f4){0.f, 0.f, 0.f, 0.f};
                    if (n < a.n_out) store4(a, row, n, v);
                }
            }
        }
        if (KW > 1) __syncthreads();   // (the sums have been read)
    }
}

template <int TYPE, bool FLOAT, bool GATED, bool EXACT, int NS, int MS, int KW>
int launch(const DenseArgs& a, hipStream_t stream) {
    const long long tiles = (a.n_rows + 16LL * MS - 1) / (16 * MS) + (a.starts ? std::min(a.n_groups, a.n_rows) : 0);
    const long long outs = (a.n_out + 16 * NS - 1) / (16 * NS);
    // (a grid holds less than 2^32 threads; tiles that it has no workgroup for are taken in turn)
    const dim3 grid((unsigned)outs, (unsigned)std::min({tiles, 4096LL, (1LL << 31) / (outs * 64 * KW)}));
    hipLaunchKernelGGL((dbf_dense_few_kernel<TYPE, FLOAT, GATED, EXACT, NS, MS, KW>), grid, dim3(64 * KW), 0, stream, a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}
template <int TYPE, bool FLOAT, bool GATED, bool EXACT>
int launch(const DenseArgs& a, hipStream_t stream) {
    const long long each = a.starts ? (a.n_rows + a.n_groups - 1) / a.n_groups : a.n_rows;
    const long long units = (a.n_out + 15) / 16 * (a.starts ? std::min(a.n_groups, a.n_rows) : 1);   // of 16 outputs
    if (each > 16) return launch<TYPE, FLOAT, GATED, EXACT, 1, 2, 4>(a, stream);
    if (units >= 2048) return launch<TYPE, FLOAT, GATED, EXACT, GATED ? 1 : 2, 1, 4>(a, stream);
    return launch<TYPE, FLOAT, GATED, EXACT, 1, 1, 8>(a, stream);
}
template <int TYPE, bool FLOAT, bool GATED>
int launch(const DenseArgs& a, hipStream_t stream) {
    if constexpr (TYPE == DBF_E4M3)
        if (a.out_dtype == DBF_F32) return launch<TYPE, FLOAT, GATED, true>(a, stream);
    return launch<TYPE, FLOAT, GATED, false>(a, stream);
}
template <int TYPE, bool FLOAT>
int launch(const DenseArgs& a, hipStream_t stream) {
    return a.w_up ? launch<TYPE, FLOAT, true>(a, stream) : launch<TYPE, FLOAT, false>(a, stream);
}

constexpr long long MOST_STRIDE = 1 << 22;   // values of a row of x, weights or x's scales: a tile's bytes have 32-bit offsets
constexpr long long MOST_GATHERED = 1LL << 32;   // bytes of x whose rows are given, or of its scales: the same

bool types_ok(const dbf_dense* p) {
    if (p->dtype != DBF_E4M3 && p->dtype != DBF_F16 && p->dtype != DBF_BF16) return false;
    if (p->out_dtype != DBF_F16 && p->out_dtype != DBF_BF16 && p->out_dtype != DBF_F32) return false;
    return p->dtype != DBF_E4M3 || p->w_scale_type == DBF_E8M0 || p->w_scale_type == DBF_F32;
}

// DBF_OK, or what is wrong with a product; the workspaces' sizes need no pointers
int check(const dbf_dense* p, bool grouped) {
    if (!p || !p->x || !p->w || !p->y || !types_ok(p)) return DBF_EINVAL;
    if (p->n_in < 1 || p->n_in > DBF_MAX_DIM || p->n_out < 1 || p->n_out > DBF_MAX_DIM) return DBF_ESHAPE;
    if (p->n_rows < 0 || p->n_x_rows < 0 || (!p->x_rows && p->n_x_rows < p->n_rows) || (p->n_rows && !p->n_x_rows)) return DBF_EINVAL;
    if (grouped ? !p->starts || p->n_groups < 1 || p->n_groups > DBF_MAX_GROUPS : p->starts || p->n_groups) return DBF_EINVAL;
    const int per = p->dtype == DBF_E4M3 ? 16 : 8, kb = (p->n_in + DBF_SCALE_BLOCK - 1) / DBF_SCALE_BLOCK;
    if (p->x_stride < p->n_in || p->x_stride % per || p->w_stride < p->n_in || p->w_stride % per || p->y_stride < p->n_out) return DBF_EINVAL;
    if (p->x_stride > MOST_STRIDE || p->w_stride > MOST_STRIDE || p->x_scale_stride > MOST_STRIDE || p->y_stride > (1LL << 32)) return DBF_EINVAL;
    if (p->x_rows && (p->n_x_rows * p->x_stride * (p->dtype == DBF_E4M3 ? 1 : 2) > MOST_GATHERED || p->n_x_rows * p->x_scale_stride > MOST_GATHERED)) return DBF_EINVAL;
    if (grouped && (p->w_group_stride < 0 || p->w_group_stride % per)) return DBF_EINVAL;
    if (dbf_misaligned(p->x, 16) || dbf_misaligned(p->w, 16) || dbf_misaligned(p->w_up, 16) || dbf_misaligned(p->x_rows, 4) || dbf_misaligned(p->starts, 4)) return DBF_EINVAL;
    if (dbf_misaligned(p->y, p->out_dtype == DBF_F32 ? 4 : 2)) return DBF_EINVAL;
    if (p->dtype != DBF_E4M3) return p->x_scale || p->w_scale || p->w_up_scale ? DBF_EINVAL : DBF_OK;
    if (!p->x_scale || !p->w_scale || !p->w_up_scale != !p->w_up) return DBF_EINVAL;
    if (dbf_misaligned(p->x_scale, 4) || p->x_scale_stride % 4 || p->x_scale_stride < kb) return DBF_EINVAL;
    if (p->w_scale_stride < kb || (grouped && p->w_scale_group_stride < 0)) return DBF_EINVAL;
    if (p->w_scale_type == DBF_F32 && (dbf_misaligned(p->w_scale, 4) || dbf_misaligned(p->w_up_scale, 4))) return DBF_EINVAL;
    return DBF_OK;
}

// Whether rows, `each` to a matrix, are few enough that operands come straight from memory, and not by tiles.  Of few rows tiles are few too and walk the long axis one step behind the other,
// half a microsecond each and more the more there are, where eight wavefronts share it here; but here each 32 rows read the weights again, at 2.8 TB/s.  us, few rows for tiles, weights that no cache holds:
//   4096 x 4096, 8 bits     24 rows 9.6 / 10.0   64 rows 15.3 / 24.1   128 rows 27.1 / 23.9        4096 x 16384, 8 bits    24 rows 24.4 / 23.7   64 rows 50.0 / 25.9
//   11008 x 4096, 8 bits    24 rows 17.0 / 53.6  64 rows 32.6 / 55.9   128 rows 61.7 / 56.3        11008 x 4096, bf16      24 rows 35 / 118      96 rows 94 / 118
//   8192 x 8192, bf16       24 rows 48 / 93      64 rows 96 / 96                                   28672 x 8192, 8 bits    24 rows 79 / 182      64 rows 170 / 192
// (to fp32 from 8 bits, by instructions for fp16, tiles take half as long again: 8192 x 8192, 64 rows 52 / 66)
bool few_rows(const DenseArgs& a, long long each, double weights, bool eight_bits) {
    if (each <= (a.starts ? 4 : 16) || (each <= 32 && weights <= (32 << 20))) return true;
    const double steps = a.k_bytes / (double)STEP, tiles = (double)(a.starts ? std::min(a.n_groups, a.n_rows) : 1) * ((a.n_out + 63) / 64) * (a.w_up ? 2 : 1);
    const double by_tiles = 5 + steps * (0.5 + tiles / 1024) * (eight_bits && a.out_dtype == DBF_F32 ? 1.5 : 1), straight = 2.5 + (each + 31) / 32 * weights / 2.8e6;
    return each <= 128 && straight < by_tiles;
}

int run(const dbf_dense* p, bool grouped, hipStream_t stream) {
    const int wrong = check(p, grouped);
    if (wrong != DBF_OK) return wrong;
    if (!p->n_rows) return DBF_OK;
    const int size = p->dtype == DBF_E4M3 ? 1 : 2, quad = p->out_dtype == DBF_F32 ? 16 : 8;
    DenseArgs a = {};
    a.x = static_cast<const uint8_t*>(p->x);
    a.x_scale = static_cast<const uint8_t*>(p->x_scale);
    a.w = static_cast<const uint8_t*>(p->w);
    a.w_up = static_cast<const uint8_t*>(p->w_up);
    a.w_scale = p->w_scale;
    a.w_up_scale = p->w_up_scale;
    a.x_rows = p->x_rows;
    a.starts = p->starts;
    a.y = p->y;
    a.x_row = p->x_stride * size;
    a.x_scale_row = p->x_scale_stride;
    a.w_row = p->w_stride * size;
    a.w_group = grouped ? p->w_group_stride * size : 0;
    a.w_scale_row = p->w_scale_stride;
    a.w_scale_group = grouped ? p->w_scale_group_stride : 0;
    a.y_stride = p->y_stride;
    a.out_dtype = p->out_dtype;
    a.n_rows = p->n_rows;
    a.n_x_rows = p->n_x_rows;
    a.k_bytes = p->n_in * size;
    a.n_out = p->n_out;
    a.n_groups = grouped ? p->n_groups : 0;
    a.quads = p->y_stride % 4 == 0 && !dbf_misaligned(p->y, quad);
    const bool fp32_scales = p->w_scale_type == DBF_F32;
    const double weights = (double)std::min(std::max(a.n_groups, 1), a.n_rows) * a.n_out * a.k_bytes * (a.w_up ? 2 : 1);
    // (us, 8 bits)  Weights that no cache holds stream past few rows: 4 rows, 64 MB 15.4 for 17.1 by the kernel for few rows, 134 MB 25 for 33, but 32 MB 10.1 for 10.0.  Of groups with 4 rows on
    // average some have more than 16, whose weights are read twice: 268 MB of 64 groups with 4 rows each 44.2 for 43.8 by tiles, with 8 49 for 45, with 1 26.5 for 28 (147 MB).
    const long long each = a.starts ? (a.n_rows + a.n_groups - 1LL) / a.n_groups : a.n_rows;
    if (each <= (a.starts ? 4 : 16) && weights >= (64 << 20) && dbf_dense_streams(a.k_bytes)) return dbf_dense_stream(&a, p->dtype, fp32_scales, stream);
    if (!few_rows(a, each, weights, p->dtype == DBF_E4M3)) return dbf_dense_tiles(&a, p->dtype, fp32_scales, stream);
    if (p->dtype == DBF_F16) return launch<DBF_F16, false>(a, stream);
    if (p->dtype == DBF_BF16) return launch<DBF_BF16, false>(a, stream);
    return fp32_scales ? launch<DBF_E4M3, true>(a, stream) : launch<DBF_E4M3, false>(a, stream);
}

}  // namespace

extern "C" size_t dbf_dense_gemm_workspace_bytes(const dbf_dense*) { return 0; }
extern "C" size_t dbf_grouped_gemm_workspace_bytes(const dbf_dense*) { return 0; }

extern "C" int dbf_dense_gemm(const dbf_dense* product, void*, size_t, void* hip_stream) { return run(product, false, static_cast<hipStream_t>(hip_stream)); }
extern "C" int dbf_grouped_gemm(const dbf_dense* product, void*, size_t, void* hip_stream) { return run(product, true, static_cast<hipStream_t>(hip_stream)); }
