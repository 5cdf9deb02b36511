// Products with ordinary weights, in 8 bits with a scale for each block of 128 or in 16 bits, of one matrix or of a matrix for each group of rows
// (include/dbf.h: dbf_dense_gemm, dbf_grouped_gemm).
//
// y^T = W x^T on the matrix cores: the weights are the operand of the result's rows, so that a lane has four neighbouring outputs of one row of y.  A step is 128 bytes of
// a row: in 8 bits one instruction over a block of 128 (exactly one scale of each operand, powers of two applied by the instruction; fp32 scales of weights on its
// result), in 16 bits two over 32 values each.  Of a step's eight 16-byte pieces lane group q = lane / 16 has pieces q and q + 4, of both operands: any order of k does.
#include "dbf_dense.h"

namespace {

// 16 outputs of 16 rows to a wavefront.
constexpr int ROWS = 16, WAVES = 4;
template <int TYPE, bool FLOAT, bool GATED>
__global__ __launch_bounds__(64 * WAVES) void dbf_dense_kernel(const DenseArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, q = lane >> 4;
    const int n0 = 16 * (WAVES * blockIdx.x + wave);
    for (int t = blockIdx.y;; t += gridDim.y) {
        const Tile tile = tile_of(a, t, ROWS);
        if (!tile.rows) return;
        if (n0 >= a.n_out) continue;
        const int row = tile.row + min(c, tile.rows - 1);
        int from = a.x_rows ? a.x_rows[row] : row;
        const bool known = (unsigned)from < (unsigned)a.n_x_rows;
        if (!known) from = 0;
        const uint8_t* x = a.x + from * a.x_row;
        const uint8_t* x_scale = a.x_scale + from * a.x_scale_row;
        const long long n = min(n0 + c, a.n_out - 1), block = tile.group * a.w_scale_group + (n0 / DBF_SCALE_BLOCK) * a.w_scale_row;
        const uint8_t* w = a.w + tile.group * a.w_group + n * a.w_row;
        const uint8_t* up = GATED ? a.w_up + tile.group * a.w_group + n * a.w_row : nullptr;
        auto scale = [&](const void* s, int b) -> int {
            return FLOAT ? static_cast<const int*>(s)[block + b] : static_cast<const uint8_t*>(s)[block + b];
        };
        dbf_f4 acc = {0.f, 0.f, 0.f, 0.f}, acc_up = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0, b = 0; k < a.k_bytes; k += STEP, ++b) {
            const int at0 = k + 16 * q, at1 = at0 + 64;
            const v8i xs = both(piece(x, at0, a.k_bytes), piece(x, at1, a.k_bytes)), ws = both(piece(w, at0, a.k_bytes), piece(w, at1, a.k_bytes));
            const int sx = TYPE == DBF_E4M3 ? x_scale[b] : 0;
            multiply<TYPE, FLOAT>(acc, ws, xs, TYPE == DBF_E4M3 ? scale(a.w_scale, b) : 0, sx);
            if constexpr (GATED) {
                const v8i us = both(piece(up, at0, a.k_bytes), piece(up, at1, a.k_bytes));
                multiply<TYPE, FLOAT>(acc_up, us, xs, TYPE == DBF_E4M3 ? scale(a.w_up_scale, b) : 0, sx);
            }
        }
        if constexpr (GATED)
            for (int i = 0; i < 4; ++i) acc[i] = gate(acc[i], acc_up[i]);
        if (!known) acc = (dbf_f4){0.f, 0.f, 0.f, 0.f};
        if (c < tile.rows && n0 + 4 * q < a.n_out) store4(a, tile.row + c, n0 + 4 * q, acc);
    }
}

template <int TYPE, bool FLOAT, bool GATED>
int launch(const DenseArgs& a, hipStream_t stream) {
    const long long tiles = (a.n_rows + ROWS - 1LL) / ROWS + (a.starts ? std::min(a.n_groups, a.n_rows) : 0);
    const dim3 grid((unsigned)((a.n_out + 16 * WAVES - 1) / (16 * WAVES)), (unsigned)std::min(tiles, 4096LL));
    hipLaunchKernelGGL((dbf_dense_kernel<TYPE, FLOAT, GATED>), grid, dim3(64 * WAVES), 0, stream, a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}
template <int TYPE, bool FLOAT>
int launch(const DenseArgs& a, hipStream_t stream) {
    return a.w_up ? launch<TYPE, FLOAT, true>(a, stream) : launch<TYPE, FLOAT, false>(a, stream);
}

constexpr long long MOST_STRIDE = 1 << 22;   // values of a row of x or weights: a tile's bytes have 32-bit offsets
constexpr long long MOST_GATHERED = 1LL << 32;   // bytes of x whose rows are given: the same

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
    if (p->x_rows && (p->n_x_rows * p->x_stride * (p->dtype == DBF_E4M3 ? 1 : 2) > MOST_GATHERED || p->n_x_rows * p->x_scale_stride > MOST_GATHERED)) return DBF_EINVAL;
    const int per = p->dtype == DBF_E4M3 ? 16 : 8, kb = (p->n_in + DBF_SCALE_BLOCK - 1) / DBF_SCALE_BLOCK;
    if (p->x_stride < p->n_in || p->x_stride % per || p->w_stride < p->n_in || p->w_stride % per || p->y_stride < p->n_out) return DBF_EINVAL;
    if (p->x_stride > MOST_STRIDE || p->w_stride > MOST_STRIDE || p->y_stride > (1LL << 32)) return DBF_EINVAL;
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
    if (a.n_rows > 16 * std::max(a.n_groups, 1)) return dbf_dense_tiles(&a, p->dtype, p->w_scale_type == DBF_F32, stream);
    if (p->dtype == DBF_F16) return launch<DBF_F16, false>(a, stream);
    if (p->dtype == DBF_BF16) return launch<DBF_BF16, false>(a, stream);
    return p->w_scale_type == DBF_F32 ? launch<DBF_E4M3, true>(a, stream) : launch<DBF_E4M3, false>(a, stream);
}

}  // namespace

extern "C" size_t dbf_dense_gemm_workspace_bytes(const dbf_dense*) { return 0; }
extern "C" size_t dbf_grouped_gemm_workspace_bytes(const dbf_dense*) { return 0; }

extern "C" int dbf_dense_gemm(const dbf_dense* product, void*, size_t, void* hip_stream) { return run(product, false, static_cast<hipStream_t>(hip_stream)); }
extern "C" int dbf_grouped_gemm(const dbf_dense* product, void*, size_t, void* hip_stream) { return run(product, true, static_cast<hipStream_t>(hip_stream)); }
