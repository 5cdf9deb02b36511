// Rounding to 8 bits with a scale for each block of 128 values (include/dbf.h: dbf_quantize).
//
// A block's scale is the smallest power of two that brings its largest value to 448 or less, so a value over its scale is exact in fp32 and the conversion to the
// type is its only rounding: codes do not hang on how a quotient is made.
// Bound by memory where there is much (8191 rows of 11008 bf16: 271 MB in 47.4 us, 5.7 TB/s beside the 5.1 of a copy) and by the launch where there is little (7 rows of 4096 in
// 2.8 us).  Eight lanes have a block, so that its largest value takes three moves between lanes and no memory; a lane's sixteen values are loads and a store of 16 bytes, and x is
// read once.  A square of 128 x 128 stays in registers between its largest value and its codes (four turns
// of 256 lanes), for the same reason.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "dbf_cache.h"
#include "dbf_internal.h"

namespace {

constexpr int THREADS = 256, BLOCK = DBF_SCALE_BLOCK, OF_LANE = 16, LANES = BLOCK / OF_LANE;

// The byte of the scale of a block whose largest value has these bits (fp32, sign off, finite): 448 is 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(unsigned most) {
    if (!most) return 127;
    return max((int)(most >> 23) - 8 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0), 0);
}

// Sixteen values from column `at` on of a row of n_cols, zeros behind its end; their largest magnitude's bits.
template <typename T>
__device__ __forceinline__ unsigned load_values(const T* row, int at, int n_cols, float (&v)[OF_LANE]) {
    if (at + OF_LANE <= n_cols) {
        constexpr int PER = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < OF_LANE / PER; ++i) {
            const dbf_u4 w = *reinterpret_cast<const dbf_u4_any*>(row + at + PER * i);
            T e[PER];
            __builtin_memcpy(e, &w, 16);
#pragma unroll
            for (int j = 0; j < PER; ++j) v[PER * i + j] = dbf_to_float(e[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < OF_LANE; ++i) v[i] = at + i < n_cols ? dbf_to_float(row[at + i]) : 0.f;
    }
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < OF_LANE; ++i) most = max(most, __builtin_bit_cast(unsigned, v[i]) & 0x7FFFFFFFu);
    return most;
}

// The codes of sixteen values, which go where they belong in their row; its last sixteen may be fewer, and are filled up with zeros.
__device__ __forceinline__ void store_codes(const float (&v)[OF_LANE], unsigned most, int byte, uint8_t* to, int have) {
    const float up = __builtin_bit_cast(float, (unsigned)(254 - byte) << 23);   // 2^(127 - byte)
    dbf_u4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * up, v[4 * i + 1] * up, 0, false);
        w[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * up, v[4 * i + 3] * up, p, true);
    }
    if (most >= 0x7F800000u) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = have >= 4 * i + 4 ? 0x7F7F7F7Fu : have <= 4 * i ? 0u : 0x7F7F7F7Fu >> (32 - 8 * (have - 4 * i));
    }
    *reinterpret_cast<dbf_u4*>(to) = w;
}

__device__ __forceinline__ unsigned lanes8_max(unsigned v) {
    auto move = [](unsigned x, auto ctrl) { return (unsigned)__builtin_amdgcn_update_dpp((int)x, (int)x, decltype(ctrl)::value, 0xF, 0xF, false); };
    v = max(v, move(v, std::integral_constant<int, 0xB1>()));    // quad_perm [1,0,3,2]
    v = max(v, move(v, std::integral_constant<int, 0x4E>()));    // quad_perm [2,3,0,1]
    return max(v, move(v, std::integral_constant<int, 0x141>()));   // row_half_mirror
}

struct QuantizeArgs {
    const void* x;
    uint8_t *codes, *scales;
    long long x_stride, codes_stride, scales_stride;
    int n_rows, n_cols;
};

// Blocks of 128 values of a row, eight lanes each.
template <typename T>
__global__ __launch_bounds__(THREADS) void dbf_fp8_rows_kernel(const QuantizeArgs a) {
    const int kb = (a.n_cols + BLOCK - 1) / BLOCK, lane = threadIdx.x & (LANES - 1);
    const long long n = (long long)a.n_rows * kb, step = (long long)gridDim.x * (THREADS / LANES);
    for (long long i = (long long)blockIdx.x * (THREADS / LANES) + threadIdx.x / LANES; i < n; i += step) {
        const int row = (int)(i / kb), b = (int)(i - (long long)row * kb), at = b * BLOCK + OF_LANE * lane;
        float v[OF_LANE];
        const unsigned most = lanes8_max(load_values(static_cast<const T*>(a.x) + row * a.x_stride, at, a.n_cols, v));
        const int byte = most >= 0x7F800000u ? 127 : scale_byte(most);
        if (at < a.n_cols) store_codes(v, most, byte, a.codes + row * a.codes_stride + at, a.n_cols - at);
        if (lane == 0) a.scales[row * a.scales_stride + b] = (uint8_t)byte;
    }
}

// Blocks of 128 rows, a workgroup each.
template <typename T>
__global__ __launch_bounds__(THREADS) void dbf_fp8_squares_kernel(const QuantizeArgs a) {
    __shared__ unsigned all[THREADS / LANES];
    constexpr int TURNS = BLOCK * LANES / THREADS;
    const int kb = (a.n_cols + BLOCK - 1) / BLOCK, lane = threadIdx.x & (LANES - 1), line = threadIdx.x / LANES;
    const long long n = (long long)((a.n_rows - 1) / BLOCK + 1) * kb;
    for (long long i = blockIdx.x; i < n; i += gridDim.x) {
        const int rb = (int)(i / kb), b = (int)(i - (long long)rb * kb), at = b * BLOCK + OF_LANE * lane;
        float v[TURNS][OF_LANE];
        unsigned most = 0;
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const long long row = (long long)rb * BLOCK + t * (THREADS / LANES) + line;
            if (row < a.n_rows) most = max(most, load_values(static_cast<const T*>(a.x) + row * a.x_stride, at, a.n_cols, v[t]));
        }
        most = lanes8_max(most);
        __syncthreads();   // (the block before has been read)
        if (lane == 0) all[line] = most;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < THREADS / LANES; ++j) most = max(most, all[j]);
        const int byte = most >= 0x7F800000u ? 127 : scale_byte(most);
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const long long row = (long long)rb * BLOCK + t * (THREADS / LANES) + line;
            if (row < a.n_rows && at < a.n_cols) store_codes(v[t], most, byte, a.codes + row * a.codes_stride + at, a.n_cols - at);
        }
        if (threadIdx.x == 0) a.scales[rb * a.scales_stride + b] = (uint8_t)byte;
    }
}

template <typename T>
int launch(const QuantizeArgs& a, int block_rows, hipStream_t stream) {
    const long long kb = (a.n_cols + BLOCK - 1) / BLOCK;
    const long long of_rows = block_rows == 1 ? ((long long)a.n_rows * kb + THREADS / LANES - 1) / (THREADS / LANES) : ((a.n_rows - 1) / BLOCK + 1) * kb;
    const dim3 grid((unsigned)std::min(of_rows, 1LL << 22)), threads(THREADS);
    if (block_rows == 1) hipLaunchKernelGGL(dbf_fp8_rows_kernel<T>, grid, threads, 0, stream, a);
    else hipLaunchKernelGGL(dbf_fp8_squares_kernel<T>, grid, threads, 0, stream, a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}

}  // namespace

extern "C" int dbf_quantize(const void* x, int dtype, long long x_stride, int n_rows, int n_cols, int block_rows, void* codes, long long codes_stride,
                                void* scales, long long scales_stride, void* hip_stream) {
    if (!x || !codes || !scales || (dtype != DBF_F16 && dtype != DBF_BF16 && dtype != DBF_F32)) return DBF_EINVAL;
    if (n_cols < 1 || n_cols > DBF_MAX_DIM) return DBF_ESHAPE;
    if (n_rows < 0 || (block_rows != 1 && block_rows != BLOCK)) return DBF_EINVAL;
    if (x_stride < n_cols || codes_stride < n_cols || codes_stride % 16 || scales_stride < (n_cols + BLOCK - 1) / BLOCK) return DBF_EINVAL;
    if (dbf_misaligned(x, dtype == DBF_F32 ? 4 : 2) || dbf_misaligned(codes, 16)) return DBF_EINVAL;
    if (!n_rows) return DBF_OK;
    const QuantizeArgs a = {x, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), x_stride, codes_stride, scales_stride, n_rows, n_cols};
    const auto stream = static_cast<hipStream_t>(hip_stream);
    return dtype == DBF_F16 ? launch<_Float16>(a, block_rows, stream) : dtype == DBF_BF16 ? launch<dbf_bf16>(a, block_rows, stream) : launch<float>(a, block_rows, stream);
}
