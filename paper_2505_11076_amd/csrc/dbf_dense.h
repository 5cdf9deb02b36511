// What the kernels of products with ordinary weights share: arguments, tiles of ragged groups, a step of a product, the output (device code and launch rules).
#ifndef DBF_DENSE_H
#define DBF_DENSE_H

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "dbf_cache.h"
#include "dbf_internal.h"
#include "dbf_wave.h"

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

constexpr int STEP = 128;   // bytes of a row to a step

struct DenseArgs {
    const uint8_t *x, *x_scale, *w, *w_up;
    const void *w_scale, *w_up_scale;
    const int32_t *x_rows, *starts;
    void* y;
    long long x_row, x_scale_row, w_row, w_group, w_scale_row, w_scale_group, y_stride;   // bytes; of the weights' scales: scales; of y: values
    int out_dtype, n_rows, n_x_rows, k_bytes, n_out, n_groups, quads;
};

// Which rows a tile has: tiles of a group's rows, group after group.
struct Tile {
    int group, row, rows;   // rows 0: there is no such tile
};
__device__ __forceinline__ Tile tile_of(const DenseArgs& a, int tile, int of_rows) {
    if (!a.starts) {
        const long long row = (long long)tile * of_rows;
        return {0, (int)row, (int)max(min((long long)of_rows, a.n_rows - row), 0LL)};
    }
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
        const int g = g0 + lane;
        int from = 0, to = 0;
        if (g < a.n_groups) {
            from = min(max(a.starts[g], 0), a.n_rows);
            to = min(max(a.starts[g + 1], 0), a.n_rows);
        }
        const int tiles = to > from ? (to - from - 1) / of_rows + 1 : 0;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(upto, d);
            if (lane >= d) upto += other;
        }
        const unsigned long long past = __ballot(before + upto > tile);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int row = __builtin_amdgcn_readlane(from, l) + (tile - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(tiles, l))) * of_rows;
            return {g0 + l, row, min(of_rows, __builtin_amdgcn_readlane(to, l) - row)};   // (scalars)
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return {0, 0, 0};
}

// How many tiles of groups there are.
__device__ __forceinline__ int tiles_of(const DenseArgs& a, int of_rows) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int g = lane; g < a.n_groups; g += 64) {
        const int from = min(max(a.starts[g], 0), a.n_rows), to = min(max(a.starts[g + 1], 0), a.n_rows);
        n += to > from ? (to - from - 1) / of_rows + 1 : 0;
    }
    return dbf_wave_sum(n);
}

// The 16 bytes of a row from byte `at` on, of which those from byte `end` of the row on are zeros.
__device__ __forceinline__ dbf_u4 piece(const uint8_t* row, int at, int end) {
    if (at >= end) return (dbf_u4){0, 0, 0, 0};
    dbf_u4 v = *reinterpret_cast<const dbf_u4*>(row + at);
    if (at + 16 > end) {
        const int have = end - at;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = have >= 4 * i + 4 ? v[i] : have <= 4 * i ? 0u : v[i] & (0xFFFFFFFFu >> (32 - 8 * (have - 4 * i)));
    }
    return v;
}

__device__ __forceinline__ v8i both(dbf_u4 a, dbf_u4 b) { return __builtin_bit_cast(v8i, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)); }
__device__ __forceinline__ dbf_u4 first(v8i v) { return __builtin_bit_cast(dbf_u4, __builtin_shufflevector(v, v, 0, 1, 2, 3)); }
__device__ __forceinline__ dbf_u4 second(v8i v) { return __builtin_bit_cast(dbf_u4, __builtin_shufflevector(v, v, 4, 5, 6, 7)); }

// acc += w x over a step.  TYPE: DBF_E4M3, DBF_F16 or DBF_BF16; FLOAT: weights' scales are fp32 numbers.
template <int TYPE, bool FLOAT>
__device__ __forceinline__ void multiply(dbf_f4& acc, const v8i& w, const v8i& x, int w_scale, int x_scale) {
    if constexpr (TYPE == DBF_E4M3) {
        if constexpr (FLOAT) {
            const dbf_f4 none = {0.f, 0.f, 0.f, 0.f};
            // The number's power of two is the instruction's, beside the rows' scale, so that neither alone takes the sum out of fp32's range; what is left of it, 1 .. 2, comes
            // on the sum.  (0, and subnormal numbers as 0: no power; infinities and no numbers: 255, no number)
            const int power = w_scale >> 23 & 255;
            const dbf_f4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, none, 0, 0, 0, power, 0, x_scale);
            const float s = __builtin_bit_cast(float, power ? (w_scale & 0x807FFFFF) | 0x3F800000 : 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = fmaf(s, p[i], acc[i]);
        } else {
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, 0, 0, 0, w_scale, 0, x_scale);
        }
    } else if constexpr (TYPE == DBF_F16) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(dbf_h8, first(w)), __builtin_bit_cast(dbf_h8, first(x)), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(dbf_h8, second(w)), __builtin_bit_cast(dbf_h8, second(x)), acc, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, first(w)), __builtin_bit_cast(v8b, first(x)), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, second(w)), __builtin_bit_cast(v8b, second(x)), acc, 0, 0, 0);
    }
}

// The number that a byte of a scale stands for (255: no number; 0: 2^-127, a subnormal number).
__device__ __forceinline__ float scale_of(int byte) {
    return __builtin_bit_cast(float, byte == 255 ? 0x7FC00000u : byte ? (unsigned)byte << 23 : 0x00400000u);
}
// The same of values in 8 bits where the result is to have 32: of each of sixteen neighbouring products the instructions for 8 bits cut off, towards zero, what lies below 2^-13 of the
// largest, so a sum is off by 16 * 2^-13 of the largest of each sixteen at most, relative to its terms and not to itself (of random values of one size it measures 1.5e-5 of the results'
// size, 6e-5 where they span 2^12: a tenth and a third of what rounding to fp16 costs); in fp16 the values are exact, and so are the products.  For results of 16 bits it is not taken, so that a
// row has the same precision among few and among many: beside weights from memory it would cost 0 to 9 % (us, 8-bit instructions / these: 13 rows of 128256 x 4096 with fp32 scales 82.5 / 84.2, 16 of
// 32064 x 4096 25.2 / 26.4, 64 of 4096 x 4096 14.3 / 15.7, one of 16384 x 4096 14.1 / 15.4), but where there are many rows the matrix cores do a third as much (2047 rows of 11008 x 4096: 310
// us; with 8-bit instructions 180 for two such matrices).
template <bool FLOAT>
__device__ __forceinline__ void multiply_exactly(dbf_f4& acc, v8i w, v8i x, int w_scale, int x_scale) {
    auto widen = [](v8i v, int k) -> dbf_h8 {   // codes 8 k .. 8 k + 7
        typedef _Float16 v2h __attribute__((ext_vector_type(2)));
        const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[2 * k], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[2 * k], 1.f, true);
        const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[2 * k + 1], 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[2 * k + 1], 1.f, true);
        return (dbf_h8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    };
    dbf_f4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(w, k), widen(x, k), p, 0, 0, 0);
    // Sums are multiples of 2^-18, so that each times the first factor, a power of two, is exact, and what rounds is the addition alone.
    float a, b;
    if constexpr (FLOAT) {
        // The power of two of a number goes together with the row's, and half of both comes on the sum first: neither alone takes it out of fp32's range where the result does not leave
        // it (with all of a number below 2^-126, or of a sum of small codes by one near it, first, digits were lost that the row's scale brings back into range)
        const float number = __builtin_bit_cast(float, w_scale);
        const int power = __builtin_amdgcn_frexp_expf(number) + x_scale - 127, half = power >> 1;
        a = x_scale == 255 ? scale_of(255) : __builtin_ldexpf(1.f, half);
        b = __builtin_ldexpf(__builtin_amdgcn_frexp_mantf(number), power - half);
    } else {
        // (the smaller one first: the other way round a sum of 2^25 leaves fp32's range where the result does not; 2^-127 of a sum is exact)
        const float by = scale_of(w_scale), of_row = scale_of(x_scale);
        const bool first = by < of_row;   // (not a minimum: no number has to stay one)
        a = first ? by : of_row, b = first ? of_row : by;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e] * a, b, acc[e]);
}

__device__ __forceinline__ float gate(float g, float up) { return g / (1.f + expf(-g)) * up; }

// Four neighbouring outputs of a row, from column n on.
template <typename T>
__device__ __forceinline__ void store4_as(T* at, const dbf_f4& v, int have, bool whole) {
    T out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = dbf_from_float<T>(v[i]);
    if (whole && have >= 4) {
        typedef std::conditional_t<sizeof(T) == 4, dbf_u4, dbf_u2> Words;
        Words w;
        __builtin_memcpy(&w, out, sizeof(w));
        *reinterpret_cast<Words*>(at) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) at[i] = out[i];
    }
}
__device__ __forceinline__ void store4(const DenseArgs& a, int row, int n, const dbf_f4& v) {
    const long long at = row * a.y_stride + n;
    const int have = a.n_out - n;
    if (a.out_dtype == DBF_F16) store4_as(static_cast<_Float16*>(a.y) + at, v, have, a.quads);
    else if (a.out_dtype == DBF_BF16) store4_as(static_cast<dbf_bf16*>(a.y) + at, v, have, a.quads);
    else store4_as(static_cast<float*>(a.y) + at, v, have, a.quads);
}

}  // namespace

// What launches them: `args` is a DenseArgs, `type` that of the operands.
int dbf_dense_tiles(const void* args, int type, bool float_scales, hipStream_t stream);
int dbf_dense_stream(const void* args, int type, bool float_scales, hipStream_t stream);
bool dbf_dense_streams(int k_bytes);   // whether rows of so many bytes fit the latter

#endif  // DBF_DENSE_H
