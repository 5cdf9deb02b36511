// A router's choice of experts, the order of rows by experts, and the sum that brings rows back to their tokens (include/dbf.h: dbf_route, dbf_combine).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "dbf_cache.h"
#include "dbf_internal.h"
#include "dbf_wave.h"

namespace {

typedef unsigned long long u64;

// ---- the choice ------------------------------------------------------------------------------------------------

constexpr int THREADS = 1024, CHOOSERS = 512, CHUNK = 32, MOST_TOP = 32;   // CHUNK: tokens of a workgroup; a bit of a word for each
constexpr int MOST_TOKENS = CHUNK * ((1 << 22) - 1);   // of 2^32 threads or more only the remainder would run: chunks of THREADS
constexpr int MOST_CHUNKS = 256;   // whose counts every workgroup of the second launch adds up itself; from more a launch between makes sums

struct RouteArgs {
    const void* logits;
    const float* bias;
    long long stride;
    int32_t* ids;
    float* weights;
    int32_t *starts, *row_token, *token_rows;
    uint8_t* counts;    // [chunks][padded]: tokens of a chunk that chose an expert
    int32_t* before;    // [chunks + 1][padded]: those of the chunks before; NULL: not made
    int n_tokens, n_experts, n_top, padded, renormalise;
    float scale;
};

template <int CTRL>
__device__ __forceinline__ u64 move64(u64 v) {
    const unsigned lo = (unsigned)dbf_dpp_move<CTRL>((int)(unsigned)v), hi = (unsigned)dbf_dpp_move<CTRL>((int)(unsigned)(v >> 32));
    return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 lane64(u64 v, int lane) {
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, lane);
}
// Of the L lanes (16 or 64) of a token, the same in all of them.
template <int L>
__device__ __forceinline__ u64 most_of(u64 v) {
    v = max(v, move64<0xB1>(v));
    v = max(v, move64<0x4E>(v));
    v = max(v, move64<0x124>(v));
    v = max(v, move64<0x128>(v));
    return L == 16 ? v : max(max(lane64(v, 0), lane64(v, 16)), max(lane64(v, 32), lane64(v, 48)));
}
template <int L>
__device__ __forceinline__ unsigned most_of(unsigned v) {
    v = max(v, (unsigned)dbf_dpp_move<0xB1>((int)v));
    v = max(v, (unsigned)dbf_dpp_move<0x4E>((int)v));
    v = max(v, (unsigned)dbf_dpp_move<0x124>((int)v));
    v = max(v, (unsigned)dbf_dpp_move<0x128>((int)v));
    if (L == 16) return v;
    auto lane = [&](int l) { return (unsigned)__builtin_amdgcn_readlane((int)v, l); };
    return max(max(lane(0), lane(16)), max(lane(32), lane(48)));
}
template <int L>
__device__ __forceinline__ double sum_of(double d) {
    auto sum = [](double a, u64 b) { return a + __builtin_bit_cast(double, b); };
    d = sum(d, move64<0xB1>(__builtin_bit_cast(u64, d)));
    d = sum(d, move64<0x4E>(__builtin_bit_cast(u64, d)));
    d = sum(d, move64<0x124>(__builtin_bit_cast(u64, d)));
    d = sum(d, move64<0x128>(__builtin_bit_cast(u64, d)));
    if (L == 16) return d;
    const u64 b = __builtin_bit_cast(u64, d);
    return (__builtin_bit_cast(double, lane64(b, 0)) + __builtin_bit_cast(double, lane64(b, 16))) +
           (__builtin_bit_cast(double, lane64(b, 32)) + __builtin_bit_cast(double, lane64(b, 48)));
}
// Numbers in their order as whole ones, above 0; -0 is 0.
__device__ __forceinline__ u64 in_order(double v) {
    const u64 b = __builtin_bit_cast(u64, v + 0.0);
    return b >> 63 ? ~b : b | 1ULL << 63;
}

// The experts of a token, L lanes to it: lane l has l, l + L, ... .  Lane l comes back with the l-th choice, and with 16 lanes with the (l + 16)-th too (-1: there is none),
// and their weights.  (Bound by chains of dependent maxima, n_top of them one behind the other: 8191 tokens of 256 experts, 8 each, 8.4 MB of logits, in 14.8 us, where their
// bytes take 1.6 by a copy's rate.  A wavefront to a token took 20, whose chains wait for themselves: 16 lanes to each of four share them.)
template <typename T, int L, int PER, bool SIGMOID>
__device__ __forceinline__ void choose(const RouteArgs& a, int token, int l, int (&id)[2], float (&weight)[2]) {
    const T* row = static_cast<const T*>(a.logits) + token * a.stride;
    const float none = -__builtin_inff();
    float x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = l + L * i;
        x[i] = e < a.n_experts ? dbf_to_float(row[e]) : none;
    }
    float most = none;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (!(x[i] > none)) x[i] = none;
        most = fmaxf(most, x[i]);
    }
    if (!SIGMOID) most = L == 16 ? dbf_row16_max(most) : dbf_wave_max(most);
    // (an infinite logit has all there is, shared with others of its kind)
    auto score = [&](float v) -> double { return SIGMOID ? 1.0 / (1.0 + exp(-(double)v)) : v == most ? 1.0 : exp((double)v - (double)most); };
    // Where there is no bias the order is that of the logits, and only the chosen ones' scores are needed but for a softmax's sum.
    double total = 1.0;
    u64 key[PER];
    if (!SIGMOID && (a.bias || !a.renormalise)) {
        total = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) total += x[i] > none ? score(x[i]) : 0.0;
        total = sum_of<L>(total);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        key[i] = 0;
        if (x[i] > none) {
            const double v = a.bias ? score(x[i]) / total + (double)a.bias[l + L * i] : (double)x[i];
            if (v > -__builtin_inf()) key[i] = in_order(v);
        }
    }
    id[0] = id[1] = -1;
    unsigned last = ~0u;
    for (int j = 0; j < a.n_top; ++j) {
        u64 best = 0;
        unsigned e = 0;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) {
            if (last == (unsigned)(l + L * i)) key[i] = 0;
            if (key[i] >= best) best = key[i], e = l + L * i;
        }
        const u64 top = most_of<L>(best);
        // of equal ones the lowest index
        last = ~most_of<L>(best == top ? ~e : 0u);
        const int now = top ? (int)last : -1;
        if (j == l) id[0] = now;
        if (L == 16 && j == l + 16) id[1] = now;
    }
    double mine[2], chosen = 0.0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        mine[h] = 0.0;
        if (id[h] >= 0) mine[h] = score(dbf_to_float(row[id[h]])) / total;
        chosen += mine[h];
    }
    chosen = sum_of<L>(chosen);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (a.renormalise) mine[h] = chosen > 0.0 ? mine[h] / chosen : 0.0;
        weight[h] = (float)(mine[h] * (double)a.scale);
    }
}

// ---- the order by experts -----------------------------------------------------------------------------------------

// A row's place is the rows of the experts before, plus the expert's in the chunks before, plus its tokens before in the chunk: counts and bits, no atomic whose order
// could show, and no sort.  A chunk's counts are bytes; up to 256 chunks every workgroup adds all of them up itself (8191 tokens of 256 experts: 64 KB, 7.1 us), which spares a
// launch; one workgroup's tokens need no second launch at all (a token 4.5 us).

struct Places {
    unsigned tokens[DBF_MAX_GROUPS];   // a chunk's tokens that chose an expert, a bit each
    int first[DBF_MAX_GROUPS];         // an expert's first row of the chunk
    int total[DBF_MAX_GROUPS];
    int all;
    int ids[CHUNK * MOST_TOP];            // the chunk's choices
};

// total[e] -> the rows of the experts before e; returns the number of all.  first[e] grows by it.
__device__ __forceinline__ int add_up(const RouteArgs& a, Places& p) {
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x, each = (a.n_experts + 63) / 64, from = min(each * lane, a.n_experts), to = min(from + each, a.n_experts);
        int sum = 0;
        for (int e = from; e < to; ++e) sum += p.total[e];
        int upto = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(upto, d);
            if (lane >= d) upto += other;
        }
        int at = upto - sum;
        for (int e = from; e < to; ++e) {
            const int n = p.total[e];
            p.total[e] = at;
            p.first[e] += at;
            at += n;
        }
        if (lane == 63) p.all = upto;
    }
    __syncthreads();
    return p.all;
}

__device__ __forceinline__ void mark(const RouteArgs& a, Places& p, int token0) {
    for (int e = threadIdx.x; e < a.n_experts; e += blockDim.x) p.tokens[e] = 0;
    __syncthreads();
    const int entries = min(CHUNK, a.n_tokens - token0) * a.n_top;
    for (int i = threadIdx.x; i < entries; i += blockDim.x) {
        const int id = a.ids[(long long)token0 * a.n_top + i];
        p.ids[i] = id;
        if (id >= 0) atomicOr(&p.tokens[id], 1u << (i / a.n_top));
    }
    __syncthreads();
}

__device__ __forceinline__ void place(const RouteArgs& a, const Places& p, int token0, int all) {
    const int entries = min(CHUNK, a.n_tokens - token0) * a.n_top;
    for (int i = threadIdx.x; i < entries; i += blockDim.x) {
        const long long at = (long long)token0 * a.n_top + i;
        const int id = p.ids[i], t = i / a.n_top;
        int row = -1;
        if (id >= 0) {
            row = p.first[id] + __popc(p.tokens[id] & ((1u << t) - 1));
            a.row_token[row] = token0 + t;
        }
        a.token_rows[at] = row;
        if (at >= all) a.row_token[at] = -1;
    }
    if (token0 == 0)
        for (int e = threadIdx.x; e <= a.n_experts; e += blockDim.x) a.starts[e] = e < a.n_experts ? p.total[e] : all;
}

template <typename T, int L, int PER, bool SIGMOID>
__global__ __launch_bounds__(CHOOSERS) void dbf_route_choose_kernel(const RouteArgs a) {
    __shared__ Places p;
    const int l = threadIdx.x & (L - 1), at_once = blockDim.x / L, token0 = blockIdx.x * CHUNK;
    for (int e = threadIdx.x; e < a.n_experts; e += blockDim.x) p.tokens[e] = 0;
    __syncthreads();
    // (all lanes of a wavefront go on while one of its tokens is there)
    for (int t0 = 0; t0 < CHUNK; t0 += at_once) {
        const int t = t0 + threadIdx.x / L;
        if (token0 + t0 + (int)(threadIdx.x & ~63) / L >= a.n_tokens) break;
        int id[2];
        float weight[2];
        choose<T, L, PER, SIGMOID>(a, min(token0 + t, a.n_tokens - 1), l, id, weight);
        if (token0 + t < a.n_tokens) {
#pragma unroll
            for (int h = 0; h < (L == 16 ? 2 : 1); ++h) {
                const int j = l + 16 * h;
                if (j >= a.n_top) continue;
                const long long at = (long long)(token0 + t) * a.n_top + j;
                a.ids[at] = id[h];
                a.weights[at] = weight[h];
                p.ids[t * a.n_top + j] = id[h];
                if (id[h] >= 0) atomicOr(&p.tokens[id[h]], 1u << t);
            }
        }
    }
    __syncthreads();
    if (gridDim.x > 1) {
        for (int e = threadIdx.x; e < a.padded; e += blockDim.x) a.counts[(long long)blockIdx.x * a.padded + e] = e < a.n_experts ? (uint8_t)__popc(p.tokens[e]) : 0;
        return;
    }
    for (int e = threadIdx.x; e < a.n_experts; e += blockDim.x) {
        p.total[e] = __popc(p.tokens[e]);
        p.first[e] = 0;
    }
    const int all = add_up(a, p);
    place(a, p, token0, all);
}

// Sums over the chunks before each, for four experts a workgroup.
__global__ __launch_bounds__(THREADS) void dbf_route_sums_kernel(const RouteArgs a, int chunks) {
    __shared__ int part[THREADS][4];
    const int tid = threadIdx.x, each = (chunks + THREADS - 1) / THREADS, from = min(tid * each, chunks), to = min(from + each, chunks);
    const uint8_t* counts = a.counts + 4 * blockIdx.x;
    int sum[4] = {0, 0, 0, 0};
    for (int c = from; c < to; ++c)
        for (int i = 0; i < 4; ++i) sum[i] += counts[(long long)c * a.padded + i];
    for (int i = 0; i < 4; ++i) part[tid][i] = sum[i];
    __syncthreads();
    for (int d = 1; d < THREADS; d <<= 1) {
        int other[4] = {0, 0, 0, 0};
        if (tid >= d)
            for (int i = 0; i < 4; ++i) other[i] = part[tid - d][i];
        __syncthreads();
        for (int i = 0; i < 4; ++i) part[tid][i] += other[i];
        __syncthreads();
    }
    int at[4];
    for (int i = 0; i < 4; ++i) at[i] = part[tid][i] - sum[i];
    for (int c = from; c < to; ++c)
        for (int i = 0; i < 4; ++i) {
            a.before[(long long)c * a.padded + 4 * blockIdx.x + i] = at[i];
            at[i] += counts[(long long)c * a.padded + i];
        }
    if (tid == THREADS - 1)
        for (int i = 0; i < 4; ++i) a.before[(long long)chunks * a.padded + 4 * blockIdx.x + i] = part[tid][i];
}

__global__ __launch_bounds__(THREADS) void dbf_route_place_kernel(const RouteArgs a) {
    __shared__ Places p;
    const int chunk = blockIdx.x, chunks = gridDim.x;
    for (int e = threadIdx.x; e < a.padded; e += THREADS) {
        p.first[e] = a.before ? a.before[(long long)chunk * a.padded + e] : 0;
        p.total[e] = a.before ? a.before[(long long)chunks * a.padded + e] : 0;
    }
    __syncthreads();
    if (!a.before) {
        // four experts a thread, the chunks dealt out to as many threads as there are
        const int words = a.padded / 4, slices = THREADS / words, w = threadIdx.x % words, slice = threadIdx.x / words;
        if (slice < slices) {
            int sum[4] = {0, 0, 0, 0}, mine[4] = {0, 0, 0, 0};
            constexpr int AT_ONCE = 8;
            for (int c0 = slice; c0 < chunks; c0 += AT_ONCE * slices) {
                unsigned v[AT_ONCE];
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) v[k] = c0 + k * slices < chunks ? *reinterpret_cast<const unsigned*>(a.counts + (long long)(c0 + k * slices) * a.padded + 4 * w) : 0;
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int n = v[k] >> (8 * i) & 255;
                        sum[i] += n;
                        mine[i] += c0 + k * slices < chunk ? n : 0;
                    }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                atomicAdd(&p.total[4 * w + i], sum[i]);
                atomicAdd(&p.first[4 * w + i], mine[i]);
            }
        }
    }
    mark(a, p, chunk * CHUNK);
    const int all = add_up(a, p);
    place(a, p, chunk * CHUNK, all);
}

bool sizes_ok(const dbf_router* r) {
    return r->n_tokens >= 0 && r->n_tokens <= MOST_TOKENS && r->n_experts >= 1 && r->n_experts <= DBF_MAX_GROUPS && r->n_top >= 1 && r->n_top <= MOST_TOP &&
           r->n_top <= r->n_experts && (long long)r->n_tokens * r->n_top <= INT_MAX;
}
struct Room {
    size_t counts, before;
};
Room room_of(const dbf_router* r) {
    const size_t chunks = ((size_t)r->n_tokens + CHUNK - 1) / CHUNK, padded = (r->n_experts + 3) / 4 * 4;
    if (chunks <= 1) return {0, 0};
    return {(chunks * padded + 255) / 256 * 256, chunks > MOST_CHUNKS ? (chunks + 1) * padded * 4 : 0};
}

template <typename T, int L, int PER>
void choose(const RouteArgs& a, int score, dim3 grid, hipStream_t stream) {
    const dim3 threads(std::min(CHOOSERS, (std::min(a.n_tokens, CHUNK) * L + 63) / 64 * 64));   // (no more wavefronts than a chunk's tokens need)
    if (score == DBF_SCORE_SIGMOID) hipLaunchKernelGGL((dbf_route_choose_kernel<T, L, PER, true>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((dbf_route_choose_kernel<T, L, PER, false>), grid, threads, 0, stream, a);
}
template <typename T>
void choose(const RouteArgs& a, int score, dim3 grid, hipStream_t stream) {
    if (a.n_experts <= 64) choose<T, 16, 4>(a, score, grid, stream);
    else if (a.n_experts <= 128) choose<T, 16, 8>(a, score, grid, stream);
    else if (a.n_experts <= 256) choose<T, 16, 16>(a, score, grid, stream);
    else choose<T, 64, 16>(a, score, grid, stream);
}

__global__ void dbf_route_nothing_kernel(int32_t* starts, int n) {
    for (int i = threadIdx.x; i <= n; i += blockDim.x) starts[i] = 0;
}

// ---- rows back to their tokens ---------------------------------------------------------------------------------------

struct CombineArgs {
    const void *rows, *residual;
    const int32_t* token_rows;
    const float* weights;
    void* out;
    long long row_stride, residual_stride, out_stride;
    int n_rows, n_tokens, n_top, n_cols;
};

// N neighbouring values of a token to a thread.  Bound by memory: 4095 tokens, a residual and four rows each of 4096 fp16 values, 201 MB in 41.2 us (4.9 TB/s,
// where a copy has 5.1; 30.6 where the last cache holds them); a token's rows
// are n_top loads that do not wait for each other, and nothing is read twice but ids and weights, which the caches hold.
constexpr int SUM_THREADS = 256;
template <typename T, int N>
__global__ __launch_bounds__(SUM_THREADS) void dbf_combine_kernel(const CombineArgs a, int pieces) {
    const long long n = (long long)a.n_tokens * pieces, step = (long long)gridDim.x * SUM_THREADS;
    for (long long i = (long long)blockIdx.x * SUM_THREADS + threadIdx.x; i < n; i += step) {
        const int token = (int)(i / pieces), at = (int)(i - (long long)token * pieces) * N;
        float sum[N];
        T v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] = 0.f;
        if (a.residual) {
            __builtin_memcpy(v, __builtin_assume_aligned(static_cast<const T*>(a.residual) + token * a.residual_stride + at, sizeof(T) * N), sizeof(v));
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] = dbf_to_float(v[k]);
        }
        for (int j = 0; j < a.n_top; ++j) {
            const int row = a.token_rows[(long long)token * a.n_top + j];
            if ((unsigned)row >= (unsigned)a.n_rows) continue;
            const float w = a.weights[(long long)token * a.n_top + j];
            __builtin_memcpy(v, __builtin_assume_aligned(static_cast<const T*>(a.rows) + row * a.row_stride + at, sizeof(T) * N), sizeof(v));
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] = fmaf(w, dbf_to_float(v[k]), sum[k]);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = dbf_from_float<T>(sum[k]);
        __builtin_memcpy(__builtin_assume_aligned(static_cast<T*>(a.out) + token * a.out_stride + at, sizeof(T) * N), v, sizeof(v));
    }
}

template <typename T>
int combine(const CombineArgs& a, hipStream_t stream) {
    constexpr int N = 16 / sizeof(T);
    const bool whole = a.n_cols % N == 0 && a.row_stride % N == 0 && a.out_stride % N == 0 && (!a.residual || a.residual_stride % N == 0) && !dbf_misaligned(a.rows, 16) &&
                       !dbf_misaligned(a.residual, 16) && !dbf_misaligned(a.out, 16);
    const int pieces = whole ? a.n_cols / N : a.n_cols;
    const long long n = (long long)a.n_tokens * pieces;
    const dim3 grid((unsigned)std::min((n + SUM_THREADS - 1) / SUM_THREADS, 1LL << 22)), threads(SUM_THREADS);
    if (whole) hipLaunchKernelGGL((dbf_combine_kernel<T, N>), grid, threads, 0, stream, a, pieces);
    else hipLaunchKernelGGL((dbf_combine_kernel<T, 1>), grid, threads, 0, stream, a, pieces);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}

bool float_type(int dtype) { return dtype == DBF_F16 || dtype == DBF_BF16 || dtype == DBF_F32; }

}  // namespace

extern "C" size_t dbf_route_workspace_bytes(const dbf_router* r) {
    if (!r || !sizes_ok(r)) return 0;
    const Room room = room_of(r);
    return room.counts + room.before;
}

extern "C" int dbf_route(const dbf_router* r, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    if (!r || !r->logits || !r->expert_ids || !r->weights || !r->starts || !r->row_token || !r->token_rows || !float_type(r->dtype)) return DBF_EINVAL;
    if (r->n_experts < 1 || r->n_experts > DBF_MAX_GROUPS) return DBF_ESHAPE;
    if (!sizes_ok(r) || r->row_stride < r->n_experts || (r->score != DBF_SCORE_SOFTMAX && r->score != DBF_SCORE_SIGMOID)) return DBF_EINVAL;
    if (dbf_misaligned(r->logits, r->dtype == DBF_F32 ? 4 : 2)) return DBF_EINVAL;
    for (const void* p : {static_cast<const void*>(r->bias), static_cast<const void*>(r->expert_ids), static_cast<const void*>(r->weights), static_cast<const void*>(r->starts),
                          static_cast<const void*>(r->row_token), static_cast<const void*>(r->token_rows)})
        if (dbf_misaligned(p, 4)) return DBF_EINVAL;
    const auto stream = static_cast<hipStream_t>(hip_stream);
    if (!r->n_tokens) {
        hipLaunchKernelGGL(dbf_route_nothing_kernel, dim3(1), dim3(THREADS), 0, stream, r->starts, r->n_experts);
        return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
    }
    const Room room = room_of(r);
    if (room.counts + room.before && (!workspace_dev || dbf_misaligned(workspace_dev, 256) || workspace_bytes < room.counts + room.before)) return DBF_EWORKSPACE;
    const int chunks = (int)((r->n_tokens + (long long)CHUNK - 1) / CHUNK);
    RouteArgs a = {};
    a.logits = r->logits;
    a.bias = r->bias;
    a.stride = r->row_stride;
    a.ids = r->expert_ids;
    a.weights = r->weights;
    a.starts = r->starts;
    a.row_token = r->row_token;
    a.token_rows = r->token_rows;
    a.counts = static_cast<uint8_t*>(workspace_dev);
    a.before = room.before ? reinterpret_cast<int32_t*>(static_cast<char*>(workspace_dev) + room.counts) : nullptr;
    a.n_tokens = r->n_tokens;
    a.n_experts = r->n_experts;
    a.n_top = r->n_top;
    a.padded = (r->n_experts + 3) / 4 * 4;
    a.renormalise = r->renormalise;
    a.scale = r->scale;
    const dim3 grid((unsigned)chunks);
    if (r->dtype == DBF_F16) choose<_Float16>(a, r->score, grid, stream);
    else if (r->dtype == DBF_BF16) choose<dbf_bf16>(a, r->score, grid, stream);
    else choose<float>(a, r->score, grid, stream);
    if (a.before) hipLaunchKernelGGL(dbf_route_sums_kernel, dim3(a.padded / 4), dim3(THREADS), 0, stream, a, chunks);
    if (chunks > 1) hipLaunchKernelGGL(dbf_route_place_kernel, grid, dim3(THREADS), 0, stream, a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}

extern "C" int dbf_combine(const dbf_combine_rows* s, void* hip_stream) {
    if (!s || !s->out || !s->token_rows || !s->weights || !float_type(s->dtype) || (!s->rows && s->n_rows)) return DBF_EINVAL;
    if (s->n_cols < 1 || s->n_cols > DBF_MAX_DIM) return DBF_ESHAPE;
    if (s->n_rows < 0 || s->n_tokens < 0 || s->n_top < 1 || s->n_top > MOST_TOP) return DBF_EINVAL;
    if (s->row_stride < s->n_cols || s->out_stride < s->n_cols || (s->residual && s->residual_stride < s->n_cols)) return DBF_EINVAL;
    const unsigned size = s->dtype == DBF_F32 ? 4 : 2;
    if (dbf_misaligned(s->rows, size) || dbf_misaligned(s->residual, size) || dbf_misaligned(s->out, size) || dbf_misaligned(s->token_rows, 4) || dbf_misaligned(s->weights, 4))
        return DBF_EINVAL;
    if (!s->n_tokens) return DBF_OK;
    const CombineArgs a = {s->rows, s->residual, s->token_rows, s->weights, s->out, s->row_stride, s->residual_stride, s->out_stride, s->n_rows, s->n_tokens, s->n_top, s->n_cols};
    const auto stream = static_cast<hipStream_t>(hip_stream);
    return s->dtype == DBF_F16 ? combine<_Float16>(a, stream) : s->dtype == DBF_BF16 ? combine<dbf_bf16>(a, stream) : combine<float>(a, stream);
}
