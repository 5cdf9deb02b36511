// Attention over the cache in 4 bits (include/dbf.h, dbf_cache_attend).
#include <algorithm>
#include <initializer_list>

#include "dbf_cache.h"
#include "dbf_wave.h"

namespace {

struct alignas(16) Piece {   // an item that was cut: its head (-1: it was not), shares, rows
    int head, share, last, row0, rows, unused[3];
};
struct AttendArgs {
    const void* q;
    void* out;
    long long q_stride, out_stride;
    const int *q_start, *kv_len, *table;
    const uint8_t* cache;
    int n_tokens, n_seq, n_q, n_kv, max_q, max_kv, table_stride, causal, n_pages, page_shift, dim;
    int group;             // query heads of a key head
    int chunk, parts;      // many rows: tokens of a part of the long axis, and parts
    float scale;
    float *part_out, *part_stat;   // of a share's first and last piece: sums [share][2][row][head_dim], maximum and sum of the row's weights [..][2]
                                   // (many rows: [request][head][part][row])
    Piece* cut;                    // of each item, or of each share the item that begins in it and goes on in others
    int by_item;
};
constexpr float LOWEST = -3.0e38f;   // of a running maximum: below all scores, and its difference from one is a number
constexpr int MOST_SHARES = 1024;
constexpr int BESIDE = 8;            // records' time that an item takes beside its records (4: batch of 64 in 88 us for 81; 12 and 16 the same)
constexpr int TILE = 64;             // tokens of a step of many rows
constexpr int MANY_WAVES = 4;       // wavefronts of a workgroup of many rows, 32 rows each
constexpr long long MOST_ROWS = 65535LL * 32 * MANY_WAVES;   // of a request and key head: a launch's third dimension
constexpr int AHEAD = 4;             // operands read from LDS ahead of their products
constexpr int LEAST_CHUNK = 512;     // tokens of a part, of many rows, at least: its first tile and the join are paid for
constexpr int FEW = 16;              // rows (tokens times heads) of a request and key head that are few

// A word that no workgroup of the launch writes, at an address that is the same for all lanes, through the scalar cache.
__device__ __forceinline__ int scalar(const int* p) { return *(const __attribute__((address_space(4))) int*)p; }

// A request's rows and tokens; ok: they are what the call allows.
struct Request {
    int row0, rows, kv;
    bool ok;
};
__device__ __forceinline__ Request request(const AttendArgs& a, int i) {
    Request r;
    const int from = a.q_start ? a.q_start[i] : i, to = a.q_start ? a.q_start[i + 1] : i + 1;
    r.row0 = min(max(from, 0), a.n_tokens);
    const int end = min(max(to, r.row0), a.n_tokens);
    r.rows = end - r.row0;
    r.kv = a.kv_len[i];
    r.ok = r.kv >= 0 && r.kv <= a.max_kv && r.kv <= (long long)a.table_stride << a.page_shift && r.rows <= a.max_q && r.row0 == from && end == to;   // (rows cut off at the tensor's ends are others than they seem)
    return r;
}

// The wavefront's lanes l, l + 16, l + 32, l + 48 hold parts of one column: their maximum or sum, in all of them.
__device__ __forceinline__ float column_max(float v) {
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    const unsigned c = __builtin_bit_cast(unsigned, fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])));
    const auto t = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)t[0]), __builtin_bit_cast(float, (unsigned)t[1]));
}
__device__ __forceinline__ float column_sum(float v) {
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    const unsigned c = __builtin_bit_cast(unsigned, __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]));
    const auto t = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    return __builtin_bit_cast(float, (unsigned)t[0]) + __builtin_bit_cast(float, (unsigned)t[1]);
}

template <typename T>
__device__ __forceinline__ void load8(const T* at, float (&v)[8]) {   // of any alignment
    const dbf_u4 w = *reinterpret_cast<const dbf_u4_any*>(at);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = dbf_to_float(__builtin_bit_cast(T, (uint16_t)(w[e >> 1] >> 16 * (e & 1))));
}

// The 16 codes of a lane's 8 bytes as two operands of the 16x16x32 product, the even and the odd ones.  A code is left where it lies in an fp16: as the
// subnormal number c 2^-24, or 16 c 2^-24 for the odd ones, which the matrix cores take as they are.
__device__ __forceinline__ void operands(unsigned w0, unsigned w1, dbf_h8& even, dbf_h8& odd) {
    const dbf_u4 e = {w0 & 0x000F000Fu, w0 >> 8 & 0x000F000Fu, w1 & 0x000F000Fu, w1 >> 8 & 0x000F000Fu};
    const dbf_u4 o = {w0 & 0x00F000F0u, w0 >> 8 & 0x00F000F0u, w1 & 0x00F000F0u, w1 >> 8 & 0x00F000F0u};
    even = __builtin_bit_cast(dbf_h8, e);
    odd = __builtin_bit_cast(dbf_h8, o);
}

// Four codes' bytes of a word, tokens 0 .. 3 with a value in the low and one in the high half of a byte, as fp16 values s c - s z (exact: 7 bits times 4), the
// pairs of tokens 0, 2 and 1, 3 of the low value and of the high one.  s and b: the pairs' scales and zeros.  (1024 + c is fp16's 1024 with c in its last bits.)
__device__ __forceinline__ void values(unsigned u, dbf_h2 s02, dbf_h2 b02, dbf_h2 s13, dbf_h2 b13, unsigned& lo02, unsigned& lo13, unsigned& hi02, unsigned& hi13) {
    const dbf_h2 less = {(_Float16)-1024.f, (_Float16)-1024.f}, part = {(_Float16)0.0625f, (_Float16)0.0625f}, less_part = {(_Float16)-64.f, (_Float16)-64.f};
    unsigned thousand = 0x64006400u;
    asm("" : "+v"(thousand));   // (in a register, so that and-or is one instruction: it takes one scalar operand)
    auto code = [=](unsigned v) { return __builtin_bit_cast(dbf_h2, v | thousand); };
    auto value = [](dbf_h2 c, dbf_h2 s, dbf_h2 b) { return __builtin_bit_cast(unsigned, __builtin_elementwise_fma(c, s, b)); };
    lo02 = value(code(u & 0x000F000Fu) + less, s02, b02);
    lo13 = value(code(u >> 8 & 0x000F000Fu) + less, s13, b13);
    hi02 = value(__builtin_elementwise_fma(code(u & 0x00F000F0u), part, less_part), s02, b02);
    hi13 = value(__builtin_elementwise_fma(code(u >> 8 & 0x00F000F0u), part, less_part), s13, b13);
}
__device__ __forceinline__ dbf_h2 word(unsigned w) { return __builtin_bit_cast(dbf_h2, w); }
// The low or the high halves of two words.
__device__ __forceinline__ dbf_h2 lows(unsigned a, unsigned b) { return __builtin_bit_cast(dbf_h2, __builtin_amdgcn_perm(b, a, 0x05040100u)); }
__device__ __forceinline__ dbf_h2 highs(unsigned a, unsigned b) { return __builtin_bit_cast(dbf_h2, __builtin_amdgcn_perm(b, a, 0x07060302u)); }

// What a lane holds of a record's keys: of tokens 16 t + (lane & 15), the bytes of its 16 N values; the groups' words of tokens 16 t + 4 (lane >> 4) ..
template <int N>
struct Keys {
    unsigned k[2][2 * N];
    dbf_u4 words[2][N];
    __device__ __forceinline__ void load(const uint8_t* rec, int lane) {
        const int g = lane >> 4, r = lane & 15;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint8_t* at = rec + (16 * t + r) * 32 * N + 8 * N * g;
            if constexpr (N == 1) {
                const dbf_u2 w = *reinterpret_cast<const dbf_u2*>(at);
                k[t][0] = w[0], k[t][1] = w[1];
            } else {
#pragma unroll
                for (int e = 0; e < N / 2; ++e) {
                    const dbf_u4 w = *reinterpret_cast<const dbf_u4*>(at + 16 * e);
#pragma unroll
                    for (int f = 0; f < 4; ++f) k[t][4 * e + f] = w[f];
                }
            }
#pragma unroll
            for (int p = 0; p < N; ++p) words[t][p] = *reinterpret_cast<const dbf_u4*>(rec + 2048 * N + 128 * p + 64 * t + 16 * g);
        }
    }
};
// ... and of its values: both runs of 16 tokens of its place in a group, and the words as above.
template <int N>
struct Values {
    dbf_u4 v[N], words[2][N];
    __device__ __forceinline__ void load(const uint8_t* rec, int lane) {
        const int g = lane >> 4;
#pragma unroll
        for (int p = 0; p < N; ++p) v[p] = *reinterpret_cast<const dbf_u4*>(rec + 1024 * N + 1024 * p + 16 * lane);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int p = 0; p < N; ++p) words[t][p] = *reinterpret_cast<const dbf_u4*>(rec + 2176 * N + 128 * p + 64 * t + 16 * g);
    }
};

// A wavefront's sums for its 16 columns, and a step over one record.
template <int N>
struct Columns {
    dbf_h8 qe[N], qo[N];         // the queries' even and odd values, the odd ones over 16
    float Q[N], kappa, m, l;     // their sums; from sums of products to scores in powers of two; largest score so far, or a little less; sum of the weights
    dbf_f4 o[4 * N];
    int seen, kv;                // tokens that the column sees, and that there are

    // x: the scores of tokens 16 t + 4 g + i
    __device__ __forceinline__ void scores(const Keys<N>& keys, float kappa, float (&x)[2][4]) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[t][i] = 0.f;
#pragma unroll
            for (int p = 0; p < N; ++p) {
                dbf_h8 even, odd;
                operands(keys.k[t][2 * p], keys.k[t][2 * p + 1], even, odd);
                dbf_f4 acc = {0.f, 0.f, 0.f, 0.f};
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, qe[p], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, qo[p], acc, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const dbf_h2 sb = word(keys.words[t][p][i]);
                    x[t][i] = fmaf((float)sb[0], acc[i], x[t][i]);
                    x[t][i] = fmaf((float)sb[1], Q[p], x[t][i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) x[t][i] *= kappa;
        }
    }
    // Tokens from `first` on that are not there for all: no scores, and no words (what lies there may be no number).
    __device__ __forceinline__ void mask(int first, bool known, float (&x)[2][4], Values<N>& values) const {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = first + 16 * t + i;
                x[t][i] = j < seen ? (known ? x[t][i] : __builtin_nanf("")) : -__builtin_inff();
#pragma unroll
                for (int p = 0; p < N; ++p) values.words[t][p][i] = known && j < kv ? values.words[t][p][i] : 0u;
            }
    }
    __device__ __forceinline__ void raise(const float (&x)[2][4]) {
        float most = LOWEST;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, x[t][i]);
        if (__any(most > m + 8.f)) {
            const float to = fmaxf(m, column_max(most)), keep = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= keep;
#pragma unroll
            for (int j = 0; j < 4 * N; ++j) o[j] *= keep;
        }
    }
    __device__ __forceinline__ void add(const float (&x)[2][4], const Values<N>& in) {
        dbf_h8 weights;
        const float from = m - 7.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = __builtin_amdgcn_exp2f(x[t][i] - from);
                l += w;
                weights[4 * t + 2 * (i & 1) + (i >> 1)] = (_Float16)w;
            }
#pragma unroll
        for (int p = 0; p < N; ++p) {
            dbf_h2 s02[2], s13[2], b02[2], b13[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const dbf_u4 w = in.words[t][p];
                s02[t] = lows(w[0], w[2]);
                s13[t] = lows(w[1], w[3]);
                b02[t] = highs(w[0], w[2]);
                b13[t] = highs(w[1], w[3]);
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                unsigned lo[4], hi[4];
#pragma unroll
                for (int t = 0; t < 2; ++t) values(in.v[p][2 * q + t], s02[t], b02[t], s13[t], b13[t], lo[2 * t], lo[2 * t + 1], hi[2 * t], hi[2 * t + 1]);
                const dbf_h8 low = __builtin_bit_cast(dbf_h8, (dbf_u4){lo[0], lo[1], lo[2], lo[3]}), high = __builtin_bit_cast(dbf_h8, (dbf_u4){hi[0], hi[1], hi[2], hi[3]});
                o[p + N * (2 * q)] = __builtin_amdgcn_mfma_f32_16x16x32_f16(low, weights, o[p + N * (2 * q)], 0, 0, 0);
                o[p + N * (2 * q + 1)] = __builtin_amdgcn_mfma_f32_16x16x32_f16(high, weights, o[p + N * (2 * q + 1)], 0, 0, 0);
            }
        }
    }
};

// Few rows: those of a request and key head are columns of one 16-wide product (the rows' tokens times the heads that share the keys), the long axis is cut
// into parts, a workgroup's part goes by records of 32 tokens to its four wavefronts, each with statistics of its own.
//   scores:  K q^T, 16 tokens x 16 columns x the 64 values of a group; x = sum over groups of s (c . q) - s z sum q: the scale and the zero come on the sums,
//            so codes go to the matrix cores as they are.  q is scaled by a power of two to the top of fp16's range, and exact there.
//   weights: e^(x - m) with m a maximum that may lag: it is raised when some score is more than 2^8 above it, so that a step that raises none
//            (nearly all) joins no lanes and touches no sums.  Rounded to fp16 for the product, times 2^7: a weight 2^-21 of the largest still has all its bits.
//   output:  V^T p^T, 16 values of a group x 16 columns x 32 tokens, of values made exact in fp16.  (Scales on the weights instead of the values were fewer
//            instructions, but their rounding does not cancel between c and z: values near zero lost three bits.)
// The sum of the weights is of the unrounded ones, which costs what that of the rounded ones would; many rows have the latter from a dot product of two.  Each is within a rounding of the other.
// It has the cache to read, 36 bytes a value of head_dim for 32 tokens: one token over 131071 of 8 heads of 128, 151 MB in 31 us (4.9 TB/s), and 5 of the join; 64 requests of 1 .. 8192 tokens, 327 MB
// in 64 (5.1) and 5.  A read of as many bytes and nothing else has 24 and 50 us (6.3 and 6.6 TB/s): between them lie the vector instructions, 66 and 70 % of the time, and waits for their issue.
// One request of 333 tokens: 7.1 us, latencies.
// A record from memory to LDS as it is, under way until vmcnt says that it is not.  (2: read once, so it need not stay in the caches: 75 -> 68 us for the batch of 64.)
template <int N>
__device__ __forceinline__ void fetch(const uint8_t* rec, uint8_t* to, int lane) {
    constexpr int BYTES = 36 * 64 * N;
#pragma unroll
    for (int k = 0; k < BYTES; k += 1024)
        if (k + 1024 <= BYTES || lane < (BYTES - k) / 16)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(rec + k + 16 * lane), (__attribute__((address_space(3))) void*)(to + k), 16, 0, 2);
}

template <int N>
struct Shared {
    union {
        alignas(16) uint8_t stage[4][2][36 * 64 * N];        // two records of each wavefront
        alignas(16) float sums[4][FEW][N == 1 ? 64 : 128];   // then its sums
    };
    float stats[4][2][FEW];
};
// Records from .. to of a request and key head: into the output, or, of a piece, into its place among the parts.
template <typename T, int N>
__device__ __forceinline__ void few_rows(const AttendArgs& a, const Request& r, int req, int head, int from, int to, long long piece, Shared<N>& shared) {
    constexpr int D = 64 * N;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15, G = a.group;
    const int cols = min(r.rows, a.max_q) * G;
    if (!cols) return;
    const int all_see = a.causal ? r.kv - r.rows + 1 : r.kv;   // tokens that all columns see
    const int* table = a.table + (long long)req * a.table_stride;
    const int first = from + wave, last = to - 1, per_page = a.page_shift - 5;
    bool known = true, known_next = true;
    auto at = [&](int b, bool& is) {
        const int page = scalar(table + (b >> per_page));
        is = (unsigned)page < (unsigned)a.n_pages;
        return a.cache + ((((long long)(is ? page : 0) * a.n_kv + head) << per_page) + (b & ((1 << per_page) - 1))) * dbf_record_bytes(D);
    };
    // A record is in registers while the next one is under way to LDS.  (From memory to registers, half a step ahead, took 12 loads a record, most of them of words that
    // 16 lanes share, for 5; and 38.9 us for 131071 tokens, 74.8 for the batch of 64.)
    uint8_t (*stage)[36 * D] = shared.stage[wave];
    __syncthreads();   // (the piece before has been read)
    if (first <= last) fetch<N>(at(first, known_next), stage[0], lane);
    // the column's query, by groups
    Columns<N> s = {};
    {
        const bool live = c < cols;
        const T* at = static_cast<const T*>(a.q) + (long long)(r.row0 + (live ? c / G : 0)) * a.q_stride + (long long)(head * G + (live ? c % G : 0)) * D + 16 * N * g;
        float v[N][16], most = 0.f;
#pragma unroll
        for (int p = 0; p < N; ++p) {
            float x[2][8];
            load8(at + 16 * p, x[0]);
            load8(at + 16 * p + 8, x[1]);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                v[p][e] = live ? x[e >> 3][e & 7] : 0.f;
                most = fmaxf(most, fabsf(v[p][e]));
            }
        }
        most = column_max(most);
        const int up = most > 0.f && most < __builtin_inff() ? 14 - __builtin_amdgcn_frexp_expf(most) : 0;
        // (no more than 2^100: sums of products are below 2^20 and, where they differ, 2^-72 apart at least, so that no score passes fp32 and those that a larger one would
        // tell apart are 2^28 apart)
        s.kappa = fminf(fmaxf(ldexpf(a.scale * 1.44269504089f, 24 - up), -0x1p100f), 0x1p100f);
#pragma unroll
        for (int p = 0; p < N; ++p) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int d = 8 * (e >> 2) + 4 * (e & 1) + (e & 2);
                const _Float16 lo = (_Float16)ldexpf(v[p][d], up), hi = (_Float16)ldexpf(v[p][d + 1], up);
                s.qe[p][e] = lo;
                s.qo[p][e] = hi * (_Float16)0.0625f;
                sum += (float)lo + (float)hi;
            }
            s.Q[p] = column_sum(sum) * 0x1p-24f;
        }
    }
    s.seen = a.causal ? r.kv - r.rows + c / G + 1 : r.kv;
    s.kv = r.kv;
    s.m = LOWEST;
    int turn = 0;
    auto step = [&](int b, bool all) {
        float x[2][4];
        Keys<N> keys;
        Values<N> in;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        keys.load(stage[turn], lane);
        in.load(stage[turn], lane);
        known = known_next;
        turn ^= 1;
        if (b + 4 <= last) fetch<N>(at(b + 4, known_next), stage[turn], lane);   // (what was there has been used)
        s.scores(keys, known ? s.kappa : __builtin_nanf(""), x);
        if (!all) s.mask(32 * b + 4 * g, known, x, in);
        s.raise(x);
        s.add(x, in);
    };
    // (two loops: the masks as a branch in one became selects, a sixth of every step's instructions)
    int b = first;
    for (; b <= last && 32 * b + 32 <= all_see; b += 4) step(b, true);
    for (; b <= last; b += 4) step(b, false);
    // the four wavefronts' sums
    s.l = column_sum(s.l);
    __syncthreads();   // (no record is needed any more)
    if (g == 0) {
        shared.stats[wave][0][c] = s.m;
        shared.stats[wave][1][c] = s.l;
    }
    constexpr int SPAN = N == 1 ? 64 : 128;
    for (int d0 = 0; d0 < D; d0 += SPAN) {
        if (d0) __syncthreads();
#pragma unroll
        for (int j = 0; j < 4 * N; ++j)
            if (16 * j >= d0 && 16 * j < d0 + SPAN) *reinterpret_cast<dbf_f4*>(&shared.sums[wave][c][16 * j - d0 + 4 * g]) = s.o[j];
        __syncthreads();
        for (int e = threadIdx.x; e < cols * SPAN; e += 256) {
            const int col = e / SPAN, d = e % SPAN;
            float most = shared.stats[0][0][col];
            for (int w = 1; w < 4; ++w) most = fmaxf(most, shared.stats[w][0][col]);
            float y = 0.f, sum = 0.f;
            for (int w = 0; w < 4; ++w) {
                const float keep = __builtin_amdgcn_exp2f(shared.stats[w][0][col] - most);
                y = fmaf(keep, shared.sums[w][col][d], y);
                sum = fmaf(keep, shared.stats[w][1][col], sum);
            }
            if (piece < 0) {
                T* out = static_cast<T*>(a.out) + (long long)(r.row0 + col / G) * a.out_stride + (long long)(head * G + col % G) * D + d0 + d;
                *out = dbf_from_float<T>(!r.ok ? __builtin_nanf("") : sum == 0.f ? 0.f : y / sum);
            } else {
                a.part_out[(piece * FEW + col) * D + d0 + d] = y;
                if (d0 + d == 0) {
                    a.part_stat[2 * (piece * FEW + col)] = most;
                    a.part_stat[2 * (piece * FEW + col) + 1] = sum;
                }
            }
        }
    }
}
__device__ __forceinline__ int records(const Request& r) { return r.ok && r.rows > 0 ? (r.kv + 31) / 32 : 0; }

constexpr int few_waves(int N) { return N == 1 ? 4 : N == 2 ? 3 : 2; }   // wavefronts of a SIMD that have registers
#define DBF_FEW_KERNEL(N) __global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(few_waves(N))))

// A workgroup to an item: a request and key head.
template <typename T, int N>
DBF_FEW_KERNEL(N) void dbf_attend_items_kernel(const AttendArgs a) {
    __shared__ Shared<N> shared;
    const Request r = request(a, blockIdx.y);
    few_rows<T, N>(a, r, blockIdx.y, blockIdx.x, 0, records(r), -1, shared);
}

// An equal share of the whole call to each of as many workgroups as the chip holds at once: items lie one after the other, each its records and a constant for what it
// costs beside them, and are cut where the shares end.  Lengths are only known here, so each workgroup makes the sums over the requests itself.  (Parts of a length chosen on the host,
// a workgroup to each: 64 requests of 1 .. 8192 tokens 103 us at the best length, in shares 83 then, 69 now; 131071 tokens of 8 heads 39 and 36.)
template <typename T, int N>
DBF_FEW_KERNEL(N) void dbf_attend_shares_kernel(const AttendArgs a) {
    __shared__ Shared<N> shared;
    __shared__ int waves[4], found_start, found;   // (costs of a call are below 2^30)
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, share = blockIdx.x;
    auto cost_of = [&](int i) { return records(request(a, i)) + BESIDE; };
    const int run = (a.n_seq + 255) / 256, from = min(tid * run, a.n_seq), to = min(from + run, a.n_seq);
    int own = 0;
    for (int i = from; i < to; ++i) own += cost_of(i);
    int sum = own;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    int before = sum - own, total = 0;
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += waves[w];
        total += waves[w];
    }
    before *= a.n_kv;
    total *= a.n_kv;
    total = __builtin_amdgcn_readfirstlane(total);
    const int size = (unsigned)(total + gridDim.x - 1) / gridDim.x, lo = share * size, hi = min(lo + size, total);
    if (tid == 0 && !a.by_item) a.cut[share].head = -1;
    if (lo >= total) return;
    if (lo >= before && lo < before + own * a.n_kv) {
        int i = from;
        if (run > 1)   // (else it is the thread's one)
            for (int c = cost_of(i) * a.n_kv; lo >= before + c; c = cost_of(i) * a.n_kv) {
                before += c;
                ++i;
            }
        found = i;
        found_start = before;
    }
    __syncthreads();
    int i = __builtin_amdgcn_readfirstlane(found);
    const int begins = __builtin_amdgcn_readfirstlane(found_start);
    Request r = request(a, i);
    int n = records(r), cost = n + BESIDE, head = (unsigned)(lo - begins) / (unsigned)cost;
    int item = begins + head * cost;   // where the item begins
    while (item < hi) {
        const int first = max(lo - item - BESIDE, 0), last = min(hi - item - BESIDE, n);
        if (n ? last > first : item >= lo) {
            const bool whole = !n || (first == 0 && last == n);   // (an item without records is answered in the share that it begins in, also where its cost goes on in the next)
            if (tid == 0 && first == 0 && (!whole || a.by_item)) {   // it begins here
                Piece& piece = a.cut[a.by_item ? i * a.n_kv + head : share];
                piece.head = whole ? -1 : head;
                piece.share = share, piece.last = (unsigned)(item + cost - 1) / (unsigned)size, piece.row0 = r.row0, piece.rows = r.rows;
            }
            few_rows<T, N>(a, r, i, head, __builtin_amdgcn_readfirstlane(first), __builtin_amdgcn_readfirstlane(last), whole ? -1 : 2LL * share + (first == 0), shared);
        }
        item += cost;
        if (++head == a.n_kv) {
            head = 0;
            if (++i == a.n_seq) break;
            r = request(a, i);
            n = records(r);
            cost = n + BESIDE;
        }
    }
}

// The pieces of a row of an item that was cut, joined in their order: a workgroup to a row of an item, or of the item that begins in a share.  How much of each piece counts is made
// first.  (5 us, a launch and the reads of the record, the statistics and the pieces, which wait for each other.)
template <typename T>
__global__ __launch_bounds__(256) void dbf_attend_join_kernel(const AttendArgs a) {
    __shared__ float keep[MOST_SHARES], total[8];
    __shared__ dbf_f4 sums[256];
    const int tid = threadIdx.x, col = blockIdx.x, D = a.dim, G = a.group, per = D / 4, lanes = 256 / per;
    const Piece item = a.cut[blockIdx.y];
    const int head = item.head, share = item.share, parts = item.last - share + 1;
    if (head < 0 || col >= item.rows * G) return;   // (rows: not more than max_q, or there were no records)
    const int d = tid % per, turn = tid / per;
    auto piece = [&](int p) { return (long long)(2 * (share + p) + (p == 0)) * FEW + col; };
    float m[MOST_SHARES / 256], l[MOST_SHARES / 256], most = LOWEST, sum = 0.f;
#pragma unroll
    for (int k = 0; k < MOST_SHARES / 256; ++k) {
        const int p = tid + 256 * k;
        const float* at = a.part_stat + 2 * piece(min(p, parts - 1));
        m[k] = p < parts ? at[0] : LOWEST;
        l[k] = p < parts ? at[1] : 0.f;
        most = fmaxf(most, m[k]);
    }
    const bool many = parts > 4 * lanes;   // then the first are asked for before it is known how much they count: 131071 tokens 38.5 -> 37.4 us (batch of 64, of few pieces: 69 -> 73)
    constexpr int EARLY = 13;   // (8 key heads of 128 in 768 shares are 96 or 97 pieces, 8 lanes of 12 or 13.  Other sizes have the rest of theirs read below; only this one was timed)
    dbf_f4 early[EARLY], y = {0.f, 0.f, 0.f, 0.f};
    if (many)
#pragma unroll
        for (int k = 0; k < EARLY; ++k) early[k] = *reinterpret_cast<const dbf_f4*>(a.part_out + piece(min(turn + k * lanes, parts - 1)) * D + 4 * d);
    most = dbf_wave_max(most);
    if ((tid & 63) == 0) total[tid >> 6] = most;
    __syncthreads();
    most = fmaxf(fmaxf(total[0], total[1]), fmaxf(total[2], total[3]));
#pragma unroll
    for (int k = 0; k < MOST_SHARES / 256; ++k) {
        const float f = __builtin_amdgcn_exp2f(m[k] - most);
        keep[tid + 256 * k] = f;
        sum = fmaf(f, l[k], sum);
    }
    sum = dbf_wave_sum_f(sum);
    if ((tid & 63) == 0) total[4 + (tid >> 6)] = sum;
    __syncthreads();
    sum = (total[4] + total[5]) + (total[6] + total[7]);
    if (many)
#pragma unroll
        for (int k = 0; k < EARLY; ++k) {
            const int p = turn + k * lanes;
            const float f = p < parts ? keep[p] : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = fmaf(f, p < parts ? early[k][i] : 0.f, y[i]);
        }
#pragma unroll 4
    for (int p = many ? turn + EARLY * lanes : turn; p < parts; p += lanes) {
        const dbf_f4 x = *reinterpret_cast<const dbf_f4*>(a.part_out + piece(p) * D + 4 * d);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = fmaf(keep[p], x[i], y[i]);
    }
    sums[tid] = y;
    __syncthreads();
    if (turn) return;
    for (int k = 1; k < lanes; ++k) y += sums[k * per + d];
    T* out = static_cast<T*>(a.out) + (long long)(item.row0 + col / G) * a.out_stride + (long long)(head * G + col % G) * D + 4 * d;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = dbf_from_float<T>(sum == 0.f ? 0.f : y[i] / sum);
}

// Many rows.  A workgroup takes 32 rows of a request and key head (tokens times the heads that share the keys) to each of its WAVES wavefronts, and walks the tokens in tiles
// of 64: codes from memory to registers while the tile before is worked on, from there as exact fp16 values to LDS, once for all rows.
//   scores:  K q^T, 32 tokens x 32 columns a product; a lane has 32 of a column's 64, the lane 32 on has the others.  The tokens' order is such that the 8 of a lane that
//            follow each other are those of a lane's 16 bytes of values in the cache.
//   output:  V^T p^T, 32 values x 32 columns: the scores' places are the product's operand as they are, since the values' tokens are laid out in that order.
// Both operands lie in LDS as the lanes take them, 16 bytes a lane one after the other.
// Measured: 3 prompts of 2048 causal rows of 32 heads of 128 on 2048 .. 3001 tokens, 165 GFLOP in 204 us, 808 TFLOP/s (a large library product of fp16: 1360).  A SIMD's products take 39 %
// of the time, its vector instructions 55 %, operands' reads from LDS half of what LDS gives: a product of 32 clocks takes 8 clocks of LDS for each of four SIMDs, so that products alone
// keep it busy.  Eight wavefronts a workgroup 214 for 219 us then, and 1.5 times as long for heads of 64 and 256; tiles of 32 tokens for three wavefronts a SIMD 207 for 204; 64 rows a
// wavefront, one a SIMD, 325 for 222; two halves of a workgroup half a step apart 222 for 211; products and vector instructions of a wavefront alternating 227 for 214.

template <int N, int WAVES>
struct Tiles {
    dbf_u4 k[2][2][4 * N][64], v[2][2 * N][4][64];   // [which][record][16 values][lane], [which][32 values][16 tokens][lane]
};

// A thread's share of a tile's bytes, all of one record: keys of a token, runs of 16 values; values of groups, 16 places by 8 tokens of the four.
template <int N, int WAVES>
struct Share {
    static constexpr int RUNS = 4 * N / WAVES > 0 ? 4 * N / WAVES : 1, UNITS = 2 * N / WAVES > 0 ? 2 * N / WAVES : 1;
    static constexpr bool ALL_KEYS = 4 * N >= WAVES, ALL_VALUES = 2 * N >= WAVES;   // whether all wavefronts have some
    dbf_u2 k[RUNS];
    unsigned kw[RUNS];
    dbf_u4 v[UNITS], vw[UNITS][2];

    __device__ __forceinline__ void load(const uint8_t* rec, int lane, int wave) {
        const int token = lane & 31, g = lane >> 4;
        if (ALL_KEYS || wave < 4 * N) {
#pragma unroll
            for (int e = 0; e < RUNS; ++e) {
                const int run = 2 * ((wave >> 1) * RUNS + e) + (lane >> 5);
                k[e] = *reinterpret_cast<const dbf_u2*>(rec + (unsigned)(token * 32 * N + 8 * run));
                kw[e] = *reinterpret_cast<const unsigned*>(rec + (unsigned)(2048 * N + 128 * (run % N) + 4 * token));
            }
        }
        if (ALL_VALUES || wave < 2 * N) {
#pragma unroll
            for (int e = 0; e < UNITS; ++e) {
                const int p = (wave >> 1) * UNITS + e;
                v[e] = *reinterpret_cast<const dbf_u4*>(rec + (unsigned)(1024 * N + 1024 * p + 16 * lane));
#pragma unroll
                for (int t = 0; t < 2; ++t) vw[e][t] = *reinterpret_cast<const dbf_u4*>(rec + (unsigned)(2176 * N + 128 * p + 64 * t + 16 * g));
            }
        }
    }
    // Tokens that are not there (from `there` on, counted from the record's first) and pages that are not: no values, and keys that are no numbers where the page is missing.
    __device__ __forceinline__ void blank(int there, bool known, int lane) {
        if (!known)
#pragma unroll
            for (int e = 0; e < RUNS; ++e) kw[e] = 0x7E007E00u;
#pragma unroll
        for (int e = 0; e < UNITS; ++e)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!known || 16 * t + 4 * (lane >> 4) + i >= there) vw[e][t][i] = 0;
    }
    __device__ __forceinline__ void store(Tiles<N, WAVES>& tiles, int which, int lane, int wave) const {
        if (ALL_KEYS || wave < 4 * N) {
            const int place = (lane & 3) | (lane >> 2 & 1) << 2 | (lane >> 4 & 1) << 3 | (lane >> 3 & 1) << 4;   // the token's among the product's 32
#pragma unroll
            for (int e = 0; e < RUNS; ++e) {
                const dbf_h2 s = lows(kw[e], kw[e]), b = highs(kw[e], kw[e]);
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    unsigned x[4];
                    values(k[e][hf], s, b, s, b, x[0], x[1], x[2], x[3]);
                    tiles.k[which][wave & 1][2 * ((wave >> 1) * RUNS + e) + (lane >> 5)][place + 32 * hf] = (dbf_u4){x[0], x[1], x[2], x[3]};
                }
            }
        }
        const int l = lane & 15, g = lane >> 4, m = 2 * (wave & 1) + (g >> 1);
        if (ALL_VALUES || wave < 2 * N) {
#pragma unroll
            for (int e = 0; e < UNITS; ++e) {
                const int p = (wave >> 1) * UNITS + e;
                dbf_h2 s02[2], b02[2], s13[2], b13[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const dbf_u4 w = vw[e][t];
                    s02[t] = lows(w[0], w[2]), b02[t] = highs(w[0], w[2]), s13[t] = lows(w[1], w[3]), b13[t] = highs(w[1], w[3]);
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    unsigned lo[4], hi[4];
#pragma unroll
                    for (int t = 0; t < 2; ++t) values(v[e][2 * q + t], s02[t], b02[t], s13[t], b13[t], lo[2 * t], lo[2 * t + 1], hi[2 * t], hi[2 * t + 1]);
                    const int low = p + N * 2 * q, high = low + N;
                    tiles.v[which][low >> 1][m][16 * (low & 1) + l + 32 * (g & 1)] = (dbf_u4){lo[0], lo[1], lo[2], lo[3]};
                    tiles.v[which][high >> 1][m][16 * (high & 1) + l + 32 * (g & 1)] = (dbf_u4){hi[0], hi[1], hi[2], hi[3]};
                }
            }
        }
    }
};

// Order of a block's products and reads of operands from LDS: so many reads ahead of all products, then a read behind each product.
template <int PRODUCTS, int READS, int AHEAD>
__device__ __forceinline__ void in_turn() {
    if constexpr (AHEAD > 0) __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int k = 0; k < READS - AHEAD; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS - (READS - AHEAD), 0);
}

__device__ __forceinline__ float both_max(float v) {   // of a lane and the one 32 on
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float both_sum(float v) {
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

template <typename T, int N, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(N == 4 ? 1 : 2))) void dbf_attend_many_kernel(const AttendArgs a) {
    // The values' first operands are under way while the weights are made: 202 -> 199 us for the prompts of 2048, 278 -> 266 for 512 rows on 30000 tokens (heads of 256 have no registers for it)
    constexpr int D = 64 * N, EARLY = N == 4 ? 0 : AHEAD;
    __shared__ Tiles<N, WAVES> tiles;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hf = lane >> 5, G = a.group;
    // (a request's later rows see more: they come first)
    const int head = blockIdx.x % a.n_kv, part = blockIdx.x / a.n_kv, req = blockIdx.y, block = gridDim.z - 1 - blockIdx.z;
    const Request r = request(a, req);
    const int rows = min(r.rows, a.max_q) * G, row0 = block * 32 * WAVES;
    if (row0 >= rows) return;
    const int row = row0 + 32 * wave + (lane & 31), t = row / G;   // the column's row, of the request's token t
    const bool live = row < rows;
    T* out = static_cast<T*>(a.out) + (long long)(r.row0 + (live ? t : 0)) * a.out_stride + (long long)(head * G + (live ? row % G : 0)) * D;
    if (!r.ok) {
        if (live && part == 0)
            for (int d = 4 * hf; d < D; d += 8)
                for (int i = 0; i < 4; ++i) out[d + i] = dbf_from_float<T>(__builtin_nanf(""));
        return;
    }
    // tokens of the workgroup's part that some of its rows see; those that all rows and those that some rows of the wavefront see
    const int last_t = min(row0 + 32 * WAVES, rows) - 1;
    const int begin = part * a.chunk, end = min(a.causal ? r.kv - r.rows + last_t / G + 1 : r.kv, a.parts > 1 ? min(begin + a.chunk, r.kv) : r.kv);
    const int seen = !live ? 0 : a.causal ? r.kv - r.rows + t + 1 : r.kv;
    const int wave_all = a.causal ? r.kv - r.rows + (row0 + 32 * wave) / G + 1 : r.kv;
    const int wave_some = row0 + 32 * wave >= rows ? 0 : a.causal ? r.kv - r.rows + (min(row0 + 32 * wave + 32, rows) - 1) / G + 1 : r.kv;
    const int* table = a.table + (long long)req * a.table_stride;
    const int per_page = a.page_shift - 5, last = (end + 31) / 32 - 1;
    bool known = true;
    auto at = [&](int b, bool& is) {
        b = min(b, last);
        const int page = scalar(table + (b >> per_page));
        is = (unsigned)page < (unsigned)a.n_pages;
        return a.cache + ((((long long)(is ? page : 0) * a.n_kv + head) << per_page) + (b & ((1 << per_page) - 1))) * dbf_record_bytes(D);
    };
    Share<N, WAVES> share;
    auto load = [&](int first) { share.load(at(first / 32 + (wave & 1), known), lane, wave); };
    auto store = [&](int first, int which) {
        if (first + TILE > r.kv || !known) {
            asm volatile("");
            share.blank(r.kv - first - 32 * (wave & 1), known, lane);
        }
        share.store(tiles, which, lane, wave);
    };
    if (begin < end) load(begin);
    // the column's query: of each 16 values the lane's 8, in the order of a word's codes
    dbf_h8 q[4 * N];
    float kappa;
    {
        const T* x = static_cast<const T*>(a.q) + (long long)(r.row0 + (live ? t : 0)) * a.q_stride + (long long)(head * G + (live ? row % G : 0)) * D + 8 * hf;
        float most = 0.f;
        for (int k = 0; k < 4 * N; ++k) {
            float v[8];
            load8(x + 16 * k, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, live ? fabsf(v[e]) : 0.f);
        }
        most = both_max(most);
        const int up = most > 0.f && most < __builtin_inff() ? 15 - __builtin_amdgcn_frexp_expf(most) : 0;
        // (not 0: what is masked is -infinity times it; no more than 2^80: sums of products are below 2^40 and, where they differ, 2^-48 apart at least, as for few rows)
        kappa = fminf(fmaxf(ldexpf(fabsf(a.scale) * 1.44269504089f, -up), 0x1p-126f), 0x1p80f);
#pragma unroll
        for (int k = 0; k < 4 * N; ++k) {
            float v[8];
            load8(x + 16 * k, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = live ? ldexpf(v[4 * (e & 1) + (e & 2) + (e >> 2)], up) : 0.f;
                q[k][e] = (_Float16)(a.scale < 0.f ? -y : y);
            }
        }
    }
    dbf_f16 o[2 * N] = {};
    float m = LOWEST, l = 0.f;
    // A weight's exponent is one rounding of x kappa + (7 - m), so what m's own rounding lost comes into all weights alike: a factor of 2^(half a unit of m), which nothing notices unless it takes them
    // out of fp16's range.  So once some |m| is above FAR, x is rounded to the score first, as m is: the largest is then m itself.
    constexpr float FAR = 0x1p20f;
    bool far = false;
    float by = kappa;   // from what x holds to scores
    if (begin < end) store(begin, 0);
    int which = 0;
    for (int first = begin; first < end; first += TILE, which ^= 1) {
        __syncthreads();
        const bool more = first + TILE < end;
        if (more) load(first + TILE);
        if (first < wave_some) {
            dbf_f16 x[2] = {};
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int k = 0; k < 4 * N; ++k)
                    x[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(dbf_h8, tiles.k[which][b][k][lane]), q[k], x[b], 0, 0, 0);
            dbf_h8 early[EARLY + 1];
#pragma unroll
            for (int n = 0; n < EARLY; ++n) early[n] = __builtin_bit_cast(dbf_h8, tiles.v[which][n % (2 * N)][n / (2 * N)][lane]);
            in_turn<8 * N, 8 * N + EARLY, AHEAD>();
            if (first + TILE > wave_all) {
                asm volatile("");
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[b][i] = first + 32 * b + 16 * (i >> 2 & 1) + 8 * (i >> 3) + 4 * hf + (i & 3) < seen ? x[b][i] : -__builtin_inff();
            }
            if (far) {
                asm volatile("");
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[b][i] *= kappa;
            }
            // Weights by the maximum so far, times 2^7; their sum says whether one of them is too large for fp16 or far above the others' place: then the maximum is raised and they
            // are made again, else nobody looks for it.  (Sums of the rounded weights, which the product below has: subnormal ones count here as they do there.)
            unsigned weights[4][4];
            auto weigh = [&] {
                const float from = 7.f - m;
                float sum[4] = {};   // (one after the other they wait for each other: 206 -> 203 us)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; i += (i & 1) ? 3 : 1) {
                        const dbf_h2 w = {(_Float16)__builtin_amdgcn_exp2f(fmaf(x[b][i], by, from)), (_Float16)__builtin_amdgcn_exp2f(fmaf(x[b][i + 2], by, from))};
                        sum[2 * b + (i & 1)] = __builtin_amdgcn_fdot2(w, (dbf_h2){(_Float16)1.f, (_Float16)1.f}, sum[2 * b + (i & 1)], false);
                        weights[2 * b + (i >> 3)][2 * (i >> 2 & 1) + (i & 1)] = __builtin_bit_cast(unsigned, w);
                    }
                return (sum[0] + sum[1]) + (sum[2] + sum[3]);
            };
            float sum = weigh();
            if (__any(!(sum <= 0x1p15f))) {   // (also where it is no number)
                float most = x[0][0];
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most = fmaxf(most, x[b][i]);
                const float to = fmaxf(m, both_max(most * by)), keep = __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= keep;
#pragma unroll
                for (int j = 0; j < 2 * N; ++j) o[j] *= keep;
                if (!far && __any(fabsf(m) > FAR && m != LOWEST)) {
                    far = true;
                    by = 1.f;
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[b][i] *= kappa;
                }
                sum = weigh();
            }
            l += sum;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 2 * N; ++j)
                    o[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(2 * N * k + j < EARLY ? early[2 * N * k + j] : __builtin_bit_cast(dbf_h8, tiles.v[which][j][k][lane]), __builtin_bit_cast(dbf_h8, (dbf_u4){weights[k][0], weights[k][1], weights[k][2], weights[k][3]}), o[j], 0, 0, 0);
            in_turn<8 * N, 8 * N - EARLY, EARLY ? 0 : AHEAD>();
        }
        if (more) store(first + TILE, which ^ 1);
    }
    l = both_sum(l);
    if (!live) return;
    if (a.parts == 1) {
        const float by = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int j = 0; j < 2 * N; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) out[32 * j + 8 * (i >> 2) + 4 * hf + (i & 3)] = dbf_from_float<T>(o[j][i] * by);
        return;
    }
    const long long piece = (((long long)req * a.n_kv + head) * a.parts + part) * (a.max_q * G) + row;
    if (hf == 0) {
        a.part_stat[2 * piece] = m;
        a.part_stat[2 * piece + 1] = l;
    }
#pragma unroll
    for (int j = 0; j < 2 * N; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *reinterpret_cast<dbf_f4*>(a.part_out + piece * D + 32 * j + 8 * k + 4 * hf) = (dbf_f4){o[j][4 * k], o[j][4 * k + 1], o[j][4 * k + 2], o[j][4 * k + 3]};
}

// The parts of the rows of such a call: head_dim / 4 lanes to a row.
template <typename T>
__global__ __launch_bounds__(256) void dbf_attend_parts_kernel(const AttendArgs a) {
    const int D = a.dim, per = D / 4, G = a.group, head = blockIdx.y, req = blockIdx.z, row = blockIdx.x * (256 / per) + threadIdx.x / per, d = 4 * (threadIdx.x % per);
    const Request r = request(a, req);
    if (row >= min(r.rows, a.max_q) * G || !r.ok) return;
    const long long step = (long long)a.max_q * G, first = ((long long)req * a.n_kv + head) * a.parts * step + row;
    const int parts = min(a.parts, (r.kv + a.chunk - 1) / a.chunk);   // (those behind have no token of the request)
    float m = LOWEST, l = 0.f;
    dbf_f4 y = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; ++p) m = fmaxf(m, a.part_stat[2 * (first + p * step)]);
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
        const long long at = first + p * step;
        const float keep = __builtin_amdgcn_exp2f(a.part_stat[2 * at] - m);
        l = fmaf(keep, a.part_stat[2 * at + 1], l);
        const dbf_f4 x = *reinterpret_cast<const dbf_f4*>(a.part_out + at * D + d);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = fmaf(keep, x[i], y[i]);
    }
    T* out = static_cast<T*>(a.out) + (long long)(r.row0 + row / G) * a.out_stride + (long long)(head * G + row % G) * D + d;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = dbf_from_float<T>(l == 0.f ? 0.f : y[i] / l);
}

int check_attend(const dbf_attend* a, const dbf_cache* c) {   // (sizes: a workspace may be asked for before there are pointers)
    if (!a) return DBF_EINVAL;
    if (const int bad = dbf_cache_check_sizes(c)) return bad;
    if (a->dtype != DBF_F16 && a->dtype != DBF_BF16) return DBF_EINVAL;
    if (a->n_seq < 1 || a->n_seq > 65535 || a->n_tokens < 0 || a->max_q < 0 || a->max_kv < 0 || a->max_kv > 1 << 30 || a->table_stride < 1) return DBF_EINVAL;
    if (a->n_q_heads < 1 || a->n_q_heads > 65535) return DBF_EINVAL;
    if (a->n_q_heads % c->n_kv_heads) return DBF_ESHAPE;
    if ((long long)a->max_q * (a->n_q_heads / c->n_kv_heads) > MOST_ROWS) return DBF_EINVAL;
    if (!(a->scale > -3.0e38f && a->scale < 3.0e38f)) return DBF_EINVAL;
    return DBF_OK;
}

// How a call is run, and what its workspace holds.
struct Cut {
    bool few;
    int shares, joins;  // few rows; 0: a workgroup to an item; of a join's launch, items where they are fewer than shares
    int chunk, parts;   // many rows
    size_t cut_bytes, stat_bytes, out_bytes;
};
Cut cut_of(const dbf_attend* a, const dbf_cache* c) {
    Cut k = {};
    // One form for the whole call: lengths are not known here.  Single tokens beside a prompt pay for that, 63 of 1 .. 8192 tokens and 512 rows on 8192 (32 heads on 8) take 489 us, and 69 and 95 in two calls.
    k.few = (long long)a->max_q * (a->n_q_heads / c->n_kv_heads) <= FEW;
    // Items are shared out where the longest may be more than a workgroup should have: 1200 tokens, and more the more items there are to fill the chip beside it.  us, an item to a
    // workgroup and shared out: 8 items of 1000 tokens 10.7 and 11.4, of 1500 14.1 and 12.6, of 4000 29 and 14; 64 of 2500 20 and 17; 256 of 2500 22 and 27, of 4000 32 and 37; 512 of 1 .. 4000
    // 43 and 39 (the rule leaves them unshared: it knows the longest request only), of 4000 52 and 62, of 1 .. 8192 79 and 63; 1600 of 1 .. 3000 77 and 84; 2400 of 1 .. 2500 90 and 114.
    const long long items = (long long)a->n_seq * c->n_kv_heads;
    if (k.few && a->max_kv > 1200 + 11 * items && items * (a->max_kv / 32 + 1 + BESIDE) < 1 << 30) {   // (and the sum of all costs fits: no memory holds more, but tables may say so)
        k.shares = 256 * few_waves(c->head_dim / 64);
        k.joins = (int)std::min<long long>(k.shares, items);
        k.cut_bytes = ((size_t)k.joins * sizeof(Piece) + 255) / 256 * 256;
        k.stat_bytes = (size_t)k.shares * 2 * FEW * 8;
        k.out_bytes = (size_t)k.shares * 2 * FEW * c->head_dim * 4;
    }
    k.chunk = INT_MAX;
    k.parts = 1;
    if (!k.few && a->max_q > 0) {
        // The long axis in parts where the rows alone are few workgroups, of LEAST_CHUNK tokens at least
        const long long rows = (long long)a->max_q * (a->n_q_heads / c->n_kv_heads), groups = (rows + 32 * MANY_WAVES - 1) / (32 * MANY_WAVES) * c->n_kv_heads * a->n_seq;
        const long long parts = std::min<long long>((512 + groups - 1) / groups, (a->max_kv + LEAST_CHUNK - 1) / LEAST_CHUNK);
        if (parts > 1) {
            k.chunk = (int)(((a->max_kv + parts - 1) / parts + TILE - 1) / TILE * TILE);
            k.parts = (a->max_kv + k.chunk - 1) / k.chunk;
        }
        if (k.parts > 1) {
            const size_t n = (size_t)rows * c->n_kv_heads * a->n_seq * k.parts;
            k.stat_bytes = (n * 8 + 255) / 256 * 256;
            k.out_bytes = n * c->head_dim * 4;
        }
    }
    return k;
}

template <typename T, int N>
void launch_few(const AttendArgs& a, int shares, int joins, hipStream_t stream) {
    if (!shares) {
        hipLaunchKernelGGL((dbf_attend_items_kernel<T, N>), dim3(a.n_kv, a.n_seq), dim3(256), 0, stream, a);
        return;
    }
    hipLaunchKernelGGL((dbf_attend_shares_kernel<T, N>), dim3(shares), dim3(256), 0, stream, a);
    hipLaunchKernelGGL(dbf_attend_join_kernel<T>, dim3(a.max_q * a.group, joins), dim3(256), 0, stream, a);
}
template <typename T>
void launch_many(const AttendArgs& a, hipStream_t stream) {
    const int rows = a.max_q * a.group, blocks = (rows + 32 * MANY_WAVES - 1) / (32 * MANY_WAVES), across = a.n_kv * a.parts;   // (parts: one where the blocks of all heads are 512)
    const auto kernel = a.dim == 64 ? dbf_attend_many_kernel<T, 1, MANY_WAVES> : a.dim == 128 ? dbf_attend_many_kernel<T, 2, MANY_WAVES> : dbf_attend_many_kernel<T, 4, MANY_WAVES>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)across, a.n_seq, (unsigned)blocks), dim3(64 * MANY_WAVES), 0, stream, a);
    const int of = 256 / (a.dim / 4);
    if (a.parts > 1) hipLaunchKernelGGL(dbf_attend_parts_kernel<T>, dim3((unsigned)((rows + of - 1) / of), a.n_kv, a.n_seq), dim3(256), 0, stream, a);
}
template <typename T>
int launch_attend(const AttendArgs& a, const Cut& cut, hipStream_t stream) {
    if (!cut.few) launch_many<T>(a, stream);
    else if (a.dim == 64) launch_few<T, 1>(a, cut.shares, cut.joins, stream);
    else if (a.dim == 128) launch_few<T, 2>(a, cut.shares, cut.joins, stream);
    else launch_few<T, 4>(a, cut.shares, cut.joins, stream);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}

}  // namespace

extern "C" size_t dbf_cache_attend_workspace_bytes(const dbf_attend* attend, const dbf_cache* cache) {
    if (check_attend(attend, cache)) return 0;
    const Cut cut = cut_of(attend, cache);
    return cut.cut_bytes + cut.stat_bytes + cut.out_bytes;
}

extern "C" int dbf_cache_attend(const dbf_attend* attend, const dbf_cache* cache, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    if (const int bad = dbf_cache_check(cache)) return bad;
    if (const int bad = check_attend(attend, cache)) return bad;
    const long long row = (long long)attend->n_q_heads * cache->head_dim;
    if (!attend->q || !attend->out || !attend->kv_len || !attend->block_table || attend->q_stride < row || attend->out_stride < row) return DBF_EINVAL;
    if (dbf_misaligned(attend->q, 2) || dbf_misaligned(attend->out, 2)) return DBF_EINVAL;
    for (const int32_t* p : {attend->q_start, attend->kv_len, attend->block_table})
        if (dbf_misaligned(p, 4)) return DBF_EINVAL;
    if (!attend->n_tokens || !attend->max_q) return DBF_OK;
    AttendArgs a = {};
    a.q = attend->q;  a.out = attend->out;  a.q_stride = attend->q_stride;  a.out_stride = attend->out_stride;
    a.q_start = attend->q_start;  a.kv_len = attend->kv_len;  a.table = attend->block_table;
    a.cache = static_cast<const uint8_t*>(cache->data);
    a.n_tokens = attend->n_tokens;  a.n_seq = attend->n_seq;  a.n_q = attend->n_q_heads;  a.n_kv = cache->n_kv_heads;
    a.max_q = attend->max_q;  a.max_kv = attend->max_kv;  a.table_stride = attend->table_stride;  a.causal = attend->causal;
    a.n_pages = cache->n_pages;  a.page_shift = dbf_page_shift(cache->page_tokens);  a.dim = cache->head_dim;  a.scale = attend->scale;
    const Cut cut = cut_of(attend, cache);
    if (cut.out_bytes) {
        if (!workspace_dev || dbf_misaligned(workspace_dev, 256) || workspace_bytes < cut.cut_bytes + cut.stat_bytes + cut.out_bytes) return DBF_EWORKSPACE;
        char* at = static_cast<char*>(workspace_dev);
        a.cut = reinterpret_cast<Piece*>(at);
        a.part_stat = reinterpret_cast<float*>(at + cut.cut_bytes);
        a.part_out = reinterpret_cast<float*>(at + cut.cut_bytes + cut.stat_bytes);
    }
    a.group = a.n_q / a.n_kv;  a.chunk = cut.chunk;  a.parts = cut.parts;  a.by_item = cut.joins < cut.shares;
    const auto stream = static_cast<hipStream_t>(hip_stream);
    return attend->dtype == DBF_F16 ? launch_attend<_Float16>(a, cut, stream) : launch_attend<dbf_bf16>(a, cut, stream);
}
