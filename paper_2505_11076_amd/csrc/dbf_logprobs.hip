// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits (include/dbf.h, dbf_token_logprobs).
//
// One read of the logits, with a maximum m that may lag and the sums s = sum e^(x - m), t = sum e^(x - m) (x - m) of what has been read, in fp32:
//     log sum e^x = m + log s,      entropy = log s - t / s.
// 32 terms make a sum of their own, and what is rounded off where that is added is kept for the next.
// The likeliest tokens: all values have keys (value, then the lower index) that differ.  A thread keeps its largest, four threads theirs; the n-th largest of these 64 is a
// bound that the n largest of all are not below, and only threads whose largest key is not below it can hold any: their values are read once more (from the cache), the
// few that pass are put in order.
// A row is one workgroup's, or where rows are few the slices of several, whose sums and lists a second launch joins.
// Where rows are many the read and the vector instructions share the time: 2048 rows of 32000 fp16, 131 MB in 27 us (4.85 TB/s), where a read alone has 20; a value costs about nine issue slots (its
// exponential four), vector units are 77 % busy and waves wait 45 % of their time for issue.  With 20 alternatives 43 us.  One row of 128256 with 20 alternatives: 7.6 us and 4.2 of the join, latencies.
// Rows of more than ROOM values, but fewer than 32 for each alternative, have no bound: everything passes, there is no room for it, and the likeliest are looked for one by one (2048 rows of 1500
// with 64: 145 us).
#include <algorithm>
#include <climits>

#include "dbf_cache.h"
#include "dbf_wave.h"

namespace {

constexpr int THREADS = 256, MOST_TOP = 64, RUN = 8;   // values of a thread's load
constexpr int ROOM = 1024;                             // values that may pass
typedef unsigned long long u64;

struct Sums {
    float m, s, t;
};
struct LogprobArgs {
    const void* x;
    long long stride;
    const int* targets;
    float *logprob, *entropy, *top_logprobs;
    int* top_ids;
    int n_rows, vocab, n_top, slices, slice;   // slices of a row, and values of one (a multiple of RUN)
    Sums* part_sums;                           // [row][slice]
    u64* part_top;                             // [row][slice][n_top], largest first; 0: there is none
};

// Larger values first, no numbers before all, then lower indexes; never 0.  (+ 0: -0 is 0.)
__device__ __forceinline__ u64 key_of(float v, int i) {
    const unsigned b = __builtin_bit_cast(unsigned, v + 0.0f);
    const unsigned order = v != v ? 0xFFFFFFFFu : (b >> 31) ? ~b : b | 0x80000000u;
    return (u64)order << 32 | (unsigned)~i;
}
__device__ __forceinline__ float value_of(u64 key) {
    const unsigned order = (unsigned)(key >> 32);
    if (order == 0xFFFFFFFFu) return __builtin_nanf("");
    return __builtin_bit_cast(float, (order >> 31) ? order & 0x7FFFFFFFu : ~order);
}

constexpr float LEAST = -3.402823466e38f;   // of a maximum: no finite value is below it (or above -LEAST), and -infinity less it is not a number's absence
// A difference from the maximum, whose exponential is nothing below -104: held to what a product with nothing leaves nothing.
__device__ __forceinline__ float below(float d) { return fmaxf(d, -200.f); }

// Of two parts.  (A part of nothing has s = t = 0.  s that is no number stays that.)
__device__ __forceinline__ Sums join(Sums a, Sums b) {
    Sums r;
    r.m = fmaxf(a.m, b.m);
    const float da = below(a.m - r.m), db = below(b.m - r.m), ea = __builtin_amdgcn_exp2f(da * 1.44269504089f), eb = __builtin_amdgcn_exp2f(db * 1.44269504089f);
    r.s = a.s * ea + b.s * eb;
    r.t = fmaf(a.s, da, a.t) * ea + fmaf(b.s, db, b.t) * eb;
    return r;
}
__device__ __forceinline__ float log_of(float s) { return s > 0.f ? __builtin_amdgcn_logf(s) * 0.693147181f : __builtin_nanf(""); }
__device__ __forceinline__ Sums wave_join(Sums v) {
    Sums r;
    r.m = dbf_wave_max(v.m);
    const float d = below(v.m - r.m), e = __builtin_amdgcn_exp2f(d * 1.44269504089f);
    r.s = dbf_wave_sum_f(v.s * e);
    r.t = dbf_wave_sum_f(fmaf(v.s, d, v.t) * e);
    return r;
}

// Values i .. i + 7 of n values that end a row, or a slice of one, of RUN at least: a run that overlaps the end is read as the last eight (also of the slice before), and
// what is not there is -infinity.  The loads have no use of their own, so several may be under way.
template <typename T>
struct Run {
    dbf_u4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* x, int i, int n) {
        const T* at = x + min(i, n - RUN);
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) w[k] = reinterpret_cast<const dbf_u4_any*>(at)[k];
    }
    __device__ __forceinline__ void get(int i, int n, float (&v)[RUN]) const {
#pragma unroll
        for (int e = 0; e < RUN; ++e) {
            if constexpr (sizeof(T) == 4) v[e] = __builtin_bit_cast(float, (unsigned)w[e >> 2][e & 3]);
            else v[e] = dbf_to_float(__builtin_bit_cast(T, (uint16_t)(w[0][e >> 1] >> 16 * (e & 1))));
        }
        if (i + RUN > n) {   // (the row's last eight values, of which the last n - i are wanted; or none)
            const int skip = i + RUN - n;
#pragma unroll
            for (int e = 0; e < RUN; ++e) v[e] = e < skip ? -__builtin_inff() : v[e];
        }
    }
};
// The keys of run i of x[0 .. n) to out; base: the index of x[0].
template <typename T, typename Out>
__device__ __forceinline__ void keys_of_run(const T* x, int i, int n, int base, Out out) {
    Run<T> run;
    run.load(x, i, n);
    float v[RUN];
    run.get(i, n, v);
    const int at = min(i, n - RUN);
#pragma unroll
    for (int e = 0; e < RUN; ++e)
        if (at + e >= i) out(key_of(v[e], base + at + e));
}
typedef u64 two __attribute__((ext_vector_type(2)));
// The n-th largest of 64 keys in LDS (0: none); 1 if there are no n.  Every wavefront for itself.  (For 256 keys 64-bit comparisons were 4 us, and a search bit by bit as much: a step of it
// is a chain from vector compare to scalar count and back.)
__device__ __forceinline__ u64 bound_of(const u64* keys, int n) {
    const u64 own = keys[threadIdx.x & 63];
    int larger = 0;
#pragma unroll 8
    for (int k = 0; k < 32; ++k) {
        const two v = reinterpret_cast<const two*>(keys)[k];
        larger += (v[0] > own) + (v[1] > own);
    }
    const u64 at = __ballot(own && larger == n - 1);
    if (!at) return 1;
    return __shfl(own, __ffsll((unsigned long long)at) - 1);
}

// The n largest of keys[0 .. count) (LDS, all different), in order, by how many are larger; out(place, key).  (Sixteen to a step, those behind the last looked at for nothing: read one
// by one 260 keys took 9 us.)
template <typename Out>
__device__ __forceinline__ void in_order(const u64* keys, int count, int n, Out out) {
    for (int i = threadIdx.x; i < count; i += THREADS) {
        const u64 own = keys[i];
        int larger = 0;
        for (int k = 0; k < count; k += 16) {
            two v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = reinterpret_cast<const two*>(keys + k)[e];
#pragma unroll
            for (int e = 0; e < 16; ++e) larger += (v[e >> 1][e & 1] > own) & (k + e < count);
        }
        if (larger < n) out(larger, own);
    }
}

struct Work {
    alignas(16) u64 groups[64];   // largest of four threads each
    u64 keys[THREADS];
    alignas(16) u64 passed[ROOM];   // (a multiple of 16)
    int chosen[THREADS], holders, count;
    Sums sums[THREADS / 64];
};

// The n_top largest keys of x[0 .. n), in order; `best` is the thread's largest, of its runs tid, tid + THREADS, ...; base: the index of x[0] in its row.
template <typename T, typename Out>
__device__ __forceinline__ void likeliest(const T* x, int n, int base, u64 best, int n_top, Work& work, Out out) {
    const int tid = threadIdx.x, wanted = min(n_top, n);
    u64 four = max(best, __shfl_xor(best, 1));
    four = max(four, __shfl_xor(four, 2));
    if ((tid & 3) == 0) work.groups[tid >> 2] = four;
    if (tid == 0) work.count = work.holders = 0;
    __syncthreads();
    const u64 bound = bound_of(work.groups, wanted);
    if (best >= bound) work.chosen[atomicAdd(&work.holders, 1)] = tid;   // (in any order: it is only a list)
    __syncthreads();
    const int holders = work.holders;
    const int runs = (n + RUN - 1) / RUN, each = (runs + THREADS - 1) / THREADS;
    for (int k = tid; k < holders * each; k += THREADS) {
        const int run = work.chosen[k % holders] + k / holders * THREADS;
        if (run >= runs) continue;
        auto pass = [&](u64 key) {
            if (key < bound) return;
            const int at = atomicAdd(&work.count, 1);   // (in any order: they are put in order by their keys)
            if (at < ROOM) work.passed[at] = key;
        };
        keys_of_run(x, run * RUN, n, base, pass);
    }
    __syncthreads();
    const int count = work.count;
    if (__builtin_expect(count <= ROOM, 1)) {
        in_order(work.passed, count, wanted, out);
    } else {   // rows made so that few threads hold thousands of the largest: one after the other
        u64 last = ~0ull;
#pragma unroll 1
        for (int k = 0; k < wanted; ++k) {
            u64 top = 0;
#pragma unroll 1
            for (int i = tid; i < n; i += THREADS) {
                const u64 key = key_of(dbf_to_float(x[i]), base + i);
                if ((k == 0 || key < last) && key > top) top = key;
            }
            __syncthreads();
            work.keys[tid] = top;
            __syncthreads();
            for (int d = THREADS / 2; d; d /= 2) {
                if (tid < d) work.keys[tid] = max(work.keys[tid], work.keys[tid + d]);
                __syncthreads();
            }
            last = work.keys[0];
            if (tid == 0) out(k, last);
        }
    }
}

// A sum and what it has lost so far: with one more term, whose rounding goes there.  (Added one by one, equal terms lose the same each time: 3e-5 of a sum of 586, 1e-3 of 65536.)
__device__ __forceinline__ float add(float sum, float term, float& lost) {
    const float wanted = term - lost, next = sum + wanted;
    lost = (next - sum) - wanted;
    return next;
}

// A row's target and its logit, asked for before anything else.
struct Target {
    int id;
    float value;
    template <typename T>
    __device__ __forceinline__ Target(const LogprobArgs& a, int row, const T* x, bool asked) : id(-1), value(0.f) {
        if (!asked || !a.logprob) return;
        id = a.targets[row];
        if (id >= 0 && id < a.vocab) value = dbf_to_float(x[id]);
    }
};
__device__ __forceinline__ void finish(const LogprobArgs& a, int row, Sums s, const Target& target, float log_s) {
    if (a.logprob) a.logprob[row] = target.id < 0 ? 0.f : target.id >= a.vocab ? __builtin_nanf("") : (target.value - s.m) - log_s;
    if (a.entropy) a.entropy[row] = log_s - s.t / s.s;
}

template <typename T, bool TOP>
__global__ __launch_bounds__(THREADS) void dbf_logprobs_kernel(const LogprobArgs a) {
    __shared__ Work work;
    const int tid = threadIdx.x, row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices, base = slice * a.slice, n = min(a.slice, a.vocab - base);
    const T* x = static_cast<const T*>(a.x) + row * a.stride + base;
    const Target target(a, row, static_cast<const T*>(a.x) + row * a.stride, tid == 0 && a.slices == 1);
    Sums s = {LEAST, 0.f, 0.f};
    float most = -__builtin_inff(), lost_s = 0.f, lost_t = 0.f;
    int most_run = INT_MAX;   // the first run that holds it
    constexpr int AHEAD = 4, STEP = THREADS * RUN * AHEAD;
    Run<T> run[AHEAD];
    for (int i0 = tid * RUN; i0 < n; i0 += STEP) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) run[k].load(x, i0 + k * THREADS * RUN, n);
        float v[AHEAD][RUN], top = -__builtin_inff();
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k * THREADS * RUN;
            run[k].get(i, n, v[k]);
            float largest = v[k][0];
#pragma unroll
            for (int e = 1; e < RUN; ++e) largest = fmaxf(largest, v[k][e]);
            if (TOP && i < n && (largest > most || most_run == INT_MAX)) {
                most = largest;
                most_run = i;
            }
            top = fmaxf(top, largest);
        }
        if (top > s.m + 8.f) {   // (rarely, once the first run is read)
            const Sums o = s;
            s = join(o, (Sums){fminf(top, -LEAST), 0.f, 0.f});   // (of a finite row the largest is its maximum as it is)
            lost_s = lost_t = 0.f;
        }
        float add_s = 0.f, add_t = 0.f;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int e = 0; e < RUN; ++e) {
                const float d = v[k][e] - s.m, w = __builtin_amdgcn_exp2f(d * 1.44269504089f);
                add_s += w;
                add_t = fmaf(w, below(d), add_t);
            }
        s.s = add(s.s, add_s, lost_s);
        s.t = add(s.t, add_t, lost_t);
    }
    const bool number = s.s < __builtin_inff() && s.t == s.t;   // (a logit of +infinity makes the sum that)
    s = wave_join(s);
    if ((tid & 63) == 0) work.sums[tid >> 6] = s;
    const bool numbers = !__syncthreads_or(!number);   // of the workgroup's part
    s = join(join(work.sums[0], work.sums[1]), join(work.sums[2], work.sums[3]));
    if (!numbers) s.s = s.t = __builtin_nanf("");
    const float log_s = log_of(s.s);
    if (tid == 0) {
        if (a.slices == 1) {
            finish(a, row, s, target, log_s);
        } else {
            a.part_sums[(long long)row * a.slices + slice] = s;
        }
    }
    if (!TOP) return;
    // the thread's largest key: the first of its values that is as large as any (or is no number)
    u64 best = 0;
    auto keep = [&](u64 key) { best = max(best, key); };
    if (__builtin_expect(numbers, 1)) {
        if (most_run != INT_MAX) keys_of_run(x, most_run, n, base, keep);
    } else {
#pragma unroll 1
        for (int i = tid * RUN; i < n; i += THREADS * RUN) keys_of_run(x, i, n, base, keep);
    }
    const long long list = ((long long)row * a.slices + slice) * a.n_top;   // (of the row itself if it has one slice)
    if (a.slices > 1)
        for (int k = n + tid; k < a.n_top; k += THREADS) a.part_top[list + k] = 0;
    likeliest(x, n, base, best, a.n_top, work, [&](int k, u64 key) {
        if (a.slices > 1) {
            a.part_top[list + k] = key;
        } else {
            a.top_ids[list + k] = (int)~(unsigned)key;
            a.top_logprobs[list + k] = (value_of(key) - s.m) - log_s;
        }
    });
}

// Rows of fewer than RUN tokens: a thread to each.
template <typename T>
__global__ __launch_bounds__(THREADS) void dbf_logprobs_short_kernel(const LogprobArgs a) {
    const int row = blockIdx.x * THREADS + threadIdx.x;
    if (row >= a.n_rows) return;
    const T* x = static_cast<const T*>(a.x) + row * a.stride;
    Sums s = {LEAST, 0.f, 0.f};
    for (int i = 0; i < a.vocab; ++i) {
        const float v = dbf_to_float(x[i]);
        s = join(s, (Sums){fminf(fmaxf(v, LEAST), -LEAST), v - v == 0.f ? 1.f : v == -__builtin_inff() ? 0.f : __builtin_nanf(""), 0.f});
    }
    const float log_s = log_of(s.s);
    finish(a, row, s, Target(a, row, x, true), log_s);
    u64 last = ~0ull;
    for (int k = 0; k < a.n_top; ++k) {
        u64 top = 0;
        for (int i = 0; i < a.vocab; ++i) {
            const u64 key = key_of(dbf_to_float(x[i]), i);
            if ((k == 0 || key < last) && key > top) top = key;
        }
        last = top;
        a.top_ids[(long long)row * a.n_top + k] = (int)~(unsigned)top;
        a.top_logprobs[(long long)row * a.n_top + k] = (value_of(top) - s.m) - log_s;
    }
}

// The slices of a row.
template <typename T>
__global__ __launch_bounds__(THREADS) void dbf_logprobs_join_kernel(const LogprobArgs a) {
    __shared__ Work work;
    const int tid = threadIdx.x, row = blockIdx.x;
    const Sums nothing = {LEAST, 0.f, 0.f};
    Sums s = tid < a.slices ? a.part_sums[(long long)row * a.slices + tid] : nothing;   // (slices <= THREADS)
    const u64* lists = a.part_top + (long long)row * a.slices * a.n_top;
    const Target target(a, row, static_cast<const T*>(a.x) + row * a.stride, tid == 0);
    u64 first = 0, listed[ROOM / THREADS];
    if (a.n_top) {
        const int of_each = min(64 / a.slices, a.n_top);   // (slices <= 64)
        if (tid < a.slices * of_each) first = lists[(long long)(tid / of_each) * a.n_top + tid % of_each];
#pragma unroll
        for (int k = 0; k < ROOM / THREADS; ++k) listed[k] = tid + k * THREADS < a.slices * a.n_top ? lists[tid + k * THREADS] : 0;
    }
    const bool number = s.s == s.s;
    s = wave_join(s);
    if ((tid & 63) == 0) work.sums[tid >> 6] = s;
    const bool numbers = !__syncthreads_or(!number);
    s = join(join(work.sums[0], work.sums[1]), join(work.sums[2], work.sums[3]));
    if (!numbers) s.s = s.t = __builtin_nanf("");
    const float log_s = log_of(s.s);
    if (tid == 0) {
        finish(a, row, s, target, log_s);
    }
    if (!a.n_top) return;
    // the same bound again: of the slices' largest, as many of each as there is room for (of the largest alone there is none for 13 slices and 20 alternatives: 4 rows of 53000 20.7 us)
    if (tid < 64) work.groups[tid] = first;
    if (tid == 0) work.count = 0;
    __syncthreads();
    const u64 bound = bound_of(work.groups, a.n_top);
#pragma unroll
    for (int k = 0; k < ROOM / THREADS; ++k)
        if (listed[k] >= bound) work.passed[atomicAdd(&work.count, 1)] = listed[k];   // (all lists together have room)
    __syncthreads();
    in_order(work.passed, work.count, a.n_top, [&](int k, u64 key) {
        a.top_ids[(long long)row * a.n_top + k] = (int)~(unsigned)key;
        a.top_logprobs[(long long)row * a.n_top + k] = (value_of(key) - s.m) - log_s;
    });
}

bool sizes_ok(int n_rows, int vocab, int n_top) { return n_rows >= 0 && vocab >= 1 && vocab <= (1 << 24) && n_top >= 0 && n_top <= MOST_TOP && n_top <= vocab; }

// Slices of a row: one where the rows alone fill the chip.  A slice has 4096 values at least, and there are no more than ROOM / n_top of them, so that a join's lists have room.
int slices_of(int n_rows, int vocab, int n_top) {
    const int fill = (768 + n_rows - 1) / std::max(n_rows, 1);
    return std::max(1, std::min({fill, (vocab + 4095) / 4096, 64, n_top ? ROOM / n_top : 64}));
}
struct Room {
    size_t sums, top;
};
Room room_of(int n_rows, int vocab, int n_top) {
    const int slices = slices_of(n_rows, vocab, n_top);
    if (slices == 1) return {0, 0};
    const size_t n = (size_t)n_rows * slices;
    return {(n * sizeof(Sums) + 255) / 256 * 256, n * n_top * sizeof(u64)};
}

template <typename T>
int launch(const LogprobArgs& all, hipStream_t stream) {
    constexpr long long MOST_ROWS = 1 << 23;   // of a launch: of 2^32 threads or more only the remainder would run (more than one slice have only fewer rows)
    for (long long row = 0; row < all.n_rows; row += MOST_ROWS) {
        LogprobArgs a = all;
        a.n_rows = (int)std::min(MOST_ROWS, all.n_rows - row);
        a.x = static_cast<const T*>(a.x) + row * a.stride;
        if (a.targets) a.targets += row, a.logprob += row;
        if (a.entropy) a.entropy += row;
        if (a.n_top) a.top_ids += row * a.n_top, a.top_logprobs += row * a.n_top;
        const dim3 grid((unsigned)(a.slices * a.n_rows)), threads(THREADS);
        if (a.vocab < RUN) hipLaunchKernelGGL(dbf_logprobs_short_kernel<T>, dim3((a.n_rows + THREADS - 1) / THREADS), threads, 0, stream, a);
        else if (a.n_top) hipLaunchKernelGGL((dbf_logprobs_kernel<T, true>), grid, threads, 0, stream, a);
        else hipLaunchKernelGGL((dbf_logprobs_kernel<T, false>), grid, threads, 0, stream, a);
        if (a.slices > 1) hipLaunchKernelGGL(dbf_logprobs_join_kernel<T>, dim3(a.n_rows), threads, 0, stream, a);
        if (hipGetLastError() != hipSuccess) return DBF_EHIP;
    }
    return DBF_OK;
}

}  // namespace

extern "C" size_t dbf_token_logprobs_workspace_bytes(int n_rows, int vocab, int n_top) {
    if (!sizes_ok(n_rows, vocab, n_top)) return 0;
    const Room room = room_of(n_rows, vocab, n_top);
    return room.sums + room.top;
}

extern "C" int dbf_token_logprobs(const void* logits, int dtype, long long row_stride, int n_rows, int vocab, const int32_t* targets, int n_top,
                                  float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs, void* workspace_dev, size_t workspace_bytes,
                                  void* hip_stream) {
    if (!logits || (dtype != DBF_F16 && dtype != DBF_BF16 && dtype != DBF_F32)) return DBF_EINVAL;
    if (vocab < 1 || vocab > (1 << 24)) return DBF_ESHAPE;
    if (!sizes_ok(n_rows, vocab, n_top) || row_stride < vocab) return DBF_EINVAL;
    if (!targets != !logprob || (n_top && (!top_ids || !top_logprobs))) return DBF_EINVAL;
    if (dbf_misaligned(logits, dtype == DBF_F32 ? 4 : 2) || dbf_misaligned(targets, 4) || dbf_misaligned(logprob, 4) || dbf_misaligned(entropy, 4) ||
        dbf_misaligned(top_ids, 4) || dbf_misaligned(top_logprobs, 4))
        return DBF_EINVAL;
    if (!n_rows) return DBF_OK;
    LogprobArgs a = {logits, row_stride, targets, logprob, entropy, top_logprobs, top_ids, n_rows, vocab, n_top, slices_of(n_rows, vocab, n_top), 0, nullptr, nullptr};
    a.slice = ((vocab + a.slices - 1) / a.slices + RUN - 1) / RUN * RUN;
    a.slices = (vocab + a.slice - 1) / a.slice;   // (rounding up may leave the last without a value)
    if (a.slices > 1) {
        const Room room = room_of(n_rows, vocab, n_top);
        if (!workspace_dev || dbf_misaligned(workspace_dev, 256) || workspace_bytes < room.sums + room.top) return DBF_EWORKSPACE;
        a.part_sums = static_cast<Sums*>(workspace_dev);
        a.part_top = reinterpret_cast<u64*>(static_cast<char*>(workspace_dev) + room.sums);
    }
    const auto stream = static_cast<hipStream_t>(hip_stream);
    return dtype == DBF_F16 ? launch<_Float16>(a, stream) : dtype == DBF_BF16 ? launch<dbf_bf16>(a, stream) : launch<float>(a, stream);
}
