// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits (include/dbf.h, dbf_token_logprobs).
//
// One read of the logits, with a maximum m that may lag and the sums s = sum e^(x - m), t = sum e^(x - m) (x - m) of what has been read, in fp32:
//     log sum e^x = m + log s,      entropy = log s - t / s.
// The likeliest tokens: all values have keys (value, then the lower index) that differ.  A thread keeps its largest; the n-th largest of these is a bound that the n largest of all
// are not below, and only the n threads whose largest keys are not below it can hold any: their values are read once more (from the cache), the few that pass are put in order.
// A row is one workgroup's, or where rows are few the slices of several, whose sums and lists a second launch joins.
// Bound by the read where rows are many: a value costs about nine issue slots (its exponential four), half of what the memory takes.
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

constexpr float LEAST = -3.402823466e38f;   // of a maximum: no finite value is below it, and -infinity less it is not a number's absence
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
__device__ __forceinline__ Sums wave_join(Sums v) {
#pragma unroll
    for (int d = 32; d; d /= 2) {
        const Sums o = {__shfl_xor(v.m, d), __shfl_xor(v.s, d), __shfl_xor(v.t, d)};
        v = join(v, o);
    }
    return v;
}

// Values i .. i + 7 of a row of n, whose end a run may overlap: what is not there is -infinity.  The loads have no use of their own, so several may be under way.
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
    // the index of value e
    static __device__ __forceinline__ int index(int i, int n, int e) { return min(i, n - RUN) + e; }
};

// The n largest of keys[0 .. count) (LDS, all different), in order, by how many are larger; out(place, key).
template <typename Out>
__device__ __forceinline__ void in_order(const u64* keys, int count, int n, Out out) {
    for (int i = threadIdx.x; i < count; i += THREADS) {
        const u64 own = keys[i];
        int larger = 0;
        for (int k = 0; k < count; ++k) larger += keys[k] > own;
        if (larger < n) out(larger, own);
    }
}

struct Work {
    u64 keys[THREADS], passed[ROOM];
    int chosen[MOST_TOP], count;
    u64 bound;
    Sums sums[THREADS / 64];
};

// The n_top largest keys of x[0 .. n), in order; `best` is the thread's largest, of its runs tid, tid + THREADS, ...; base: the index of x[0] in its row.
template <typename T, typename Out>
__device__ __forceinline__ void likeliest(const T* x, int n, int base, u64 best, int n_top, Work& work, Out out) {
    const int tid = threadIdx.x, wanted = min(n_top, n);
    work.keys[tid] = best;
    if (tid == 0) {
        work.count = 0;
        work.bound = 1;   // (fewer threads than tokens wanted: all pass)
    }
    __syncthreads();
    int larger = 0;
    for (int k = 0; k < THREADS; ++k) larger += work.keys[k] > best;
    if (best && larger < wanted) work.chosen[larger] = tid;
    if (best && larger == wanted - 1) work.bound = best;
    const int holders = __syncthreads_count(best && larger < wanted);
    const u64 bound = work.bound;
    const int runs = (n + RUN - 1) / RUN, each = (runs + THREADS - 1) / THREADS;
    for (int k = tid; k < holders * each; k += THREADS) {
        const int run = work.chosen[k % holders] + k / holders * THREADS;
        if (run >= runs) continue;
        for (int e = 0; e < RUN; ++e) {
            const int i = run * RUN + e;
            const u64 key = i < n ? key_of(dbf_to_float(x[i]), base + i) : 0;
            if (key >= bound) {
                const int at = atomicAdd(&work.count, 1);   // (in any order: they are put in order by their keys)
                if (at < ROOM) work.passed[at] = key;
            }
        }
    }
    __syncthreads();
    const int count = work.count;
    if (count <= ROOM) {
        in_order(work.passed, count, wanted, out);
    } else {   // rows made so that few threads hold thousands of the largest: one after the other
        u64 last = ~0ull;
        for (int k = 0; k < wanted; ++k) {
            u64 top = 0;
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

__device__ __forceinline__ void finish(const LogprobArgs& a, int row, Sums s, float target_value, int target, float log_s) {
    if (a.logprob) a.logprob[row] = target < 0 ? 0.f : target >= a.vocab ? __builtin_nanf("") : (target_value - s.m) - log_s;
    if (a.entropy) a.entropy[row] = log_s - s.t / s.s;
}

template <typename T, bool TOP>
__global__ __launch_bounds__(THREADS) void dbf_logprobs_kernel(const LogprobArgs a) {
    __shared__ Work work;
    const int tid = threadIdx.x, row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices, base = slice * a.slice, n = min(a.slice, a.vocab - base);
    const T* x = static_cast<const T*>(a.x) + row * a.stride + base;
    Sums s = {LEAST, 0.f, 0.f};
    float most = -__builtin_inff();
    int most_run = INT_MAX;   // the first run that holds it
    constexpr int AHEAD = 4, STEP = THREADS * RUN * AHEAD;
    if (n >= RUN) {
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
                s = join(o, (Sums){fminf(top, 3.4e38f), 0.f, 0.f});
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int e = 0; e < RUN; ++e) {
                    const float d = v[k][e] - s.m, w = __builtin_amdgcn_exp2f(d * 1.44269504089f);
                    s.s += w;
                    s.t = fmaf(w, below(d), s.t);
                }
        }
    } else {
        for (int i = tid; i < n; i += THREADS) {
            const float v = dbf_to_float(x[i]);
            s = (Sums){fminf(fmaxf(v, LEAST), 3.4e38f), 1.f, 0.f};
            if (v - v != 0.f) s.s = s.t = v == -__builtin_inff() ? 0.f : __builtin_nanf("");
            most = v;
            most_run = i / RUN * RUN;
        }
    }
    const bool number = s.s < __builtin_inff() && s.t == s.t;   // (a logit of +infinity makes the sum that)
    s = wave_join(s);
    if ((tid & 63) == 0) work.sums[tid >> 6] = s;
    const bool numbers = !__syncthreads_or(!number);   // of the workgroup's part
    s = join(join(work.sums[0], work.sums[1]), join(work.sums[2], work.sums[3]));
    if (!numbers) s.s = s.t = __builtin_nanf("");
    const float log_s = s.s > 0.f ? logf(s.s) : __builtin_nanf("");
    if (tid == 0) {
        if (a.slices == 1) {
            const int target = a.logprob ? a.targets[row] : -1;
            finish(a, row, s, target >= 0 && target < a.vocab ? dbf_to_float(x[target]) : 0.f, target, log_s);
        } else {
            a.part_sums[(long long)row * a.slices + slice] = s;
        }
    }
    if (!TOP) return;
    // the thread's largest key: the first of its values that is as large as any (or is no number)
    u64 best = 0;
    if (most_run != INT_MAX) {
        const int runs = (n + RUN - 1) / RUN;
        if (numbers) {
            for (int e = 0; e < RUN && most_run + e < n; ++e) best = max(best, key_of(dbf_to_float(x[most_run + e]), base + most_run + e));
        } else {
            for (int r = tid; r < runs; r += THREADS)
                for (int e = 0; e < RUN && r * RUN + e < n; ++e) best = max(best, key_of(dbf_to_float(x[r * RUN + e]), base + r * RUN + e));
        }
    }
    if (n < RUN && tid) best = 0;   // (one run: the first thread's)
    if (n < RUN && tid == 0)
        for (int e = 0; e < n; ++e) best = max(best, key_of(dbf_to_float(x[e]), base + e));
    if (a.slices == 1) {
        likeliest(x, n, base, best, a.n_top, work, [&](int k, u64 key) {
            a.top_ids[(long long)row * a.n_top + k] = (int)~(unsigned)key;
            a.top_logprobs[(long long)row * a.n_top + k] = (value_of(key) - s.m) - log_s;
        });
    } else {
        u64* list = a.part_top + ((long long)row * a.slices + slice) * a.n_top;
        for (int k = n + tid; k < a.n_top; k += THREADS) list[k] = 0;
        likeliest(x, n, base, best, a.n_top, work, [&](int k, u64 key) { list[k] = key; });
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
    const u64 first = a.n_top && tid < a.slices ? lists[(long long)tid * a.n_top] : 0;
    const bool number = s.s == s.s;
    s = wave_join(s);
    if ((tid & 63) == 0) work.sums[tid >> 6] = s;
    const bool numbers = !__syncthreads_or(!number);
    s = join(join(work.sums[0], work.sums[1]), join(work.sums[2], work.sums[3]));
    if (!numbers) s.s = s.t = __builtin_nanf("");
    const float log_s = s.s > 0.f ? logf(s.s) : __builtin_nanf("");
    if (tid == 0) {
        const int target = a.logprob ? a.targets[row] : -1;
        finish(a, row, s, target >= 0 && target < a.vocab ? dbf_to_float((static_cast<const T*>(a.x) + row * a.stride)[target]) : 0.f, target, log_s);
    }
    if (!a.n_top) return;
    // the same bound again: of slices' largest; at most n_top slices have keys that pass
    work.keys[tid] = first;
    if (tid == 0) {
        work.count = 0;
        work.bound = 1;
    }
    __syncthreads();
    int larger = 0;
    for (int k = 0; k < a.slices; ++k) larger += work.keys[k] > first;
    if (first && larger == a.n_top - 1) work.bound = first;
    __syncthreads();
    const u64 bound = work.bound;
    for (int k = tid; k < a.slices * a.n_top; k += THREADS) {
        const u64 key = lists[k];
        if (key >= bound) work.passed[atomicAdd(&work.count, 1)] = key;   // (at most n_top lists: MOST_LISTED)
    }
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
int launch(const LogprobArgs& a, hipStream_t stream) {
    const long long groups = (long long)a.slices * a.n_rows;
    if (groups > INT_MAX) return DBF_EINVAL;
    const dim3 grid((unsigned)groups), threads(THREADS);
    if (a.n_top) hipLaunchKernelGGL((dbf_logprobs_kernel<T, true>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((dbf_logprobs_kernel<T, false>), grid, threads, 0, stream, a);
    if (a.slices > 1) hipLaunchKernelGGL(dbf_logprobs_join_kernel<T>, dim3(a.n_rows), threads, 0, stream, a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
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
