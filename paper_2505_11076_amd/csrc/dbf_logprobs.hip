// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits (include/dbf.h, dbf_token_logprobs).
//
// One pass with a running maximum m and the sums s = sum e^(x - m), t = sum e^(x - m) (x - m) of what has been read:
//     log sum e^x = m + log s,      entropy = log s - t / s.
// The likeliest tokens: a thread keeps its largest key (value, then the lower index; all keys differ).  The n largest of the row are in the
// threads whose largest keys are the n largest of those: only these threads' values are read again.
#include <climits>

#include "dbf_cache.h"

namespace {

constexpr int THREADS = 256, MOST_TOP = 64;
typedef unsigned long long u64;

struct LogprobArgs {
    const void* x;
    long long stride;
    const int* targets;
    float *logprob, *entropy, *top_logprobs;
    int* top_ids;
    int n_rows, vocab, n_top;
};

// Larger values first, no numbers before all, then lower indexes.  (+ 0: -0 is 0.)
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

// A difference from the maximum, whose exponential is nothing below -104: held to what a product with nothing leaves nothing (a type's lowest value
// less the maximum is -infinity).
__device__ __forceinline__ float below(float d) { return fmaxf(d, -200.f); }

struct Sums {
    float m, s, t;
};
// Of two parts.  (A part of nothing, or of tokens that cannot be only, has m = -infinity and s = t = 0.)
__device__ __forceinline__ Sums join(Sums a, Sums b) {
    Sums r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.m == r.m ? 0.f : below(a.m - r.m), db = b.m == r.m ? 0.f : below(b.m - r.m);
    const float ea = expf(da), eb = expf(db);
    r.s = a.s * ea + b.s * eb;
    r.t = (a.s > 0.f ? (a.t + a.s * da) * ea : 0.f) + (b.s > 0.f ? (b.t + b.s * db) * eb : 0.f);
    if (a.s != a.s || b.s != b.s) r.s = r.t = __builtin_nanf("");
    return r;
}
__device__ __forceinline__ void take(Sums& a, float x) {
    if (x != x || x == __builtin_inff()) {
        a.s = a.t = __builtin_nanf("");
        return;
    }
    if (x == -__builtin_inff()) return;
    if (x > a.m) {
        const float d = below(a.m - x), e = a.s > 0.f ? expf(d) : 0.f;
        a.t = a.s > 0.f ? (a.t + a.s * d) * e : a.s;    // (a.s that is no number stays that)
        a.s = a.s * (a.s > 0.f ? e : 1.f) + 1.f;
        a.m = x;
    } else {
        const float d = below(x - a.m), e = expf(d);
        a.s += e;
        a.t = fmaf(e, d, a.t);
    }
}

template <typename T>
__global__ __launch_bounds__(THREADS) void dbf_logprobs_kernel(const LogprobArgs a) {
    __shared__ Sums parts[THREADS];
    __shared__ u64 keys[THREADS];
    const int tid = threadIdx.x, row = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + row * a.stride;
    Sums s = {-__builtin_inff(), 0.f, 0.f};
    for (int i = tid; i < a.vocab; i += THREADS) take(s, dbf_to_float(x[i]));
    parts[tid] = s;
    __syncthreads();
    for (int n = THREADS / 2; n; n /= 2) {
        if (tid < n) parts[tid] = join(parts[tid], parts[tid + n]);
        __syncthreads();
    }
    s = parts[0];
    const float log_s = s.s > 0.f ? logf(s.s) : __builtin_nanf("");
    if (tid == 0) {
        if (a.logprob) {
            const int target = a.targets[row];
            a.logprob[row] = target < 0 ? 0.f : target >= a.vocab ? __builtin_nanf("") : (dbf_to_float(x[target]) - s.m) - log_s;
        }
        if (a.entropy) a.entropy[row] = log_s - s.t / s.s;
    }
    // one after the other
    u64 last = ~0ull;
    for (int k = 0; k < a.n_top; ++k) {
        u64 best = 0;
        for (int i = tid; i < a.vocab; i += THREADS) {
            const u64 key = key_of(dbf_to_float(x[i]), i);
            if ((k == 0 || key < last) && key > best) best = key;
        }
        keys[tid] = best;
        __syncthreads();
        for (int n = THREADS / 2; n; n /= 2) {
            if (tid < n) keys[tid] = max(keys[tid], keys[tid + n]);
            __syncthreads();
        }
        last = keys[0];
        if (tid == 0) {
            a.top_ids[(long long)row * a.n_top + k] = ~(unsigned)last;
            a.top_logprobs[(long long)row * a.n_top + k] = (value_of(last) - s.m) - log_s;
        }
        __syncthreads();
    }
}

bool sizes_ok(int n_rows, int vocab, int n_top) { return n_rows >= 0 && vocab >= 1 && vocab <= (1 << 24) && n_top >= 0 && n_top <= MOST_TOP && n_top <= vocab; }

}  // namespace

extern "C" size_t dbf_token_logprobs_workspace_bytes(int n_rows, int vocab, int n_top) {
    if (!sizes_ok(n_rows, vocab, n_top)) return 0;
    return 0;
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
    const LogprobArgs a = {logits, row_stride, targets, logprob, entropy, top_logprobs, top_ids, n_rows, vocab, n_top};
    const auto kernel = dtype == DBF_F16 ? dbf_logprobs_kernel<_Float16> : dtype == DBF_BF16 ? dbf_logprobs_kernel<dbf_bf16> : dbf_logprobs_kernel<float>;
    hipLaunchKernelGGL(kernel, dim3(n_rows), dim3(THREADS), 0, static_cast<hipStream_t>(hip_stream), a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}
