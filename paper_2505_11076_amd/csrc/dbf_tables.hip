// Pages and slots for the new tokens of a pass's requests (include/dbf.h, dbf_block_tables).
//
// With c_i tokens held, n_i new ones and pages of P: request i has h_i = ceil(c_i / P) pages and takes ceil((c_i + n_i) / P) - h_i from the
// free list, behind those of the requests before it; its tokens lie behind theirs in the common order.  Both are prefix sums over the requests.
// One launch: a workgroup takes 1024 tokens and makes the sums itself, from lengths that all workgroups read (8 bytes a request, from L2
// after the first): a step between workgroups or launches costs more.  A new page begins with a new token, whose thread enters it
// in the table; entries that were there are only read, so nothing waits for the table.
// Bound by latencies: a read of the lengths, the sums, a read of the free list, the stores: 61 requests with a token each 3.5 us, 4096 with 127 000 new tokens 9.2.  (Lengths read one by one,
// tokens of a thread next to each other: 16.6.)
#include "dbf_cache.h"

namespace {

constexpr int THREADS = 256, PER = 4, TOKENS = THREADS * PER;

struct TablesArgs {
    const int *cached, *fresh, *free_pages;
    int *table, *q_start, *kv_len, *positions, *slots, *status;
    int n_seq, page_shift, n_free, table_stride, max_tokens;
};

__device__ __forceinline__ long long wave_scan(long long v, int lane) {   // of the lanes up to this one
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const long long o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// AHEAD: lengths of a thread at once, 1 for up to 256 requests (with 16 their launch took 5.1 us for 4.0: more code than work), 16 above.
template <int AHEAD>
__global__ __launch_bounds__(THREADS) void dbf_block_tables_kernel(const TablesArgs a) {
    __shared__ long long sums[2][THREADS / 64];
    __shared__ int head[TOKENS], first[TOKENS], pages[TOKENS], held[TOKENS], nearest[TOKENS], before[THREADS / 64];
    __shared__ unsigned cached[THREADS * (AHEAD + 1)], fresh[THREADS * (AHEAD + 1)];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long t0 = (long long)blockIdx.x * TOKENS;
    const int P = 1 << a.page_shift;
    auto pages_of = [&](unsigned tokens) { return (tokens >> a.page_shift) + ((tokens & (P - 1)) != 0); };   // (two lengths together are below 2^32)
    for (int e = tid; e < TOKENS; e += THREADS) head[e] = -1;
    const bool writes = blockIdx.x == 0;
    long long all_tokens = 0, all_pages = 0;   // of the requests before
    for (int i0 = 0; i0 < a.n_seq; i0 += THREADS * AHEAD) {
        // lengths as they lie, neighbours to neighbouring threads; then a run of AHEAD requests to a thread (a word apart for each, so that runs begin in different banks)
        unsigned c[AHEAD], n[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = min(i0 + tid + k * THREADS, a.n_seq - 1);
            c[k] = a.cached[i];
            n[k] = a.fresh[i];
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int e = tid + k * THREADS, i = i0 + e;
            c[k] = max((int)c[k], 0);
            n[k] = i < a.n_seq ? max((int)n[k], 0) : 0;
            cached[e + e / AHEAD] = c[k];
            fresh[e + e / AHEAD] = n[k];
            if (writes && i < a.n_seq) a.kv_len[i] = (int)min(c[k] + n[k], (unsigned)INT_MAX);
        }
        __syncthreads();
        const int run = tid * (AHEAD + 1), from = i0 + tid * AHEAD;
        long long n_tokens = 0, n_pages = 0;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            c[k] = cached[run + k];
            n[k] = fresh[run + k];
            n_tokens += n[k];
            n_pages += pages_of(c[k] + n[k]) - pages_of(c[k]);
        }
        long long token = wave_scan(n_tokens, lane), page = wave_scan(n_pages, lane);
        if (lane == 63) {
            sums[0][wave] = token;
            sums[1][wave] = page;
        }
        __syncthreads();
        token += all_tokens - n_tokens;
        page += all_pages - n_pages;
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) {
                token += sums[0][w];
                page += sums[1][w];
            }
            all_tokens += sums[0][w];
            all_pages += sums[1][w];
        }
        // where a request's tokens begin among the workgroup's: its number, its first token, its first page of the free list and what it held (nearly all threads have none)
        if (writes || (token < t0 + TOKENS && token + n_tokens > t0)) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (writes) fresh[run + k] = (unsigned)min(token, (long long)INT_MAX);
                if (n[k] > 0 && token < t0 + TOKENS && token + n[k] > t0) {
                    const int at = (int)max(token - t0, 0LL);
                    head[at] = from + k;
                    first[at] = (int)(token - t0);                  // (negative: it began in an earlier workgroup's)
                    pages[at] = (int)min(page, (long long)INT_MAX);
                    held[at] = (int)c[k];
                }
                token += n[k];
                page += pages_of(c[k] + n[k]) - pages_of(c[k]);
            }
        }
        __syncthreads();
        if (writes)
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int e = tid + k * THREADS;
                if (i0 + e < a.n_seq) a.q_start[i0 + e] = (int)fresh[e + e / AHEAD];
            }
        if (i0 + THREADS * AHEAD < a.n_seq) __syncthreads();
    }
    if (writes && tid == 0) {
        a.q_start[a.n_seq] = (int)min(all_tokens, (long long)INT_MAX);
        a.status[0] = (int)min(all_pages, (long long)a.n_free);
        a.status[1] = (int)min(max(all_pages - a.n_free, 0LL), (long long)INT_MAX);
    }
    // the nearest beginning at or before each token
    int at[PER], last = -1;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        if (head[tid * PER + e] >= 0) last = tid * PER + e;
        at[e] = last;
    }
    int scan = last;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(scan, d);
        if (lane >= d) scan = max(scan, o);
    }
    if (lane == 63) before[wave] = scan;
    int prior = __shfl_up(scan, 1);
    if (lane == 0) prior = -1;
    __syncthreads();
    for (int w = 0; w < wave; ++w) prior = max(prior, before[w]);
#pragma unroll
    for (int e = 0; e < PER; ++e) nearest[tid * PER + e] = max(at[e], prior);
    __syncthreads();
    // from here on a thread's tokens are THREADS apart: neighbours' stores and look-ups lie together
    int position[PER], id[PER], i[PER];
    long long r[PER];
    bool fresh_page[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int t = tid + e * THREADS, h = max(nearest[t], 0);
        const bool is = t0 + t < all_tokens && t0 + t < a.max_tokens;
        const long long place = is ? held[h] + ((long long)t - first[h]) : 0, have = is ? pages_of(held[h]) : 0;
        i[e] = is ? head[h] : 0;
        r[e] = place >> a.page_shift;
        position[e] = (int)min(place, (long long)INT_MAX);
        fresh_page[e] = r[e] >= have;
        id[e] = -1;
        if (is) {
            const long long k = pages[h] + (r[e] - have);
            if (!fresh_page[e]) {
                if (r[e] < a.table_stride) id[e] = a.table[(long long)i[e] * a.table_stride + r[e]];
            } else if (k < a.n_free) {
                id[e] = a.free_pages[k];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const long long t = t0 + tid + e * THREADS;
        if (t >= a.max_tokens) continue;
        if (r[e] >= a.table_stride) id[e] = -1;
        else if (t < all_tokens && fresh_page[e] && (position[e] & (P - 1)) == 0) a.table[(long long)i[e] * a.table_stride + r[e]] = id[e];
        const long long s = ((long long)id[e] << a.page_shift) + (position[e] & (P - 1));
        a.positions[t] = position[e];
        a.slots[t] = id[e] >= 0 && s <= INT_MAX ? (int)s : -1;
    }
}

}  // namespace

extern "C" int dbf_block_tables(const int32_t* cached_len, const int32_t* new_len, int n_seq, int page_tokens, const int32_t* free_pages, int n_free,
                                int32_t* block_table, int table_stride, int max_tokens, int32_t* q_start, int32_t* kv_len, int32_t* positions,
                                int32_t* slots, int32_t* status, void* hip_stream) {
    if (!cached_len || !new_len || !block_table || !q_start || !kv_len || !status) return DBF_EINVAL;
    if (n_seq < 1 || n_seq > DBF_MAX_DIM || n_free < 0 || max_tokens < 0 || table_stride < 1) return DBF_EINVAL;
    if (page_tokens != 32 && page_tokens != 64 && page_tokens != 128 && page_tokens != 256) return DBF_EINVAL;
    if ((n_free && !free_pages) || (max_tokens && (!positions || !slots))) return DBF_EINVAL;
    for (const void* p : {(const void*)cached_len, (const void*)new_len, (const void*)free_pages, (const void*)block_table, (const void*)q_start,
                          (const void*)kv_len, (const void*)positions, (const void*)slots, (const void*)status})
        if (dbf_misaligned(p, 4)) return DBF_EINVAL;
    const TablesArgs a = {cached_len, new_len, free_pages, block_table, q_start, kv_len, positions, slots, status,
                          n_seq, dbf_page_shift(page_tokens), n_free, table_stride, max_tokens};
    const unsigned groups = max_tokens ? (unsigned)(((long long)max_tokens + TOKENS - 1) / TOKENS) : 1u;
    hipLaunchKernelGGL(n_seq <= THREADS ? dbf_block_tables_kernel<1> : dbf_block_tables_kernel<16>, dim3(groups), dim3(THREADS), 0, static_cast<hipStream_t>(hip_stream), a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}
