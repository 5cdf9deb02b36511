// Pages and slots for the new tokens of a pass's requests (include/dbf.h, dbf_block_tables).
//
// With c_i tokens held, n_i new ones and pages of P: request i has h_i = ceil(c_i / P) pages and takes ceil((c_i + n_i) / P) - h_i from the
// free list, behind those of the requests before it; its tokens lie behind theirs in the common order.  Both are prefix sums over the requests.
// One launch: a workgroup takes 1024 tokens and makes the sums itself, from lengths that all workgroups read (8 bytes a request, from L2
// after the first): a step between workgroups or launches costs more.  A new page begins with a new token, whose thread enters it
// in the table; entries that were there are only read, so nothing waits for the table.
// Bound by latencies: a read of the lengths, the sums, a read of the free list, the stores.
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

__global__ __launch_bounds__(THREADS) void dbf_block_tables_kernel(const TablesArgs a) {
    __shared__ long long sums[2][THREADS / 64];
    __shared__ int head[TOKENS], first[TOKENS], pages[TOKENS], before[THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long t0 = (long long)blockIdx.x * TOKENS;
    const int P = 1 << a.page_shift;
    auto lengths = [&](int i, long long& c, long long& n) {
        c = max(a.cached[i], 0);
        n = max(a.fresh[i], 0);
    };
    auto pages_of = [&](long long tokens) { return (tokens + P - 1) >> a.page_shift; };
    // a run of requests to a thread: its tokens and pages, then those before it
    const int run = (a.n_seq + THREADS - 1) / THREADS, from = min(tid * run, a.n_seq), to = min(from + run, a.n_seq);
    long long n_tokens = 0, n_pages = 0, c, n;
    for (int i = from; i < to; ++i) {
        lengths(i, c, n);
        n_tokens += n;
        n_pages += pages_of(c + n) - pages_of(c);
    }
    long long token = wave_scan(n_tokens, lane), page = wave_scan(n_pages, lane);
    if (lane == 63) {
        sums[0][wave] = token;
        sums[1][wave] = page;
    }
    for (int e = tid; e < TOKENS; e += THREADS) head[e] = -1;
    __syncthreads();
    long long all_tokens = 0, all_pages = 0;
    token -= n_tokens;
    page -= n_pages;
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) {
            token += sums[0][w];
            page += sums[1][w];
        }
        all_tokens += sums[0][w];
        all_pages += sums[1][w];
    }
    // where a request's tokens begin among the workgroup's: its number, its first token and its first page of the free list
    const bool writes = blockIdx.x == 0;
    for (int i = from; i < to; ++i) {
        lengths(i, c, n);
        if (writes) {
            a.q_start[i] = (int)min(token, (long long)INT_MAX);
            a.kv_len[i] = (int)min(c + n, (long long)INT_MAX);
        }
        if (n > 0 && token < t0 + TOKENS && token + n > t0) {
            const int at = (int)max(token - t0, 0LL);
            head[at] = i;
            first[at] = (int)(token - t0);                  // (negative: it began in an earlier workgroup's)
            pages[at] = (int)min(page, (long long)INT_MAX);
        }
        token += n;
        page += pages_of(c + n) - pages_of(c);
    }
    if (writes && tid == 0) {
        a.q_start[a.n_seq] = (int)min(all_tokens, (long long)INT_MAX);
        a.status[0] = (int)min(all_pages, (long long)a.n_free);
        a.status[1] = (int)min(max(all_pages - a.n_free, 0LL), (long long)INT_MAX);
    }
    __syncthreads();
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
    for (int e = 0; e < PER; ++e) {
        const long long t = t0 + tid * PER + e;
        if (t >= a.max_tokens) break;
        int slot = -1, position = 0;
        if (t < all_tokens) {
            const int h = max(at[e], prior), i = head[h];
            lengths(i, c, n);
            const long long place = c + (tid * PER + e - first[h]), r = place >> a.page_shift, have = pages_of(c);
            position = (int)min(place, (long long)INT_MAX);
            long long id = -1;
            if (r >= have) {
                const long long k = pages[h] + (r - have);
                if (k < a.n_free) id = a.free_pages[k];
                if (r >= a.table_stride) id = -1;
                else if ((place & (P - 1)) == 0) a.table[(long long)i * a.table_stride + r] = (int)id;
            } else if (r < a.table_stride) {
                id = a.table[(long long)i * a.table_stride + r];
            }
            const long long s = (id << a.page_shift) + (place & (P - 1));
            if (id >= 0 && s <= INT_MAX) slot = (int)s;
        }
        a.positions[t] = position;
        a.slots[t] = slot;
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
    hipLaunchKernelGGL(dbf_block_tables_kernel, dim3(groups), dim3(THREADS), 0, static_cast<hipStream_t>(hip_stream), a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}
