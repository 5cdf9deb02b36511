// Attention over the cache in 4 bits (include/dbf.h, dbf_cache_attend).
#include <initializer_list>

#include "dbf_cache.h"
#include "dbf_wave.h"

namespace {

struct AttendArgs {
    const void* q;
    void* out;
    long long q_stride, out_stride;
    const int *q_start, *kv_len, *table;
    const uint8_t* cache;
    int n_tokens, n_seq, n_q, n_kv, max_q, max_kv, table_stride, causal, n_pages, page_shift, dim;
    float scale;
};

// A request's rows and tokens; ok: they are what the call allows.
struct Request {
    int row0, rows, kv;
    bool ok;
};
__device__ __forceinline__ Request request(const AttendArgs& a, int i) {
    Request r;
    const long long from = a.q_start ? a.q_start[i] : i, to = a.q_start ? a.q_start[i + 1] : i + 1;
    r.row0 = (int)min(max(from, 0LL), (long long)a.n_tokens);
    r.rows = (int)min(max(to - r.row0, 0LL), (long long)a.n_tokens - r.row0);
    r.kv = a.kv_len[i];
    r.ok = r.kv >= 0 && r.kv <= a.max_kv && r.kv <= (long long)a.table_stride << a.page_shift && r.rows <= a.max_q;
    return r;
}

// A workgroup to a row and head.
template <typename T>
__global__ __launch_bounds__(256) void dbf_attend_simple_kernel(const AttendArgs a) {
    __shared__ float q[256], p[256], part[4];
    const int tid = threadIdx.x, head = blockIdx.y, D = a.dim, n = D / 64;
    const Request r = request(a, blockIdx.z);
    const int t = blockIdx.x;
    if (t >= r.rows) return;
    T* out = static_cast<T*>(a.out) + (long long)(r.row0 + t) * a.out_stride + (long long)head * D;
    if (!r.ok) {
        if (tid < D) out[tid] = dbf_from_float<T>(__builtin_nanf(""));
        return;
    }
    if (tid < D) q[tid] = dbf_to_float((static_cast<const T*>(a.q) + (long long)(r.row0 + t) * a.q_stride + (long long)head * D)[tid]) * a.scale;
    const int kv_head = head / (a.n_q / a.n_kv), seen = a.causal ? min(r.kv, r.kv - r.rows + t + 1) : r.kv;
    const int* table = a.table + (long long)blockIdx.z * a.table_stride;
    float m = -__builtin_inff(), l = 0.f, o = 0.f;
    auto record = [&](int j, bool& known) {
        const int page = table[j >> a.page_shift];
        known = page >= 0 && page < a.n_pages;
        const long long slot = ((long long)(known ? page : 0) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        return a.cache + dbf_record_at((int)slot, kv_head, a.n_kv, a.page_shift, D);
    };
    for (int j0 = 0; j0 < seen; j0 += 256) {
        __syncthreads();
        const int j = j0 + tid;
        float x = -__builtin_inff();
        if (j < seen) {
            bool known;
            const uint8_t* rec = record(j, known);
            x = known ? 0.f : __builtin_nanf("");
            const dbf_h2* w = reinterpret_cast<const dbf_h2*>(rec + 32 * D) + (j & 31);
            for (int d = 0; d < D; ++d) {
                const dbf_h2 sb = w[32 * ((d >> 4) % n)];
                const unsigned c = rec[(j & 31) * (D / 2) + (d >> 1)] >> 4 * (d & 1) & 15;
                x = fmaf(q[d], fmaf((float)sb[0], (float)c, (float)sb[1]), x);
            }
        }
        float top = dbf_wave_max(x != x ? 0.f : x);
        if ((tid & 63) == 0) part[tid >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
        const float now = fmaxf(m, top), keep = m == now ? 1.f : expf(m - now);
        const float e = x == -__builtin_inff() ? 0.f : expf(x - now);
        p[tid] = e;
        __syncthreads();
        const float sum = dbf_wave_sum_f(e);
        if ((tid & 63) == 0) part[tid >> 6] = sum;
        __syncthreads();
        l = l * keep + ((part[0] + part[1]) + (part[2] + part[3]));
        o *= keep;
        m = now;
        if (tid < D) {
            const int run = tid >> 4, g = run % n, k = run / n;
            for (int i = 0; i < min(256, seen - j0); ++i) {
                bool known;
                const uint8_t* rec = record(j0 + i, known);
                const int u = (j0 + i) & 31;
                const dbf_h2 sb = reinterpret_cast<const dbf_h2*>(rec + 34 * D)[32 * g + u];
                const unsigned c = rec[16 * D + 1024 * g + 16 * (16 * (u >> 2 & 3) + (tid & 15)) + 4 * (2 * (k >> 1) + (u >> 4)) + (u & 3)] >> 4 * (k & 1) & 15;
                o = fmaf(p[i], known ? fmaf((float)sb[0], (float)c, (float)sb[1]) : 0.f, o);
            }
        }
    }
    if (tid < D) out[tid] = dbf_from_float<T>(l == 0.f ? 0.f : o / l);
}

int check_attend(const dbf_attend* a, const dbf_cache* c) {
    if (!a) return DBF_EINVAL;
    if (const int bad = dbf_cache_check(c)) return bad;
    if (a->dtype != DBF_F16 && a->dtype != DBF_BF16) return DBF_EINVAL;
    if (a->n_seq < 1 || a->n_seq > 65535 || a->n_tokens < 0 || a->max_q < 0 || a->max_kv < 0 || a->table_stride < 1) return DBF_EINVAL;
    if (a->n_q_heads < 1 || a->n_q_heads > 65535) return DBF_EINVAL;
    if (a->n_q_heads % c->n_kv_heads) return DBF_ESHAPE;
    if (!(a->scale > -3.0e38f && a->scale < 3.0e38f)) return DBF_EINVAL;
    return DBF_OK;
}

}  // namespace

extern "C" size_t dbf_cache_attend_workspace_bytes(const dbf_attend* attend, const dbf_cache* cache) {
    if (check_attend(attend, cache)) return 0;
    return 0;
}

extern "C" int dbf_cache_attend(const dbf_attend* attend, const dbf_cache* cache, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
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
    const auto kernel = attend->dtype == DBF_F16 ? dbf_attend_simple_kernel<_Float16> : dbf_attend_simple_kernel<dbf_bf16>;
    hipLaunchKernelGGL(kernel, dim3(a.max_q, a.n_q, a.n_seq), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}
