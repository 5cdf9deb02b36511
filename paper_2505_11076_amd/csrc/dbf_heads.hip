// Norms and rotation of query and key heads, and the write of keys and values to the cache in 4 bits (include/dbf.h: dbf_qk_norm_rope,
// dbf_cache_append, dbf_cache_read).
//
// A wavefront takes one head of one token.  Norm: x w / sqrt(mean x^2 + eps); rotation: pairs (a cos - b sin, b cos + a sin); all of a head is in fp32 in LDS
// when it is rounded, once: to 16 bits, or to a code per value with a scale and a zero per 64.
#include <initializer_list>

#include "dbf_cache.h"
#include "dbf_wave.h"

namespace {

constexpr int WAVES = 4, MOST_DIM = 1024;

struct HeadsArgs {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    void *q_out, *k_out;
    long long q_out_stride, k_out_stride;
    const void *q_weight, *k_weight;
    const float* rope;
    const int *positions, *slots;
    uint8_t* cache;
    int n_tokens, n_q, n_kv, dim, rope_len, rot, interleaved, n_slots, page_shift;
    float eps;
};

// What the wavefront's lanes have written to LDS is there for all of them.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A head's norm and rotation, from memory to `row` in LDS, by one wavefront.
template <typename T>
__device__ __forceinline__ void turn(const HeadsArgs& a, const T* x, const T* weight, int token, int lane, float* row) {
    float sum = 0.f;
    for (int d = lane; d < a.dim; d += 64) {
        const float v = dbf_to_float(x[d]);
        row[d] = v;
        sum = fmaf(v, v, sum);
    }
    wave_sync();
    float scale = 1.f;
    if (weight) scale = 1.f / sqrtf(dbf_wave_sum_f(sum) / (float)a.dim + a.eps);
    if (a.rope) {
        const int p = a.positions[token], half = a.rot >> 1;
        const bool known = p >= 0 && p < a.rope_len;
        const float* table = a.rope + (long long)(known ? p : 0) * a.rot;
        for (int i = lane; i < half; i += 64) {
            const int d0 = a.interleaved ? 2 * i : i, d1 = a.interleaved ? 2 * i + 1 : i + half;
            float u = row[d0] * scale, w = row[d1] * scale;
            if (weight) {
                u *= dbf_to_float(weight[d0]);
                w *= dbf_to_float(weight[d1]);
            }
            float c = table[i], s = table[half + i];
            if (!known) c = __builtin_nanf("");
            row[d0] = u * c - w * s;
            row[d1] = w * c + u * s;
        }
    }
    if (weight)
        for (int d = (a.rope ? a.rot : 0) + lane; d < a.dim; d += 64) row[d] = row[d] * scale * dbf_to_float(weight[d]);
    wave_sync();
}

// A head's values, n = dim / 64 to a lane (values n lane ..), as codes; its group's scale and zero.  Lanes of a group: all that agree in the bits that
// number the groups (values n lane are of run n lane / 16, groups are the runs' numbers modulo n).
template <int N>
__device__ __forceinline__ bool quantise(const float* row, int lane, unsigned (&code)[N], float& s, float& z) {
    float x[N], lo = 0.f, hi = 0.f;
    bool fine = true;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        x[e] = row[N * lane + e];
        const bool finite = fabsf(x[e]) < __builtin_inff();
        fine = fine && finite;
        x[e] = finite ? fminf(fmaxf(x[e], -DBF_CACHE_MOST), DBF_CACHE_MOST) : 0.f;
        lo = fminf(lo, x[e]);
        hi = fmaxf(hi, x[e]);
    }
    constexpr int low = 16 / N, which = low * (N - 1);   // the bits of a lane that number its group
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        if (!(d & which)) {
            lo = fminf(lo, __shfl_xor(lo, d));
            hi = fmaxf(hi, __shfl_xor(hi, d));
        }
    s = dbf_group_scale(hi - lo);
    const float by = s > 0.f ? s : 1.f;
    z = rintf(-lo / by);
#pragma unroll
    for (int e = 0; e < N; ++e) code[e] = (unsigned)fminf(fmaxf(rintf(x[e] / by) + z, 0.f), 15.f);
    return !__any(!fine);   // of the whole head
}

template <int N>
__device__ __forceinline__ void store_cache(const HeadsArgs& a, const float* k_row, const float* v_row, int slot, int head, int lane) {
    uint8_t* rec = a.cache + dbf_record_at(slot, head, a.n_kv, a.page_shift, 64 * N);
    const int t = slot & 31, tile = t >> 4, g = (t >> 2) & 3, i = t & 3, group = (N * lane >> 4) % N;
    unsigned kc[N], vc[N];
    float ks, kz, vs, vz;
    const bool k_fine = quantise<N>(k_row, lane, kc, ks, kz), fine = quantise<N>(v_row, lane, vc, vs, vz) && k_fine;
    // keys: two values to a byte
    if constexpr (N == 1) {
        const unsigned other = __shfl_xor(kc[0], 1);
        if (!(lane & 1)) rec[t * 32 + (lane >> 1)] = (uint8_t)(kc[0] | other << 4);
    } else {
#pragma unroll
        for (int e = 0; e < N; e += 2) rec[t * 32 * N + ((N * lane + e) >> 1)] = (uint8_t)(kc[e] | kc[e + 1] << 4);
    }
    // values: a value and the one 16 N further, 16 lanes on
    const int q = lane >> 5;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const unsigned other = __shfl_xor(vc[e], 16);
        const int l = (N * lane + e) & 15;
        if (!(lane & 16)) rec[1024 * N + 1024 * group + 16 * (16 * g + l) + 4 * (2 * q + tile) + i] = (uint8_t)(vc[e] | other << 4);
    }
    if (lane < 16 && (N * lane & 15) == 0) {   // the first lane of each group
        dbf_h2* kw = reinterpret_cast<dbf_h2*>(rec + 2048 * N) + 32 * group + t;
        dbf_h2* vw = kw + 32 * N;
        const float bias = fine ? -ks * kz : __builtin_nanf("");
        *kw = (dbf_h2){(_Float16)ks, (_Float16)bias};
        *vw = fine ? (dbf_h2){(_Float16)vs, (_Float16)(-vs * vz)} : (dbf_h2){(_Float16)0.f, (_Float16)0.f};
    }
}

template <typename T>
__global__ __launch_bounds__(64 * WAVES) void dbf_heads_kernel(const HeadsArgs a) {
    __shared__ float rows[WAVES][2][MOST_DIM];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n_q = a.q ? a.n_q : 0, n_k = a.k ? a.n_kv : 0;
    const long long item = (long long)blockIdx.x * WAVES + wave, per = n_q + n_k;
    const int token = (int)(item / per), h = (int)(item % per);
    if (token >= a.n_tokens) return;
    float* row = rows[wave][0];
    if (h < n_q) {
        turn<T>(a, static_cast<const T*>(a.q) + token * a.q_stride + (long long)h * a.dim, static_cast<const T*>(a.q_weight), token, lane, row);
        T* out = static_cast<T*>(a.q_out) + token * a.q_out_stride + (long long)h * a.dim;
        for (int d = lane; d < a.dim; d += 64) out[d] = dbf_from_float<T>(row[d]);
        return;
    }
    const int head = h - n_q;
    int slot = 0;
    if (a.cache) {
        slot = a.slots[token];
        if (slot < 0 || slot >= a.n_slots) return;
    }
    turn<T>(a, static_cast<const T*>(a.k) + token * a.k_stride + (long long)head * a.dim, static_cast<const T*>(a.k_weight), token, lane, row);
    if (!a.cache) {
        T* out = static_cast<T*>(a.k_out) + token * a.k_out_stride + (long long)head * a.dim;
        for (int d = lane; d < a.dim; d += 64) out[d] = dbf_from_float<T>(row[d]);
        return;
    }
    float* v_row = rows[wave][1];
    const T* v = static_cast<const T*>(a.v) + token * a.v_stride + (long long)head * a.dim;
    for (int d = lane; d < a.dim; d += 64) v_row[d] = dbf_to_float(v[d]);
    wave_sync();
    if (a.dim == 64) store_cache<1>(a, row, v_row, slot, head, lane);
    else if (a.dim == 128) store_cache<2>(a, row, v_row, slot, head, lane);
    else store_cache<4>(a, row, v_row, slot, head, lane);
}

template <typename T>
__global__ __launch_bounds__(64 * WAVES) void dbf_cache_read_kernel(const uint8_t* cache, const int* slots, int n_tokens, int n_slots, int n_kv, int dim,
                                                                    int page_shift, T* k_out, T* v_out) {
    const int lane = threadIdx.x & 63;
    const long long item = (long long)blockIdx.x * WAVES + (threadIdx.x >> 6);
    const int token = (int)(item / n_kv), head = (int)(item % n_kv), n = dim / 64;
    if (token >= n_tokens) return;
    const int slot = slots[token];
    const bool held = slot >= 0 && slot < n_slots;
    const uint8_t* rec = cache + dbf_record_at(held ? slot : 0, head, n_kv, page_shift, dim);
    const int t = slot & 31, tile = t >> 4, g = (t >> 2) & 3, i = t & 3;
    for (int d = lane; d < dim; d += 64) {
        const int run = d >> 4, p = run % n, r = run / n;
        float kx = 0.f, vx = 0.f;
        if (held) {
            const dbf_h2 kw = reinterpret_cast<const dbf_h2*>(rec + 32 * dim)[32 * p + t], vw = reinterpret_cast<const dbf_h2*>(rec + 34 * dim)[32 * p + t];
            const unsigned kb = rec[t * (dim / 2) + (d >> 1)], vb = rec[16 * dim + 1024 * p + 16 * (16 * g + (d & 15)) + 4 * (2 * (r >> 1) + tile) + i];
            kx = fmaf((float)kw[0], (float)(kb >> 4 * (d & 1) & 15), (float)kw[1]);
            vx = fmaf((float)vw[0], (float)(vb >> 4 * (r & 1) & 15), (float)vw[1]);
        }
        const long long at = ((long long)token * n_kv + head) * dim + d;
        k_out[at] = dbf_from_float<T>(kx);
        v_out[at] = dbf_from_float<T>(vx);
    }
}

// What is wrong with a call's heads: the same for both entry points.
int check_heads(const dbf_heads* h) {
    if (!h || (h->dtype != DBF_F16 && h->dtype != DBF_BF16) || h->n_tokens < 0 || (!h->q && !h->k)) return DBF_EINVAL;
    if (h->head_dim < 2 || h->head_dim > MOST_DIM || (h->head_dim & 1)) return DBF_ESHAPE;
    if (h->q && (h->n_q_heads < 1 || h->n_q_heads > 65535 || !h->q_out || h->q_stride < (long long)h->n_q_heads * h->head_dim ||
                 h->q_out_stride < (long long)h->n_q_heads * h->head_dim))
        return DBF_EINVAL;
    if (h->k && (h->n_kv_heads < 1 || h->n_kv_heads > 65535 || h->k_stride < (long long)h->n_kv_heads * h->head_dim)) return DBF_EINVAL;
    if (h->rope && (!h->positions || h->rope_len < 1 || h->rot_dim < 2 || (h->rot_dim & 1) || h->rot_dim > h->head_dim)) return DBF_EINVAL;
    if (!(h->eps >= 0.f) || h->eps > 3.0e38f) return DBF_EINVAL;
    for (const void* p : {h->q, h->k, h->v, (const void*)h->q_out, (const void*)h->k_out, h->q_weight, h->k_weight})
        if (dbf_misaligned(p, 2)) return DBF_EINVAL;
    return dbf_misaligned(h->rope, 4) || dbf_misaligned(h->positions, 4) ? DBF_EINVAL : DBF_OK;
}

HeadsArgs heads_args(const dbf_heads* h) {
    HeadsArgs a = {};
    a.q = h->q;  a.k = h->k;  a.v = h->v;
    a.q_stride = h->q_stride;  a.k_stride = h->k_stride;  a.v_stride = h->v_stride;
    a.q_out = h->q_out;  a.k_out = h->k_out;
    a.q_out_stride = h->q_out_stride;  a.k_out_stride = h->k_out_stride;
    a.q_weight = h->q_weight;  a.k_weight = h->k_weight;
    a.rope = static_cast<const float*>(h->rope);  a.positions = h->positions;
    a.n_tokens = h->n_tokens;  a.n_q = h->n_q_heads;  a.n_kv = h->n_kv_heads;  a.dim = h->head_dim;
    a.rope_len = h->rope_len;  a.rot = h->rope ? h->rot_dim : 0;  a.interleaved = h->interleaved;  a.eps = h->eps;
    return a;
}

int launch_heads(const HeadsArgs& a, int dtype, void* hip_stream) {
    if (!a.n_tokens) return DBF_OK;
    const long long items = (long long)a.n_tokens * ((a.q ? a.n_q : 0) + (a.k ? a.n_kv : 0)), groups = (items + WAVES - 1) / WAVES;
    if (groups > INT_MAX) return DBF_EINVAL;
    const auto kernel = dtype == DBF_F16 ? dbf_heads_kernel<_Float16> : dbf_heads_kernel<dbf_bf16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * WAVES), 0, static_cast<hipStream_t>(hip_stream), a);
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}

}  // namespace

extern "C" size_t dbf_cache_bytes(int n_pages, int page_tokens, int n_kv_heads, int head_dim) {
    if (!dbf_cache_shape_ok(n_pages, page_tokens, n_kv_heads, head_dim)) return 0;
    return (size_t)n_pages * (page_tokens / DBF_CACHE_BLOCK) * n_kv_heads * (size_t)dbf_record_bytes(head_dim);
}

extern "C" int dbf_qk_norm_rope(const dbf_heads* heads, void* hip_stream) {
    if (const int bad = check_heads(heads)) return bad;
    if (heads->k && (!heads->k_out || heads->k_out_stride < (long long)heads->n_kv_heads * heads->head_dim)) return DBF_EINVAL;
    return launch_heads(heads_args(heads), heads->dtype, hip_stream);
}

extern "C" int dbf_cache_append(const dbf_heads* heads, const dbf_cache* cache, const int32_t* slots, void* hip_stream) {
    if (const int bad = check_heads(heads)) return bad;
    if (const int bad = dbf_cache_check(cache)) return bad;
    if (heads->head_dim != cache->head_dim || heads->n_kv_heads != cache->n_kv_heads) return DBF_ESHAPE;
    if (!heads->k || !heads->v || !slots || dbf_misaligned(slots, 4)) return DBF_EINVAL;
    if (heads->v_stride < (long long)heads->n_kv_heads * heads->head_dim) return DBF_EINVAL;
    HeadsArgs a = heads_args(heads);
    a.slots = slots;
    a.cache = static_cast<uint8_t*>(cache->data);
    a.n_slots = cache->n_pages * cache->page_tokens;
    a.page_shift = dbf_page_shift(cache->page_tokens);
    return launch_heads(a, heads->dtype, hip_stream);
}

extern "C" int dbf_cache_read(const dbf_cache* cache, const int32_t* slots, int n_tokens, void* k_out, void* v_out, int dtype, void* hip_stream) {
    if (const int bad = dbf_cache_check(cache)) return bad;
    if (!slots || !k_out || !v_out || n_tokens < 0 || (dtype != DBF_F16 && dtype != DBF_BF16 && dtype != DBF_F32)) return DBF_EINVAL;
    const unsigned size = dtype == DBF_F32 ? 4 : 2;
    if (dbf_misaligned(slots, 4) || dbf_misaligned(k_out, size) || dbf_misaligned(v_out, size)) return DBF_EINVAL;
    if (!n_tokens) return DBF_OK;
    const long long groups = ((long long)n_tokens * cache->n_kv_heads + WAVES - 1) / WAVES;
    if (groups > INT_MAX) return DBF_EINVAL;
    const dim3 grid((unsigned)groups), threads(64 * WAVES);
    const auto stream = static_cast<hipStream_t>(hip_stream);
    const uint8_t* data = static_cast<const uint8_t*>(cache->data);
    const int n_slots = cache->n_pages * cache->page_tokens, shift = dbf_page_shift(cache->page_tokens);
    if (dtype == DBF_F16)
        hipLaunchKernelGGL(dbf_cache_read_kernel<_Float16>, grid, threads, 0, stream, data, slots, n_tokens, n_slots, cache->n_kv_heads, cache->head_dim, shift,
                           static_cast<_Float16*>(k_out), static_cast<_Float16*>(v_out));
    else if (dtype == DBF_BF16)
        hipLaunchKernelGGL(dbf_cache_read_kernel<dbf_bf16>, grid, threads, 0, stream, data, slots, n_tokens, n_slots, cache->n_kv_heads, cache->head_dim, shift,
                           static_cast<dbf_bf16*>(k_out), static_cast<dbf_bf16*>(v_out));
    else
        hipLaunchKernelGGL(dbf_cache_read_kernel<float>, grid, threads, 0, stream, data, slots, n_tokens, n_slots, cache->n_kv_heads, cache->head_dim, shift,
                           static_cast<float*>(k_out), static_cast<float*>(v_out));
    return hipGetLastError() == hipSuccess ? DBF_OK : DBF_EHIP;
}
