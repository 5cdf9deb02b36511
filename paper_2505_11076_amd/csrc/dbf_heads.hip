// Norms and rotation of query and key heads, and the write of keys and values to the cache in 4 bits (include/dbf.h: dbf_qk_norm_rope,
// dbf_cache_append, dbf_cache_read).
//
// Norm: x w / sqrt(mean x^2 + eps); rotation: pairs (a cos - b sin, b cos + a sin).  In fp32, rounded once: to 16 bits, or to a code per value with a scale and
// a zero per 64.
#include <algorithm>
#include <initializer_list>

#include "dbf_cache.h"
#include "dbf_wave.h"

namespace {

constexpr int WAVES = 4, MOST_DIM = 1024;
constexpr long long MOST_ITEMS = (1LL << 23) * WAVES;   // wavefronts of a launch: of 2^32 threads or more only the remainder would run

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

// Any even head size: a wavefront takes one head of one token, by LDS.  (8191 tokens of 40 heads of 96, 129 MB: 192 us.)
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

// Heads of 64 N values with pairs of whole quads: a head is 8 N lanes' with two quads (four values) each, so that a pair of quads that turn into each other is one lane's, and
// 8 / N heads a wavefront's.  Query heads come first, then the key heads (with their values, where those go to the cache); a wavefront has one kind.
// Without a cache bound by the read and the write: 8191 tokens of 32 + 8 heads of 128, 170 MB in 36.5 us (4.65 TB/s; a large copy has 4.95).  (A wavefront to a head, values of a lane 64
// apart and through LDS: 238 us.)
// Into the cache: 2047 tokens of 32 + 32 heads of 128 in 29 us, 11 of them the queries' norms and rotation; the rest are the groups' scales and codes (610 vector instructions of a wavefront with
// keys and values, 16 of them a lane; 187 of one with queries) and stores: codes of values written a byte at a time were 38 us, divisions and maxima as they are written in C one more.
template <typename T>
struct Quad {
    dbf_u2 w;
    __device__ __forceinline__ void load(const T* x, int quad) { w = *reinterpret_cast<const dbf_u2_any*>(x + 4 * quad); }
    __device__ __forceinline__ float operator[](int e) const { return dbf_to_float(__builtin_bit_cast(T, (uint16_t)(w[e >> 1] >> 16 * (e & 1)))); }
    static __device__ __forceinline__ void store(T* x, int quad, const float* v) {
        dbf_u2 out = {0u, 0u};
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e >> 1] |= (unsigned)__builtin_bit_cast(uint16_t, dbf_from_float<T>(v[e])) << 16 * (e & 1);
        *reinterpret_cast<dbf_u2_any*>(x + 4 * quad) = out;
    }
};
template <int N>   // of the 8 N lanes of a head, in all of them
__device__ __forceinline__ float head_sum(float v) {
    if constexpr (N == 1) return dbf_row8_sum_f(v);
    v = dbf_row16_sum_f(v);
    if constexpr (N == 2) return v;
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
// The largest of values that are not negative, by their bits (as numbers a maximum makes each of its operands a quiet one first): of the lanes of a head ...
__device__ __forceinline__ unsigned larger(unsigned v, unsigned w) { return v > w ? v : w; }
template <int CTRL>   // (nothing stays of the register written, so that the move is part of the maximum's instruction)
__device__ __forceinline__ unsigned moved(unsigned v) {
    return (unsigned)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true);
}
template <int N>
__device__ __forceinline__ float head_max(float x) {
    unsigned v = __builtin_bit_cast(unsigned, x);
    v = larger(v, moved<0xB1>(v));    // 1 away
    v = larger(v, moved<0x4E>(v));    // 2
    v = larger(v, moved<0x141>(v));   // 4: the other half of eight lanes, which has one value by now
    if constexpr (N > 1) v = larger(v, moved<0x128>(v));   // 8
    if constexpr (N > 2) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = larger(r[0], r[1]);
    }
    return __builtin_bit_cast(float, v);
}
// ... and of those that agree in bits 2 .. of their place but the top one.
template <int N>
__device__ __forceinline__ float group_max(float x) {
    unsigned v = __builtin_bit_cast(unsigned, x);
    v = larger(v, moved<0xB1>(v));
    v = larger(v, moved<0x4E>(v));
    if constexpr (N == 1) v = larger(v, moved<0x141>(v));
    if constexpr (N == 2) v = larger(v, moved<0x128>(v));
    if constexpr (N == 4) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = larger(r[0], r[1]);
    }
    return __builtin_bit_cast(float, v);
}
// A value's code, as a number.  Its quotient has to be correctly rounded: a value of few bits may lie halfway between two codes.
__device__ __forceinline__ float code_of(float x, const DbfInverse& inverse, float z) { return __builtin_amdgcn_fmed3f(rintf(dbf_quotient(x, inverse)) + z, 0.f, 15.f); }
// Of a scale (1 for 0), which has at most 7 bits: its product with the approximate inverse is exact in the remainder.
__device__ __forceinline__ DbfInverse inverse_of(float scale) {
    const float by = scale > 0.f ? scale : 1.f, near = __builtin_amdgcn_rcpf(by), most = fmaf(fmaf(-by, near, 1.f), near, near);
    return {most, fmaf(-by, most, 1.f) * most};
}
// Values within what the cache holds; whether all are finite.  (The sum of their sizes says that nothing is to be done, nearly always.)
__device__ __forceinline__ bool hold(float* x) {
    const float size = ((fabsf(x[0]) + fabsf(x[1])) + (fabsf(x[2]) + fabsf(x[3]))) + ((fabsf(x[4]) + fabsf(x[5])) + (fabsf(x[6]) + fabsf(x[7])));
    bool fine = true;
    if (__any(!(size <= DBF_CACHE_MOST))) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool finite = fabsf(x[e]) < __builtin_inff();
            fine = fine && finite;
            x[e] = finite ? fminf(fmaxf(x[e], -DBF_CACHE_MOST), DBF_CACHE_MOST) : 0.f;
        }
    }
    return fine;
}

// Tokens of a wavefront's key heads on their way to the cache: in a row of slots, four tokens' codes of a value share a word, which one lane writes.
constexpr int tokens_together(int N, bool cache) { return !cache ? 1 : N == 4 ? 2 : 4; }
template <typename T, int N, bool CACHE>
__global__ __launch_bounds__(64 * WAVES) void dbf_heads_quads_kernel(const HeadsArgs a) {
    constexpr int D = 64 * N, LANES = 8 * N, HEADS = 8 / N, TOKENS = tokens_together(N, CACHE);
    const int lane = threadIdx.x & 63, sub = lane % LANES;
    const int q_steps = a.q ? (a.n_q + HEADS - 1) / HEADS : 0, k_steps = a.k ? (a.n_kv * TOKENS + HEADS - 1) / HEADS : 0;
    // (neighbouring tokens, whose values share the cache's bytes and lines, to one compute die: workgroups are dealt out to the eight one by one)
    const unsigned each = gridDim.x / 8, group = CACHE && blockIdx.x < 8 * each ? blockIdx.x % 8 * each + blockIdx.x / 8 : blockIdx.x;
    const unsigned item = group * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), per = TOKENS * q_steps + k_steps;
    const int first = (int)(item / per) * TOKENS, step = (int)(item % per);   // first of its tokens
    const bool query = step < TOKENS * q_steps;
    const int turn = query ? step / q_steps : lane / LANES % TOKENS, there = first + turn;
    if (query ? there >= a.n_tokens : first >= a.n_tokens) return;
    const int n = query ? a.n_q : a.n_kv, head = query ? step % q_steps * HEADS + lane / LANES : (step - TOKENS * q_steps) * (HEADS / TOKENS) + lane / LANES / TOKENS;
    const bool live = head < n && there < a.n_tokens;
    const int at = min(head, n - 1), token = min(there, a.n_tokens - 1);
    // the lane's quads
    const int hq = a.interleaved ? 0 : a.rot >> 3;   // quads of half the rotated values
    const int qa = sub < hq ? sub : 2 * sub, qb = sub < hq ? sub + hq : 2 * sub + 1;
    const bool turns = a.rope && (a.interleaved ? 8 * sub < a.rot : sub < hq);
    const T* x = query ? static_cast<const T*>(a.q) + token * a.q_stride : static_cast<const T*>(a.k) + token * a.k_stride;
    const T* weight = static_cast<const T*>(query ? a.q_weight : a.k_weight);
    Quad<T> xa, xb, wa, wb;
    xa.load(x + (long long)at * D, qa);
    xb.load(x + (long long)at * D, qb);
    if (weight) {
        wa.load(weight, qa);
        wb.load(weight, qb);
    }
    // values of the cache: a quad and the one that shares its bytes
    const int vq = sub / (4 * N), vp = (sub >> 2) % N, vu = sub & 3, va = 4 * (vp + 2 * N * vq) + vu;
    int slot = -1;
    Quad<T> ya, yb;
    if (CACHE && !query) {
        const T* v = static_cast<const T*>(a.v) + token * a.v_stride + (long long)at * D;
        ya.load(v, va);
        yb.load(v, va + 4 * N);
        slot = a.slots[token];
    }
    dbf_f4 c = {1.f, 1.f, 1.f, 1.f}, sn = {0.f, 0.f, 0.f, 0.f};
    if (a.rope) {
        const int p = a.positions[token];
        const bool known = p >= 0 && p < a.rope_len;
        if (turns) {
            typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
            const float* table = a.rope + (long long)(known ? p : 0) * a.rot + 4 * sub;
            c = *reinterpret_cast<const f4_any*>(table);
            sn = *reinterpret_cast<const f4_any*>(table + (a.rot >> 1));
            if (!known) c[0] = c[1] = c[2] = c[3] = __builtin_nanf("");
        }
    }
    float v[8];   // quad a, quad b
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = xa[e];
        v[4 + e] = xb[e];
        sum = fmaf(v[e], v[e], fmaf(v[4 + e], v[4 + e], sum));
    }
    if (weight) {
        const float scale = 1.f / sqrtf(head_sum<N>(sum) / (float)D + a.eps);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] *= scale * wa[e];
            v[4 + e] *= scale * wb[e];
        }
    }
    if (!turns) {   // (also no product with 0: its partner may be infinite)
    } else if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float s = v[2 * e], t = v[2 * e + 1];
            v[2 * e] = s * c[e] - t * sn[e];
            v[2 * e + 1] = t * c[e] + s * sn[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float s = v[e], t = v[4 + e];
            v[e] = s * c[e] - t * sn[e];
            v[4 + e] = t * c[e] + s * sn[e];
        }
    }
    if (query || !CACHE) {
        T* out = query ? static_cast<T*>(a.q_out) + token * a.q_out_stride : static_cast<T*>(a.k_out) + token * a.k_out_stride;
        if (live) {
            Quad<T>::store(out + (long long)head * D, qa, v);
            Quad<T>::store(out + (long long)head * D, qb, v + 4);
        }
        return;
    }
    if constexpr (!CACHE) return;
    const bool held = live && slot >= 0 && slot < a.n_slots;
    if (!__any(held)) return;
    const int slot0 = __shfl(slot, lane & ~(LANES * (TOKENS - 1)));   // the first token's
    const bool row = __all(there < a.n_tokens && slot >= 0 && slot < a.n_slots && slot == slot0 + turn);
    float y[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        y[e] = ya[e];
        y[4 + e] = yb[e];
    }
    const bool k_fine = hold(v), own_fine = hold(y) && k_fine;
    const bool fine = !((__ballot(!own_fine) >> (lane & ~(LANES - 1))) & ((N == 4 ? 0xFFFFFFFFull : (1ull << LANES) - 1)));
    // the keys' groups: a quad's group is that of its run of four quads
    const int ga = (qa >> 2) % N, gb = (qb >> 2) % N;
    float ks[N];
    float lo_a = fminf(fminf(v[0], v[1]), fminf(v[2], v[3])), hi_a = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
    float lo_b = fminf(fminf(v[4], v[5]), fminf(v[6], v[7])), hi_b = fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7]));
    DbfInverse ia = {}, ib = {};
    float za = 0.f, zb = 0.f, s_own = 0.f, z_own = 0.f;
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const float low = head_max<N>(fmaxf(fmaxf(ga == p ? -lo_a : 0.f, gb == p ? -lo_b : 0.f), 0.f)), high = head_max<N>(fmaxf(fmaxf(ga == p ? hi_a : 0.f, gb == p ? hi_b : 0.f), 0.f));
        ks[p] = dbf_group_scale(high + low);
        const DbfInverse inverse = inverse_of(ks[p]);
        const float zero = rintf(dbf_quotient(low, inverse));
        if (ga == p) ia = inverse, za = zero;
        if (gb == p) ib = inverse, zb = zero;
        if (sub == p) s_own = ks[p], z_own = zero;
    }
    // the values' group: lanes of the same vp
    float vlo = 0.f, vhi = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        vlo = fmaxf(vlo, -y[e]);
        vhi = fmaxf(vhi, y[e]);
    }
    vlo = group_max<N>(vlo);
    vhi = group_max<N>(vhi);
    const float vs = dbf_group_scale(vhi + vlo);
    const DbfInverse v_inverse = inverse_of(vs);
    const float vz = rintf(dbf_quotient(vlo, v_inverse));
    unsigned bytes = 0;   // of four places, the group's first 4 vu
#pragma unroll
    for (int e = 0; e < 4; ++e) bytes |= (unsigned)fmaf(code_of(y[4 + e], v_inverse, vz), 16.f, code_of(y[e], v_inverse, vz)) << 8 * e;
    if (TOKENS > 1 && row) {   // lane of a token: one place (two of two tokens), its tokens' bytes
        unsigned others = 0;
#pragma unroll
        for (int j = 0; j < TOKENS; ++j) {
            const unsigned w = __shfl(bytes, (lane & ~(LANES * (TOKENS - 1))) + j * LANES);
            if constexpr (TOKENS == 4) others |= (w >> 8 * turn & 255) << 8 * j;
            else others |= (w >> 16 * turn & 255) << 8 * j | (w >> (16 * turn + 8) & 255) << (8 * j + 16);
        }
        bytes = others;
    }
    if (!held) return;
    uint8_t* rec = a.cache + dbf_record_at(slot, head, a.n_kv, a.page_shift, D);
    const int t = slot & 31;
    auto place = [&](int slot, int l) {   // of a token's byte of the group's place l
        return a.cache + dbf_record_at(slot, head, a.n_kv, a.page_shift, D) + 1024 * N + 1024 * vp + 16 * (16 * (slot >> 2 & 3) + l) + 4 * (2 * vq + (slot >> 4 & 1)) + (slot & 3);
    };
    auto pack = [](const float* x, const DbfInverse& inverse, float zero) {   // four codes, 16 bits: whole numbers below 2^16 in fp32
        return (uint16_t)(unsigned)fmaf(fmaf(fmaf(code_of(x[3], inverse, zero), 16.f, code_of(x[2], inverse, zero)), 16.f, code_of(x[1], inverse, zero)), 16.f,
                                        code_of(x[0], inverse, zero));
    };
    *reinterpret_cast<uint16_t*>(rec + t * 32 * N + 2 * qa) = pack(v, ia, za);
    *reinterpret_cast<uint16_t*>(rec + t * 32 * N + 2 * qb) = pack(v + 4, ib, zb);
    const int row0 = __builtin_amdgcn_readfirstlane(slot0), i0 = row0 & 3;   // (of a row it is all lanes' first)
    if (TOKENS == 1 || !row || (TOKENS == 2 && (i0 & 1))) {
        if (TOKENS == 2 && row) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                *place(row0, 4 * vu + 2 * turn + e) = (uint8_t)(bytes >> 16 * e);
                *place(row0 + 1, 4 * vu + 2 * turn + e) = (uint8_t)(bytes >> (16 * e + 8));
            }
        } else {
            uint8_t* own = place(slot, 4 * vu);
#pragma unroll
            for (int e = 0; e < 4; ++e) own[16 * e] = (uint8_t)(bytes >> 8 * e);
        }
    } else if (TOKENS == 2) {
#pragma unroll
        for (int e = 0; e < 2; ++e) *reinterpret_cast<uint16_t*>(place(row0, 4 * vu + 2 * turn + e)) = (uint16_t)(bytes >> 16 * e);
    } else {   // from i0 on in one word of four tokens, the rest in the next one
        uint8_t *one = place(row0, 4 * vu + turn), *next = place(row0 + 4 - i0, 4 * vu + turn);
        if (i0 == 0) *reinterpret_cast<unsigned*>(one) = bytes;
        else if (i0 == 1) *one = (uint8_t)bytes, *reinterpret_cast<uint16_t*>(one + 1) = (uint16_t)(bytes >> 8), *next = (uint8_t)(bytes >> 24);
        else if (i0 == 2) *reinterpret_cast<uint16_t*>(one) = (uint16_t)bytes, *reinterpret_cast<uint16_t*>(next) = (uint16_t)(bytes >> 16);
        else *one = (uint8_t)bytes, *reinterpret_cast<uint16_t*>(next) = (uint16_t)(bytes >> 8), next[2] = (uint8_t)(bytes >> 24);
    }
    dbf_h2* words = reinterpret_cast<dbf_h2*>(rec + 2048 * N);
    if (sub < N) words[32 * sub + t] = (dbf_h2){(_Float16)s_own, (_Float16)(fine ? -s_own * z_own : __builtin_nanf(""))};
    if (vq == 0 && vu == 0) words[32 * N + 32 * vp + t] = fine ? (dbf_h2){(_Float16)vs, (_Float16)(-vs * vz)} : (dbf_h2){(_Float16)0.f, (_Float16)0.f};
}

template <typename T>
__device__ __forceinline__ void store4(T* out, const float* v) {
    if constexpr (sizeof(T) == 4) {
        typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
        *reinterpret_cast<f4_any*>(out) = (f4_any){v[0], v[1], v[2], v[3]};
    } else {
        Quad<T>::store(out, 0, v);
    }
}
// Lanes as in the kernel above: a lane has two neighbouring quads of the keys, and of the values a quad and the one that shares its bytes.
template <typename T, int N>
__global__ __launch_bounds__(64 * WAVES) void dbf_cache_read_kernel(const uint8_t* cache, const int* slots, int n_tokens, int n_slots, int n_kv, int page_shift, T* k_out, T* v_out) {
    constexpr int D = 64 * N, LANES = 8 * N, HEADS = 8 / N;
    const int lane = threadIdx.x & 63, sub = lane % LANES, steps = (n_kv + HEADS - 1) / HEADS;
    const unsigned item = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = (int)(item / steps), head = (int)(item % steps) * HEADS + lane / LANES;
    if (token >= n_tokens || head >= n_kv) return;
    const int slot = slots[token];
    float k[8] = {}, v[8] = {};
    const int vq = sub / (4 * N), vp = (sub >> 2) % N, vu = sub & 3, va = 4 * (vp + 2 * N * vq) + vu;
    if (slot >= 0 && slot < n_slots) {
        const uint8_t* rec = cache + dbf_record_at(slot, head, n_kv, page_shift, D);
        const int t = slot & 31, tile = t >> 4, g = (t >> 2) & 3, i = t & 3;
        const dbf_h2* words = reinterpret_cast<const dbf_h2*>(rec + 2048 * N);
        const dbf_h2 kw = words[32 * ((sub >> 1) % N) + t], vw = words[32 * N + 32 * vp + t];
        const unsigned codes = *reinterpret_cast<const unsigned*>(rec + t * 32 * N + 4 * sub);
        const uint8_t* bytes = rec + 1024 * N + 1024 * vp + 16 * (16 * g + 4 * vu) + 4 * (2 * vq + tile) + i;
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] = fmaf((float)kw[0], (float)(codes >> 4 * e & 15), (float)kw[1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned b = bytes[16 * e];
            v[e] = fmaf((float)vw[0], (float)(b & 15), (float)vw[1]);
            v[4 + e] = fmaf((float)vw[0], (float)(b >> 4), (float)vw[1]);
        }
    }
    const long long at = ((long long)token * n_kv + head) * D;
    store4(k_out + at + 8 * sub, k);
    store4(k_out + at + 8 * sub + 4, k + 4);
    store4(v_out + at + 4 * va, v);
    store4(v_out + at + 4 * (va + 4 * N), v + 4);
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

template <typename T, int N>
void launch_quads(const HeadsArgs& a, unsigned groups, hipStream_t stream) {
    const auto kernel = a.cache ? dbf_heads_quads_kernel<T, N, true> : dbf_heads_quads_kernel<T, N, false>;
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(64 * WAVES), 0, stream, a);
}
template <typename T>
int launch_heads(const HeadsArgs& all, hipStream_t stream) {
    // heads of 64, 128 and 256 values that turn by whole quads; any other by the general kernel
    const bool quads = (all.dim == 64 || all.dim == 128 || all.dim == 256) && all.rot % 8 == 0;
    const int heads = quads ? 512 / all.dim : 1, together = quads ? tokens_together(all.dim / 64, all.cache) : 1;   // of a wavefront
    const long long per = (all.q ? together * ((all.n_q + heads - 1) / heads) : 0) + (all.k ? (all.n_kv * together + heads - 1) / heads : 0);   // items of so many tokens
    const long long most = MOST_ITEMS / per * together;
    for (long long t = 0; t < all.n_tokens; t += most) {
        HeadsArgs a = all;
        a.n_tokens = (int)std::min(most, all.n_tokens - t);
        if (a.q) a.q = static_cast<const T*>(a.q) + t * a.q_stride, a.q_out = static_cast<T*>(a.q_out) + t * a.q_out_stride;
        if (a.k) a.k = static_cast<const T*>(a.k) + t * a.k_stride;
        if (a.k_out) a.k_out = static_cast<T*>(a.k_out) + t * a.k_out_stride;
        if (a.v) a.v = static_cast<const T*>(a.v) + t * a.v_stride;
        if (a.positions) a.positions += t;
        if (a.slots) a.slots += t;
        const unsigned groups = (unsigned)(((a.n_tokens + (long long)together - 1) / together * per + WAVES - 1) / WAVES);
        if (!quads) hipLaunchKernelGGL(dbf_heads_kernel<T>, dim3(groups), dim3(64 * WAVES), 0, stream, a);
        else if (a.dim == 64) launch_quads<T, 1>(a, groups, stream);
        else if (a.dim == 128) launch_quads<T, 2>(a, groups, stream);
        else launch_quads<T, 4>(a, groups, stream);
        if (hipGetLastError() != hipSuccess) return DBF_EHIP;
    }
    return DBF_OK;
}

int launch_heads(const HeadsArgs& a, int dtype, hipStream_t stream) {
    return dtype == DBF_F16 ? launch_heads<_Float16>(a, stream) : launch_heads<dbf_bf16>(a, stream);
}

template <typename T>
int launch_read(const dbf_cache* c, const int32_t* slots, int n_tokens, void* k_out, void* v_out, hipStream_t stream) {
    const int heads = 512 / c->head_dim;   // of a wavefront
    const long long steps = (c->n_kv_heads + heads - 1) / heads, most = MOST_ITEMS / steps, row = (long long)c->n_kv_heads * c->head_dim;
    const auto kernel = c->head_dim == 64 ? dbf_cache_read_kernel<T, 1> : c->head_dim == 128 ? dbf_cache_read_kernel<T, 2> : dbf_cache_read_kernel<T, 4>;
    for (long long t = 0; t < n_tokens; t += most) {
        const int n = (int)std::min(most, n_tokens - t);
        hipLaunchKernelGGL(kernel, dim3((unsigned)((n * steps + WAVES - 1) / WAVES)), dim3(64 * WAVES), 0, stream, static_cast<const uint8_t*>(c->data), slots + t, n, c->n_pages * c->page_tokens,
                           c->n_kv_heads, dbf_page_shift(c->page_tokens), static_cast<T*>(k_out) + t * row, static_cast<T*>(v_out) + t * row);
        if (hipGetLastError() != hipSuccess) return DBF_EHIP;
    }
    return DBF_OK;
}

}  // namespace

extern "C" size_t dbf_cache_bytes(int n_pages, int page_tokens, int n_kv_heads, int head_dim) {
    if (!dbf_cache_shape_ok(n_pages, page_tokens, n_kv_heads, head_dim)) return 0;
    return (size_t)n_pages * (page_tokens / DBF_CACHE_BLOCK) * n_kv_heads * (size_t)dbf_record_bytes(head_dim);
}

extern "C" int dbf_qk_norm_rope(const dbf_heads* heads, void* hip_stream) {
    if (const int bad = check_heads(heads)) return bad;
    if (heads->k && (!heads->k_out || heads->k_out_stride < (long long)heads->n_kv_heads * heads->head_dim)) return DBF_EINVAL;
    return launch_heads(heads_args(heads), heads->dtype, static_cast<hipStream_t>(hip_stream));
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
    return launch_heads(a, heads->dtype, static_cast<hipStream_t>(hip_stream));
}

extern "C" int dbf_cache_read(const dbf_cache* cache, const int32_t* slots, int n_tokens, void* k_out, void* v_out, int dtype, void* hip_stream) {
    if (const int bad = dbf_cache_check(cache)) return bad;
    if (!slots || !k_out || !v_out || n_tokens < 0 || (dtype != DBF_F16 && dtype != DBF_BF16 && dtype != DBF_F32)) return DBF_EINVAL;
    const unsigned size = dtype == DBF_F32 ? 4 : 2;
    if (dbf_misaligned(slots, 4) || dbf_misaligned(k_out, size) || dbf_misaligned(v_out, size)) return DBF_EINVAL;
    if (!n_tokens) return DBF_OK;
    const auto stream = static_cast<hipStream_t>(hip_stream);
    return dtype == DBF_F16    ? launch_read<_Float16>(cache, slots, n_tokens, k_out, v_out, stream)
           : dtype == DBF_BF16 ? launch_read<dbf_bf16>(cache, slots, n_tokens, k_out, v_out, stream)
                               : launch_read<float>(cache, slots, n_tokens, k_out, v_out, stream);
}
