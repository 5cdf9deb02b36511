// The cache in 4 bits and the element types of the entry points around it: layout, conversions, checks (include/dbf.h describes the layout).
#ifndef DBF_CACHE_H
#define DBF_CACHE_H

#include <hip/hip_runtime.h>

#include <climits>
#include <cstdint>

#include "../../include/dbf.h"

typedef _Float16 dbf_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 dbf_h4 __attribute__((ext_vector_type(4)));
typedef _Float16 dbf_h8 __attribute__((ext_vector_type(8)));
typedef float dbf_f4 __attribute__((ext_vector_type(4)));
typedef float dbf_f16 __attribute__((ext_vector_type(16)));
typedef unsigned int dbf_u2 __attribute__((ext_vector_type(2)));
typedef unsigned int dbf_u4 __attribute__((ext_vector_type(4)));
typedef unsigned int dbf_u4_any __attribute__((ext_vector_type(4), aligned(2)));   // read or written at any even address
typedef unsigned int dbf_u2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef unsigned int dbf_u1_any __attribute__((aligned(2)));

struct dbf_bf16 {
    uint16_t bits;
};

__device__ __forceinline__ float dbf_to_float(_Float16 v) { return (float)v; }
__device__ __forceinline__ float dbf_to_float(float v) { return v; }
__device__ __forceinline__ float dbf_to_float(dbf_bf16 v) { return __builtin_bit_cast(float, (unsigned)v.bits << 16); }
template <typename T>
__device__ __forceinline__ T dbf_from_float(float v) {
    return (T)v;
}
template <>
__device__ __forceinline__ dbf_bf16 dbf_from_float<dbf_bf16>(float v) {   // to the nearest, ties to even; no numbers stay that
    const __bf16 b = (__bf16)v;
    return __builtin_bit_cast(dbf_bf16, b);
}

// Sizes of a cache.  A record is 32 tokens of one head: 36 bytes a value of head_dim.
__host__ __device__ __forceinline__ long long dbf_record_bytes(int head_dim) { return 36LL * head_dim; }
static inline bool dbf_cache_shape_ok(int n_pages, int page_tokens, int n_kv_heads, int head_dim) {
    if (n_pages < 1 || n_kv_heads < 1 || n_kv_heads > 65535) return false;
    if (page_tokens != 32 && page_tokens != 64 && page_tokens != 128 && page_tokens != 256) return false;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return false;
    return (long long)n_pages * page_tokens <= INT_MAX;   // (slots are 32-bit)
}
// DBF_OK, or what is wrong with its sizes, or with it
static inline int dbf_cache_check_sizes(const dbf_cache* c) {
    if (!c) return DBF_EINVAL;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return DBF_ESHAPE;
    return dbf_cache_shape_ok(c->n_pages, c->page_tokens, c->n_kv_heads, c->head_dim) ? DBF_OK : DBF_EINVAL;
}
static inline int dbf_cache_check(const dbf_cache* c) {
    if (!c || !c->data || (reinterpret_cast<uintptr_t>(c->data) & 15)) return DBF_EINVAL;
    return dbf_cache_check_sizes(c);
}
static inline bool dbf_misaligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// Byte offset of the record that holds a slot's token.
__device__ __forceinline__ long long dbf_record_at(int slot, int head, int n_heads, int page_shift, int head_dim) {
    const long long page = slot >> page_shift;
    const int blocks = 1 << (page_shift - 5), block = (slot & ((1 << page_shift) - 1)) >> 5;
    return ((page * n_heads + head) * blocks + block) * dbf_record_bytes(head_dim);
}
static inline int dbf_page_shift(int page_tokens) { return page_tokens == 32 ? 5 : page_tokens == 64 ? 6 : page_tokens == 128 ? 7 : 8; }

// 1 / by as the sum of two fp32, and x times it: two instructions for ten of a division, and as correctly rounded where `by` has at most 7 significant bits: the sum is
// exact to 2^-47, and no quotient by so few bits lies nearer than 2^-33 of itself to the middle of two fp32.
struct DbfInverse {
    float most, rest;
};
__device__ __forceinline__ float dbf_quotient(float x, const DbfInverse& inverse) { return fmaf(x, inverse.most, x * inverse.rest); }
// The scale of a group whose values and zero span `range`: over 15, rounded up to 7 significant bits, and to a multiple of 2^-24.
__device__ __forceinline__ float dbf_group_scale(float range) {
    constexpr DbfInverse fifteenth = {1.0f / 15.0f, (float)(1.0 / 15.0 - (double)(1.0f / 15.0f))};
    const unsigned bits = (__builtin_bit_cast(unsigned, dbf_quotient(range, fifteenth)) + 0x1FFFFu) & ~0x1FFFFu;
    return ceilf(__builtin_bit_cast(float, bits) * 16777216.0f) * (1.0f / 16777216.0f);
}
constexpr float DBF_CACHE_MOST = 57344.0f;   // larger values are held as this: every value held, s / 2 beyond it at most, is finite in fp16

#endif  // DBF_CACHE_H
