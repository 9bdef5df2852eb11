// What all device code of libcusa shares: a layer's cache as the kernels see it, vector types, a rounding.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cusa {

constexpr int D = 128;        // head_dim
constexpr int PAGE = 16;      // tokens per page of a paged cache

struct KvView {
    const uint16_t* k;
    const uint16_t* v;
    int64_t sb, sh, st;       // contiguous: element strides (batch, kv head, token)
    const int32_t* bt;        // paged: block table [B][max_pages]
    int32_t max_pages;
    int32_t G;                // kv heads
    const int32_t* seq_lens;  // [B]
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct CacheArgs {
    KvView kv;
    int32_t n_pages;                       // paged: pages of the pool
    int32_t max_len;                       // positions that may be touched
};

// The row of one position (its number in the pool, or in the sequence's own rows), or -1 for an entry that names no page.
template <bool PAGED>
__device__ __forceinline__ int cache_row(const CacheArgs& c, int b, int kvh, int pos) {
    if (!PAGED) return pos;
    const int page = c.kv.bt[(int64_t)b * c.kv.max_pages + (pos >> 4)];
    return (uint32_t)page < (uint32_t)c.n_pages ? (page * c.kv.G + kvh) * PAGE + (pos & (PAGE - 1)) : -1;
}
// Elements between the cache's start and its row: 64 bits, a cache may be longer than 32 count.
template <bool PAGED>
__device__ __forceinline__ int64_t cache_offset(const CacheArgs& c, int b, int kvh, int row) {
    return PAGED ? (int64_t)row * D : (int64_t)b * c.kv.sb + (int64_t)kvh * c.kv.sh + (int64_t)row * c.kv.st;
}

// A value at a wave-uniform address that no kernel of the launch writes: a scalar load.
__device__ __forceinline__ int32_t uniform_load(const int32_t* p) {
    return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
}

// Where a running maximum of scores starts: no score of a tile needs to be finite.  (From -infinity, a first tile whose scores are all
// -infinity makes NaN of its weights; from here they are 2^-infinity = 0.)
constexpr float LOWEST = -3.402823466e38f;

__device__ __forceinline__ uint16_t f32_to_bf16_rne(float f) {
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7fc0;   // NaN
    u += 0x7fffu + ((u >> 16) & 1u);
    return (uint16_t)(u >> 16);
}

}  // namespace cusa
