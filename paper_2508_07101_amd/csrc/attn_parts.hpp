// What attention kernels of several files share: operands, loads to LDS, weights.
#pragma once
#include "cache_view.hpp"

namespace cusa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

// Of the lane's value and that of its counterpart in the other half of the wave.
__device__ __forceinline__ float other_half_max(float v) {
    const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}

// 16 bytes a lane from memory to LDS at `lds` + 16 * lane, past the registers.  Not the builtin: for that, the compiler lets every later
// LDS read wait for all such loads, which leaves one tile under way at most.  Whoever uses the bytes waits for them (wait_tiles) and, where
// another wave asked for them, meets it at a barrier.
// m0 is a reserved register: the compiler keeps nothing in it.  With the streaming hint: the caches need not keep what is read once (a copy of 128 MB to LDS by 256 workgroups: 24.4 us, so 19.7).
__device__ __forceinline__ void load_to_lds(const uint16_t* from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(lds), "v"(from) : "memory");
}
// The same from a uniform address and 32 bits of offset a lane.
__device__ __forceinline__ void load_to_lds(const uint16_t* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}

// A weight 2^(scale x - m).  The instruction makes 0 of results below 2^-126, which beside a value of 2^120 are not nothing: it makes the weight's 2^64-fold.
// (With the sums of the rounded weights 1 to 2 % of tree_attn_kernel for 128 to 512 rows.)
__device__ __forceinline__ float weight(float m, float x, float scale_log2e) {
    return __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale_log2e, 64.0f - m)) * 0x1p-64f;
}

}  // namespace cusa
