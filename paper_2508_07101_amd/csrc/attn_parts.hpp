// What attention kernels of several files share: operands, loads to LDS, weights, the merge of a row's pieces.
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

// A row's pieces by one wave: a lane for each piece's weight, then two columns a lane.
__device__ __forceinline__ void merge_pieces(const float* part_acc, const float* part_ml, int pieces, uint16_t* out, int lane) {
    float m = LOWEST, l = 0.0f;
    if (lane < pieces) {
        const f32x2 ml = *reinterpret_cast<const f32x2*>(part_ml + lane * 2);
        m = ml[0];
        l = ml[1];
    }
    float top = m;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float w = exp2f(m - top);
    float sum = lane < pieces ? w * l : 0.0f;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    f32x2 acc = {0.0f, 0.0f};
    // (a sum that is infinite stays so whatever its piece weighs: the weight is not 0, also where 32 bits hold nothing of it)
    auto add = [&](float wp, f32x2 v) {
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[j] += __builtin_isfinite(v[j]) ? wp * v[j] : v[j];
    };
    const float* part = part_acc + lane * 2;
    int p = 0;
    for (; p + 8 <= pieces; p += 8) {                         // eight at a time under way
        f32x2 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const f32x2*>(part + (p + i) * D);
#pragma unroll
        for (int i = 0; i < 8; ++i) add(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p + i)), v[i]);
    }
    for (; p < pieces; ++p) {
        const f32x2 v = *reinterpret_cast<const f32x2*>(part + p * D);
        add(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p)), v);
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    *reinterpret_cast<uint32_t*>(out + lane * 2) = (uint32_t)f32_to_bf16_rne(acc[0] * inv) | (uint32_t)f32_to_bf16_rne(acc[1] * inv) << 16;
}

}  // namespace cusa
