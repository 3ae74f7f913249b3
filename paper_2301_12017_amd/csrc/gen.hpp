// What the kernels of token generation share (gfx950): the two 16-bit types, fragments of the matrix instructions.
#pragma once
#include "common.hpp"

namespace w4a4 {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

template <bool BF16>
__device__ __forceinline__ float4_t mfma16(u32x4_t a, u32x4_t b, float4_t c) {       // [16 x 32] x [32 x 16], fp32 sums
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}

template <bool BF16>
__device__ __forceinline__ float to_float(uint16_t x) {
    if constexpr (BF16) return __builtin_bit_cast(float, (uint32_t)x << 16);
    else return (float)__builtin_bit_cast(_Float16, x);
}
template <bool BF16>
__device__ __forceinline__ uint16_t from_float(float x) {                            // to nearest even
    if constexpr (BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    else return __builtin_bit_cast(uint16_t, (_Float16)x);
}

// Blocks of the 8-bit cache: 16, 32, 64 or 128 tokens.
inline bool kv8_block_ok(int block) { return block >= 16 && block <= 128 && (block & (block - 1)) == 0; }

}  // namespace w4a4
