// Device helpers of the serving-step kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace tl {

typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// two floats to bf16, to nearest even, in one instruction (a NaN stays one)
__device__ inline uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// two of a word's four E4M3 values times a power of two, exact in bf16
template <bool HIGH>
__device__ inline uint32_t fp8_to_bf16(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}

// 2^(e - 127) of a biased exponent
__device__ inline float exp_scale(uint32_t e) { return __uint_as_float(e << 23); }

}  // namespace tl
