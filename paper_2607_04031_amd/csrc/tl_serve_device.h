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

// two of a word's eight E2M1 values, of byte BYTE, times a power of two, of which
// the instruction takes the exponent's bits alone: exact in bf16, infinity past
// it, NaN if the bits are all ones
template <int BYTE>
__device__ inline uint32_t fp4_to_bf16(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, BYTE));
}
// all eight
__device__ inline u32x4 fp4_to_bf16x8(uint32_t w, float scale) {
    return u32x4{fp4_to_bf16<0>(w, scale), fp4_to_bf16<1>(w, scale), fp4_to_bf16<2>(w, scale), fp4_to_bf16<3>(w, scale)};
}

// 2^(e - 127) of a biased exponent
__device__ inline float exp_scale(uint32_t e) { return __uint_as_float(e << 23); }

// a / b of a >= 0, b > 0 below 2^53.  A workgroup of the attention kernels makes six
// such divisions in a row before its first load.  Below 2^31: by way of a float's reciprocal, off by at
// most 2^-21 of itself, and of that of what is left (below 2^10 b, so that the
// second is off by less than one): 20 instructions; else by way of a double, 50,
// and a sixth of a 64-bit integer division's.
__device__ inline int64_t quotient(int64_t a, int64_t b) {
    if (uint64_t(a) < 0x80000000u && uint64_t(b) < 0x80000000u) {
        const float inv = __builtin_amdgcn_rcpf(float(int(b)));
        int q = int(float(int(a)) * inv);
        q += int(float(int(uint32_t(a) - uint32_t(q) * uint32_t(b))) * inv);
        const int r = int(uint32_t(a) - uint32_t(q) * uint32_t(b));
        return q + (r >= int(b)) - (r < 0);
    }
    const int64_t q = int64_t(double(a) / double(b)), r = a - q * b;
    return q + (r >= b) - (r < 0);
}

// Sums over the lanes up to each one: six moves between lanes inside the vector
// unit (through LDS each takes about 60 ns more, one after the other).
template <int CTRL, int ROWS>
__device__ inline int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ inline int64_t moved(int64_t x) {
    return int64_t(uint64_t(uint32_t(moved<CTRL, ROWS>(int(x >> 32)))) << 32 | uint32_t(moved<CTRL, ROWS>(int(x))));
}
template <typename T>
__device__ inline T upto_lane(T x) {
    x += moved<0x111, 0xf>(x);      // the lanes 1, 2, 4, 8 before, of 16
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);      // the last one of the 16, and of the 32, before
    x += moved<0x143, 0xc>(x);
    return x;
}
__device__ inline int of_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ inline int64_t of_lane(int64_t x, int lane) {
    return int64_t(uint64_t(uint32_t(of_lane(int(x >> 32), lane))) << 32 | uint32_t(of_lane(int(x), lane)));
}
template <typename T>
__device__ inline T over_lanes(T x) { return of_lane(upto_lane(x), 63); }

}  // namespace tl
