// Values in 8 bits (e4m3: 1 sign, 4 exponent, 3 mantissa bits, largest 448) with a power-of-two scale per block, held as
// its biased exponent in a byte.
//
// The scale of a block is the smallest power of two, 2^-100 at least, that brings its finite values to 448 at most.  A
// finer scale would gain nothing but a little of the subnormals' range, as e4m3 has an exponent of its own, and a power of
// two costs nothing later: value times scale is exact in bf16, the matrix core takes such scales beside its 8-bit
// operands, and a block's values move to a larger scale exactly, but into subnormals.
#pragma once

#include "common.hpp"

namespace trajspec {

constexpr uint32_t kScaleLowest = 27;    // 2^-100: the smallest e4m3 subnormal times it is a normal bf16
constexpr uint32_t kScaleHighest = 247;  // 2^120: bf16's largest is below 448 times it
constexpr uint32_t kScaleOne = 127;

// Magnitude of a value for the scale, as fp32 bits: infinities and NaN don't count.
__device__ __forceinline__ uint32_t magnitude_bits(float x) {
    const uint32_t a = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}

// Scale byte of the largest magnitude: 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t scale_byte(uint32_t magnitude) {
    const int e = (int)(magnitude >> 23) - 8 + ((magnitude & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < (int)kScaleLowest ? kScaleLowest : (uint32_t)e;
}

// 2^(byte - 127), and its inverse for a byte up to 253.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// Four values, scaled already, to e4m3: nearest, even on ties; infinities and NaN become NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// 16 e4m3 values times a power of two as bf16 (exact).  The pairs stay whole words: taking them apart by element makes this
// compiler use the first value twice.
__device__ __forceinline__ void unpack_e4m3(const u32x4_t& x, float scale, u32x4_t& lo, u32x4_t& hi) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        lo[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, false));
        lo[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, true));
        hi[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 + i], scale, false));
        hi[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 + i], scale, true));
    }
}

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef short s16x2_t __attribute__((ext_vector_type(2)));

// Largest magnitudes of bf16 pairs, by halves: bf16 magnitudes order like their bits.
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b)));
}

// Magnitude (fp32 bits) for the scale of N words of bf16 pairs: two instructions a pair, four where any is not finite.
template <int N>
__device__ __forceinline__ uint32_t magnitude_of(const uint32_t (&x)[N]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max_pair(m, x[i] & 0x7fff7fffu);
    uint32_t top = max(m & 0xffffu, m >> 16);
    if (ballot64(top >= 0x7f80u) != 0ull) {  // rare
        top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t a = x[i] & 0x7fffu, b = x[i] >> 16 & 0x7fffu;
            top = max(top, max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u));
        }
    }
    return top << 16;
}

// Two bf16 pairs divided by a power of two, to e4m3.
__device__ __forceinline__ uint32_t pack_e4m3(uint32_t a, uint32_t b, float scale) {
    s16x2_t w = {};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2_t, a), scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2_t, b), scale, true));
}

}  // namespace trajspec
