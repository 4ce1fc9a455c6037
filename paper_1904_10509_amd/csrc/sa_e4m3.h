// e4m3 (OCP: sign, 4 exponent bits, 3 of mantissa, largest 448, 0x7f / 0xff NaN) with
// power-of-two scales.
//
// Why powers of two: code * scale is exact (in bf16 as well: 4 significant bits), so is
// x * 2^-e ahead of the one rounding, and moving a code to a larger scale is exact
// unless it turns subnormal.  A finer scale would gain nothing: a floating format's
// relative step is the same wherever in its range a block lies.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sa_mfma.h"

namespace sa {

constexpr int kMinExp = -100, kMaxExp = 120;  // of a scale

// Least e with amax <= 448 * 2^e, clamped; amax as the bits of a finite float >= 0.
// amax = m 2^x, 1 <= m < 2, and 448 = 1.75 * 2^8: e = x - 8, one more for m > 1.75.
__host__ __device__ inline int scale_exponent(uint32_t amax) {
    const int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < kMinExp ? kMinExp : (e > kMaxExp ? kMaxExp : e);
}
// The exponent of a stored scale (clamped: memory that was never stored to holds anything).
__host__ __device__ inline int exponent_of(uint32_t scale) {
    const int e = (int)(scale >> 23 & 0xffu) - 127;
    return e < kMinExp ? kMinExp : (e > kMaxExp ? kMaxExp : e);
}
// Bits of 2^e, -126 <= e <= 127.
__host__ __device__ inline uint32_t power_bits(int e) { return (uint32_t)(e + 127) << 23; }

#ifdef __HIP_DEVICE_COMPILE__
// Four floats of magnitude <= 448 as codes, nearest, ties to even; x[0] in the low byte.
__device__ inline uint32_t encode4(const float* x) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], r, true);
    return (uint32_t)r;
}
// Four codes as floats.
__device__ inline void decode4(uint32_t u, float* x) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, true);
    x[0] = lo[0];
    x[1] = lo[1];
    x[2] = hi[0];
    x[3] = hi[1];
}
// Four elements over a power of two as codes, nearest, ties to even, straight from words
// of two bf16 or from floats; the first element in the low byte.  Magnitudes of at most
// 448 scales.
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ inline uint32_t encode_word(uint32_t ab, uint32_t cd, float scale) {
    s16x2 r{0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, ab), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, cd), scale, true);
    return __builtin_bit_cast(uint32_t, r);
}
__device__ inline uint32_t encode_word(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float scale) {
    s16x2 r{0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(a), __uint_as_float(b), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(c), __uint_as_float(d), scale, true);
    return __builtin_bit_cast(uint32_t, r);
}
// Two codes of a word (its upper half if HI) times a power of two, as two bf16: exact.
template <bool HI>
__device__ inline uint32_t scaled2(uint32_t u, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, scale, HI));
}
#else
__device__ inline uint32_t encode4(const float*) { return 0; }
__device__ inline void decode4(uint32_t, float*) {}
__device__ inline uint32_t encode_word(uint32_t, uint32_t, float) { return 0; }
__device__ inline uint32_t encode_word(uint32_t, uint32_t, uint32_t, uint32_t, float) { return 0; }
template <bool HI>
__device__ inline uint32_t scaled2(uint32_t, float) {
    return 0;
}
#endif
// Eight codes times a power of two, as eight bf16.
__device__ inline bf16x8 scaled8(uint32_t lo, uint32_t hi, float scale) {
    return __builtin_bit_cast(bf16x8, u32x4{scaled2<false>(lo, scale), scaled2<true>(lo, scale),
                                            scaled2<false>(hi, scale), scaled2<true>(hi, scale)});
}

}  // namespace sa
