// e4m3 values with an exponent for each row of head_dim: conversions between them and bf16.  gfx950.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spa {

// Biased exponent (127 + e) of a row whose largest finite magnitude is amax: the least e with amax <= 448 * 2^e, at least -126.  448 = 1.75 * 2^8, so it goes by
// the bits of amax: mantissas up to 1.75 take its own exponent less 8, larger ones one more.  bf16 inputs leave at most 247.
__device__ __forceinline__ uint32_t row_exponent(float amax) {
    const uint32_t bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(e < 1 ? 1 : e);
}
// 2^(biased - 127) and its inverse, for exponents 1 .. 253
__device__ __forceinline__ float two_to(uint32_t biased) { return __uint_as_float(biased << 23); }
__device__ __forceinline__ float finite_or_zero(float x) { return fabsf(x) < INFINITY ? x : 0.f; }
__device__ __forceinline__ float finite_or_nan(float x) { return fabsf(x) < INFINITY ? x : NAN; }

// four values to e4m3, to the nearest, ties to even; NaN stays NaN
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}
typedef __attribute__((ext_vector_type(2))) __bf16 bf16_pair;
// values 0, 1 (HI: 2, 3) of a word times 2^(biased - 127), scale = two_to(biased): exact
template <bool HI>
__device__ __forceinline__ uint32_t to_bf16_pair(uint32_t word, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale, HI));
}

}  // namespace spa
