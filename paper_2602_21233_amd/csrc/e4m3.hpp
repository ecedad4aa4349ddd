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

// bytes of 8 rows of 8 the other way round
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&out)[4]) {
    const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab2 = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd2 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    out[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(cd2, ab2, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(cd2, ab2, 0x07060302u);
}
__device__ __forceinline__ void transpose8(const uint2 (&in)[8], uint2 (&out)[8]) {
    uint32_t t[4];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        transpose4(in[4 * x].x, in[4 * x + 1].x, in[4 * x + 2].x, in[4 * x + 3].x, t);
#pragma unroll
        for (int y = 0; y < 4; ++y) (x ? out[y].y : out[y].x) = t[y];
        transpose4(in[4 * x].y, in[4 * x + 1].y, in[4 * x + 2].y, in[4 * x + 3].y, t);
#pragma unroll
        for (int y = 0; y < 4; ++y) (x ? out[4 + y].y : out[4 + y].x) = t[y];
    }
}

}  // namespace spa
