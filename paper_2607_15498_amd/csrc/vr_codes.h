// e4m3 codes and the powers of two of their blocks: shared by the operators that write them.
#pragma once
#include "vr_internal.h"

namespace vr {

constexpr int BLOCK = VARRATE_BLOCK8;                      // tokens of a scale
constexpr int E_LO = -110, E_HI = 119;                     // exponents of scales: every value stays a normal bf16 number

typedef float f32x2 __attribute__((ext_vector_type(2)));

// |x|'s bits where x is a number, 0 for infinities and NaN, which do not count in a block's scale
__device__ __forceinline__ uint32_t magnitude(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
    return u < 0x7F800000u ? u : 0u;
}
// the smallest e that takes magnitudes up to `most` (bits) to 448 = 1.75 x 2^8 or less
__device__ __forceinline__ int exponent_for(uint32_t most) {
    const int e = (int)(most >> 23) - 127 - 8 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < E_LO ? E_LO : e > E_HI ? E_HI : e;
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// a stored scale's exponent, within what this library stores
__device__ __forceinline__ int exponent_of(uint8_t b) {
    const int e = (int)b - 127;
    return e < E_LO ? E_LO : e > E_HI ? E_HI : e;
}
// 8 numbers times s, rounded to the nearest codes; infinities become NaN.  ALL: beyond 448 it is 448 (what blocks of E_HI alone hold)
template <bool ALL>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float s) {
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        y[k] = x[k] * s;
        if (ALL && fabsf(y[k]) > 448.f && fabsf(y[k]) < INFINITY) y[k] = copysignf(448.f, y[k]);
    }
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k], y[4 * k + 1], 0, false);
        w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k + 2], y[4 * k + 3], v, true);
    }
    return uint2{w[0], w[1]};
}
// 8 codes times s
__device__ __forceinline__ void values8(uint2 w, float s, float (&x)[8]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int v = (int)(k ? w.y : w.x);
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(v, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(v, true);
        x[4 * k] = a[0] * s;
        x[4 * k + 1] = a[1] * s;
        x[4 * k + 2] = b[0] * s;
        x[4 * k + 3] = b[1] * s;
    }
}
// the largest of a wave's values, in every lane
__device__ __forceinline__ uint32_t wave_most(uint32_t v) {
#pragma unroll
    for (int m = 1; m < WAVE; m <<= 1) {
        const uint32_t y = __shfl_xor(v, m, WAVE);
        v = y > v ? y : v;
    }
    return v;
}

}  // namespace vr
