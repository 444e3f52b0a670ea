// fff_pack.hpp -- rows in 8 bits: e4m3 values (four exponent bits, three of mantissa, largest
// 448, no infinities) with one power of two for every 32 columns of a row, kept as its exponent
// + 127 in a byte (255: NaN).
//
// The scale of a block is the smallest power of two that brings its largest finite value to
// at most 448, so no value is cut off; a power of two, since it moves no mantissa bit: what a block holds
// are e4m3's own roundings (half a step, 2^-4 of a value; below 2^-15 of the block's largest at worst,
// where e4m3 has no more exponents, 2^-10 of the scale).  Packed values are exact in fp32, and in bf16 from scale code 3 on:
// e4m3's smallest value is 2^-9, bf16's 2^-133.
#pragma once

#include "fff_rows.hpp"

#include <hip/hip_runtime.h>

#include <cstdint>

namespace fff {

constexpr int PACK_BLOCK = 32;  // columns that share a scale

__host__ __device__ __forceinline__ int64_t pack_blocks(int64_t hidden) { return (hidden + PACK_BLOCK - 1) / PACK_BLOCK; }

// The bits of |v|, 0 where v is infinite or NaN: ordered as the values are.
__device__ __forceinline__ uint32_t finite_bits(float v) {
    const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0;
}
// The scale's code for the largest of those: exponents are one up where the mantissa is past 448's 1.75.
__device__ __forceinline__ uint32_t scale_code(uint32_t most) {
    const uint32_t e = (most + 0x1fffffu) >> 23;
    return e > 8 ? e - 8 : 0;
}
// 1 / scale (codes that scale_code gives: at most 247), and the scale of any code.
__device__ __forceinline__ float scale_inverse(uint32_t code) { return __uint_as_float((254 - code) << 23); }
constexpr uint32_t INFINITE_CODE = 247;  // 448 times 2^120 is past fp32: values of this scale and of larger ones may be infinite
__device__ __forceinline__ float scale_value(uint32_t code) {
    return __uint_as_float(code == 255 ? 0x7fc00000u : code ? code << 23 : 0x00400000u);
}
// v / scale.  Beside the largest scale, 256 times it is past fp32: what would round to that becomes 240 times
// it, so that finite values stay finite.
__device__ __forceinline__ float scaled(float v, uint32_t code, float inverse) {
    v *= inverse;
    if (code == 247 && __builtin_fabsf(v) > 240.0f && __builtin_fabsf(v) <= 256.0f) v = __builtin_copysignf(240.0f, v);
    return v;
}
// Four values in e4m3, to the nearest, even at ties.  The conversion makes infinities NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return uint32_t(w);
}
// Four values times their scale, which is a power of two (the conversion adds its exponent) or NaN.
__device__ __forceinline__ void unpack_e4m3(float* f, uint32_t w, float scale) {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
    f[0] = lo[0];
    f[1] = lo[1];
    f[2] = hi[0];
    f[3] = hi[1];
}

// The larger of v and the value of the lane whose number differs in bit 0, 1 or 2 of eight lanes' (DPP).
__device__ __forceinline__ uint32_t max_quad(uint32_t v) {
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0xb1, 0xf, 0xf, false)));  // quad_perm 1 0 3 2
    return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x4e, 0xf, 0xf, false)));  // quad_perm 2 3 0 1
}
__device__ __forceinline__ uint32_t max_eight(uint32_t v) {
    v = max_quad(v);
    return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x141, 0xf, 0xf, false)));  // row_half_mirror
}

}  // namespace fff
