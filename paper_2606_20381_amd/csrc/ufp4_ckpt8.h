// Activation checkpoints in 8 bits: E4M3 levels and a power of two 2^e per 32 values of a row, stored as the byte e + 127.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ufp4_rows.h"

namespace ufp4 {

constexpr int kCkpt8Block = 32;
// The smallest scale: with it the lowest place of a level (2^-9) is that of bf16's subnormal numbers (2^-133), so every
// value is a bf16 number.
constexpr int kCkpt8MinExp = -124;
constexpr uint32_t kCkpt8MaxScale = 247;  // of magnitudes above 1.75 2^127

typedef float v2f __attribute__((ext_vector_type(2)));

// Scale byte of a block whose largest finite magnitude is the bits `top`: the smallest e >= kCkpt8MinExp with top <= 448 2^e
// (448 = 1.75 2^8, E4M3's largest number), so that nothing is cut and a level is off by at most 2^-4 of the value. top < 2^128: at
// most byte 247.
__device__ __forceinline__ uint32_t ckpt8_scale(uint32_t top) {
    const int e = (int)(top >> 23) - 135 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)((e < kCkpt8MinExp ? kCkpt8MinExp : e) + 127);
}

// 2^-e of a scale byte: 3 .. 247, so the result is a normal number.
__device__ __forceinline__ float ckpt8_inverse(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }
__device__ __forceinline__ float ckpt8_factor(uint32_t scale) { return __uint_as_float(scale << 23); }

// Four codes of four values. x 2^-e is exact (or far below the smallest level), the conversion rounds to nearest even; infinities
// and NaN become NaN, the format has no infinity.
__device__ __forceinline__ uint32_t ckpt8_encode(float a, float b, float c, float d, float inverse) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, r, true);
}

// The values of four codes, exact.
__device__ __forceinline__ void ckpt8_decode(uint32_t codes, float factor, float (&f)[4]) {
    const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    f[0] = lo[0] * factor;
    f[1] = lo[1] * factor;
    f[2] = hi[0] * factor;
    f[3] = hi[1] * factor;
}

// 16 codes of one block as bf16, exact: the upper halves of the fp32 numbers.
__device__ __forceinline__ void ckpt8_to_bf16(const u32x4_any& codes, uint32_t scale, u32x4_any& lo, u32x4_any& hi) {
    const float factor = ckpt8_factor(scale);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float f[4];
        ckpt8_decode(codes[q], factor, f);
        const uint32_t x = __builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u);
        const uint32_t y = __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u);
        (q < 2 ? lo : hi)[q % 2 * 2] = x;
        (q < 2 ? lo : hi)[q % 2 * 2 + 1] = y;
    }
}

}  // namespace ufp4
