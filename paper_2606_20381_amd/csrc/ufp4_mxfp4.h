// Shared by the kernels on microscaled 4-bit operands.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ufp4 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kNaNScale = 255;

// Two bf16 values to byte BYTE of c.
template <int BYTE>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t c, uint32_t w, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w), scale, BYTE);
}

// Two maxima of 16-bit patterns at once.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// The scale byte of a block whose largest magnitude has the fp32 exponent field ef (255: not finite).
__device__ __forceinline__ uint32_t scale_byte(uint32_t ef) { return ef == 255u ? kNaNScale : ef > 2u ? ef - 2u : 0u; }

// A block's 32 bf16 values (pairs, element 2j in the low half of w[j]) to 16 bytes of codes, to nearest; returns the scale
// byte.
__device__ __forceinline__ uint32_t micro_block_bf16(const uint32_t (&w)[16], uint4& codes) {
    uint32_t m = 0, c[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max_u16x2(m, w[i] & 0x7FFF7FFFu);
    const uint32_t lo = m & 0xFFFFu, hi = m >> 16;
    const uint32_t e8 = scale_byte((lo > hi ? lo : hi) >> 7);
    const float scale = __uint_as_float(e8 << 23);
    if (e8 != kNaNScale) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[i] = fp4_pair<0>(c[i], w[4 * i], scale);
            c[i] = fp4_pair<1>(c[i], w[4 * i + 1], scale);
            c[i] = fp4_pair<2>(c[i], w[4 * i + 2], scale);
            c[i] = fp4_pair<3>(c[i], w[4 * i + 3], scale);
        }
    }
    codes = make_uint4(c[0], c[1], c[2], c[3]);
    return e8;
}

// Where position `pos` of the groups' concatenation, each group padded to a multiple of PAD, lies: its row among the
// unpadded ones and how many of its group's rows remain from there (0 or less: padding). False past the last group. Every
// lane of a wave calls this with the same arguments and gets the same answer: 64 groups per step, by a sum over the lanes.
template <int PAD>
__device__ __forceinline__ bool padded_position(const int64_t* off, int G, int64_t pos, int64_t& src, int64_t& left) {
    const int lane = threadIdx.x & 63;
    int64_t base = 0;
    for (int g0 = 0; g0 < G; g0 += 64) {
        const int g = g0 + lane;
        const int64_t start = g < G ? off[g] : 0;
        int64_t m = g < G ? off[g + 1] - start : 0;
        if (m < 0) m = 0;
        const int64_t pad = (m + PAD - 1) / PAD * PAD;
        int64_t inc = pad;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t v = __shfl_up(inc, d, 64);
            if (lane >= d) inc += v;
        }
        const int64_t first = base + inc - pad;
        const uint64_t hit = __ballot(pos >= first && pos < first + pad);
        if (hit) {
            const int at = __builtin_ctzll(hit);
            src = __shfl(start + (pos - first), at, 64);
            left = __shfl(m - (pos - first), at, 64);
            return true;
        }
        base += __shfl(inc, 63, 64);
    }
    src = 0;
    left = 0;
    return false;
}

}  // namespace ufp4
