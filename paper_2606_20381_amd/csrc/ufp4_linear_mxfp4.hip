// y [M, N] = Q(x) W^T for few tokens: x bf16, W kept as a microscaled 4-bit operand (layout of ufp4_mxfp4.hip).
//
// Bound by reading W once, so the tokens are quantized by the workgroup that needs them and the product is one launch: a
// workgroup takes R rows of W (all of K) and its eight waves split K; each first quantizes its share of x into LDS in the
// layout of W, with the first loads of W already in flight. W goes from memory straight to the registers that the matrix
// instruction reads (runs of R * 16 bytes), and the waves' sums are added through LDS in a fixed order.
// R = 16 (16 x 16 x 128 instruction) gives a narrow W twice the workgroups; R = 32 (32 x 32 x 64) halves the times that x
// is read and quantized.

#include "ufp4_internal.h"
#include "ufp4_mxfp4.h"

#include <type_traits>

namespace ufp4 {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8;
constexpr int kAhead = 4;             // groups of 128 of the reduction that a wave has in flight
constexpr int kLdsBytes = 60 * 1024;  // of quantized x: two workgroups per CU

template <int R>
struct Frag {  // W's part of one group: R = 32: blocks h and 2 + h of the lane's row; R = 16: block q of it
    static constexpr int kCodes = R == 32 ? 2 : 1;
    uint4 c[kCodes];
    uint32_t s;
};

// M <= 16 tokens; M tokens' codes of `groups` groups in LDS at a time: [block][token] 16 bytes, then scales [group][b % 2]
// [token][2].
template <int OUT, int R>
__global__ __launch_bounds__(64 * kWaves) void linear_mxfp4_kernel(LinearJob j, int chunk) {
    extern __shared__ __align__(16) uint8_t smem[];
    const int M = j.M, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * R;
    const int nkb = (int)j.nkb, groups = (nkb + 3) / 4;
    uint8_t* const xc = smem;
    uint8_t* const xs = smem + (size_t)chunk * 4 * M * 16;

    const int row = lane & (R - 1), part = lane / R;  // part: h (R = 32) or q (R = 16)
    const int64_t panel = n0 / 128;
    const uint8_t* const wc = j.w + panel * j.w_pld + ((n0 & 127) + row) * 16;
    const uint8_t* const ws = j.ws + panel * j.ws_pld + (part & 1) * 256 + ((n0 & 127) + row) * 2;
    auto load = [&](int g, Frag<R>& f) {
#pragma unroll
        for (int k = 0; k < Frag<R>::kCodes; ++k) {
            int b = 4 * g + (R == 32 ? 2 * k : 0) + part;
            b = b < nkb ? b : nkb - 1;  // past the end: any codes, the scale is 0
            f.c[k] = *reinterpret_cast<const uint4*>(wc + (int64_t)b * 2048);
        }
        if constexpr (R == 32) f.s = *reinterpret_cast<const uint16_t*>(ws + (int64_t)g * 512);
        else f.s = ws[(int64_t)g * 512 + (part >> 1)];
    };
    typedef typename std::conditional<R == 32, v16f, v4f>::type Acc;
    Acc acc;
#pragma unroll
    for (int i = 0; i < R * R / 64; ++i) acc[i] = 0.0f;
    const int token = row < M ? row : M - 1;  // the instruction's columns past M repeat the last token
    auto multiply = [&](int lg, const Frag<R>& f) {  // lg: group within the chunk
        auto operand = [](const uint4& x) {
            const v8i v = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
            return v;
        };
        const uint8_t* const s = xs + (lg * 2 + (part & 1)) * M * 2 + token * 2;
        if constexpr (R == 32) {
            const int sx = *reinterpret_cast<const uint16_t*>(s);
            const uint4 x0 = *reinterpret_cast<const uint4*>(xc + ((4 * lg + part) * M + token) * 16);
            const uint4 x1 = *reinterpret_cast<const uint4*>(xc + ((4 * lg + 2 + part) * M + token) * 16);
            acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(f.c[0]), operand(x0), acc, 4, 4, 0, f.s, 0, sx);
            acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(f.c[1]), operand(x1), acc, 4, 4, 1, f.s, 1, sx);
        } else {
            const uint4 x0 = *reinterpret_cast<const uint4*>(xc + ((4 * lg + part) * M + token) * 16);
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(f.c[0]), operand(x0), acc, 4, 4, 0, f.s, 0,
                                                                   (int)s[part >> 1]);
        }
    };

    for (int g0 = 0; g0 < groups; g0 += chunk) {
        const int n = groups - g0 < chunk ? groups - g0 : chunk;
        Frag<R> f[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (wave + k * kWaves < n) load(g0 + wave + k * kWaves, f[k]);
        if (g0 > 0) __syncthreads();  // the last chunk's x has been read
        // x's blocks of the chunk, a thread each; blocks past the end: codes and scale 0
        for (int i = tid; i < n * 4 * M; i += 64 * kWaves) {
            const int t = i / (n * 4), lb = i - t * (n * 4), b = g0 * 4 + lb;
            uint32_t w[16], e8 = 0;
            uint4 c = make_uint4(0, 0, 0, 0);
            if (b < nkb) {
                const uint4* const src = reinterpret_cast<const uint4*>(j.x + (int64_t)t * j.ldx + (int64_t)b * 32);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint4 v = src[k];
                    w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
                }
                e8 = micro_block_bf16(w, c);
            }
            *reinterpret_cast<uint4*>(xc + (lb * M + t) * 16) = c;
            xs[((lb >> 2) * 2 + (lb & 1)) * M * 2 + t * 2 + ((lb >> 1) & 1)] = (uint8_t)e8;
        }
        __syncthreads();
        for (int lg = wave; lg < n; lg += kAhead * kWaves) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int g = lg + k * kWaves;
                if (g < n) {
                    multiply(g, f[k]);
                    if (g + kAhead * kWaves < n) load(g0 + g + kAhead * kWaves, f[k]);
                }
            }
        }
    }
    // The waves' sums [wave][token][R], added in the order of the waves. A lane holds token `row` and R^2 / 64 rows of W.
    __syncthreads();
    float* const red = reinterpret_cast<float*>(smem);
    if (row < M) {
#pragma unroll
        for (int q = 0; q < R * R / 256; ++q) {
            const int at = R == 32 ? 8 * q + 4 * part : 4 * part;
            *reinterpret_cast<float4*>(red + (wave * M + row) * R + at) =
                make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
        }
    }
    __syncthreads();
    for (int i = tid; i < M * R; i += 64 * kWaves) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += red[w * M * R + i];
        const int t = i / R;
        const int64_t n = n0 + (i - t * R), at = t * j.ldc + n;
        if (n < j.N) {
            if constexpr (OUT == kOutF32) static_cast<float*>(j.y)[at] = v;
            else static_cast<uint16_t*>(j.y)[at] = __builtin_bit_cast(uint16_t, (__bf16)v);
        }
    }
}

template <int OUT, int R>
hipError_t launch_linear_t(const LinearJob& j, hipStream_t s) {
    const int groups = (int)((j.nkb + 3) / 4);
    int chunk = kLdsBytes / (68 * j.M);  // 68 bytes per token and group
    if (chunk > groups) chunk = groups;
    const int need = chunk * 68 * j.M, sums = kWaves * j.M * R * 4;
    linear_mxfp4_kernel<OUT, R><<<(unsigned)((j.N + R - 1) / R), 64 * kWaves, need > sums ? need : sums, s>>>(j, chunk);
    return hipGetLastError();
}

template <int OUT>
hipError_t launch_linear_r(const LinearJob& j, hipStream_t s) {
    return j.N <= 8192 ? launch_linear_t<OUT, 16>(j, s) : launch_linear_t<OUT, 32>(j, s);
}

}  // namespace

hipError_t launch_linear_mxfp4(const LinearJob& j, hipStream_t s) {
    return j.out_dtype == kOutBF16 ? launch_linear_r<kOutBF16>(j, s) : launch_linear_r<kOutF32>(j, s);
}

}  // namespace ufp4
