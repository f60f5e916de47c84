// y [M, N] = Q(x) W^T for few tokens: x bf16, W kept as a microscaled 4-bit operand (layout of ufp4_mxfp4.hip).
//
// Bound by reading W once, so the tokens are quantized by the workgroup that needs them and the product is one launch: a
// workgroup takes R rows of W at a time (all of K) and its waves split K. It quantizes x into LDS in the layout of W, once if
// all of it fits, with the first loads of W already in flight. W goes from memory straight to the registers that the matrix
// instruction reads (runs of R * 16 bytes), and the waves' sums are added through LDS in a fixed order.
// Up to 8 MiB of W it takes about 4-6 us whatever its size (launch, one read's latency, the waves' sums); 32768 x 4096 14 us = 5.2
// TB/s, 16384 x 16384 25 us = 5.8 TB/s for one token.
// R = 16 (16 x 16 x 128 instruction) gives a narrow W twice the workgroups; R = 32 (32 x 32 x 64) halves what each reads of x.

#include "ufp4_internal.h"
#include "ufp4_mxfp4.h"

#include <type_traits>

namespace ufp4 {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));

constexpr int kAhead = 4;           // groups of 128 of the reduction that a wave has in flight
constexpr int kGroupBytes = 4 * 17;  // a token's codes and scales of a group

template <int R>
struct Frag {  // W's part of one group: R = 32: blocks h and 2 + h of the lane's row; R = 16: block q of it
    static constexpr int kCodes = R == 32 ? 2 : 1;
    uint4 c[kCodes];
    uint32_t s;
};

// M <= 16 tokens. LDS: `chunk` groups of x at a time, [block][token] 16 bytes, then scales [group][b % 2][token][2]; the waves'
// sums [wave][token][R].
template <int OUT, int R, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 4) void linear_mxfp4_kernel(LinearJob j, int chunk) {
    extern __shared__ __align__(16) uint8_t smem[];
    const int M = j.M, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nkb = (int)j.nkb, groups = (nkb + 3) / 4;
    uint8_t* const xc = smem;
    uint8_t* const xs = smem + (size_t)chunk * 4 * M * 16;
    float* const sums = reinterpret_cast<float*>(smem + ((size_t)chunk * kGroupBytes * M + 15) / 16 * 16);

    const int row = lane & (R - 1), part = lane / R;  // part: h (R = 32) or q (R = 16)
    const int64_t tiles = (j.N + R - 1) / R;
    auto load = [&](int64_t tile, int g, Frag<R>& f) {
        const int64_t n0 = tile * R, panel = n0 / 128;
        const uint8_t* const wc = j.w + panel * j.w_pld + ((n0 & 127) + row) * 16;
        const uint8_t* const ws = j.ws + panel * j.ws_pld + (part & 1) * 256 + ((n0 & 127) + row) * 2;
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
    // x's blocks of the n groups from g0, a thread each; blocks past the end: codes and scale 0
    auto quantize = [&](int g0, int n) {
        for (int i = tid; i < n * 4 * M; i += 64 * WAVES) {
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
    };

    Frag<R> f[kAhead];
    auto begin = [&](int64_t tile, int g0, int n) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (wave + k * WAVES < n) load(tile, g0 + wave + k * WAVES, f[k]);
    };
    const int first = groups < chunk ? groups : chunk;
    int64_t tile = blockIdx.x;
    begin(tile, 0, first);
    bool have = false;  // all of x is in LDS
    for (; tile < tiles; tile += gridDim.x) {
#pragma unroll
        for (int i = 0; i < R * R / 64; ++i) acc[i] = 0.0f;
        for (int g0 = 0; g0 < groups; g0 += chunk) {
            const int n = groups - g0 < chunk ? groups - g0 : chunk;
            if (g0 > 0) begin(tile, g0, n);
            if (!have) {
                __syncthreads();  // the last chunk of x has been read
                quantize(g0, n);
                __syncthreads();
                have = chunk >= groups;
            }
            for (int lg = wave; lg < n; lg += kAhead * WAVES) {
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int g = lg + k * WAVES;
                    if (g < n) {
                        multiply(g, f[k]);
                        if (g + kAhead * WAVES < n) load(tile, g0 + g + kAhead * WAVES, f[k]);
                    }
                }
            }
        }
        if (tile + gridDim.x < tiles) begin(tile + gridDim.x, 0, first);  // on its way while the sums are added
        // The waves' sums, added in the order of the waves. A lane holds token `row` and R^2 / 64 rows of W.
        __syncthreads();  // the last tile's sums have been read
        if (row < M) {
#pragma unroll
            for (int q = 0; q < R * R / 256; ++q) {
                const int at = R == 32 ? 8 * q + 4 * part : 4 * part;
                *reinterpret_cast<float4*>(sums + (wave * M + row) * R + at) =
                    make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
            }
        }
        __syncthreads();
        for (int i = tid; i < M * R; i += 64 * WAVES) {
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v += sums[w * M * R + i];
            const int t = i / R;
            const int64_t n = tile * R + (i - t * R), at = t * j.ldc + n;
            if (n < j.N) {
                if constexpr (OUT == kOutF32) static_cast<float*>(j.y)[at] = v;
                else static_cast<uint16_t*>(j.y)[at] = __builtin_bit_cast(uint16_t, (__bf16)v);
            }
        }
    }
}

// Eight waves and two workgroups per CU where all of x fits half of a CU's LDS; sixteen waves and one where it fits the whole, or
// comes in chunks.
constexpr int kHalfLds = 80 * 1024, kWholeLds = 160 * 1024;
bool fits(const LinearJob& j, int R, int waves, int lds) {
    return (j.nkb + 3) / 4 * kGroupBytes * j.M + waves * j.M * R * 4 + 16 <= lds;
}

template <int OUT, int R, int WAVES>
hipError_t launch_linear_w(const LinearJob& j, int lds, hipStream_t s) {
    const int groups = (int)((j.nkb + 3) / 4), sums = WAVES * j.M * R * 4;
    int chunk = (lds - sums - 16) / (kGroupBytes * j.M);
    if (chunk > groups) chunk = groups;
    const int64_t tiles = (j.N + R - 1) / R, resident = WAVES == 8 ? 512 : 256;
    const int need = (chunk * kGroupBytes * j.M + 15) / 16 * 16 + sums;
    linear_mxfp4_kernel<OUT, R, WAVES><<<(unsigned)(tiles < resident ? tiles : resident), 64 * WAVES, need, s>>>(j, chunk);
    return hipGetLastError();
}

template <int OUT, int R>
hipError_t launch_linear_t(const LinearJob& j, hipStream_t s) {
    return fits(j, R, 8, kHalfLds) ? launch_linear_w<OUT, R, 8>(j, kHalfLds, s) : launch_linear_w<OUT, R, 16>(j, kWholeLds, s);
}

// R = 32 where W has tiles for every workgroup and x need not come in chunks for it (the smaller sums of R = 16 leave more room).
// Measured in a graph, us, 1 / 3 / 8 / 16 tokens: 2048 x 8192 5.5 / 6.0 / 7.5 / 9.8 (R = 16), 32768 x 4096 13.9 / 13.7 / 15.5 / 18.4
// (R = 32; W alone at 5.1 TB/s 14.0).
template <int OUT>
hipError_t launch_linear_r(const LinearJob& j, hipStream_t s) {
    return j.N >= 16384 && fits(j, 32, 16, kWholeLds) ? launch_linear_t<OUT, 32>(j, s) : launch_linear_t<OUT, 16>(j, s);
}

}  // namespace

hipError_t launch_linear_mxfp4(const LinearJob& j, hipStream_t s) {
    return j.out_dtype == kOutBF16 ? launch_linear_r<kOutBF16>(j, s) : launch_linear_r<kOutF32>(j, s);
}

}  // namespace ufp4
