// Microscaled 4-bit floating point (the OCP Microscaling format MXFP4): E2M1 levels with one E8M0 scale per 32 values along
// the reduction axis, the operands that gfx950's scaled matrix instruction takes as they are.
//
//   E = max(floor(log2 amax) - 2, -127), level = nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 to x 2^-E (ties to the even code, cut
//   at 6), or stochastically one of its two neighbours; a block that holds an infinity or a NaN gets the scale NaN.
//
// Layout (panels of 128 rows): block b of row 128 p + i has its 16 code bytes at p * code_panel_ld + b * 2048 + i * 16 -- what
// one lane of the 32 x 32 x 64 matrix instruction holds, so the GEMM's LDS reads are 16 bytes of consecutive rows -- and its
// scale at p * scale_panel_ld + (b / 4) * 512 + (b % 2) * 256 + i * 2 + (b / 2) % 2: the two scales that a lane needs over
// four blocks (128 of the reduction) lie together. Scale bytes of the blocks that fill up the last four are 0.
//
// HBM bound: 2 bytes read and 17/32 written per value. amax is a packed 16-bit integer maximum of the bf16 patterns (their
// order is that of the magnitudes) and the conversion one instruction per two values, so the plain form has little to compute (4
// vector instructions a value). Stochastic it has 27 (28 transposed) and is bound by their issue; Philox's draws are part of them, but
// the quantizer of the uniform grid, with the same draws and a rotation, has 24 (21): the rest goes into two ranges of every value
// (fp4_sr) and into codes merged one at a time. Rotated (fp64 sums, as the other quantizers) and stochastic it has 35 (36).
// Measured, 32768 x 16384 (1 GiB), us: rowwise 230 (5.9 TB/s), transposed 256 (5.3), both 306 (5.4), rowwise / transposed rotated
// 230-244 / 315, stochastic 350-380 / 404-411, both of these 453 / 526, back to bf16 243-251 (5.6).

#include "ufp4_internal.h"
#include "ufp4_device.h"
#include "ufp4_mxfp4.h"
#include "ufp4_rows.h"

#include <type_traits>

namespace ufp4 {

namespace {

// The E2M1 code of v (|v| < 8, cut at 6) between its neighbours by a 16-bit draw: the upper one of the signed pair
// g_a <= v < g_b iff u / 2^16 < (v - g_a) / (g_b - g_a). On integers, exact, and a level never moves.
// |v| >= 1: the levels are the fp32 numbers with one fraction bit, F the 22 bits below it. A positive v goes up iff U = 2^6 u <
// F, that is if F + (2^22 - 1 - U) carries; a negative one goes away from zero unless U < 2^22 - F, that is if F + U carries.
// |v| < 1: steps of 0.5; the upper level is ceil(2 v - u / 2^16) = -floor((u + floor(-2^17 v)) / 2^16).
__device__ __forceinline__ uint32_t fp4_sr(float v, uint32_t u16) {
    const uint32_t bits = __float_as_uint(v);
    const float a = __builtin_fminf(__builtin_fabsf(v), 6.0f);
    const uint32_t flip = (uint32_t)((int32_t)~bits >> 31) & 0x3FFFFFu;  // positive: 2^22 - 1 - U
    const uint32_t big = ((__float_as_uint(a) + ((u16 << 6) ^ flip)) >> 22) - 252u;
    int32_t f;
    asm("v_cvt_flr_i32_f32 %0, %1" : "=v"(f) : "v"(v * -131072.0f));
    const int32_t lower = ((int32_t)u16 + f) >> 16;  // minus the level's steps
    const uint32_t small = (uint32_t)(lower < 0 ? -lower : lower);
    return (a >= 1.0f ? big : small) | ((bits >> 28) & 8u);
}

// Sixteen values of a block (half of it) on their way to codes.
template <bool RHT>
struct Half {
    uint32_t w[8];  // bf16 pairs
    float y[RHT ? 16 : 1];

    // `unit` times the sums of the block-16 RHT, in fp64 as in the other quantizers, rounded once
    __device__ __forceinline__ void rotate(const QuantArgs& qa, double unit) {
        double d[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t p = w[j] ^ qa.sign_xor[j];
            d[2 * j] = (double)bf16_lo(p);
            d[2 * j + 1] = (double)bf16_hi(p);
        }
#pragma unroll
        for (int s = 1; s < 16; s <<= 1)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!(i & s)) {
                    const double a = d[i], b = d[i + s];
                    d[i] = a + b;
                    d[i + s] = a - b;
                }
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = (float)(d[i] * unit);
    }

    // exponent field of the largest magnitude
    __device__ __forceinline__ uint32_t exponent() const {
        uint32_t m = 0;
        if constexpr (RHT) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t b = __float_as_uint(y[i]) & 0x7FFFFFFFu;
                m = b > m ? b : m;
            }
            return m >> 23;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max_u16x2(m, w[j] & 0x7FFF7FFFu);
            const uint32_t lo = m & 0xFFFFu, hi = m >> 16;
            return (lo > hi ? lo : hi) >> 7;
        }
    }

    __device__ __forceinline__ bool finite_inputs() const {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max_u16x2(m, w[j] & 0x7FFF7FFFu);
        return (m & 0xFFFFu) < 0x7F80u && (m >> 16) < 0x7F80u;
    }

    // 16 codes at the scale 2^(e8 - 127), element 2j in the low nibble of byte j
    template <int ROUND>
    __device__ __forceinline__ uint2 encode(uint32_t e8, const QuantArgs& qa, uint32_t blk16, uint32_t row) const {
        uint32_t c[2] = {0, 0};
        if constexpr (ROUND == kRoundSR) {
            const Philox4 p0 = philox4x32_10(blk16, row, 0u, qa.stream, qa.key0, qa.key1);
            const Philox4 p1 = philox4x32_10(blk16, row, 1u, qa.stream, qa.key0, qa.key1);
            const uint32_t u[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
            const float mult = __uint_as_float((254u - e8) << 23);  // 2^-E: a normal number (e8 <= 252)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float v;
                if constexpr (RHT) v = y[i];
                else v = i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
                const uint32_t draw = i & 1 ? u[i >> 1] >> 16 : u[i >> 1] & 0xFFFFu;
                c[i >> 3] |= fp4_sr(__fmul_rn(v, mult), draw) << (4 * (i & 7));
            }
        } else {
            const float scale = __uint_as_float(e8 << 23);  // the instruction reads the exponent field only
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (RHT) {
                    c[h] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[h], y[8 * h], y[8 * h + 1], scale, 0);
                    c[h] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[h], y[8 * h + 2], y[8 * h + 3], scale, 1);
                    c[h] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[h], y[8 * h + 4], y[8 * h + 5], scale, 2);
                    c[h] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[h], y[8 * h + 6], y[8 * h + 7], scale, 3);
                } else {
                    c[h] = fp4_pair<0>(c[h], w[4 * h], scale);
                    c[h] = fp4_pair<1>(c[h], w[4 * h + 1], scale);
                    c[h] = fp4_pair<2>(c[h], w[4 * h + 2], scale);
                    c[h] = fp4_pair<3>(c[h], w[4 * h + 3], scale);
                }
            }
        }
        return make_uint2(c[0], c[1]);
    }
};

constexpr double kUnit = 0.25;            // 1/4 = 1/sqrt(16)
constexpr int kOverflowShift = 8;         // rotated values past FLT_MAX are taken 2^-8 as large
constexpr double kUnitSmall = 0x1p-10;

// One 32-block of two neighbouring columns, m[i] the pair of row i: codes and scale bytes of each.
template <int ROUND, bool RHT>
__device__ __forceinline__ void quantize_columns(const uint32_t (&m)[32], const QuantArgs& qa, int64_t b, int64_t col,
                                                 uint4 (&out)[2], uint32_t (&e8c)[2]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        Half<RHT> v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[h].w[j] = c == 0 ? __builtin_amdgcn_perm(m[16 * h + 2 * j + 1], m[16 * h + 2 * j], 0x05040100u)
                                   : __builtin_amdgcn_perm(m[16 * h + 2 * j + 1], m[16 * h + 2 * j], 0x07060302u);
        uint32_t ef[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (RHT) v[h].rotate(qa, kUnit);
            ef[h] = v[h].exponent();
        }
        uint32_t top = ef[0] > ef[1] ? ef[0] : ef[1];
        uint32_t e8 = scale_byte(top), at = e8;
        if constexpr (RHT) {
            if (__builtin_expect(top == 255u, 0)) {
                const bool fine = v[0].finite_inputs() && v[1].finite_inputs();
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v[h].rotate(qa, kUnitSmall);
                    ef[h] = v[h].exponent();
                }
                if (fine) {
                    at = scale_byte(ef[0] > ef[1] ? ef[0] : ef[1]);
                    e8 = at + kOverflowShift;
                }
            }
        }
        const uint2 lo = v[0].template encode<ROUND>(at, qa, (uint32_t)(2 * b), (uint32_t)(col + c));
        const uint2 hi = v[1].template encode<ROUND>(at, qa, (uint32_t)(2 * b + 1), (uint32_t)(col + c));
        out[c] = e8 == kNaNScale ? make_uint4(0, 0, 0, 0) : make_uint4(lo.x, lo.y, hi.x, hi.y);
        e8c[c] = e8;
    }
}

// The scale of a row's block whose two halves lie in neighbouring lanes: the byte stored, and in `at` the scale that the values in
// hand are taken at.
template <bool RHT>
__device__ __forceinline__ uint32_t pair_scale(Half<RHT>& v, const QuantArgs& qa, uint32_t& at) {
    if constexpr (RHT) v.rotate(qa, kUnit);
    uint32_t ef = v.exponent();
    uint32_t other = __shfl_xor(ef, 1, 64);
    ef = ef > other ? ef : other;
    uint32_t e8 = scale_byte(ef);
    at = e8;
    if constexpr (RHT) {
        if (__builtin_expect(ef == 255u, 0)) {  // a rotated value past FLT_MAX (or an input that is not finite)
            const int fine = v.finite_inputs() ? 1 : 0;
            v.rotate(qa, kUnitSmall);
            uint32_t e = v.exponent();
            other = __shfl_xor(e, 1, 64);
            e = e > other ? e : other;
            if (fine & __shfl_xor(fine, 1, 64)) {
                at = scale_byte(e);
                e8 = at + kOverflowShift;
            }
        }
    }
    return e8;
}

// ------------------------------------------------------------------------------------------------
// Rowwise: a workgroup takes 64 rows x 256 columns (8 blocks). A thread takes 16 values of a row, its neighbour the block's
// other half; loads are 512-byte runs, and codes and scales go through LDS, so that stores are runs of a block's rows (1 KiB
// of codes) instead of 8 bytes each.
// ------------------------------------------------------------------------------------------------
constexpr int kRowsTile = 64, kColsTile = 256;
constexpr int kCodeStride = kRowsTile * 16 + 64;  // a block's codes in LDS: 64 bytes apart in the banks

struct MicroOut {
    uint8_t* codes;
    int64_t code_pld;
    uint8_t* scales;
    int64_t scale_pld;
};

template <int ROUND, bool RHT, bool GROUPED>
__global__ __launch_bounds__(256) void micro_rows_kernel(const uint16_t* __restrict__ x, int64_t xrows, int64_t cols,
                                                         int64_t ld, int64_t col_tiles, const int64_t* offsets, int G,
                                                         QuantArgs qa, MicroOut o) {
    __shared__ __align__(16) uint8_t s_codes[8 * kCodeStride];
    __shared__ __align__(16) uint8_t s_scales[kRowsTile * 8];  // [group of 4][b % 2][row][2]
    const int tid = threadIdx.x;
    const int64_t rt = blockIdx.x / col_tiles, ct = blockIdx.x - rt * col_tiles;
    const int64_t row0 = rt * kRowsTile, c0 = ct * kColsTile;
    int64_t src = row0, left = xrows - row0;  // first row of x, rows that exist
    if constexpr (GROUPED) {
        if (!padded_position<128>(offsets, G, row0, src, left)) left = 0;
        if (src < 0 || src >= xrows) left = 0;
        if (left > xrows - src) left = xrows - src;
    }
    const int part = tid & 15, r0 = tid >> 4;  // 16 columns, row within 16
    const int64_t col = c0 + part * 16;
    Half<RHT> v[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int r = p * 16 + r0;
        uint4 a = make_uint4(0, 0, 0, 0), b = a;
        if (r < left && col < cols) {
            const uint4* const q = reinterpret_cast<const uint4*>(x + (src + r) * ld + col);
            a = q[0];
            b = q[1];
        }
        v[p].w[0] = a.x; v[p].w[1] = a.y; v[p].w[2] = a.z; v[p].w[3] = a.w;
        v[p].w[4] = b.x; v[p].w[5] = b.y; v[p].w[6] = b.z; v[p].w[7] = b.w;
    }
    const int blk = part >> 1, half = part & 1;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int r = p * 16 + r0;
        uint32_t at;
        const uint32_t e8 = pair_scale(v[p], qa, at);
        const int64_t grow = GROUPED ? src + r : row0 + r;  // the SR counters number x's rows
        uint2 c = v[p].template encode<ROUND>(at, qa, (uint32_t)(col >> 4), (uint32_t)grow);
        if (e8 == kNaNScale || r >= left) c = make_uint2(0, 0);  // padding: some signs rotate its zeros to -0
        *reinterpret_cast<uint2*>(s_codes + blk * kCodeStride + r * 16 + half * 8) = c;
        if (half == 0) s_scales[(blk >> 2) * 256 + (blk & 1) * 128 + r * 2 + ((blk >> 1) & 1)] = (uint8_t)e8;
    }
    __syncthreads();
    const int64_t nkb = cols / 32, b0 = c0 / 32;
    const int64_t panel = row0 / 128;
    const int half_panel = (int)(row0 / 64) & 1;
    uint8_t* const codes = o.codes + panel * o.code_pld + half_panel * 1024;
    uint8_t* const scales = o.scales + panel * o.scale_pld + half_panel * 128;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int u = k * 256 + tid, b = u >> 6, r = u & 63;
        if (b0 + b < nkb)
            *reinterpret_cast<uint4*>(codes + (b0 + b) * 2048 + r * 16) =
                *reinterpret_cast<const uint4*>(s_codes + b * kCodeStride + r * 16);
    }
    if (tid < 32) {
        const int g = tid >> 4, h = (tid >> 3) & 1, k = tid & 7;
        if (b0 + g * 4 < nkb)
            *reinterpret_cast<uint4*>(scales + (b0 / 4 + g) * 512 + h * 256 + k * 16) =
                *reinterpret_cast<const uint4*>(s_scales + g * 256 + h * 128 + k * 16);
    }
}

// ------------------------------------------------------------------------------------------------
// Transposed, and both operands from one read (DO_R): a workgroup takes 128 x 128 of x, which is four blocks of one panel of
// either output (8 KiB of codes and 512 bytes of scales each, both contiguous). x comes in 256-byte runs of rows, 16 values a
// thread, and goes to LDS (and, DO_R, through the rowwise quantization); then each wave takes one block of 32 rows of the LDS
// tile, two columns a lane. (Without LDS, a wave loading two columns a lane from memory: 1 GiB 276 us instead of 257.)
// ------------------------------------------------------------------------------------------------
constexpr int kTileStride = 2048 + 32;  // a block's row codes in LDS: 32 bytes apart in the banks

// Eight columns of a row of which `left` exist.
__device__ __forceinline__ uint4 load_columns(const uint16_t* p, int64_t left) {
    if (left >= 8) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < left) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int ROUND, bool RHT_R, bool RHT_C, bool DO_R, bool GROUPED>
__global__ __launch_bounds__(256) void micro_tile_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t cols, int64_t ld,
                                                         int64_t nkb_c, int64_t col_tiles, const int64_t* offsets, int G,
                                                         QuantArgs qr, QuantArgs qc, MicroOut o_r, MicroOut o_c) {
    __shared__ __align__(16) uint16_t s_x[128 * 128];
    __shared__ __align__(16) uint8_t s_codes[DO_R ? 4 * kTileStride : 16];
    __shared__ __align__(16) uint8_t s_scales[2][512];  // of Q_r, of Q_c
    __shared__ int64_t s_place[4][2];                   // grouped: each block's first row of x, rows that exist
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t pr = blockIdx.x / col_tiles, pc = blockIdx.x - pr * col_tiles;
    if constexpr (GROUPED) {
        int64_t src = 0, left = 0;
        const int64_t b = pr * 4 + wave;
        if (b >= nkb_c || !padded_position<32>(offsets, G, b * 32, src, left)) left = 0;
        if (src < 0 || src >= rows) left = 0;
        if (lane == 0) {
            s_place[wave][0] = src;
            s_place[wave][1] = left < rows - src ? left : rows - src;
        }
        __syncthreads();
    }
    const int part = tid & 7, r0 = tid >> 3;  // 16 columns, row within 32
    const int64_t col = pc * 128 + part * 16;
    const bool whole = (pc + 1) * 128 <= cols;  // no thread tests its columns
    Half<RHT_R> v[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int64_t src = GROUPED ? s_place[p][0] : pr * 128 + p * 32, left = GROUPED ? s_place[p][1] : rows - src;
        uint4 a = make_uint4(0, 0, 0, 0), b = a;
        const uint16_t* const q = x + (src + r0) * ld + col;
        if (whole) {
            if (r0 < left) {
                a = reinterpret_cast<const uint4*>(q)[0];
                b = reinterpret_cast<const uint4*>(q)[1];
            }
        } else if (r0 < left && col < cols) {
            a = load_columns(q, cols - col);
            if (col + 8 < cols) b = load_columns(q + 8, cols - col - 8);
        }
        v[p].w[0] = a.x; v[p].w[1] = a.y; v[p].w[2] = a.z; v[p].w[3] = a.w;
        v[p].w[4] = b.x; v[p].w[5] = b.y; v[p].w[6] = b.z; v[p].w[7] = b.w;
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint4* const d = reinterpret_cast<uint4*>(s_x + (p * 32 + r0) * 128 + part * 16);
        d[0] = make_uint4(v[p].w[0], v[p].w[1], v[p].w[2], v[p].w[3]);
        d[1] = make_uint4(v[p].w[4], v[p].w[5], v[p].w[6], v[p].w[7]);
    }
    if constexpr (DO_R) {
        const int blk = part >> 1, half = part & 1;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int r = p * 32 + r0;
            uint32_t at;
            const uint32_t e8 = pair_scale(v[p], qr, at);
            uint2 c = v[p].template encode<ROUND>(at, qr, (uint32_t)(col >> 4), (uint32_t)(pr * 128 + r));
            if (e8 == kNaNScale || pr * 128 + r >= rows) c = make_uint2(0, 0);
            *reinterpret_cast<uint2*>(s_codes + blk * kTileStride + r * 16 + half * 8) = c;
            if (half == 0) s_scales[0][(blk & 1) * 256 + r * 2 + (blk >> 1)] = (uint8_t)e8;
        }
    }
    __syncthreads();
    if constexpr (DO_R) {
        uint8_t* const cr = o_r.codes + pr * o_r.code_pld + pc * 8192;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int u = k * 256 + tid, b = u >> 7, r = u & 127;
            if (pc * 4 + b < cols / 32)
                *reinterpret_cast<uint4*>(cr + b * 2048 + r * 16) =
                    *reinterpret_cast<const uint4*>(s_codes + b * kTileStride + r * 16);
        }
    }
    uint32_t m[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) m[i] = *reinterpret_cast<const uint32_t*>(s_x + (wave * 32 + i) * 128 + lane * 2);
    const int64_t bc = pr * 4 + wave;
    uint4 out[2];
    uint32_t e8c[2];
    quantize_columns<ROUND, RHT_C>(m, qc, bc, pc * 128 + 2 * lane, out, e8c);
    if constexpr (RHT_C) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
            if (pc * 128 + 2 * lane + c >= cols) out[c] = make_uint4(0, 0, 0, 0);
    }
    if (bc < nkb_c) {
        uint4* const d = reinterpret_cast<uint4*>(o_c.codes + pc * o_c.code_pld + bc * 2048 + lane * 32);
        d[0] = out[0];
        d[1] = out[1];
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) s_scales[1][(wave & 1) * 256 + (2 * lane + c) * 2 + (wave >> 1)] = (uint8_t)e8c[c];
    __syncthreads();
    if (DO_R && tid < 32)
        *reinterpret_cast<uint4*>(o_r.scales + pr * o_r.scale_pld + pc * 512 + tid * 16) =
            *reinterpret_cast<const uint4*>(s_scales[0] + tid * 16);
    else if (tid >= 32 && tid < 64)
        *reinterpret_cast<uint4*>(o_c.scales + pc * o_c.scale_pld + pr * 512 + (tid - 32) * 16) =
            *reinterpret_cast<const uint4*>(s_scales[1] + (tid - 32) * 16);
}

// ------------------------------------------------------------------------------------------------
// Codes and scales to bf16 (exact: a level has two significant bits; 6 * 2^127 is infinity): a lane takes 8 values, 32 lanes a
// run of 512 bytes of a row. Outputs of kStreamBytes and more are stored nontemporally (us, so / plainly: 1 GiB 243 / 258, 512 MiB
// 99 / 131, 369 MB 67 / 92, 134 MB 26 / 26).
// ------------------------------------------------------------------------------------------------
template <bool STREAM>
__global__ __launch_bounds__(256) void micro_decode_kernel(MicroOut q, int64_t rows, int64_t red, int64_t col_tiles,
                                                           uint16_t* __restrict__ out, int64_t ldo) {
    const int64_t rt = blockIdx.x / col_tiles, ct = blockIdx.x - rt * col_tiles;
    const int part = threadIdx.x & 31;
    const int64_t col = ct * kColsTile + part * 8, b = col / 32;
    if (col >= red) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t row = rt * 32 + k * 8 + (threadIdx.x >> 5);
        if (row >= rows) return;
        const int64_t p = row / 128;
        const int i = (int)(row & 127);
        const uint32_t c = *reinterpret_cast<const uint32_t*>(q.codes + p * q.code_pld + b * 2048 + i * 16 + (part & 3) * 4);
        const uint32_t e8 = q.scales[p * q.scale_pld + (b / 4) * 512 + (b & 1) * 256 + i * 2 + ((b >> 1) & 1)];
        const float scale = __uint_as_float(e8 << 23);
        u32x4_any r;
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
        Piece<uint16_t>::store<STREAM>(out + row * ldo + col, 8, r);
    }
}

template <int ROUND, bool RHT, bool GROUPED>
hipError_t launch_micro_t(const MxQuantJob& j, hipStream_t s) {
    const MicroOut o{static_cast<uint8_t*>(j.codes), j.code_pld, static_cast<uint8_t*>(j.scales), j.scale_pld};
    const uint16_t* const x = static_cast<const uint16_t*>(j.x);
    const int64_t tiles = micro_quant_tiles(j.transpose, j.qrows, j.red);
    if (tiles == 0) return hipSuccess;
    if (j.transpose) {
        micro_tile_kernel<ROUND, false, RHT, false, GROUPED><<<(unsigned)tiles, 256, 0, s>>>(
            x, j.xrows, j.qrows, j.ld, j.red / 32, padded_rows(j.qrows) / 128, j.group_off, j.num_groups, j.qa, j.qa, o, o);
    } else {
        micro_rows_kernel<ROUND, RHT, GROUPED><<<(unsigned)tiles, 256, 0, s>>>(x, j.xrows, j.red, j.ld,
                                                                              (j.red + kColsTile - 1) / kColsTile, j.group_off,
                                                                              j.num_groups, j.qa, o);
    }
    return hipGetLastError();
}

template <int ROUND, bool RHT>
hipError_t launch_micro_g(const MxQuantJob& j, hipStream_t s) {
    return j.group_off ? launch_micro_t<ROUND, RHT, true>(j, s) : launch_micro_t<ROUND, RHT, false>(j, s);
}

template <int ROUND>
hipError_t launch_micro_r(const MxQuantJob& j, hipStream_t s) {
    return j.rht ? launch_micro_g<ROUND, true>(j, s) : launch_micro_g<ROUND, false>(j, s);
}

template <int ROUND>
hipError_t launch_micro_dual_r(const MxDualJob& j, hipStream_t s) {
    const int64_t row_tiles = padded_rows(j.rows) / 128, col_tiles = padded_rows(j.cols) / 128;
    const unsigned g = (unsigned)(row_tiles * col_tiles);
    const uint16_t* const x = static_cast<const uint16_t*>(j.x);
    const MicroOut r{static_cast<uint8_t*>(j.codes_r), j.code_pld_r, static_cast<uint8_t*>(j.scales_r), j.scale_pld_r};
    const MicroOut c{static_cast<uint8_t*>(j.codes_c), j.code_pld_c, static_cast<uint8_t*>(j.scales_c), j.scale_pld_c};
    auto go = [&](auto rht_r, auto rht_c) {
        micro_tile_kernel<ROUND, decltype(rht_r)::value, decltype(rht_c)::value, true, false>
            <<<g, 256, 0, s>>>(x, j.rows, j.cols, j.ld, j.rows / 32, col_tiles, nullptr, 0, j.qr, j.qc, r, c);
    };
    if (j.rht_r) j.rht_c ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
    else j.rht_c ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_mxfp4_dual(const MxDualJob& j, hipStream_t s) {
    return j.rounding == kRoundSR ? launch_micro_dual_r<kRoundSR>(j, s) : launch_micro_dual_r<kRoundRTNE>(j, s);
}

int64_t micro_quant_tiles(int transpose, int64_t qrows, int64_t red) {
    if (transpose) return padded_rows(qrows) / 128 * ((red / 32 + 3) / 4);
    return padded_rows(qrows) / kRowsTile * ((red + kColsTile - 1) / kColsTile);
}

int64_t micro_decode_tiles(int64_t rows, int64_t red) { return (rows + 31) / 32 * ((red + kColsTile - 1) / kColsTile); }

hipError_t launch_quantize_mxfp4(const MxQuantJob& j, hipStream_t s) {
    return j.rounding == kRoundSR ? launch_micro_r<kRoundSR>(j, s) : launch_micro_r<kRoundRTNE>(j, s);
}

hipError_t launch_dequantize_mxfp4(const void* codes, int64_t code_pld, const void* scales, int64_t scale_pld, int64_t rows,
                                   int64_t red, void* out, int64_t ldo, hipStream_t s) {
    const MicroOut q{static_cast<uint8_t*>(const_cast<void*>(codes)), code_pld,
                     static_cast<uint8_t*>(const_cast<void*>(scales)), scale_pld};
    const int64_t tiles = micro_decode_tiles(rows, red);
    if (tiles == 0) return hipSuccess;
    const auto kernel = rows * red * 2 >= kStreamBytes ? micro_decode_kernel<true> : micro_decode_kernel<false>;
    kernel<<<(unsigned)tiles, 256, 0, s>>>(q, rows, red, (red + kColsTile - 1) / kColsTile, static_cast<uint16_t*>(out), ldo);
    return hipGetLastError();
}

}  // namespace ufp4
