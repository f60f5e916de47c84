// Activation checkpoints in 8 bits (format in ufp4_ckpt8.h) and the experts' activation around them:
//   save: x -> codes, scales; load: back to bf16 or fp32, exact
//   activation: a = f(u), and u's checkpoint from the same read; f(u) = max(u, 0)^2, or g / (1 + e^-g) v of the halves g, v of u
//   its gradient from the checkpoint (or from u): du = f'(u) da, and a once more, which the next product's weights need
// Bound by memory: every tensor is read or written once, all arithmetic is on registers.
//
// A thread takes 16 values at a time (half a block: its codes are one 16-byte store), the other half's maximum comes from the
// neighbouring lane.

#include "ufp4_ckpt8.h"
#include "ufp4_internal.h"
#include "ufp4_rows.h"
#include "ufp4_tiles.h"

namespace ufp4 {

namespace {

constexpr int kThreads = 256;
constexpr int kHalf = kCkpt8Block / 2;  // values of a thread's unit

// 16 values of a row, in pieces of 16 bytes.
template <typename T>
struct Unit {
    using P = Piece<T>;
    static constexpr int kPieces = kHalf / P::V;
    u32x4_any raw[kPieces];

    __device__ __forceinline__ void load(const T* p, int64_t left) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) raw[i] = P::load(p + i * P::V, left - i * P::V);
    }
    __device__ __forceinline__ void values(float (&f)[kHalf]) const {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            float v[P::V];
            P::unpack(raw[i], v);
#pragma unroll
            for (int e = 0; e < P::V; ++e) f[i * P::V + e] = v[e];
        }
    }
    template <bool STREAM>
    static __device__ __forceinline__ void store(T* p, int64_t left, const float (&f)[kHalf]) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            float v[P::V];
#pragma unroll
            for (int e = 0; e < P::V; ++e) v[e] = f[i * P::V + e];
            P::template store<STREAM>(p + i * P::V, left - i * P::V, P::pack(v));
        }
    }
};

// Units [64 N w, 64 N (w + 1)) of wave w, N a lane: unit i of row i / per, values 16 (i % per) .. of it; `per` is even, so that a
// block's halves are in neighbouring lanes.
template <int N>
struct Where {
    int64_t row[N];
    int col[N];
    bool some[N];

    __device__ __forceinline__ Where(int64_t rows, uint32_t per) {
        const int64_t total = rows * per, base = ((int64_t)blockIdx.x * (kThreads / 64) + uniform(threadIdx.x >> 6)) * (64 * N);
        const int64_t row0 = total <= UINT32_MAX ? (int64_t)((uint32_t)base / per) : base / per;
        const uint32_t unit0 = (uint32_t)(base - row0 * per), lane = threadIdx.x & 63;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const uint32_t u = unit0 + t * 64 + lane, q = u / per;
            row[t] = row0 + q;
            col[t] = (int)(u - q * per) * kHalf;
            some[t] = base + t * 64 + lane < total;
        }
    }
};

// The scale byte of the block whose halves this lane and its neighbour hold.
__device__ __forceinline__ uint32_t block_scale(const float (&f)[kHalf]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kHalf; ++i) {
        const uint32_t b = __float_as_uint(f[i]) & 0x7FFFFFFFu;
        top = b < 0x7F800000u && b > top ? b : top;  // infinities and NaN do not set a scale
    }
    const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false);  // lanes 1, 0, 3, 2
    return ckpt8_scale(top > other ? top : other);
}

// A half block to its codes, and its scale from the block's first lane. Columns past the row are zeros, which the codes hold, too.
template <bool STREAM>
__device__ __forceinline__ void keep(float (&f)[kHalf], uint8_t* codes, uint8_t* scale, int col) {
    const uint32_t s = block_scale(f);
    if (s == kCkpt8MaxScale) {  // 1.9375 2^127 and more would become 2^128, which no load could give back: 1.875 2^127, the level below
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            const uint32_t b = __float_as_uint(f[i]), m = b & 0x7FFFFFFFu;
            if (m >= 0x7F780000u && m < 0x7F800000u) f[i] = __uint_as_float((b & 0x80000000u) | 0x7F700000u);
        }
    }
    const float inverse = ckpt8_inverse(s);
    u32x4_any c;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = ckpt8_encode(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3], inverse);
    u32x4_any* const to = reinterpret_cast<u32x4_any*>(codes + col);
    if constexpr (STREAM) __builtin_nontemporal_store(c, to);
    else *to = c;
    if (!(col & kHalf)) scale[col / kCkpt8Block] = (uint8_t)s;
}

struct Codes {
    u32x4_any raw;
    uint32_t scale;
    __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int col) {
        raw = *reinterpret_cast<const u32x4_any*>(codes + col);
        scale = scales[col / kCkpt8Block];
    }
    __device__ __forceinline__ void values(float (&f)[kHalf]) const {
        const float factor = ckpt8_factor(scale);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v[4];
            ckpt8_decode(raw[i], factor, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[4 * i + e] = v[e];
        }
    }
};

template <typename T, int N, bool STREAM>
__global__ __launch_bounds__(kThreads) void save_kernel(Ckpt8Job j) {
    const Where<N> w(j.rows, (uint32_t)((j.cols + kCkpt8Block - 1) / kCkpt8Block * 2));
    Unit<T> u[N];
#pragma unroll
    for (int t = 0; t < N; ++t)
        if (w.some[t]) u[t].load(static_cast<const T*>(j.x) + w.row[t] * j.ldx + w.col[t], j.cols - w.col[t]);
#pragma unroll
    for (int t = 0; t < N; ++t) {
        if (!w.some[t]) continue;
        float f[kHalf];
        u[t].values(f);
        keep<STREAM>(f, j.codes + w.row[t] * j.ldc, j.scales + w.row[t] * j.lds, w.col[t]);
    }
}

template <typename T, int N, bool STREAM>
__global__ __launch_bounds__(kThreads) void load_kernel(Ckpt8Job j) {
    const Where<N> w(j.rows, (uint32_t)((j.cols + kCkpt8Block - 1) / kCkpt8Block * 2));
    Codes c[N];
#pragma unroll
    for (int t = 0; t < N; ++t)
        if (w.some[t]) c[t].load(j.codes + w.row[t] * j.ldc, j.scales + w.row[t] * j.lds, w.col[t]);
#pragma unroll
    for (int t = 0; t < N; ++t) {
        if (!w.some[t]) continue;
        float f[kHalf];
        c[t].values(f);
        Unit<T>::template store<STREAM>(static_cast<T*>(j.out) + w.row[t] * j.ldx + w.col[t], j.cols - w.col[t], f);
    }
}

// ------------------------------------------------------------------------------------------------
// activation
// ------------------------------------------------------------------------------------------------

// s = 1 / (1 + e^-g) and 1 - s, both without cancellation or overflow: from e^-|g| in (0, 1].
__device__ __forceinline__ void logistic(float g, float& s, float& rest) {
    const float e = expf(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.0f + e);  // within one unit of the last place
    s = g >= 0.0f ? r : e * r;
    rest = g >= 0.0f ? e * r : r;
    if (g != g) s = rest = g;
}

// NaN stays NaN
__device__ __forceinline__ float positive(float u) { return u < 0.0f ? 0.0f : u; }

// u: gate, then value of a gated activation.
template <int KIND>
__device__ __forceinline__ float act(const float (&u)[2]) {
    if constexpr (KIND == kActRelu2) {
        const float r = positive(u[0]);
        return r * r;
    } else {
        float s, rest;
        logistic(u[0], s, rest);
        return u[0] * s * u[1];
    }
}

template <int KIND>
__device__ __forceinline__ float act_grad(const float (&u)[2], float da, float (&du)[2]) {
    if constexpr (KIND == kActRelu2) {
        const float r = positive(u[0]);
        du[0] = 2.0f * r * da;
        return r * r;
    } else {
        float s, rest;
        logistic(u[0], s, rest);
        const float f = u[0] * s;
        du[0] = da * u[1] * (s * (1.0f + u[0] * rest));
        du[1] = da * f;
        return f * u[1];
    }
}

template <typename T, int KIND, bool SAVE, int N, bool STREAM>
__global__ __launch_bounds__(kThreads) void act_kernel(ActJob j) {
    constexpr int kParts = KIND == kActSwiglu ? 2 : 1;
    const int64_t blocks = (j.cols + kCkpt8Block - 1) / kCkpt8Block;
    const Where<N> w(j.rows, (uint32_t)(blocks * 2));
    Unit<T> u[N][kParts];
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int p = 0; p < kParts; ++p)
            if (w.some[t]) u[t][p].load(static_cast<const T*>(j.u) + w.row[t] * j.ldu + p * j.cols + w.col[t], j.cols - w.col[t]);
#pragma unroll
    for (int t = 0; t < N; ++t) {
        if (!w.some[t]) continue;
        float f[kParts][kHalf], a[kHalf];
#pragma unroll
        for (int p = 0; p < kParts; ++p) u[t][p].values(f[p]);
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            const float v[2] = {f[0][i], f[kParts - 1][i]};
            a[i] = act<KIND>(v);
        }
        Unit<T>::template store<STREAM>(static_cast<T*>(j.a) + w.row[t] * j.lda + w.col[t], j.cols - w.col[t], a);
        if constexpr (SAVE)
#pragma unroll
            for (int p = 0; p < kParts; ++p)
                keep<STREAM>(f[p], j.codes + w.row[t] * j.ldc + p * blocks * kCkpt8Block, j.scales + w.row[t] * j.lds + p * blocks, w.col[t]);
    }
}

template <typename T, int KIND, bool SAVED, int N, bool STREAM>
__global__ __launch_bounds__(kThreads) void act_bwd_kernel(ActJob j) {
    constexpr int kParts = KIND == kActSwiglu ? 2 : 1;
    const int64_t blocks = (j.cols + kCkpt8Block - 1) / kCkpt8Block;
    const Where<N> w(j.rows, (uint32_t)(blocks * 2));
    Unit<T> d[N], u[N][kParts];
    Codes c[N][kParts];
#pragma unroll
    for (int t = 0; t < N; ++t) {
        if (!w.some[t]) continue;
        d[t].load(static_cast<const T*>(j.da) + w.row[t] * j.ldda + w.col[t], j.cols - w.col[t]);
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            if constexpr (SAVED)
                c[t][p].load(j.codes + w.row[t] * j.ldc + p * blocks * kCkpt8Block, j.scales + w.row[t] * j.lds + p * blocks, w.col[t]);
            else
                u[t][p].load(static_cast<const T*>(j.u) + w.row[t] * j.ldu + p * j.cols + w.col[t], j.cols - w.col[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < N; ++t) {
        if (!w.some[t]) continue;
        float f[kParts][kHalf], da[kHalf], du[kParts][kHalf], a[kHalf];
        d[t].values(da);
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            if constexpr (SAVED) c[t][p].values(f[p]);
            else u[t][p].values(f[p]);
        }
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            const float v[2] = {f[0][i], f[kParts - 1][i]};
            float g[2];
            a[i] = act_grad<KIND>(v, da[i], g);
#pragma unroll
            for (int p = 0; p < kParts; ++p) du[p][i] = g[p];
        }
#pragma unroll
        for (int p = 0; p < kParts; ++p)
            Unit<T>::template store<STREAM>(static_cast<T*>(j.du) + w.row[t] * j.lddu + p * j.cols + w.col[t], j.cols - w.col[t], du[p]);
        if (j.a) Unit<T>::template store<STREAM>(static_cast<T*>(j.a) + w.row[t] * j.lda + w.col[t], j.cols - w.col[t], a);
    }
}

int64_t units(int64_t rows, int64_t cols) { return rows * ((cols + kCkpt8Block - 1) / kCkpt8Block * 2); }

unsigned grid(int64_t n, int each) { return (unsigned)((n + kThreads * each - 1) / (kThreads * each)); }

// Units a thread: several where the chip is full all the same.
constexpr int64_t kManyUnits = int64_t(256) * 2048 * 4;

template <typename T, int N>
void save_stream(const Ckpt8Job& j, bool stream, hipStream_t s) {
    const unsigned n = grid(units(j.rows, j.cols), N);
    if (stream) save_kernel<T, N, true><<<n, kThreads, 0, s>>>(j);
    else save_kernel<T, N, false><<<n, kThreads, 0, s>>>(j);
}
template <typename T, int N>
void load_stream(const Ckpt8Job& j, bool stream, hipStream_t s) {
    const unsigned n = grid(units(j.rows, j.cols), N);
    if (stream) load_kernel<T, N, true><<<n, kThreads, 0, s>>>(j);
    else load_kernel<T, N, false><<<n, kThreads, 0, s>>>(j);
}

template <typename T, int KIND, bool SAVED, int N>
void act_stream(const ActJob& j, bool bwd, bool stream, hipStream_t s) {
    const unsigned n = grid(units(j.rows, j.cols), N);
    if (bwd) {
        if (stream) act_bwd_kernel<T, KIND, SAVED, N, true><<<n, kThreads, 0, s>>>(j);
        else act_bwd_kernel<T, KIND, SAVED, N, false><<<n, kThreads, 0, s>>>(j);
    } else {
        if (stream) act_kernel<T, KIND, SAVED, N, true><<<n, kThreads, 0, s>>>(j);
        else act_kernel<T, KIND, SAVED, N, false><<<n, kThreads, 0, s>>>(j);
    }
}

template <typename T, int KIND>
void act_saved(const ActJob& j, bool bwd, bool stream, hipStream_t s) {
    const bool many = units(j.rows, j.cols) >= kManyUnits;
    if (j.codes) many ? act_stream<T, KIND, true, 2>(j, bwd, stream, s) : act_stream<T, KIND, true, 1>(j, bwd, stream, s);
    else many ? act_stream<T, KIND, false, 2>(j, bwd, stream, s) : act_stream<T, KIND, false, 1>(j, bwd, stream, s);
}

hipError_t launch_any(const ActJob& j, bool bwd, hipStream_t s) {
    const bool stream = j.rows * j.cols * (j.bf16 ? 2 : 4) >= kStreamBytes;
    if (j.kind == kActSwiglu) j.bf16 ? act_saved<uint16_t, kActSwiglu>(j, bwd, stream, s) : act_saved<float, kActSwiglu>(j, bwd, stream, s);
    else j.bf16 ? act_saved<uint16_t, kActRelu2>(j, bwd, stream, s) : act_saved<float, kActRelu2>(j, bwd, stream, s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ckpt8_save(const Ckpt8Job& j, hipStream_t s) {
    const int64_t n = units(j.rows, j.cols);
    const bool many = n >= kManyUnits, stream = n * kHalf >= kStreamBytes;
    if (j.bf16) many ? save_stream<uint16_t, 4>(j, stream, s) : save_stream<uint16_t, 1>(j, stream, s);
    else many ? save_stream<float, 2>(j, stream, s) : save_stream<float, 1>(j, stream, s);
    return hipGetLastError();
}

hipError_t launch_ckpt8_load(const Ckpt8Job& j, hipStream_t s) {
    const int64_t n = units(j.rows, j.cols);
    const bool many = n >= kManyUnits, stream = n * kHalf * (j.bf16 ? 2 : 4) >= kStreamBytes;
    if (j.bf16) many ? load_stream<uint16_t, 4>(j, stream, s) : load_stream<uint16_t, 1>(j, stream, s);
    else many ? load_stream<float, 2>(j, stream, s) : load_stream<float, 1>(j, stream, s);
    return hipGetLastError();
}

hipError_t launch_act(const ActJob& j, hipStream_t s) { return launch_any(j, false, s); }
hipError_t launch_act_bwd(const ActJob& j, hipStream_t s) { return launch_any(j, true, s); }

int64_t ckpt8_units(int64_t rows, int64_t cols) { return units(rows, cols); }

}  // namespace ufp4
