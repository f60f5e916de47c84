// Activation checkpoints in 8 bits (format in ufp4_ckpt8.h) and the experts' activation around them:
//   save: x -> codes, scales; load: back to bf16 or fp32, exact
//   activation: a = f(u), and u's checkpoint from the same read; f(u) = max(u, 0)^2, or g / (1 + e^-g) v of the halves g, v of u
//   its gradient from the checkpoint (or from u): du = f'(u) da, and a once more, which the next product's weights need
// Bound by memory: every tensor is read or written once, all arithmetic is on registers. 1 GiB of bf16 to 8 bits 265 us and back 270 us
// (6.0-6.1 TB/s; a copy runs at 5.1); squared ReLU of 98304 x 1408 bf16 with checkpoint 113 us, its gradient 153 us (6.2 TB/s); gated SiLU of
// 4099 x 1411 fp32 15 and 17 us.
//
// A lane takes a 16-byte piece of a row at a time (8 bf16 or 4 fp32 values), so that every access of a wave is one run of memory; a block's
// maximum comes from the 4 or 8 lanes that hold it.

#include "ufp4_ckpt8.h"
#include "ufp4_internal.h"
#include "ufp4_rows.h"
#include "ufp4_tiles.h"

#include <type_traits>

namespace ufp4 {

namespace {

constexpr int kThreads = 256;

// Pieces [64 N w, 64 N (w + 1)) of wave w, N a lane: piece i of row i / per, values V (i % per) .. of it. `per` is whole blocks, whose
// lanes lie side by side.
template <int N, int V>
struct Where {
    int64_t row[N];
    int col[N];
    bool some[N];

    __device__ __forceinline__ Where(int64_t rows, int64_t blocks) {
        const uint32_t per = (uint32_t)blocks * (kCkpt8Block / V);
        const int64_t total = rows * per, base = ((int64_t)blockIdx.x * (kThreads / 64) + uniform(threadIdx.x >> 6)) * (64 * N);
        const int64_t row0 = total <= UINT32_MAX ? (int64_t)((uint32_t)base / per) : base / per;
        const uint32_t unit0 = (uint32_t)(base - row0 * per), lane = threadIdx.x & 63;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const uint32_t u = unit0 + t * 64 + lane, q = u / per;
            row[t] = row0 + q;
            col[t] = (int)(u - q * per) * V;
            some[t] = base + t * 64 + lane < total;
        }
    }
};

__host__ __device__ inline int64_t blocks_of(int64_t cols) { return (cols + kCkpt8Block - 1) / kCkpt8Block; }

// The scale byte of the block that this lane and its neighbours hold.
template <int V>
__device__ __forceinline__ uint32_t block_scale(const float (&f)[V]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t b = __float_as_uint(f[i]) & 0x7FFFFFFFu;
        top = b < 0x7F800000u && b > top ? b : top;  // infinities and NaN do not set a scale
    }
    auto across = [&](auto control) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, decltype(control)::value, 0xF, 0xF, false);
        top = o > top ? o : top;
    };
    across(std::integral_constant<int, 0xB1>{});                          // lanes 1, 0, 3, 2
    across(std::integral_constant<int, 0x4E>{});                          // lanes 2, 3, 0, 1
    if constexpr (V == 4) across(std::integral_constant<int, 0x141>{});  // lanes 7 .. 0
    return ckpt8_scale(top);
}

template <int V>
struct CodeWord;
template <>
struct CodeWord<8> {
    typedef uint32_t Type __attribute__((ext_vector_type(2)));
};
template <>
struct CodeWord<4> {
    typedef uint32_t Type __attribute__((ext_vector_type(1)));
};

// A piece of a block to its codes, and its scale from the block's first lane. Columns past the row are zeros, which the codes hold, too.
template <bool STREAM, int V>
__device__ __forceinline__ void keep(float (&f)[V], uint8_t* codes, uint8_t* scale, int col) {
    const uint32_t s = block_scale(f);
    if (s == kCkpt8MaxScale) {  // 1.9375 2^127 and more would become 2^128, which no load could give back: 1.875 2^127, the level below
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t b = __float_as_uint(f[i]), m = b & 0x7FFFFFFFu;
            if (m >= 0x7F780000u && m < 0x7F800000u) f[i] = __uint_as_float((b & 0x80000000u) | 0x7F700000u);
        }
    }
    const float inverse = ckpt8_inverse(s);
    typename CodeWord<V>::Type c;
#pragma unroll
    for (int i = 0; i < V / 4; ++i) c[i] = ckpt8_encode(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3], inverse);
    auto* const to = reinterpret_cast<typename CodeWord<V>::Type*>(codes + col);
    if constexpr (STREAM) __builtin_nontemporal_store(c, to);
    else *to = c;
    if (!(col & (kCkpt8Block - 1))) scale[col / kCkpt8Block] = (uint8_t)s;
}

template <int V>
struct Codes {
    typename CodeWord<V>::Type raw;
    uint32_t scale;
    __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int col) {
        raw = *reinterpret_cast<const typename CodeWord<V>::Type*>(codes + col);
        scale = scales[col / kCkpt8Block];
    }
    __device__ __forceinline__ void values(float (&f)[V]) const {
        const float factor = ckpt8_factor(scale);
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            float v[4];
            ckpt8_decode(raw[i], factor, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[4 * i + e] = v[e];
        }
    }
};

template <typename T, int N, bool STREAM>
__global__ __launch_bounds__(kThreads) void save_kernel(Ckpt8Job j) {
    using P = Piece<T>;
    const Where<N, P::V> w(j.rows, blocks_of(j.cols));
    u32x4_any u[N];
#pragma unroll
    for (int t = 0; t < N; ++t)
        if (w.some[t]) u[t] = P::load(static_cast<const T*>(j.x) + w.row[t] * j.ldx + w.col[t], j.cols - w.col[t]);
#pragma unroll
    for (int t = 0; t < N; ++t) {
        if (!w.some[t]) continue;
        float f[P::V];
        P::unpack(u[t], f);
        keep<STREAM>(f, j.codes + w.row[t] * j.ldc, j.scales + w.row[t] * j.lds, w.col[t]);
    }
}

template <typename T, int N, bool STREAM>
__global__ __launch_bounds__(kThreads) void load_kernel(Ckpt8Job j) {
    using P = Piece<T>;
    const Where<N, P::V> w(j.rows, blocks_of(j.cols));
    Codes<P::V> c[N];
#pragma unroll
    for (int t = 0; t < N; ++t)
        if (w.some[t]) c[t].load(j.codes + w.row[t] * j.ldc, j.scales + w.row[t] * j.lds, w.col[t]);
#pragma unroll
    for (int t = 0; t < N; ++t) {
        if (!w.some[t]) continue;
        float f[P::V];
        c[t].values(f);
        P::template store<STREAM>(static_cast<T*>(j.out) + w.row[t] * j.ldx + w.col[t], j.cols - w.col[t], P::pack(f));
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

// One piece a lane (two: 98304 x 1408 bf16 forward and back 280 us instead of 267).
template <typename T, int KIND, bool SAVE, bool STREAM>
__global__ __launch_bounds__(kThreads) void act_kernel(ActJob j) {
    using P = Piece<T>;
    constexpr int kParts = KIND == kActSwiglu ? 2 : 1, V = P::V;
    const int64_t blocks = blocks_of(j.cols);
    const Where<1, V> w(j.rows, blocks);
    if (!w.some[0]) return;
    const int64_t row = w.row[0], left = j.cols - w.col[0];
    const int col = w.col[0];
    u32x4_any u[kParts];
#pragma unroll
    for (int p = 0; p < kParts; ++p) u[p] = P::load(static_cast<const T*>(j.u) + row * j.ldu + p * j.cols + col, left);
    float f[kParts][V], a[V];
#pragma unroll
    for (int p = 0; p < kParts; ++p) P::unpack(u[p], f[p]);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float v[2] = {f[0][i], f[kParts - 1][i]};
        a[i] = act<KIND>(v);
    }
    P::template store<STREAM>(static_cast<T*>(j.a) + row * j.lda + col, left, P::pack(a));
    if constexpr (SAVE)
#pragma unroll
        for (int p = 0; p < kParts; ++p)
            keep<STREAM>(f[p], j.codes + row * j.ldc + p * blocks * kCkpt8Block, j.scales + row * j.lds + p * blocks, col);
}

template <typename T, int KIND, bool SAVED, bool STREAM>
__global__ __launch_bounds__(kThreads) void act_bwd_kernel(ActJob j) {
    using P = Piece<T>;
    constexpr int kParts = KIND == kActSwiglu ? 2 : 1, V = P::V;
    const int64_t blocks = blocks_of(j.cols);
    const Where<1, V> w(j.rows, blocks);
    if (!w.some[0]) return;
    const int64_t row = w.row[0], left = j.cols - w.col[0];
    const int col = w.col[0];
    const u32x4_any d = P::load(static_cast<const T*>(j.da) + row * j.ldda + col, left);
    float f[kParts][V], da[V], du[kParts][V], a[V];
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
        if constexpr (SAVED) {
            Codes<V> c;
            c.load(j.codes + row * j.ldc + p * blocks * kCkpt8Block, j.scales + row * j.lds + p * blocks, col);
            c.values(f[p]);
        } else {
            P::unpack(P::load(static_cast<const T*>(j.u) + row * j.ldu + p * j.cols + col, left), f[p]);
        }
    }
    P::unpack(d, da);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float v[2] = {f[0][i], f[kParts - 1][i]};
        float g[2];
        a[i] = act_grad<KIND>(v, da[i], g);
#pragma unroll
        for (int p = 0; p < kParts; ++p) du[p][i] = g[p];
    }
#pragma unroll
    for (int p = 0; p < kParts; ++p)
        P::template store<STREAM>(static_cast<T*>(j.du) + row * j.lddu + p * j.cols + col, left, P::pack(du[p]));
    if (j.a) P::template store<STREAM>(static_cast<T*>(j.a) + row * j.lda + col, left, P::pack(a));
}

int64_t pieces(int64_t rows, int64_t cols, bool bf16) { return rows * blocks_of(cols) * (kCkpt8Block / (bf16 ? 8 : 4)); }

unsigned grid(int64_t n, int each) { return (unsigned)((n + kThreads * each - 1) / (kThreads * each)); }

// Two pieces a lane for tensors of 2^24 pieces and more (1 GiB of bf16 to 8 bits and back, us, one / two / four / eight a lane: 567 / 537 /
// 539 / 554; 4099 x 1411 fp32 14.2 / 15.0).
constexpr int kTwo = 2;
constexpr int64_t kTwoPieces = int64_t(1) << 24;

template <typename T, int N>
void save_stream(const Ckpt8Job& j, bool stream, hipStream_t s) {
    const unsigned n = grid(pieces(j.rows, j.cols, j.bf16), N);
    if (stream) save_kernel<T, N, true><<<n, kThreads, 0, s>>>(j);
    else save_kernel<T, N, false><<<n, kThreads, 0, s>>>(j);
}
template <typename T, int N>
void load_stream(const Ckpt8Job& j, bool stream, hipStream_t s) {
    const unsigned n = grid(pieces(j.rows, j.cols, j.bf16), N);
    if (stream) load_kernel<T, N, true><<<n, kThreads, 0, s>>>(j);
    else load_kernel<T, N, false><<<n, kThreads, 0, s>>>(j);
}

template <typename T, int KIND, bool SAVED>
void act_stream(const ActJob& j, bool bwd, bool stream, hipStream_t s) {
    const unsigned n = grid(pieces(j.rows, j.cols, j.bf16), 1);
    if (bwd) {
        if (stream) act_bwd_kernel<T, KIND, SAVED, true><<<n, kThreads, 0, s>>>(j);
        else act_bwd_kernel<T, KIND, SAVED, false><<<n, kThreads, 0, s>>>(j);
    } else {
        if (stream) act_kernel<T, KIND, SAVED, true><<<n, kThreads, 0, s>>>(j);
        else act_kernel<T, KIND, SAVED, false><<<n, kThreads, 0, s>>>(j);
    }
}

template <typename T, int KIND>
void act_saved(const ActJob& j, bool bwd, bool stream, hipStream_t s) {
    j.codes ? act_stream<T, KIND, true>(j, bwd, stream, s) : act_stream<T, KIND, false>(j, bwd, stream, s);
}

hipError_t launch_any(const ActJob& j, bool bwd, hipStream_t s) {
    const bool stream = j.rows * j.cols * (j.bf16 ? 2 : 4) >= kStreamBytes;
    if (j.kind == kActSwiglu) j.bf16 ? act_saved<uint16_t, kActSwiglu>(j, bwd, stream, s) : act_saved<float, kActSwiglu>(j, bwd, stream, s);
    else j.bf16 ? act_saved<uint16_t, kActRelu2>(j, bwd, stream, s) : act_saved<float, kActRelu2>(j, bwd, stream, s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ckpt8_save(const Ckpt8Job& j, hipStream_t s) {
    const bool many = pieces(j.rows, j.cols, j.bf16) >= kTwoPieces, stream = j.rows * j.cols >= kStreamBytes;
    if (j.bf16) many ? save_stream<uint16_t, kTwo>(j, stream, s) : save_stream<uint16_t, 1>(j, stream, s);
    else many ? save_stream<float, kTwo>(j, stream, s) : save_stream<float, 1>(j, stream, s);
    return hipGetLastError();
}

hipError_t launch_ckpt8_load(const Ckpt8Job& j, hipStream_t s) {
    const bool many = pieces(j.rows, j.cols, j.bf16) >= kTwoPieces, stream = j.rows * j.cols * (j.bf16 ? 2 : 4) >= kStreamBytes;
    if (j.bf16) many ? load_stream<uint16_t, kTwo>(j, stream, s) : load_stream<uint16_t, 1>(j, stream, s);
    else many ? load_stream<float, kTwo>(j, stream, s) : load_stream<float, 1>(j, stream, s);
    return hipGetLastError();
}

hipError_t launch_act(const ActJob& j, hipStream_t s) { return launch_any(j, false, s); }
hipError_t launch_act_bwd(const ActJob& j, hipStream_t s) { return launch_any(j, true, s); }

int64_t ckpt8_units(int64_t rows, int64_t cols) { return rows * blocks_of(cols) * (kCkpt8Block / 4); }

}  // namespace ufp4
