// Layer norm over the rows of a bf16 or fp32 tensor, forward and backward.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), h = (x - mu) r, y = h gamma + beta
//   g = dy gamma, dx = r (g - mean(g) - h mean(g h)), dgamma = sum over rows of dy h, dbeta = sum over rows of dy
//
// HBM bound: forward reads x and writes y once, backward reads x and dy and writes dx once. A row lives in the registers
// of TPR threads (an eighth of a wave up to 1024 threads), so that mean and variance are two sums over registers (no cancellation
// of E[x^2] - mu^2) without a second read. A thread keeps its columns over all rows that its workgroup takes: gamma, beta
// and, backward, the partial dgamma and dbeta stay in its registers, and the weights' gradient costs one fp32 row per
// workgroup instead of a second pass over x and dy. The partial rows are then added in a fixed order, so results repeat.
// Rows too long for the registers are read again per pass (`*_long_kernel`).
//
// Measured: forward 16384 x 5120 bf16 55 us = 6.1 TB/s with tensors in place, 65 us = 5.2 TB/s with new ones each time (a copy of
// 1 GiB runs at 5.1); backward 8192 x 2048 bf16 22.5 us in two launches (25 with new tensors; its 101 MB are 20 us at the copy's rate), 32768 x 5120
// 187 us = 5.4 TB/s; short rows, 262144 x 128 bf16, 24 and 34 us (a wave per row: 61 and 91); 4 x 2048 3.6 us, launch and two
// dependent sums.

#include "ufp4_internal.h"
#include "ufp4_rows.h"

#include <type_traits>

namespace ufp4 {

namespace {

constexpr int kLongThreads = 1024;

__device__ __forceinline__ float weight_at(const void* w, int w_bf16, int64_t c) {
    return w_bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(w)[c] << 16) : static_cast<const float*>(w)[c];
}

// A thread's pieces of a weight vector (bf16 or fp32, `otherwise` where there is none or past its end).
template <int TPR, int NP, int V>
__device__ __forceinline__ void load_weights(const void* w, int w_bf16, int64_t cols, int t, float otherwise, float (&f)[NP][V]) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) f[p][i] = otherwise;
    if (!w) return;
    auto some = [&](auto* q) {
        using W = typename std::remove_const<typename std::remove_pointer<decltype(q)>::type>::type;
        using P = Piece<W>;
        constexpr int kV = V < P::V ? V : P::V;  // of a 16-byte load
        u32x4_any raw[NP][V / kV];
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int k = 0; k < V / kV; ++k) {
                const int64_t c = ((int64_t)p * TPR + t) * V + k * kV;
                raw[p][k] = P::load(q + c, cols - c < kV ? cols - c : P::V <= cols - c ? P::V : kV);
            }
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int k = 0; k < V / kV; ++k) {
                const int64_t c = ((int64_t)p * TPR + t) * V + k * kV;
                float g[P::V];
                P::unpack(raw[p][k], g);
#pragma unroll
                for (int i = 0; i < kV; ++i)
                    if (c + i < cols) f[p][k * kV + i] = g[i];
            }
    };
    if (w_bf16) some(static_cast<const uint16_t*>(w));
    else some(static_cast<const float*>(w));
}

// Sum over the 64 lanes of a wave, or over each TPR of them.
template <int TPR>
__device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (TPR >= 64) {
        return wave_sum(v);
    } else {
#pragma unroll
        for (int d = TPR / 2; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
        return v;
    }
}

// Sums of N values over the TPR threads of a row. TPR > 64: through `s` ([wave][N], one barrier; the caller alternates
// between two such arrays, so that a wave that is ahead does not overwrite what another still reads).
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* s) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = lanes_sum<TPR>(v[n]);
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) s[wave * N + n] = v[n];
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float t = 0.0f;
#pragma unroll
            for (int w = 0; w < TPR / 64; ++w) t += s[w * N + n];
            v[n] = t;
        }
    }
}

// NP 16-byte pieces per thread. The next row is on its way while this one is computed.
template <typename T, int TPR, int NP, bool STREAM>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(NormJob j) {
    using P = Piece<T>;
    constexpr int V = P::V, kRowsWG = TPR < 256 ? 256 / TPR : 1;
    __shared__ float s_sum[2][16];
    const int t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * kRowsWG;
    int64_t row = (int64_t)blockIdx.x * kRowsWG + threadIdx.x / TPR;
    auto load = [&](int64_t r, u32x4_any (&raw)[NP]) {
        const T* const x = static_cast<const T*>(j.x) + r * j.ldx;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int64_t c = ((int64_t)p * TPR + t) * V;
            raw[p] = P::load(x + c, j.cols - c);
        }
    };
    u32x4_any raw[NP];
    if (row < j.rows) load(row, raw);
    float gm[NP][V], bt[NP][V];
    load_weights<TPR, NP, V>(j.gamma, j.w_bf16, j.cols, t, 1.0f, gm);
    load_weights<TPR, NP, V>(j.beta, j.w_bf16, j.cols, t, 0.0f, bt);
    const float inv_n = 1.0f / (float)j.cols;
    for (; row < j.rows; row += step) {
        float f[NP][V], sum[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            P::unpack(raw[p], f[p]);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0] += f[p][i];
        }
        if (row + step < j.rows) load(row + step, raw);
        row_sums<TPR, 1>(sum, s_sum[0]);
        const float mean = sum[0] * inv_n;
        float sq[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int64_t c = ((int64_t)p * TPR + t) * V + i;
                f[p][i] -= mean;
                if (c < j.cols) sq[0] = __builtin_fmaf(f[p][i], f[p][i], sq[0]);
            }
        row_sums<TPR, 1>(sq, s_sum[1]);
        const float rstd = 1.0f / sqrtf(sq[0] * inv_n + j.eps);
        if (t == 0) {
            if (j.mean) j.mean[row] = mean;
            if (j.rstd) j.rstd[row] = rstd;
        }
        T* const y = static_cast<T*>(j.y) + row * j.ldy;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int64_t c = ((int64_t)p * TPR + t) * V;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = __builtin_fmaf(f[p][i] * rstd, gm[p][i], bt[p][i]);
            P::template store<STREAM>(y + c, j.cols - c, P::pack(o));
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kLongThreads) void norm_long_kernel(NormJob j) {
    using P = Piece<T>;
    constexpr int V = P::V;
    __shared__ float s_sum[2][16];
    const int64_t step = (int64_t)kLongThreads * V;
    for (int64_t row = blockIdx.x; row < j.rows; row += gridDim.x) {
        const T* const x = static_cast<const T*>(j.x) + row * j.ldx;
        T* const y = static_cast<T*>(j.y) + row * j.ldy;
        float f[V], sum[1] = {0.0f}, sq[1] = {0.0f};
        for (int64_t c = (int64_t)threadIdx.x * V; c < j.cols; c += step) {
            P::unpack(P::load(x + c, j.cols - c), f);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0] += f[i];
        }
        row_sums<kLongThreads, 1>(sum, s_sum[0]);
        const float mean = sum[0] / (float)j.cols;
        for (int64_t c = (int64_t)threadIdx.x * V; c < j.cols; c += step) {
            P::unpack(P::load(x + c, j.cols - c), f);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i < j.cols) sq[0] = __builtin_fmaf(f[i] - mean, f[i] - mean, sq[0]);
        }
        row_sums<kLongThreads, 1>(sq, s_sum[1]);
        const float rstd = 1.0f / sqrtf(sq[0] / (float)j.cols + j.eps);
        if (threadIdx.x == 0) {
            if (j.mean) j.mean[row] = mean;
            if (j.rstd) j.rstd[row] = rstd;
        }
        for (int64_t c = (int64_t)threadIdx.x * V; c < j.cols; c += step) {
            P::unpack(P::load(x + c, j.cols - c), f);
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool in = c + i < j.cols;
                const float gm = in && j.gamma ? weight_at(j.gamma, j.w_bf16, c + i) : 1.0f;
                const float bt = in && j.beta ? weight_at(j.beta, j.w_bf16, c + i) : 0.0f;
                o[i] = __builtin_fmaf((f[i] - mean) * rstd, gm, bt);
            }
            P::store(y + c, j.cols - c, P::pack(o));
        }
    }
}

// Where workgroup `at` of `n` puts its sums of dy h (q = 0) and of dy (q = 1): in its row of `part` [n][2][cols], or, alone, where
// they are asked for (null: nowhere).
__device__ __forceinline__ float* sums_at(const NormBwdJob& j, unsigned n, unsigned at, int q) {
    return n > 1 ? j.part + ((int64_t)at * 2 + q) * j.cols : q ? j.dbeta : j.dgamma;
}

// Backward. A workgroup takes several rows at a time, as many as a CU's registers hold, at one partial row per CU. kAhead: the next
// row is on its way while this one is computed.
template <typename T, int TPR, int NP>
struct BwdShape {
    static constexpr int kRegs = NP * Piece<T>::V;  // columns per thread, about six registers each
    static constexpr int kThreads = TPR == 1024 || kRegs <= 8 ? 1024 : 512, kRows = kThreads / TPR;
    static constexpr bool kAhead = kThreads == 512 || kRegs <= 8;
    static constexpr bool kFits = TPR < 1024 || kRegs <= 16;
};
template <typename T, int TPR, int NP, bool STREAM>
__global__ __launch_bounds__((BwdShape<T, TPR, NP>::kThreads)) void norm_bwd_kernel(NormBwdJob j) {
    using P = Piece<T>;
    using B = BwdShape<T, TPR, NP>;
    constexpr int V = P::V, kRowsWG = B::kRows, kRowWaves = TPR / 64;
    constexpr int kSums = TPR < 64 ? B::kThreads / 64 : kRowsWG;  // sums of a column that are left at the end: per wave, or per row
    __shared__ float s_sum[2][B::kThreads / 64][2];
    __shared__ float s_part[kSums > 1 ? kSums - 1 : 1][kSums > 1 ? TPR * V : 1];
    const int t = threadIdx.x % TPR, rw = threadIdx.x / TPR;
    const int64_t step = (int64_t)gridDim.x * kRowsWG;
    int64_t row = (int64_t)blockIdx.x * kRowsWG + rw;
    u32x4_any rx[NP], rd[NP];
    float mean = 0.0f, rstd = 0.0f;
    auto load = [&](int64_t r) {
        const T* const x = static_cast<const T*>(j.x) + r * j.ldx;
        const T* const dy = static_cast<const T*>(j.dy) + r * j.lddy;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int64_t c = ((int64_t)p * TPR + t) * V;
            rx[p] = P::load(x + c, j.cols - c);
            rd[p] = P::load(dy + c, j.cols - c);  // zero past the row: its terms add nothing
        }
        mean = j.mean[r];
        rstd = j.rstd[r];
    };
    if (B::kAhead && row < j.rows) load(row);
    float gm[NP][V], ag[NP][V], ab[NP][V];
    load_weights<TPR, NP, V>(j.gamma, j.w_bf16, j.cols, t, 1.0f, gm);
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) ag[p][i] = ab[p][i] = 0.0f;
    const float inv_n = 1.0f / (float)j.cols;
    int buf = 0;
    for (int64_t first = (int64_t)blockIdx.x * kRowsWG; first < j.rows; first += step, row += step) {  // the same for every thread
        const bool live = row < j.rows;
        float sum[2] = {0.0f, 0.0f};
        float h[NP][V], d[NP][V];
        if (!B::kAhead && live) load(row);
        const float r = rstd;
        if (live) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                P::unpack(rx[p], h[p]);
                P::unpack(rd[p], d[p]);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    // past the row: nothing, even where the statistics are not finite
                    const bool in = ((int64_t)p * TPR + t) * V + i < j.cols;
                    h[p][i] = in ? (h[p][i] - mean) * r : 0.0f;
                    ag[p][i] = __builtin_fmaf(d[p][i], h[p][i], ag[p][i]);
                    ab[p][i] += d[p][i];
                    d[p][i] *= gm[p][i];
                    sum[0] += d[p][i];
                    sum[1] = __builtin_fmaf(d[p][i], h[p][i], sum[1]);
                }
            }
        }
        if (B::kAhead && row + step < j.rows) load(row + step);
        sum[0] = lanes_sum<TPR>(sum[0]);
        sum[1] = lanes_sum<TPR>(sum[1]);
        if constexpr (kRowWaves > 1) {  // one barrier a row: two arrays in turn, so that a wave ahead does not overwrite
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) {
                s_sum[buf][wave][0] = sum[0];
                s_sum[buf][wave][1] = sum[1];
            }
            __syncthreads();
            sum[0] = sum[1] = 0.0f;
#pragma unroll
            for (int w = 0; w < kRowWaves; ++w) {
                sum[0] += s_sum[buf][rw * kRowWaves + w][0];
                sum[1] += s_sum[buf][rw * kRowWaves + w][1];
            }
            buf ^= 1;
        }
        if (live) {
            const float c1 = sum[0] * inv_n, c2 = sum[1] * inv_n;
            T* const dx = static_cast<T*>(j.dx) + row * j.lddx;
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int64_t c = ((int64_t)p * TPR + t) * V;
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = r * (d[p][i] - c1 - h[p][i] * c2);
                P::template store<STREAM>(dx + c, j.cols - c, P::pack(o));
            }
        }
    }
    if (!j.part) return;
    // the workgroup's rows have the same columns: those of a wave are added by shuffles, then the sums in their order, piece by piece
    const int at = TPR < 64 ? (int)(threadIdx.x >> 6) : rw;
    const bool holds = TPR >= 64 || (threadIdx.x & 63) < TPR;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float* const out = sums_at(j, gridDim.x, blockIdx.x, q);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[i] = q ? ab[p][i] : ag[p][i];
#pragma unroll
                for (int d = TPR; d < 64; d <<= 1) v[i] += __shfl_xor(v[i], d, 64);
            }
            if constexpr (kSums > 1) {
                __syncthreads();
                if (at > 0 && holds) {
#pragma unroll
                    for (int i = 0; i < V; ++i) s_part[at - 1][i * TPR + t] = v[i];
                }
                __syncthreads();
            }
            if (at == 0 && holds) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if constexpr (kSums > 1) {
#pragma unroll
                        for (int w = 0; w < kSums - 1; ++w) v[i] += s_part[w][i * TPR + t];
                    }
                    const int64_t c = ((int64_t)p * TPR + t) * V + i;
                    if (c < j.cols && out) out[c] = v[i];
                }
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kLongThreads) void norm_bwd_long_kernel(NormBwdJob j) {
    using P = Piece<T>;
    constexpr int V = P::V;
    __shared__ float s_sum[2][32];
    const int64_t step = (int64_t)kLongThreads * V;
    int buf = 0;
    for (int64_t row = blockIdx.x; row < j.rows; row += gridDim.x) {
        const T* const x = static_cast<const T*>(j.x) + row * j.ldx;
        const T* const dy = static_cast<const T*>(j.dy) + row * j.lddy;
        const float mean = j.mean[row], rstd = j.rstd[row];
        float h[V], d[V], sum[2] = {0.0f, 0.0f};
        auto take = [&](int64_t c) {
            P::unpack(P::load(x + c, j.cols - c), h);
            P::unpack(P::load(dy + c, j.cols - c), d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool in = c + i < j.cols;
                h[i] = in ? (h[i] - mean) * rstd : 0.0f;
                if (in && j.gamma) d[i] *= weight_at(j.gamma, j.w_bf16, c + i);
            }
        };
        for (int64_t c = (int64_t)threadIdx.x * V; c < j.cols; c += step) {
            take(c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                sum[0] += d[i];
                sum[1] = __builtin_fmaf(d[i], h[i], sum[1]);
            }
        }
        row_sums<kLongThreads, 2>(sum, s_sum[buf]);
        buf ^= 1;
        const float c1 = sum[0] / (float)j.cols, c2 = sum[1] / (float)j.cols;
        T* const dx = static_cast<T*>(j.dx) + row * j.lddx;
        for (int64_t c = (int64_t)threadIdx.x * V; c < j.cols; c += step) {
            take(c);
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = rstd * (d[i] - c1 - h[i] * c2);
            P::store(dx + c, j.cols - c, P::pack(o));
        }
    }
}

// Partial dgamma and dbeta of long rows: a thread takes one column of a run of rows.
template <typename T>
__global__ __launch_bounds__(256) void norm_bwd_cols_kernel(NormBwdJob j) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= j.cols) return;
    float ag = 0.0f, ab = 0.0f;
    for (int64_t row = blockIdx.y; row < j.rows; row += gridDim.y) {
        const T xv = static_cast<const T*>(j.x)[row * j.ldx + c], dv = static_cast<const T*>(j.dy)[row * j.lddy + c];
        float x, d;
        if constexpr (sizeof(T) == 2) {
            x = __uint_as_float((uint32_t)xv << 16);
            d = __uint_as_float((uint32_t)dv << 16);
        } else {
            x = xv;
            d = dv;
        }
        ag = __builtin_fmaf(d, (x - j.mean[row]) * j.rstd[row], ag);
        ab += d;
    }
    float *const g = sums_at(j, gridDim.y, blockIdx.y, 0), *const b = sums_at(j, gridDim.y, blockIdx.y, 1);
    if (g) g[c] = ag;
    if (b) b[c] = ab;
}

// dgamma and dbeta from `n` partial rows of 2 * cols sums: a workgroup takes 64 columns at a time, 16 waves over the partial rows,
// then the waves' sums in order. Rows of up to kReduceGroups * 32 columns have a workgroup for each 64 sums; a grid holds fewer
// than 2^32 threads, so those of longer ones take several in turn.
constexpr int64_t kReduceGroups = int64_t(1) << 16;
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float* __restrict__ part, int n, int64_t cols, float* dgamma,
                                                           float* dbeta) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < 2 * cols; c0 += (int64_t)gridDim.x * 64) {  // the same for every thread
        const int64_t c = c0 + lane;  // of 2 * cols
        float v = 0.0f;
        if (c < 2 * cols) {
#pragma unroll 8
            for (int i = wave; i < n; i += 16) v += part[(int64_t)i * 2 * cols + c];
        }
        s[wave][lane] = v;
        __syncthreads();
        if (wave == 0 && c < 2 * cols) {
            float t = 0.0f;
#pragma unroll
            for (int w = 0; w < 16; ++w) t += s[w][lane];
            if (c < cols) {
                if (dgamma) dgamma[c] = t;
            } else if (dbeta) {
                dbeta[c - cols] = t;
            }
        }
        __syncthreads();  // the sums have been read
    }
}

// Threads and pieces that a row of `pieces` 16-byte pieces takes: few pieces a thread, so that the weights (and, backward, their
// gradient) leave registers for many waves; a wave by itself needs no barrier; short rows share a wave. A rule of kernel(threads, pieces per thread);
// false for a row that is too long.
template <typename F>
bool for_row(int64_t pieces, F&& kernel) {
    using std::integral_constant;
    if (pieces <= 8) kernel(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (pieces <= 16) kernel(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (pieces <= 32) kernel(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (pieces <= 64) kernel(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (pieces <= 128) kernel(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (pieces <= 256) kernel(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (pieces <= 512) kernel(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (pieces <= 768) kernel(integral_constant<int, 256>{}, integral_constant<int, 3>{});
    else if (pieces <= 1024) kernel(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
    else if (pieces <= 2048) kernel(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    else if (pieces <= 4096) kernel(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    else return false;
    return true;
}
template <typename T>
int64_t pieces_of(int64_t cols) {
    return (cols + Piece<T>::V - 1) / Piece<T>::V;
}

int64_t min64(int64_t a, int64_t b) { return a < b ? a : b; }

// Partial rows of the weights' gradient, one per workgroup of the backward kernel (one workgroup a CU); of long rows, the runs of
// rows whose columns are summed.
constexpr int64_t kMostParts = 256, kLongParts = 64;
template <typename T>
int64_t parts_of(int64_t rows, int64_t cols) {
    int64_t n = min64(rows, kLongParts);
    for_row(pieces_of<T>(cols), [&](auto tpr, auto np) {
        using B = BwdShape<T, decltype(tpr)::value, decltype(np)::value>;
        if (B::kFits) n = min64((rows + B::kRows - 1) / B::kRows, kMostParts);
    });
    return n;
}

// Whether `n` tensors of this shape, read and written, are kStreamBytes and more: the output is then stored nontemporally. us, so /
// plainly, bf16: forward 16384 x 5120 55 / 65, 65536 x 2048 90 / 107, 32768 x 5120 127 / 131; backward 32768 x 2048 68 / 80,
// 16384 x 5120 101 / 103.
template <typename T>
bool streams(int n, int64_t rows, int64_t cols) {
    return rows * cols * (int64_t)sizeof(T) * n >= kStreamBytes;
}

template <typename T>
hipError_t launch_norm_t(const NormJob& j, hipStream_t s) {
    const bool fits = for_row(pieces_of<T>(j.cols), [&](auto tpr, auto np) {
        constexpr int kTPR = decltype(tpr)::value, kThreads = kTPR < 256 ? 256 : kTPR, kRows = kThreads / kTPR;
        const int64_t wgs = min64((j.rows + kRows - 1) / kRows, kThreads == 1024 ? 512 : 2048);  // resident on 256 CUs
        const auto kernel = streams<T>(2, j.rows, j.cols) ? norm_kernel<T, kTPR, decltype(np)::value, true>
                                                          : norm_kernel<T, kTPR, decltype(np)::value, false>;
        kernel<<<(unsigned)wgs, kThreads, 0, s>>>(j);
    });
    if (!fits) norm_long_kernel<T><<<(unsigned)min64(j.rows, 512), kLongThreads, 0, s>>>(j);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_norm_bwd_t(const NormBwdJob& j, hipStream_t s) {
    const unsigned parts = (unsigned)parts_of<T>(j.rows, j.cols);
    if (parts > 0) {
        bool done = false;
        for_row(pieces_of<T>(j.cols), [&](auto tpr, auto np) {
            using B = BwdShape<T, decltype(tpr)::value, decltype(np)::value>;
            if constexpr (B::kFits) {
                const auto kernel = streams<T>(3, j.rows, j.cols)
                                        ? norm_bwd_kernel<T, decltype(tpr)::value, decltype(np)::value, true>
                                        : norm_bwd_kernel<T, decltype(tpr)::value, decltype(np)::value, false>;
                kernel<<<parts, B::kThreads, 0, s>>>(j);
                done = true;
            }
        });
        if (!done) {
            if (j.part)  // before dx, which may lie on x or dy
                norm_bwd_cols_kernel<T><<<dim3((unsigned)((j.cols + 255) / 256), parts), 256, 0, s>>>(j);
            norm_bwd_long_kernel<T><<<(unsigned)min64(j.rows, 512), kLongThreads, 0, s>>>(j);
        }
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!j.dgamma && !j.dbeta) || parts == 1) return e;  // a lone workgroup's sums are in place
    norm_reduce_kernel<<<(unsigned)min64((2 * j.cols + 63) / 64, kReduceGroups), 1024, 0, s>>>(j.part, (int)parts, j.cols, j.dgamma,
                                                                                            j.dbeta);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormJob& j, hipStream_t s) {
    return j.bf16 ? launch_norm_t<uint16_t>(j, s) : launch_norm_t<float>(j, s);
}

hipError_t launch_norm_bwd(const NormBwdJob& j, hipStream_t s) {
    return j.bf16 ? launch_norm_bwd_t<uint16_t>(j, s) : launch_norm_bwd_t<float>(j, s);
}

int64_t norm_bwd_parts(int bf16, int64_t rows, int64_t cols) {
    return bf16 ? parts_of<uint16_t>(rows, cols) : parts_of<float>(rows, cols);
}

}  // namespace ufp4
