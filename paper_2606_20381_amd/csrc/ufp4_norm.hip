// Layer norm over the rows of a bf16 or fp32 tensor, forward and backward.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), h = (x - mu) r, y = h gamma + beta
//   g = dy gamma, dx = r (g - mean(g) - h mean(g h)), dgamma = sum over rows of dy h, dbeta = sum over rows of dy
//
// HBM bound: forward reads x and writes y once, backward reads x and dy and writes dx once. A row lives in the registers
// of TPR threads (one wave, 256 or 1024 threads), so that mean and variance are two sums over registers (no cancellation
// of E[x^2] - mu^2) without a second read. A thread keeps its columns over all rows that its workgroup takes: gamma, beta
// and, backward, the partial dgamma and dbeta stay in its registers, and the weights' gradient costs one fp32 row per
// workgroup instead of a second pass over x and dy. The partial rows are then added in a fixed order, so results repeat.
// Rows too long for the registers are read again per pass (`*_long_kernel`).

#include "ufp4_internal.h"
#include "ufp4_rows.h"

namespace ufp4 {

namespace {

constexpr int kPieces = 4;  // 16-byte pieces per thread of a row in registers
constexpr int kLongThreads = 1024;

__device__ __forceinline__ float weight_at(const void* w, int w_bf16, int64_t c) {
    return w_bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(w)[c] << 16) : static_cast<const float*>(w)[c];
}

// Sums of N values over the TPR threads of a row. TPR > 64: through `s` ([wave][N], one barrier; the caller alternates
// between two such arrays, so that a wave that is ahead does not overwrite what another still reads).
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* s) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
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

template <typename T, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(NormJob j) {
    using P = Piece<T>;
    constexpr int V = P::V, kRowsWG = TPR < 256 ? 256 / TPR : 1;
    __shared__ float s_sum[2][16];
    const int t = threadIdx.x % TPR;
    float gm[kPieces][V], bt[kPieces][V];
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int64_t c = ((int64_t)p * TPR + t) * V + i;
            gm[p][i] = j.gamma && c < j.cols ? weight_at(j.gamma, j.w_bf16, c) : 1.0f;
            bt[p][i] = j.beta && c < j.cols ? weight_at(j.beta, j.w_bf16, c) : 0.0f;
        }
    const float inv_n = 1.0f / (float)j.cols;
    for (int64_t row = (int64_t)blockIdx.x * kRowsWG + threadIdx.x / TPR; row < j.rows; row += (int64_t)gridDim.x * kRowsWG) {
        const T* const x = static_cast<const T*>(j.x) + row * j.ldx;
        u32x4_any raw[kPieces];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int64_t c = ((int64_t)p * TPR + t) * V;
            raw[p] = P::load(x + c, j.cols - c);
        }
        float f[kPieces][V], sum[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            P::unpack(raw[p], f[p]);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0] += f[p][i];
        }
        row_sums<TPR, 1>(sum, s_sum[0]);
        const float mean = sum[0] * inv_n;
        float sq[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
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
        for (int p = 0; p < kPieces; ++p) {
            const int64_t c = ((int64_t)p * TPR + t) * V;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = __builtin_fmaf(f[p][i] * rstd, gm[p][i], bt[p][i]);
            P::store(y + c, j.cols - c, P::pack(o));
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

// Backward. `part` is [gridDim.x][2][cols]: the workgroup's sums of dy h and of dy.
template <typename T, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_bwd_kernel(NormBwdJob j) {
    using P = Piece<T>;
    constexpr int V = P::V, kRowsWG = TPR < 256 ? 256 / TPR : 1;
    __shared__ float s_sum[2][32];
    __shared__ float s_part[kRowsWG > 1 ? kRowsWG - 1 : 1][kRowsWG > 1 ? TPR * V : 1];
    const int t = threadIdx.x % TPR, rw = threadIdx.x / TPR;
    float gm[kPieces][V], ag[kPieces][V], ab[kPieces][V];
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int64_t c = ((int64_t)p * TPR + t) * V + i;
            gm[p][i] = j.gamma && c < j.cols ? weight_at(j.gamma, j.w_bf16, c) : 1.0f;
            ag[p][i] = ab[p][i] = 0.0f;
        }
    const float inv_n = 1.0f / (float)j.cols;
    int buf = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRowsWG + rw; row < j.rows; row += (int64_t)gridDim.x * kRowsWG) {
        const T* const x = static_cast<const T*>(j.x) + row * j.ldx;
        const T* const dy = static_cast<const T*>(j.dy) + row * j.lddy;
        u32x4_any rx[kPieces], rd[kPieces];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int64_t c = ((int64_t)p * TPR + t) * V;
            rx[p] = P::load(x + c, j.cols - c);
            rd[p] = P::load(dy + c, j.cols - c);  // zero past the row: its terms add nothing
        }
        const float mean = j.mean[row], rstd = j.rstd[row];
        float sum[2] = {0.0f, 0.0f};
        float h[kPieces][V], d[kPieces][V];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            P::unpack(rx[p], h[p]);
            P::unpack(rd[p], d[p]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                // past the row: nothing, even where the statistics are not finite
                const bool in = ((int64_t)p * TPR + t) * V + i < j.cols;
                h[p][i] = in ? (h[p][i] - mean) * rstd : 0.0f;
                ag[p][i] = __builtin_fmaf(d[p][i], h[p][i], ag[p][i]);
                ab[p][i] += d[p][i];
                d[p][i] *= gm[p][i];
                sum[0] += d[p][i];
                sum[1] = __builtin_fmaf(d[p][i], h[p][i], sum[1]);
            }
        }
        row_sums<TPR, 2>(sum, s_sum[buf]);
        buf ^= 1;
        const float c1 = sum[0] * inv_n, c2 = sum[1] * inv_n;
        T* const dx = static_cast<T*>(j.dx) + row * j.lddx;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int64_t c = ((int64_t)p * TPR + t) * V;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = rstd * (d[p][i] - c1 - h[p][i] * c2);
            P::store(dx + c, j.cols - c, P::pack(o));
        }
    }
    if (!j.part) return;
    // the workgroup's waves hold the same columns (TPR 64): added in the order of the waves, piece by piece
    float* const out = j.part + (int64_t)blockIdx.x * 2 * j.cols;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            if constexpr (kRowsWG > 1) {
                __syncthreads();
                if (rw > 0) {
#pragma unroll
                    for (int i = 0; i < V; ++i) s_part[rw - 1][i * TPR + t] = q ? ab[p][i] : ag[p][i];
                }
                __syncthreads();
            }
            if (rw == 0) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float v = q ? ab[p][i] : ag[p][i];
                    if constexpr (kRowsWG > 1) {
#pragma unroll
                        for (int w = 0; w < kRowsWG - 1; ++w) v += s_part[w][i * TPR + t];
                    }
                    const int64_t c = ((int64_t)p * TPR + t) * V + i;
                    if (c < j.cols) out[q * j.cols + c] = v;
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
    float* const out = j.part + (int64_t)blockIdx.y * 2 * j.cols;
    out[c] = ag;
    out[j.cols + c] = ab;
}

// dgamma and dbeta from `n` partial rows of 2 * cols sums: 64 columns per workgroup, 16 waves over the partial rows, then
// the waves' sums in order.
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float* __restrict__ part, int n, int64_t cols, float* dgamma,
                                                           float* dbeta) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;  // of 2 * cols
    float v = 0.0f;
    if (c < 2 * cols)
        for (int i = wave; i < n; i += 16) v += part[(int64_t)i * 2 * cols + c];
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
}

template <typename T>
int threads_per_row(int64_t cols) {
    const int64_t one = (int64_t)Piece<T>::V * kPieces;  // columns per thread
    return cols <= 64 * one ? 64 : cols <= 256 * one ? 256 : cols <= 1024 * one ? 1024 : 0;
}

unsigned norm_grid(int64_t rows, int tpr) {
    const int64_t wgs = tpr == 64 ? (rows + 3) / 4 : rows;
    const int64_t most = tpr == 1024 || tpr == 0 ? 512 : 2048;  // resident workgroups on 256 CUs
    return (unsigned)(wgs < most ? wgs : most);
}

// Workgroups, and so partial rows of the weights' gradient, of the backward kernel.
constexpr int64_t kMostParts = 512;
unsigned norm_bwd_grid(int64_t rows, int tpr) {
    const int64_t wgs = tpr == 64 ? (rows + 3) / 4 : rows;
    return (unsigned)(wgs < kMostParts ? wgs : kMostParts);
}
constexpr int kLongParts = 64;

template <typename T>
hipError_t launch_norm_t(const NormJob& j, hipStream_t s) {
    const int tpr = threads_per_row<T>(j.cols);
    const unsigned g = norm_grid(j.rows, tpr);
    switch (tpr) {
        case 64: norm_kernel<T, 64><<<g, 256, 0, s>>>(j); break;
        case 256: norm_kernel<T, 256><<<g, 256, 0, s>>>(j); break;
        case 1024: norm_kernel<T, 1024><<<g, 1024, 0, s>>>(j); break;
        default: norm_long_kernel<T><<<g, kLongThreads, 0, s>>>(j); break;
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch_norm_bwd_t(const NormBwdJob& j, hipStream_t s) {
    const int tpr = threads_per_row<T>(j.cols);
    unsigned g = norm_bwd_grid(j.rows, tpr);
    if (g > 0) {
        switch (tpr) {
            case 64: norm_bwd_kernel<T, 64><<<g, 256, 0, s>>>(j); break;
            case 256: norm_bwd_kernel<T, 256><<<g, 256, 0, s>>>(j); break;
            case 1024: norm_bwd_kernel<T, 1024><<<g, 1024, 0, s>>>(j); break;
            default: {
                const unsigned rows_g = g;
                if (j.part) {  // before dx, which may lie on x or dy
                    g = (unsigned)(j.rows < kLongParts ? j.rows : kLongParts);
                    norm_bwd_cols_kernel<T><<<dim3((unsigned)((j.cols + 255) / 256), g), 256, 0, s>>>(j);
                }
                norm_bwd_long_kernel<T><<<rows_g, kLongThreads, 0, s>>>(j);
            }
        }
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!j.dgamma && !j.dbeta)) return e;
    norm_reduce_kernel<<<(unsigned)((2 * j.cols + 63) / 64), 1024, 0, s>>>(j.part, (int)g, j.cols, j.dgamma, j.dbeta);
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
    const int tpr = bf16 ? threads_per_row<uint16_t>(cols) : threads_per_row<float>(cols);
    if (tpr == 0) return rows < kLongParts ? rows : kLongParts;
    return norm_bwd_grid(rows, tpr);
}

}  // namespace ufp4
