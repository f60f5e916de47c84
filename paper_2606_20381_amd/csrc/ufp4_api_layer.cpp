// C ABI of the layer norm and of the expert sort, dispatch and combine: argument validation on the host, then the launches.
// Declarations and the meaning of every argument are in include/ufp4.h.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ufp4.h"
#include "ufp4_internal.h"

using namespace ufp4;

namespace {

int status_of(hipError_t e) { return e == hipSuccess ? UFP4_OK : UFP4_ERR_HIP; }
bool known(int dtype) { return dtype == UFP4_OUT_F32 || dtype == UFP4_OUT_BF16; }
bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
uintptr_t size_of(int dtype) { return dtype == UFP4_OUT_BF16 ? 2 : 4; }

constexpr int64_t kMostCols = int64_t(1) << 30;

// A tensor [rows, cols] of `dtype` at p, rows ld elements apart; without an element it is never accessed.
int check_rows(int dtype, const void* p, int64_t rows, int64_t cols, int64_t ld) {
    if (rows == 0 || cols == 0) return UFP4_OK;
    if (!p) return UFP4_ERR_INVALID_ARG;
    if (ld < cols) return UFP4_ERR_SHAPE;
    if (!aligned(p, size_of(dtype))) return UFP4_ERR_ALIGN;
    return UFP4_OK;
}

int first(int a, int b) { return a != UFP4_OK ? a : b; }

}  // namespace

extern "C" {

int ufp4_layer_norm(int dtype, const void* x_dev, int64_t rows, int64_t cols, int64_t ldx, int w_dtype, const void* gamma_dev,
                    const void* beta_dev, float eps, void* y_dev, int64_t ldy, float* mean_dev, float* rstd_dev,
                    void* stream) {
    if (!known(dtype) || !known(w_dtype) || rows < 0 || cols < 0) return UFP4_ERR_INVALID_ARG;
    if (!(eps >= 0.0f) || isinf(eps)) return UFP4_ERR_INVALID_ARG;
    const int st = first(check_rows(dtype, x_dev, rows, cols, ldx), check_rows(dtype, y_dev, rows, cols, ldy));
    if (st != UFP4_OK) return st;
    if (!aligned(gamma_dev, size_of(w_dtype)) || !aligned(beta_dev, size_of(w_dtype)) || !aligned(mean_dev, 4) ||
        !aligned(rstd_dev, 4))
        return UFP4_ERR_ALIGN;
    if (cols > kMostCols) return UFP4_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return UFP4_OK;
    const NormJob j{dtype == UFP4_OUT_BF16, w_dtype == UFP4_OUT_BF16, x_dev, rows, cols, ldx, gamma_dev, beta_dev, eps,
                    y_dev, ldy, mean_dev, rstd_dev};
    return status_of(launch_norm(j, static_cast<hipStream_t>(stream)));
}

int ufp4_layer_norm_bwd_workspace(int dtype, int64_t rows, int64_t cols, size_t* bytes) {
    if (!known(dtype) || rows < 0 || cols < 0 || !bytes) return UFP4_ERR_INVALID_ARG;
    if (cols > kMostCols) return UFP4_ERR_UNSUPPORTED;
    *bytes = rows == 0 || cols == 0 ? 0 : (size_t)norm_bwd_parts(dtype == UFP4_OUT_BF16, rows, cols) * 2 * cols * sizeof(float);
    return UFP4_OK;
}

int ufp4_layer_norm_bwd(int dtype, const void* dy_dev, int64_t lddy, const void* x_dev, int64_t rows, int64_t cols,
                        int64_t ldx, int w_dtype, const void* gamma_dev, const float* mean_dev, const float* rstd_dev,
                        void* dx_dev, int64_t lddx, float* dgamma_dev, float* dbeta_dev, void* workspace_dev,
                        size_t workspace_bytes, void* stream) {
    if (!known(dtype) || !known(w_dtype) || rows < 0 || cols < 0) return UFP4_ERR_INVALID_ARG;
    const int st = first(first(check_rows(dtype, dy_dev, rows, cols, lddy), check_rows(dtype, x_dev, rows, cols, ldx)),
                         check_rows(dtype, dx_dev, rows, cols, lddx));
    if (st != UFP4_OK) return st;
    if (cols > kMostCols) return UFP4_ERR_UNSUPPORTED;
    const bool some = rows > 0 && cols > 0, weights = dgamma_dev || dbeta_dev;
    if (some && (!mean_dev || !rstd_dev)) return UFP4_ERR_INVALID_ARG;
    if (!aligned(gamma_dev, size_of(w_dtype)) || !aligned(mean_dev, 4) || !aligned(rstd_dev, 4) || !aligned(dgamma_dev, 4) ||
        !aligned(dbeta_dev, 4))
        return UFP4_ERR_ALIGN;
    if (some && weights) {
        size_t need = 0;
        ufp4_layer_norm_bwd_workspace(dtype, rows, cols, &need);
        if (!workspace_dev) return UFP4_ERR_INVALID_ARG;
        if (workspace_bytes < need) return UFP4_ERR_SHAPE;
        if (!aligned(workspace_dev, 16)) return UFP4_ERR_ALIGN;
    }
    if (cols == 0 || (rows == 0 && !weights)) return UFP4_OK;
    const NormBwdJob j{dtype == UFP4_OUT_BF16, w_dtype == UFP4_OUT_BF16, dy_dev, x_dev, rows, cols, lddy, ldx, gamma_dev,
                       mean_dev, rstd_dev, dx_dev, lddx, dgamma_dev, dbeta_dev,
                       some && weights ? static_cast<float*>(workspace_dev) : nullptr};
    return status_of(launch_norm_bwd(j, static_cast<hipStream_t>(stream)));
}

int ufp4_moe_sort_workspace(int64_t tokens, int32_t k, int32_t experts, size_t* bytes) {
    if (tokens < 0 || k < 1 || experts < 1 || !bytes) return UFP4_ERR_INVALID_ARG;
    if (k > kMoeMaxK || experts > kMoeMaxExperts || tokens > INT32_MAX / k) return UFP4_ERR_UNSUPPORTED;
    const int64_t runs = moe_sort_runs(tokens * k);
    *bytes = runs > 1 ? (size_t)(runs + 1) * experts * sizeof(int32_t) : 0;
    return UFP4_OK;
}

int ufp4_moe_sort(const void* ids_dev, int ids_bits, int64_t tokens, int32_t k, int32_t experts, int64_t* offsets_dev,
                  int32_t* rows_dev, int32_t* source_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    const int st = ufp4_moe_sort_workspace(tokens, k, experts, &need);
    if (st != UFP4_OK) return st;
    if (ids_bits != 32 && ids_bits != 64) return UFP4_ERR_INVALID_ARG;
    if (!offsets_dev || (tokens > 0 && (!ids_dev || !rows_dev)) || (need && !workspace_dev)) return UFP4_ERR_INVALID_ARG;
    if (workspace_bytes < need) return UFP4_ERR_SHAPE;
    if (!aligned(ids_dev, ids_bits / 8) || !aligned(offsets_dev, 8) || !aligned(rows_dev, 4) || !aligned(source_dev, 4) ||
        !aligned(workspace_dev, 4))
        return UFP4_ERR_ALIGN;
    const MoeSortJob j{ids_dev, ids_bits == 64, tokens * k, experts, offsets_dev, rows_dev, source_dev,
                       static_cast<int32_t*>(workspace_dev), moe_sort_runs(tokens * k)};
    return status_of(launch_moe_sort(j, static_cast<hipStream_t>(stream)));
}

}  // extern "C"

namespace {

// Limits of the row kernels: 2^32 threads per grid dimension at 256 threads for 4 segments of at least 1024 elements, or for
// one token.
constexpr int64_t kMostTokens = (int64_t(1) << 24) - 1;

int check_moe(int dtype, int64_t tokens, int64_t cols, int32_t k, const int32_t* rows, int64_t y_rows, const float* w) {
    if (!known(dtype) || tokens < 0 || cols < 0 || k < 1 || y_rows < 0) return UFP4_ERR_INVALID_ARG;
    if (tokens > 0 && !rows) return UFP4_ERR_INVALID_ARG;
    if (!aligned(rows, 4) || !aligned(w, 4)) return UFP4_ERR_ALIGN;
    if (k > kMoeMaxK || cols > kMostCols || y_rows > INT32_MAX || tokens > kMostTokens) return UFP4_ERR_UNSUPPORTED;
    if (tokens > 0 && tokens * ((cols + 1023) / 1024) > 4 * kMostTokens) return UFP4_ERR_UNSUPPORTED;
    return UFP4_OK;
}

}  // namespace

extern "C" {

int ufp4_moe_dispatch(int dtype, const void* x_dev, int64_t tokens, int64_t cols, int64_t ldx, const int32_t* rows_dev,
                      int32_t k, const int64_t* offsets_dev, int32_t experts, const float* weights_dev, void* y_dev,
                      int64_t y_rows, int64_t ldy, void* stream) {
    const int st = first(first(check_moe(dtype, tokens, cols, k, rows_dev, y_rows, weights_dev),
                               check_rows(dtype, x_dev, tokens, cols, ldx)), check_rows(dtype, y_dev, y_rows, cols, ldy));
    if (st != UFP4_OK) return st;
    if (experts < 1 || !offsets_dev) return UFP4_ERR_INVALID_ARG;
    if (!aligned(offsets_dev, 8)) return UFP4_ERR_ALIGN;
    if (y_rows != tokens * k) return UFP4_ERR_SHAPE;
    if (tokens == 0 || cols == 0) return UFP4_OK;
    const MoeRowsJob j{dtype == UFP4_OUT_BF16, x_dev, ldx, y_dev, ldy, tokens, cols, y_rows, k, experts, rows_dev, offsets_dev,
                       weights_dev, 0};
    return status_of(launch_moe_dispatch(j, static_cast<hipStream_t>(stream)));
}

int ufp4_moe_combine(int dtype, const void* y_dev, int64_t y_rows, int64_t cols, int64_t ldy, const int32_t* rows_dev,
                     int64_t tokens, int32_t k, const float* weights_dev, void* out_dev, int64_t ldo, void* stream) {
    const int st = first(first(check_moe(dtype, tokens, cols, k, rows_dev, y_rows, weights_dev),
                               check_rows(dtype, y_dev, y_rows, cols, ldy)), check_rows(dtype, out_dev, tokens, cols, ldo));
    if (st != UFP4_OK) return st;
    if (tokens == 0 || cols == 0) return UFP4_OK;
    const MoeRowsJob j{dtype == UFP4_OUT_BF16, y_dev, ldy, out_dev, ldo, tokens, cols, y_rows, k, 0, rows_dev, nullptr,
                       weights_dev, 0};
    return status_of(launch_moe_combine(j, static_cast<hipStream_t>(stream)));
}

int ufp4_moe_combine_bwd(int dtype, const void* dout_dev, int64_t tokens, int64_t cols, int64_t lddo, const void* y_dev,
                         int64_t y_rows, int64_t ldy, const int32_t* rows_dev, int32_t k, const int64_t* offsets_dev,
                         int32_t experts, const float* weights_dev, void* dy_dev, int64_t lddy, float* dweights_dev,
                         void* stream) {
    const int st = first(first(check_moe(dtype, tokens, cols, k, rows_dev, y_rows, weights_dev),
                               check_rows(dtype, dout_dev, tokens, cols, lddo)),
                         first(check_rows(dtype, y_dev, y_rows, cols, ldy), check_rows(dtype, dy_dev, y_rows, cols, lddy)));
    if (st != UFP4_OK) return st;
    if (experts < 1 || !offsets_dev || (tokens > 0 && !dweights_dev)) return UFP4_ERR_INVALID_ARG;
    if (!aligned(offsets_dev, 8) || !aligned(dweights_dev, 4)) return UFP4_ERR_ALIGN;
    if (y_rows != tokens * k) return UFP4_ERR_SHAPE;
    if (tokens == 0) return UFP4_OK;
    const MoeBwdJob j{dtype == UFP4_OUT_BF16, dout_dev, y_dev, lddo, ldy, dy_dev, lddy, tokens, cols, y_rows, k, experts,
                      rows_dev, offsets_dev, weights_dev, dweights_dev};
    return status_of(launch_moe_combine_bwd(j, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
