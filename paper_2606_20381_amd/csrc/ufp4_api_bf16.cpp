// C ABI of the grouped products of bf16 rows, of the 8-bit checkpoints and of the activation: argument validation on the host, then the
// launches. Declarations and the meaning of every argument are in include/ufp4.h.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ufp4.h"
#include "ufp4_ckpt8.h"
#include "ufp4_internal.h"

using namespace ufp4;

namespace {

int status_of(hipError_t e) { return e == hipSuccess ? UFP4_OK : UFP4_ERR_HIP; }
bool known(int dtype) { return dtype == UFP4_OUT_F32 || dtype == UFP4_OUT_BF16; }
bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
uintptr_t size_of(int dtype) { return dtype == UFP4_OUT_BF16 ? 2 : 4; }
int first(int a, int b) { return a != UFP4_OK ? a : b; }

constexpr int64_t kMostCols = int64_t(1) << 30;
constexpr int64_t kMostLd = int64_t(1) << 40;  // far above any tensor; keeps products of sizes within 64 bits

// A tensor [rows, cols] of `dtype` at p, rows ld elements apart; without an element it is never accessed.
int check_rows(int dtype, const void* p, int64_t rows, int64_t cols, int64_t ld) {
    if (rows == 0 || cols == 0) return UFP4_OK;
    if (!p) return UFP4_ERR_INVALID_ARG;
    if (ld < cols) return UFP4_ERR_SHAPE;
    if (ld > kMostLd) return UFP4_ERR_UNSUPPORTED;
    return aligned(p, size_of(dtype)) ? UFP4_OK : UFP4_ERR_ALIGN;
}

int64_t blocks_of(int64_t cols) { return (cols + kCkpt8Block - 1) / kCkpt8Block; }

// Codes and scales of [rows, parts * cols].
int check_codes(const uint8_t* codes, int64_t code_ld, const uint8_t* scales, int64_t scale_ld, int64_t rows, int64_t cols, int parts) {
    if (rows == 0 || cols == 0) return UFP4_OK;
    if (!codes || !scales) return UFP4_ERR_INVALID_ARG;
    if (code_ld < parts * blocks_of(cols) * kCkpt8Block || scale_ld < parts * blocks_of(cols)) return UFP4_ERR_SHAPE;
    if (code_ld > kMostLd || scale_ld > kMostLd) return UFP4_ERR_UNSUPPORTED;
    return code_ld % 16 == 0 && aligned(codes, 16) ? UFP4_OK : UFP4_ERR_ALIGN;
}

// A grid holds fewer than 2^32 threads, whole workgroups of 256 of them.
int check_size(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0) return UFP4_ERR_INVALID_ARG;
    if (cols > kMostCols || rows > int64_t(1) << 36 || ckpt8_units(rows, cols) > (int64_t(1) << 32) - 256) return UFP4_ERR_UNSUPPORTED;
    return UFP4_OK;
}

// What the four products share: sizes, offsets and the output [out_rows, out_cols].
int check_gemm(int64_t tokens, int64_t N, int64_t K, const int64_t* offsets, int32_t G, const void* c, int64_t out_rows, int64_t out_cols,
               int64_t ldc, int out_dtype) {
    if (!known(out_dtype) || tokens < 0 || N < 0 || K < 0 || G < 1 || !offsets) return UFP4_ERR_INVALID_ARG;
    if (!aligned(offsets, 8)) return UFP4_ERR_ALIGN;
    if (G > kBf16Groups || tokens > INT32_MAX || N > kMostCols || K > kMostCols) return UFP4_ERR_UNSUPPORTED;
    return check_rows(out_dtype, c, out_rows, out_cols, ldc);
}

int run(const Bf16GemmJob& j, size_t workspace_bytes, void* stream) {
    if (!bf16_gemm_fits(j)) return UFP4_ERR_UNSUPPORTED;
    const size_t need = (size_t)bf16_gemm_workspace(j);
    if (need && !j.counters) return UFP4_ERR_INVALID_ARG;
    if (workspace_bytes < need) return UFP4_ERR_SHAPE;
    if (need && !aligned(j.counters, 4)) return UFP4_ERR_ALIGN;
    return status_of(launch_gemm_bf16(j, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int ufp4_bf16_gemm_grouped_workspace(int pass, int64_t tokens, int64_t N, int64_t K, int32_t G, size_t* bytes) {
    if (pass < UFP4_PASS_FWD_Y || pass > UFP4_PASS_BWD_DW || tokens < 0 || N < 0 || K < 0 || G < 1 || !bytes) return UFP4_ERR_INVALID_ARG;
    if (G > kBf16Groups || tokens > INT32_MAX || N > kMostCols || K > kMostCols) return UFP4_ERR_UNSUPPORTED;
    Bf16GemmJob j{};
    j.pass = pass;
    j.tokens = tokens;
    j.M = pass == UFP4_PASS_BWD_DW ? N : 0;
    j.N = pass == UFP4_PASS_FWD_Y ? N : K;
    j.red = pass == UFP4_PASS_FWD_Y ? K : pass == UFP4_PASS_BWD_DX ? N : 0;
    j.G = G;
    if (!bf16_gemm_fits(j)) return UFP4_ERR_UNSUPPORTED;
    *bytes = (size_t)bf16_gemm_workspace(j);
    return UFP4_OK;
}

int ufp4_bf16_gemm_fwd_y_grouped(const void* x_dev, int64_t tokens, int64_t K, int64_t ldx, const void* w_dev, int64_t N, int64_t ldw,
                                 const int64_t* offsets_dev, int32_t G, void* y_dev, int64_t ldc, int out_dtype, void* workspace_dev, size_t workspace_bytes, void* stream) {
    const int st = first(check_gemm(tokens, N, K, offsets_dev, G, y_dev, tokens, N, ldc, out_dtype),
                         first(check_rows(UFP4_OUT_BF16, x_dev, tokens, K, ldx), check_rows(UFP4_OUT_BF16, w_dev, N, K, ldw)));
    if (st != UFP4_OK) return st;
    if (tokens == 0 || N == 0) return UFP4_OK;
    const Bf16GemmJob j{kBf16FwdY, out_dtype, static_cast<const uint16_t*>(x_dev), ldx, static_cast<const uint16_t*>(w_dev), ldw, nullptr,
                        nullptr, 0, tokens, 0, N, K, y_dev, ldc, offsets_dev, G, static_cast<uint32_t*>(workspace_dev)};
    return run(j, workspace_bytes, stream);
}

int ufp4_bf16_gemm_bwd_dx_grouped(const void* dy_dev, int64_t tokens, int64_t N, int64_t lddy, const void* w_dev, int64_t K, int64_t ldw,
                                  const int64_t* offsets_dev, int32_t G, void* dx_dev, int64_t ldc, int out_dtype, void* workspace_dev, size_t workspace_bytes, void* stream) {
    const int st = first(check_gemm(tokens, N, K, offsets_dev, G, dx_dev, tokens, K, ldc, out_dtype),
                         first(check_rows(UFP4_OUT_BF16, dy_dev, tokens, N, lddy), check_rows(UFP4_OUT_BF16, w_dev, N, K, ldw)));
    if (st != UFP4_OK) return st;
    if (tokens == 0 || K == 0) return UFP4_OK;
    const Bf16GemmJob j{kBf16BwdDx, out_dtype, static_cast<const uint16_t*>(dy_dev), lddy, static_cast<const uint16_t*>(w_dev), ldw, nullptr,
                        nullptr, 0, tokens, 0, K, N, dx_dev, ldc, offsets_dev, G, static_cast<uint32_t*>(workspace_dev)};
    return run(j, workspace_bytes, stream);
}

int ufp4_bf16_gemm_bwd_dw_grouped(const void* dy_dev, int64_t tokens, int64_t N, int64_t lddy, const void* x_dev, int64_t K, int64_t ldx,
                                  const int64_t* offsets_dev, int32_t G, void* dw_dev, int64_t ldc, int out_dtype, void* workspace_dev, size_t workspace_bytes, void* stream) {
    const int st = first(check_gemm(tokens, N, K, offsets_dev, G, dw_dev, N, K, ldc, out_dtype),
                         first(check_rows(UFP4_OUT_BF16, dy_dev, tokens, N, lddy), check_rows(UFP4_OUT_BF16, x_dev, tokens, K, ldx)));
    if (st != UFP4_OK) return st;
    if (N == 0 || K == 0) return UFP4_OK;
    const Bf16GemmJob j{kBf16BwdDw, out_dtype, static_cast<const uint16_t*>(dy_dev), lddy, static_cast<const uint16_t*>(x_dev), ldx, nullptr,
                        nullptr, 0, tokens, N, K, 0, dw_dev, ldc, offsets_dev, G, static_cast<uint32_t*>(workspace_dev)};
    return run(j, workspace_bytes, stream);
}

int ufp4_bf16_gemm_bwd_dw_grouped_ckpt8(const void* dy_dev, int64_t tokens, int64_t N, int64_t lddy, const uint8_t* codes_dev,
                                        int64_t code_ld, const uint8_t* scales_dev, int64_t scale_ld, int64_t K, const int64_t* offsets_dev,
                                        int32_t G, void* dw_dev, int64_t ldc, int out_dtype, void* workspace_dev, size_t workspace_bytes, void* stream) {
    const int st = first(check_gemm(tokens, N, K, offsets_dev, G, dw_dev, N, K, ldc, out_dtype),
                         first(check_rows(UFP4_OUT_BF16, dy_dev, tokens, N, lddy),
                               check_codes(codes_dev, code_ld, scales_dev, scale_ld, tokens, K, 1)));
    if (st != UFP4_OK) return st;
    if (N == 0 || K == 0) return UFP4_OK;
    static const uint8_t none = 0;  // never read: a checkpoint of no tokens may have no codes
    const Bf16GemmJob j{kBf16BwdDw, out_dtype, static_cast<const uint16_t*>(dy_dev), lddy, nullptr, code_ld, codes_dev ? codes_dev : &none,
                        scales_dev, scale_ld, tokens, N, K, 0, dw_dev, ldc, offsets_dev, G, static_cast<uint32_t*>(workspace_dev)};
    return run(j, workspace_bytes, stream);
}

int ufp4_ckpt8_ld(int64_t cols, int parts, int64_t* code_ld, int64_t* scale_ld) {
    if (cols < 0 || parts < 1 || parts > 2) return UFP4_ERR_INVALID_ARG;
    if (cols > kMostCols) return UFP4_ERR_UNSUPPORTED;
    if (code_ld) *code_ld = parts * blocks_of(cols) * kCkpt8Block;
    if (scale_ld) *scale_ld = (parts * blocks_of(cols) + 3) / 4 * 4;
    return UFP4_OK;
}

int ufp4_ckpt8_save(int dtype, const void* x_dev, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes_dev, int64_t code_ld,
                    uint8_t* scales_dev, int64_t scale_ld, void* stream) {
    if (!known(dtype)) return UFP4_ERR_INVALID_ARG;
    const int st = first(check_size(rows, cols), first(check_rows(dtype, x_dev, rows, cols, ldx),
                                                       check_codes(codes_dev, code_ld, scales_dev, scale_ld, rows, cols, 1)));
    if (st != UFP4_OK) return st;
    if (rows == 0 || cols == 0) return UFP4_OK;
    const Ckpt8Job j{dtype == UFP4_OUT_BF16, x_dev, nullptr, ldx, rows, cols, codes_dev, code_ld, scales_dev, scale_ld};
    return status_of(launch_ckpt8_save(j, static_cast<hipStream_t>(stream)));
}

int ufp4_ckpt8_load(int dtype, const uint8_t* codes_dev, int64_t code_ld, const uint8_t* scales_dev, int64_t scale_ld, int64_t rows,
                    int64_t cols, void* y_dev, int64_t ldy, void* stream) {
    if (!known(dtype)) return UFP4_ERR_INVALID_ARG;
    const int st = first(check_size(rows, cols), first(check_rows(dtype, y_dev, rows, cols, ldy),
                                                       check_codes(codes_dev, code_ld, scales_dev, scale_ld, rows, cols, 1)));
    if (st != UFP4_OK) return st;
    if (rows == 0 || cols == 0) return UFP4_OK;
    const Ckpt8Job j{dtype == UFP4_OUT_BF16, nullptr, y_dev, ldy, rows, cols, const_cast<uint8_t*>(codes_dev), code_ld,
                     const_cast<uint8_t*>(scales_dev), scale_ld};
    return status_of(launch_ckpt8_load(j, static_cast<hipStream_t>(stream)));
}

int ufp4_activation(int kind, int dtype, const void* u_dev, int64_t rows, int64_t cols, int64_t ldu, void* a_dev, int64_t lda,
                    uint8_t* codes_dev, int64_t code_ld, uint8_t* scales_dev, int64_t scale_ld, void* stream) {
    if ((kind != UFP4_ACT_RELU2 && kind != UFP4_ACT_SWIGLU) || !known(dtype)) return UFP4_ERR_INVALID_ARG;
    const int parts = kind == UFP4_ACT_SWIGLU ? 2 : 1;
    const int st = first(check_size(rows, cols), first(check_rows(dtype, u_dev, rows, parts * cols, ldu), check_rows(dtype, a_dev, rows, cols, lda)));
    if (st != UFP4_OK) return st;
    if (codes_dev || scales_dev) {
        const int kept = check_codes(codes_dev, code_ld, scales_dev, scale_ld, rows, cols, parts);
        if (kept != UFP4_OK) return kept;
    }
    if (rows == 0 || cols == 0) return UFP4_OK;
    const ActJob j{dtype == UFP4_OUT_BF16, kind, u_dev, ldu, a_dev, lda, nullptr, 0, nullptr, 0, rows, cols, codes_dev, code_ld, scales_dev,
                   scale_ld};
    return status_of(launch_act(j, static_cast<hipStream_t>(stream)));
}

int ufp4_activation_bwd(int kind, int dtype, const void* da_dev, int64_t rows, int64_t cols, int64_t ldda, const void* u_dev, int64_t ldu,
                        const uint8_t* codes_dev, int64_t code_ld, const uint8_t* scales_dev, int64_t scale_ld, void* du_dev,
                        int64_t lddu, void* a_dev, int64_t lda, void* stream) {
    if ((kind != UFP4_ACT_RELU2 && kind != UFP4_ACT_SWIGLU) || !known(dtype)) return UFP4_ERR_INVALID_ARG;
    const int parts = kind == UFP4_ACT_SWIGLU ? 2 : 1;
    const int st = first(first(check_size(rows, cols), check_rows(dtype, da_dev, rows, cols, ldda)),
                         first(check_rows(dtype, du_dev, rows, parts * cols, lddu), a_dev ? check_rows(dtype, a_dev, rows, cols, lda) : UFP4_OK));
    if (st != UFP4_OK) return st;
    if (u_dev && codes_dev) return UFP4_ERR_INVALID_ARG;  // one of them
    const int in = u_dev ? check_rows(dtype, u_dev, rows, parts * cols, ldu)
                         : check_codes(codes_dev, code_ld, scales_dev, scale_ld, rows, cols, parts);
    if (in != UFP4_OK) return in;
    if (rows == 0 || cols == 0) return UFP4_OK;
    const ActJob j{dtype == UFP4_OUT_BF16, kind, u_dev, ldu, a_dev, lda, da_dev, ldda, du_dev, lddu, rows, cols,
                   const_cast<uint8_t*>(codes_dev), code_ld, const_cast<uint8_t*>(scales_dev), scale_ld};
    return status_of(launch_act_bwd(j, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
