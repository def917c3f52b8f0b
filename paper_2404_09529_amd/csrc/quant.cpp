// The 8-bit integer projections' entry points: argument checks, then one launch (or two) on the
// caller's stream.  Host side only.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "kernels.h"
#include "prepack.h"
#include "status.h"

namespace {

constexpr size_t kAlign = 256;
constexpr int32_t kMaxK = 131056;          // 2^31 / 128^2, down to a multiple of 16
constexpr int32_t kMaxRows = INT32_MAX - 511;   // a row index past the last tile's end stays a 32-bit number
constexpr int64_t kMaxLd = 8388592;        // 256 rows of a tile lie within a 31-bit byte offset

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }

pp_status finish(const char* what) {
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return pp::fail(PP_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(err));
    return PP_OK;
}

}  // namespace

namespace {

// The checks pp_quantize_rows and pp_dequantize_rows share; *done: there is nothing to do.
pp_status check_rows(int32_t dtype, const void* x, int64_t ldx, int32_t rows, int32_t d, const void* q, int64_t ldq,
                     const void* scale, bool* done) {
    *done = false;
    if (dtype != PP_F32 && dtype != PP_BF16) return pp::fail(PP_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (rows < 0 || d <= 0) return pp::fail(PP_ERR_INVALID_ARG, "rows %d, d %d", rows, d);
    if (ldx < d || ldq < d)
        return pp::fail(PP_ERR_INVALID_ARG, "row strides %lld, %lld below d = %d", (long long)ldx, (long long)ldq, d);
    if (d % 16 || ldx % 16 || ldq % 16)
        return pp::fail(PP_ERR_UNSUPPORTED, "d %d, ldx %lld and ldq %lld must be multiples of 16", d, (long long)ldx,
                        (long long)ldq);
    *done = rows == 0;
    if (*done) return PP_OK;
    if (!x || !q || !scale) return pp::fail(PP_ERR_INVALID_ARG, "NULL buffer");
    if (misaligned(x) || misaligned(q)) return pp::fail(PP_ERR_UNSUPPORTED, "x and q must be 16-byte aligned");
    return PP_OK;
}

}  // namespace

extern "C" pp_status pp_quantize_rows(int32_t dtype, const void* x, int64_t ldx, int32_t rows, int32_t d, int8_t* q,
                                      int64_t ldq, float* scale, void* stream) {
    pp::clear_error();
    bool done;
    if (pp_status st = check_rows(dtype, x, ldx, rows, d, q, ldq, scale, &done)) return st;
    if (done) return PP_OK;
    (void)hipGetLastError();
    ppk::quantize_rows(dtype, x, ldx, rows, d, q, ldq, scale, static_cast<hipStream_t>(stream));
    return finish("quantize_rows");
}

extern "C" pp_status pp_dequantize_rows(int32_t dtype, const int8_t* q, int64_t ldq, const float* scale, int32_t rows,
                                        int32_t d, void* x, int64_t ldx, void* stream) {
    pp::clear_error();
    bool done;
    if (pp_status st = check_rows(dtype, x, ldx, rows, d, q, ldq, scale, &done)) return st;
    if (done) return PP_OK;
    (void)hipGetLastError();
    ppk::dequantize_rows(dtype, q, ldq, scale, rows, d, x, ldx, static_cast<hipStream_t>(stream));
    return finish("dequantize_rows");
}

extern "C" pp_status pp_rmsnorm_quant(int32_t dtype, float* x, const void* add, const float* gain, int32_t rows,
                                      int32_t d, float eps, int8_t* q, float* scale, void* stream) {
    pp::clear_error();
    if (dtype != PP_F32 && dtype != PP_BF16) return pp::fail(PP_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (rows < 0 || d <= 0) return pp::fail(PP_ERR_INVALID_ARG, "rows %d, d %d", rows, d);
    if (!(eps >= 0.f)) return pp::fail(PP_ERR_INVALID_ARG, "eps must be >= 0");
    if (d % 16) return pp::fail(PP_ERR_UNSUPPORTED, "d = %d must be a multiple of 16", d);
    if (rows == 0) return PP_OK;
    if (!x || !gain || !q || !scale) return pp::fail(PP_ERR_INVALID_ARG, "NULL buffer");
    if (misaligned(x) || misaligned(add) || misaligned(gain) || misaligned(q))
        return pp::fail(PP_ERR_UNSUPPORTED, "x, add, gain and q must be 16-byte aligned");
    (void)hipGetLastError();
    ppk::rmsnorm_quant(dtype, x, add, gain, rows, d, eps, q, scale, static_cast<hipStream_t>(stream));
    return finish("rmsnorm_quant");
}

extern "C" pp_status pp_gemm_quant_workspace_size(int32_t M, int32_t N, int32_t K, size_t* bytes) {
    pp::clear_error();
    if (M < 0 || N <= 0 || K <= 0) return pp::fail(PP_ERR_INVALID_ARG, "M %d, N %d, K %d", M, N, K);
    if (!bytes) return pp::fail(PP_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = ppk::quant_gemm_workspace(M, N, K);
    return PP_OK;
}

extern "C" pp_status pp_gemm_quant(int32_t dtype, int32_t epilogue, const int8_t* A, int64_t lda,
                                   const float* a_scale, const int8_t* B, int64_t ldb, const float* b_scale, void* C,
                                   int64_t ldc, int32_t M, int32_t N, int32_t K, const pp_dplan* plan,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    pp::clear_error();
    if (dtype != PP_F32 && dtype != PP_BF16) return pp::fail(PP_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (epilogue < PP_EPI_STORE || epilogue > PP_EPI_SWIGLU)
        return pp::fail(PP_ERR_INVALID_ARG, "unknown epilogue %d", epilogue);
    if (M < 0 || N <= 0 || K <= 0) return pp::fail(PP_ERR_INVALID_ARG, "M %d, N %d, K %d", M, N, K);
    const bool swiglu = epilogue == PP_EPI_SWIGLU;
    if (lda < K || ldb < K || ldc < (swiglu ? N / 2 : N))
        return pp::fail(PP_ERR_INVALID_ARG, "leading dimensions too small (lda %lld ldb %lld ldc %lld)",
                        (long long)lda, (long long)ldb, (long long)ldc);
    if (K % 16 || K > kMaxK || N % (swiglu ? 32 : 16))
        return pp::fail(PP_ERR_UNSUPPORTED, "8-bit GEMM needs K %% 16 == 0, K <= %d, N %% %d == 0 (N %d K %d)", kMaxK,
                        swiglu ? 32 : 16, N, K);
    if (M > kMaxRows || N > kMaxRows) return pp::fail(PP_ERR_UNSUPPORTED, "M %d or N %d above %d", M, N, kMaxRows);
    if (lda % 16 || ldb % 16 || lda > kMaxLd || ldb > kMaxLd || ldc % 4)
        return pp::fail(PP_ERR_UNSUPPORTED, "8-bit GEMM needs lda, ldb %% 16 == 0 up to %lld and ldc %% 4 == 0 "
                        "(lda %lld ldb %lld ldc %lld)", (long long)kMaxLd, (long long)lda, (long long)ldb, (long long)ldc);
    if (plan) {
        if (pp_status st = pp::validate_plan(plan)) return st;
        if (int64_t(M) != int64_t(plan->n_rows) * plan->capacity)
            return pp::fail(PP_ERR_INVALID_ARG, "M %d != n_rows * capacity of the plan", M);
        if (M > 0 && !plan->mtile_m0) return pp::fail(PP_ERR_INVALID_ARG, "plan mtile_m0 is NULL");
    }
    if (M == 0 || (plan && plan->n_mtiles == 0)) return PP_OK;
    if (!A || !a_scale || !B || !b_scale || !C) return pp::fail(PP_ERR_INVALID_ARG, "NULL buffer");
    if (misaligned(A) || misaligned(B) || misaligned(C))
        return pp::fail(PP_ERR_UNSUPPORTED, "A, B and C must be 16-byte aligned");
    const size_t need = ppk::quant_gemm_workspace(M, N, K);
    if (need) {
        if (!workspace) return pp::fail(PP_ERR_INVALID_ARG, "workspace is NULL");
        if (reinterpret_cast<uintptr_t>(workspace) % kAlign)
            return pp::fail(PP_ERR_INVALID_ARG, "workspace is not %zu-byte aligned", kAlign);
        if (workspace_bytes < need)
            return pp::fail(PP_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes < %zu needed", workspace_bytes, need);
    }
    (void)hipGetLastError();
    const int epi = epilogue == PP_EPI_STORE ? ppk::kStore : (swiglu ? ppk::kSwiGLU : ppk::kResidual);
    ppk::quant_gemm(epi, dtype == PP_F32,
                    ppk::QuantGemm{A, lda, a_scale, B, ldb, b_scale, C, ldc, M, N, K, plan ? plan->mtile_m0 : nullptr,
                                   plan ? plan->n_mtiles : 0, static_cast<int32_t*>(workspace)},
                    static_cast<hipStream_t>(stream));
    return finish("gemm_quant");
}
