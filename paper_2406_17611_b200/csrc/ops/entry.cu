// Workspace size of the residual-block operators and the weight gradient reached from outside a layer.
#include <algorithm>

#include "kernels.h"
#include "ops_common.cuh"

namespace {

using namespace vops;

// The layer's weight-gradient kernel takes at most 1024 x 256 outputs: larger ones go in pieces, each reading its columns of
// A and B again (bf16, 2.45M rows, 256 x 1024: 1.78 ms = 0.72 PFLOP/s; 169,343 rows, 256 x 256: 105 us; fp32, without tensor
// cores: 563 us = 39 TFLOP/s).
constexpr int kMaxRows = 1024, kMaxCols = 256;

size_t piece_bytes(int Fa, int Fb) {
  const int r = Fa < kMaxRows ? Fa : kMaxRows, c = Fb < kMaxCols ? Fb : kMaxCols;
  // the column sums of A run in the same scratch, in pieces of kMaxRows columns
  const size_t g = std::max(varco_gemm_scratch_bytes(r, c), varco_simt_dw_scratch_bytes(1, r));
  return (g + 255) / 256 * 256 + (Fb > kMaxCols ? (size_t)r * c * 4 : 0);
}

}  // namespace

extern "C" {

int varco_ops_workspace_bytes(int32_t F_max, size_t *bytes) {
  if (!bytes || F_max < 1) return VARCO_INVALID_ARG;
  if (F_max > 16384) return VARCO_UNSUPPORTED;
  const size_t a = norm_scratch_bytes(F_max), b = clip_scratch_bytes();
  *bytes = 256 + kStatusBytes + (a > b ? a : b);
  return VARCO_OK;
}

int varco_weight_grad_workspace_bytes(int32_t Fa, int32_t Fb, size_t *bytes) {
  if (!bytes || Fa < 1 || Fb < 1) return VARCO_INVALID_ARG;
  *bytes = 256 + kStatusBytes + piece_bytes(Fa, Fb);
  return VARCO_OK;
}

int varco_weight_grad(int64_t rows, int32_t Fa, int32_t Fb, varco_dtype_t dtype, const void *A, int64_t lda, const void *B, int64_t ldb,
                      float *dW, float *dsum, void *workspace, size_t ws_bytes, void *stream) {
  if (rows < 0 || Fa < 1 || Fb < 1 || !dtype_ok(dtype) || !dW || !workspace) return VARCO_INVALID_ARG;
  if (rows > INT32_MAX - 256) return VARCO_UNSUPPORTED;
  if (ws_bytes < 256 + kStatusBytes + piece_bytes(Fa, Fb)) return VARCO_WORKSPACE_TOO_SMALL;
  cudaStream_t st = (cudaStream_t)stream;
  if (rows == 0) {
    VARCO_CUDA_CHECK(cudaMemsetAsync(dW, 0, (size_t)Fa * Fb * 4, st));
    if (dsum) VARCO_CUDA_CHECK(cudaMemsetAsync(dsum, 0, (size_t)Fa * 4, st));
    return VARCO_OK;
  }
  const int es = elem_size(dtype);
  if (!matrix_ok(A, lda, Fa, es) || !matrix_ok(B, ldb, Fb, es)) return VARCO_INVALID_ARG;
  char *ws = ws_align(workspace);
  char *scratch = ws + kStatusBytes;
  if (dsum)
    for (int r0 = 0; r0 < Fa; r0 += kMaxRows) {
      const int r = Fa - r0 < kMaxRows ? Fa - r0 : kMaxRows;
      if (int rc = varco_colsum((int)rows, r, dtype, (const char *)A + (int64_t)r0 * es, lda, dsum + r0, (float *)scratch, st)) return rc;
    }
  for (int c0 = 0; c0 < Fb; c0 += kMaxCols)
    for (int r0 = 0; r0 < Fa; r0 += kMaxRows) {
      const int r = Fa - r0 < kMaxRows ? Fa - r0 : kMaxRows, c = Fb - c0 < kMaxCols ? Fb - c0 : kMaxCols;
      const char *a = (const char *)A + (int64_t)r0 * es, *b = (const char *)B + (int64_t)c0 * es;
      const size_t gemm = (varco_gemm_scratch_bytes(r, c) + 255) / 256 * 256;
      float *out = Fb > kMaxCols ? reinterpret_cast<float *>(scratch + gemm) : dW + (int64_t)r0 * Fb;
      int rc = dtype == VARCO_F32 ? varco_simt_gemm_dw((int)rows, r, c, dtype, a, lda, b, ldb, out, (float *)scratch, st)
                                  : varco_tc_gemm_dw((int)rows, r, c, nullptr, 0, a, lda, b, ldb, nullptr, out, scratch, (int *)ws, st);
      if (rc != VARCO_OK) return rc;
      if (Fb > kMaxCols)
        VARCO_CUDA_CHECK(cudaMemcpy2DAsync(dW + (int64_t)r0 * Fb + c0, (size_t)Fb * 4, out, (size_t)c * 4, (size_t)c * 4, (size_t)r,
                                           cudaMemcpyDeviceToDevice, st));
    }
  return VARCO_OK;
}

}  // extern "C"
