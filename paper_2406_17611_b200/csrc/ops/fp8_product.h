// The two forms of the 8-bit product behind varco_fp8_product (internal).
#ifndef VARCO_FP8_PRODUCT_H_
#define VARCO_FP8_PRODUCT_H_

#include <cuda_runtime.h>

#include "varco.h"

// Few rows take the form without tiles while its CTAs of 16 columns all run at once, four an SM with 8 rows, two with more
// (whose registers fill the SM): 8 x 9472 x 1024 3.5 against 7.6 us, 16 x 4736 x 4096 6.7 against 15, 32 x 4736 x 1024 4.7 against
// 6.4.  Beyond, every CTA reads A again and the tiles win: 32 x 6144 x 256 5.5 against 4.2, x 4096 20 against 15.
// With an 8-bit output the CTAs come in clusters of eight, which do not fill every SM: 7/8 of them are sure to run at once (8 rows:
// 8960 columns do, 9472 do not, 5.1 against 4.4 us for K = 128; 32 rows: 4096 do, 12.4 against 15.3 for K = 4096, 4480 do not, 21.2
// against 15.3).
// Only 8 rows pay for a second round: without an 8-bit output at any length (8 x 10,000 x 256 3.3 against 4.6, 18,000 x 256 3.8
// against 4.8), with one from K = 1024 (18,000 x 768 8.2 against 7.5, x 1024 8.4 against 9.7).
// With 48 rows the registers of a CTA fill an SM alone: 48 x 4096 x 1024 14.0 against 7.5.
constexpr int kFewRows = 32, kFewCols = 16;
constexpr int few_rows_ctas(int rows) { return rows <= 8 ? 4 : 2; }   // of an SM
constexpr bool few_rows_pay(int64_t M, int64_t N, int64_t K, bool quantize, int sms) {
  const int64_t ctas = (N + kFewCols - 1) / kFewCols, once = (int64_t)sms * few_rows_ctas((int)M);
  return M <= kFewRows && ctas <= (M <= 8 && (!quantize || K >= 1024) ? 2 * once : quantize ? once * 7 / 8 : once);
}
// at most kFewRows rows; arguments already checked
int varco_launch_fp8_few_rows(const varco_fp8_desc_t *d, const void *A8, const float *sA, const void *B8, const float *sB, const float *bias,
                              const void *mask, void *Y, void *Y8, float *sY, cudaStream_t st);

#endif  // VARCO_FP8_PRODUCT_H_
