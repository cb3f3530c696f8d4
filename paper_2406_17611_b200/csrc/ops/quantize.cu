// 8-bit operands of the product: e4m3 values and 32-bit scales.
//
//   rows     one scale for every row and 128 columns (activations, gradients):  s = max|x| (1/448), q = e4m3(x (1/s))
//   weight   one scale for every 128 x 128 block, and both layouts of the bytes: the product contracts over the last
//            index of both operands, so the forward reads W and the backward W transposed, each with the same scales
//
// Bound: HBM (rows: one pass, the next row's loads under the arithmetic; weight: a 128 x 128 block in registers, its
// transposed bytes through shared memory).  2.45M x 256 bf16: 390 us (4.8 TB/s); 4096 x 4096, both layouts:
// fp32 24 us (4.2 TB/s), bf16 27 (2.5: loads of single elements).
#include "ops_common.cuh"

namespace {

using namespace vops;

// 16 lanes (bf16) or a warp (fp32) walk down one 128-column block of the rows.
template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T *__restrict__ X, int64_t ldx, int64_t rows, int F,
                                                            uint8_t *__restrict__ Y8, int64_t ld8, float *__restrict__ scales,
                                                            int64_t lds) {
  constexpr int V = ElemTraits<T>::kVec, LANES = kBlock / V, GROUPS = 256 / LANES, R = 4;   // R rows on their way
  const int lane = threadIdx.x % LANES, b = blockIdx.y, c = b * LANES + lane;
  const bool col = c * V < F;
  const int chunks = chunks_of_eight<V>(F);
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  // groups of one CTA take the same number of trips: those past the last row stay for the shuffles
  for (int64_t row0 = (int64_t)blockIdx.x * GROUPS; row0 < rows; row0 += step * R) {
    const int64_t first = row0 + threadIdx.x / LANES;
    uint4 v[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      v[q] = make_uint4(0u, 0u, 0u, 0u);
      if (col && first + q * step < rows) v[q] = load_stream(reinterpret_cast<const uint4 *>(X + (first + q * step) * ldx) + c);
    }
    float f[R][V];
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < R; ++q) {
      unpack16(v[q], f[q], T());
      clear_padding<V>(f[q], c, F);
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) m = max(m, abs_bits(f[q][j]));
      m = lanes_max<LANES>(m);
      if (lane % R == q) top = m;
    }
    // lane q makes and stores row q's scale, so that its two quotients are taken once for the R rows
    const Scale s = block_scale(top);
    if (lane < R && first + lane * step < rows) scales[(int64_t)b * lds + first + lane * step] = s.s;
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const float inv = __shfl_sync(0xFFFFFFFFu, s.inv, q, LANES);
      if (c < chunks && first + q * step < rows) store_e4m3(Y8 + (first + q * step) * ld8 + (int64_t)c * V, f[q], inv);
    }
  }
}

// One CTA per 128 x 128 block: a thread holds four neighbouring columns of 16 rows.  `end` and `endt`: columns of W8 and of the
// transposed bytes with their padding, multiples of 16.
template <typename T>
__global__ void __launch_bounds__(256) quantize_weight_kernel(const T *__restrict__ W, int64_t ldw, int R, int C,
                                                              uint8_t *__restrict__ W8, int64_t ld8, int64_t end,
                                                              uint8_t *__restrict__ T8, int64_t ldt8, int64_t endt, float *__restrict__ scales, int64_t lds) {
  __shared__ uint32_t tile[kBlock][kBlock / 4 + 1];
  __shared__ uint32_t amax[8];
  const int r0 = blockIdx.y * kBlock, c0 = blockIdx.x * kBlock;
  const int x = threadIdx.x % 32, y = threadIdx.x / 32;
  float f[16][4];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = r0 + y + 8 * i;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = c0 + 4 * x + j;
      f[i][j] = r < R && c < C ? ElemTraits<T>::to_f(W[(int64_t)r * ldw + c]) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max(m, abs_bits(f[i][j]));
  m = lanes_max<32>(m);
  if (x == 0) amax[y] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) m = max(m, amax[w]);
  const Scale s = block_scale(m);
  if (threadIdx.x == 0) scales[(int64_t)blockIdx.y * lds + blockIdx.x] = s.s;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = r0 + y + 8 * i;
    const uint32_t q = pack_e4m3x4_scaled(f[i], s.inv);
    tile[y + 8 * i][x] = q;
    // a group of four bytes is inside or outside as a whole
    if (W8 && r < R && c0 + 4 * x < end) *reinterpret_cast<uint32_t *>(W8 + (int64_t)r * ld8 + c0 + 4 * x) = q;
  }
  __syncthreads();
  if (T8) {
    const uint8_t *bytes = reinterpret_cast<const uint8_t *>(tile);
    constexpr int LD = (kBlock / 4 + 1) * 4;
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int c = y + 8 * i;           // column of the block, row of the transposed matrix
      if (c0 + c < C && r0 + 4 * x < endt) {
        uint32_t q = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) q |= (uint32_t)bytes[(4 * x + j) * LD + c] << (8 * j);
        *reinterpret_cast<uint32_t *>(T8 + (int64_t)(c0 + c) * ldt8 + r0 + 4 * x) = q;
      }
    }
  }
}

}  // namespace

extern "C" {

int varco_quantize_rows(int64_t rows, int32_t F, varco_dtype_t dtype, const void *X, int64_t ldx, void *Y8, int64_t ld8,
                        float *scales, int64_t lds, void *stream) {
  if (rows < 0 || F < 1 || !dtype_ok(dtype)) return VARCO_INVALID_ARG;
  if (rows == 0) return VARCO_OK;
  if (!matrix_ok(X, ldx, F, elem_size(dtype)) || !matrix_ok(Y8, ld8, F, 1) || !scales || lds < rows) return VARCO_INVALID_ARG;
  const int64_t blocks = ((int64_t)F + kBlock - 1) / kBlock;
  if (blocks > 65535) return VARCO_UNSUPPORTED;
  const int sms = sm_count();
  if (sms <= 0) return VARCO_CUDA;
  const int groups = dtype == VARCO_F32 ? 8 : 16;
  const int64_t ctas = (rows + groups - 1) / groups, most = ((int64_t)sms * 8 + blocks - 1) / blocks;
  const dim3 grid((unsigned)(ctas < most ? ctas : most), (unsigned)blocks);
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == VARCO_F32)
    quantize_rows_kernel<float><<<grid, 256, 0, st>>>((const float *)X, ldx, rows, F, (uint8_t *)Y8, ld8, scales, lds);
  else
    quantize_rows_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>((const __nv_bfloat16 *)X, ldx, rows, F, (uint8_t *)Y8, ld8, scales, lds);
  VARCO_KERNEL_LAUNCHED();
  return VARCO_OK;
}

int varco_quantize_weight(int32_t rows, int32_t cols, varco_dtype_t dtype, const void *W, int64_t ldw, void *W8, int64_t ld8,
                          void *WT8, int64_t ldt8, float *scales, int64_t lds, void *stream) {
  if (rows < 1 || cols < 1 || !dtype_ok(dtype) || !W || ldw < cols || (!W8 && !WT8) || !scales) return VARCO_INVALID_ARG;
  const int64_t across = ((int64_t)cols + kBlock - 1) / kBlock, down = ((int64_t)rows + kBlock - 1) / kBlock;
  if ((W8 && !matrix_ok(W8, ld8, cols, 1)) || (WT8 && !matrix_ok(WT8, ldt8, rows, 1)) || lds < across) return VARCO_INVALID_ARG;
  if (down > 65535 || cols > INT32_MAX - kBlock) return VARCO_UNSUPPORTED;
  const dim3 grid((unsigned)across, (unsigned)down);
  cudaStream_t st = (cudaStream_t)stream;
  const int64_t end = round_up64(cols, 16), endt = round_up64(rows, 16);
  if (dtype == VARCO_F32)
    quantize_weight_kernel<float><<<grid, 256, 0, st>>>((const float *)W, ldw, rows, cols, (uint8_t *)W8, ld8, end, (uint8_t *)WT8, ldt8, endt, scales, lds);
  else
    quantize_weight_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>((const __nv_bfloat16 *)W, ldw, rows, cols, (uint8_t *)W8, ld8, end, (uint8_t *)WT8, ldt8, endt, scales, lds);
  VARCO_KERNEL_LAUNCHED();
  return VARCO_OK;
}

}  // extern "C"
