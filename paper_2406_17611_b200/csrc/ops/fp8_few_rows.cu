// The 8-bit product for at most 32 rows (a few nodes asked for at inference time): bound by reading B once.
//
// A 128-row tile would multiply empty rows, which costs nothing, but gives an SM a whole tile's contraction: 1 x 4096 x 4096
// keeps 32 of 148 SMs busy for 15 us, 4.9 here (5.9 with an 8-bit output; 32 rows: 10.8 and 12.2; 1 x 8192 x 256 with both outputs
// 3.4 against 4.9, 32 x 4096 x 1024 4.7 against 6.3).  A CTA owns 16 columns and its eight warps share the contraction, block by
// block; a warp's lanes read 16 bytes of B each (64 contiguous bytes of a row) straight into registers, as the first operand of
// mma.sync m16n8k32: 16 columns of the product x 8 rows of A.  The order of k inside an instruction is free as
// long as both operands agree, so lane l of a row takes bytes 16 l .. 16 l + 15 of it and uses them for two instructions.
// A block's sum is scaled and added in 32 bits, the warps' sums are added in their order.  The 8-bit output needs the
// largest magnitude of 128 columns: eight CTAs of a cluster exchange theirs through distributed shared memory.
#include "ops_common.cuh"
#include "fp8_product.h"

namespace {

using namespace vops;

constexpr int kWarps = 8, kCols = kFewCols;      // of a CTA

struct FewParams {
  const uint8_t *a, *b;
  const float *sa, *sb, *bias;
  const void *mask;
  void *y;
  uint8_t *y8;
  float *sy;
  int64_t lda, ldb, ld_sa, sb_n, sb_k, ldmask, ldy, ldy8, ld_sy;
  int M, N, K, kblocks;
};

__device__ __forceinline__ void mma_e4m3(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes of a row from column k; those from column K on are zero
__device__ __forceinline__ uint4 load_bytes(const uint8_t *row, int k, int K) {
  if (k >= K) return make_uint4(0u, 0u, 0u, 0u);
  uint4 v = __ldg(reinterpret_cast<const uint4 *>(row + k));
  if (k + 16 > K) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = K - k - 4 * i;
      if (n < 4) w[i] = n <= 0 ? 0u : w[i] & ((1u << 8 * n) - 1u);
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}

template <typename T, int TILES, bool QUANT>
__global__ void __launch_bounds__(kWarps * 32, few_rows_ctas(TILES * 8)) few_rows_kernel(const FewParams p, int relu_on) {
  constexpr int ROWS = TILES * 8;          // of A
  __shared__ float part[kWarps][ROWS][kCols + 1];
  __shared__ uint32_t amax[8][ROWS];       // of the cluster's CTAs
  // Another CTA's shared memory may be written once that CTA has started: each says so here, and who writes waits for all eight
  // behind its contraction.
  if constexpr (QUANT) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, l = lane % 4;
  const int n0 = blockIdx.x * kCols;
  const uint8_t *b0 = p.b + (int64_t)min(n0 + g, p.N - 1) * p.ldb, *b1 = p.b + (int64_t)min(n0 + g + 8, p.N - 1) * p.ldb;
  const float *sb = p.sb + (int64_t)(min(n0, p.N - 1) / kBlock) * p.sb_n;
  const uint8_t *a[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) a[t] = p.a + (int64_t)min(t * 8 + g, p.M - 1) * p.lda;
  float sum[TILES][4] = {};
  for (int kb = warp; kb < p.kblocks; kb += kWarps) {
    uint4 w0[2], w1[2], x[2][TILES];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = kb * kBlock + h * 64 + l * 16;
      w0[h] = load_bytes(b0, k, p.K);
      w1[h] = load_bytes(b1, k, p.K);
#pragma unroll
      for (int t = 0; t < TILES; ++t) x[h][t] = load_bytes(a[t], k, p.K);
    }
    const float s = __ldg(sb + (int64_t)kb * p.sb_k);
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      // the accumulator's columns are rows t * 8 + 2 l and + 1 of A
      const int m = t * 8 + 2 * l;
      const float s0 = s * __ldg(p.sa + (int64_t)kb * p.ld_sa + min(m, p.M - 1)), s1 = s * __ldg(p.sa + (int64_t)kb * p.ld_sa + min(m + 1, p.M - 1));
      float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        mma_e4m3(c, w0[h].x, w1[h].x, w0[h].y, w1[h].y, x[h][t].x, x[h][t].y);
        mma_e4m3(c, w0[h].z, w1[h].z, w0[h].w, w1[h].w, x[h][t].z, x[h][t].w);
      }
      sum[t][0] = fmaf(s0, c[0], sum[t][0]);
      sum[t][1] = fmaf(s1, c[1], sum[t][1]);
      sum[t][2] = fmaf(s0, c[2], sum[t][2]);
      sum[t][3] = fmaf(s1, c[3], sum[t][3]);
    }
  }
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    part[warp][t * 8 + 2 * l][g] = sum[t][0];
    part[warp][t * 8 + 2 * l + 1][g] = sum[t][1];
    part[warp][t * 8 + 2 * l][g + 8] = sum[t][2];
    part[warp][t * 8 + 2 * l + 1][g + 8] = sum[t][3];
  }
  __syncthreads();
  // 16 lanes a row of A, one column each
  constexpr int PER = (ROWS * kCols + kWarps * 32 - 1) / (kWarps * 32);
  float v[PER];
  const int c = threadIdx.x % kCols, n = n0 + c;
  constexpr int V = ElemTraits<T>::kVec;
  const int end = (p.N + V - 1) / V * V, end8 = (p.N + 15) / 16 * 16;     // columns with their padding, which becomes zero
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int m = threadIdx.x / kCols + i * (kWarps * 32 / kCols);
    float r = 0.f;
    if (m < ROWS) {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) r += part[w][m][c];
    }
    const bool here = m < p.M && n < p.N;
    if (!here) r = 0.f;
    if (here && p.bias) r += p.bias[n];
    if (relu_on) r = relu(r);
    if (here && p.mask) r = ElemTraits<T>::to_f(((const T *)p.mask)[(int64_t)m * p.ldmask + n]) > 0.f ? r : 0.f;
    if (m < p.M && n < end && p.y) ((T *)p.y)[(int64_t)m * p.ldy + n] = ElemTraits<T>::from_f(r);
    v[i] = r;
  }
  if constexpr (QUANT) {
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // pairs with the arrival at the start
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int m = threadIdx.x / kCols + i * (kWarps * 32 / kCols);
      const uint32_t top = lanes_max<kCols>(abs_bits(v[i]));
      if (m < ROWS && c < 8) {             // lane c of the row tells CTA c
        uint32_t to;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(&amax[rank][m])), "r"(c));
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(top) : "memory");
      }
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int m = threadIdx.x / kCols + i * (kWarps * 32 / kCols);
      if (m < p.M && m < ROWS && n < end8) {
        uint32_t top = 0;
#pragma unroll
        for (int r = 0; r < 8; ++r) top = max(top, amax[r][m]);
        const Scale s = block_scale(top);
        p.y8[(int64_t)m * p.ldy8 + n] = n < p.N ? (uint8_t)pack_e4m3x2(v[i] * s.inv, 0.f) : (uint8_t)0;
        if (rank == 0 && c == 0) p.sy[(int64_t)(n / kBlock) * p.ld_sy + m] = s.s;
      }
    }
  }
}

template <typename T, int TILES> int launch(const FewParams &p, int relu_on, cudaStream_t st) {
  const int ctas = (p.N + kCols - 1) / kCols;
  if (!p.y8) {
    few_rows_kernel<T, TILES, false><<<ctas, kWarps * 32, 0, st>>>(p, relu_on);
  } else {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((ctas + 7) / 8 * 8);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.stream = st;
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = 8, cluster.val.clusterDim.y = 1, cluster.val.clusterDim.z = 1;
    cfg.attrs = &cluster;
    cfg.numAttrs = 1;
    VARCO_CUDA_CHECK(cudaLaunchKernelEx(&cfg, few_rows_kernel<T, TILES, true>, p, relu_on));
  }
  VARCO_KERNEL_LAUNCHED();
  return VARCO_OK;
}

template <typename T> int dispatch(const FewParams &p, int relu_on, cudaStream_t st) {
  if (p.M <= 8) return launch<T, 1>(p, relu_on, st);
  if (p.M <= 16) return launch<T, 2>(p, relu_on, st);
  if (p.M <= 24) return launch<T, 3>(p, relu_on, st);
  return launch<T, 4>(p, relu_on, st);
}

}  // namespace

int varco_launch_fp8_few_rows(const varco_fp8_desc_t *d, const void *A8, const float *sA, const void *B8, const float *sB, const float *bias,
                              const void *mask, void *Y, void *Y8, float *sY, cudaStream_t st) {
  FewParams p;
  p.a = (const uint8_t *)A8, p.b = (const uint8_t *)B8, p.sa = sA, p.sb = sB, p.bias = bias, p.mask = mask, p.y = Y, p.y8 = (uint8_t *)Y8, p.sy = sY;
  p.lda = d->lda, p.ldb = d->ldb, p.ld_sa = d->ld_sa, p.sb_n = d->sb_n, p.sb_k = d->sb_k, p.ldmask = d->ldmask, p.ldy = d->ldy, p.ldy8 = d->ldy8,
  p.ld_sy = d->ld_sy;
  p.M = (int)d->M, p.N = d->N, p.K = d->K, p.kblocks = (d->K + kBlock - 1) / kBlock;
  return d->dtype == VARCO_F32 ? dispatch<float>(p, d->relu != 0, st) : dispatch<__nv_bfloat16>(p, d->relu != 0, st);
}
