// Device-side helpers of the residual-block operators: 8-bit blocks with scales, row teams, 16-byte chunks.
#ifndef VARCO_OPS_COMMON_CUH_
#define VARCO_OPS_COMMON_CUH_

#include "device_common.cuh"

namespace vops {

constexpr int kBlock = 128;               // columns (or rows and columns) that share one scale
constexpr float kTop = 448.f;             // largest e4m3 value
constexpr float kLeastScale = 0x1p-126f;  // a block of zeros or denormals keeps a normal scale

// Scale of a block from the bits of its largest magnitude.  Magnitudes are compared as integers: for non-negative
// floats the order is the same, and a NaN (bits above infinity's) wins, so that a block with a NaN is NaN as a
// whole instead of losing it.  A scale that is not finite multiplies by zero: the block is NaN through its scale, its padding
// stays zero.
// 1/s is rounded to nearest, so that the bytes are the definition's, ties included: the fast quotient (2 ulp) and one Newton step
// with a fused residual (Markstein 1990), exact over all mantissas for the s that occur here, 2^-126 to 2^120.  __frcp_rn, which
// covers every operand, makes the norm's backward 2 % slower (2.45M x 256 bf16: 974 us).
struct Scale {
  float s, inv;
};
__device__ __forceinline__ Scale block_scale(uint32_t amax_bits) {
  Scale r;
  r.s = __uint_as_float(amax_bits) * (1.f / kTop);
  if (r.s < kLeastScale) r.s = kLeastScale;
  const float q = __fdividef(1.f, r.s);
  const float n = fmaf(q, fmaf(-r.s, q, 1.f), q);
  r.inv = r.s <= 0x1p120f ? n : 0.f;
  return r;
}
// max(v, 0) that keeps a NaN
__device__ __forceinline__ float relu(float v) {
  float r;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// two e4m3 values, round to nearest even, saturating; `lo` in the lower byte.  amax * inv may exceed 448 by one
// rounding: saturation makes it 448.
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\t"
      "mov.b32 %0, {l, h};\n\t}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ uint32_t pack_e4m3x4_scaled(float2 a, float2 b, float inv) {
  a = __fmul2_rn(a, make_float2(inv, inv));
  b = __fmul2_rn(b, make_float2(inv, inv));
  return pack_e4m3x4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ uint32_t pack_e4m3x4_scaled(const float *f, float inv) {
  return pack_e4m3x4_scaled(make_float2(f[0], f[1]), make_float2(f[2], f[3]), inv);
}
__device__ __forceinline__ void store_e4m3(uint8_t *p, const float (&f)[4], float inv) {
  *reinterpret_cast<uint32_t *>(p) = pack_e4m3x4_scaled(f, inv);
}
__device__ __forceinline__ void store_e4m3(uint8_t *p, const float (&f)[8], float inv) {
  *reinterpret_cast<uint2 *>(p) = make_uint2(pack_e4m3x4_scaled(f, inv), pack_e4m3x4_scaled(f + 4, inv));
}
// Chunks of V bytes of an 8-bit row with its padding up to 16 bytes: those past the row's own hold zeros.
template <int V> __device__ __forceinline__ int chunks_of_eight(int F) { return (F + 15) / 16 * (16 / V); }

// A row is worked on by a team of TEAM threads: 2 to 32 lanes of a warp, or a whole CTA of TEAM threads.
// Lane `l` holds the 16-byte chunks l, l + TEAM, ...: neighbouring lanes read neighbouring chunks.
template <int TEAM> constexpr int threads_per_cta() { return TEAM <= 32 ? 256 : TEAM; }
template <int TEAM> constexpr int rows_per_cta() { return threads_per_cta<TEAM>() / TEAM; }

// sum over the team, the same value in every thread (fixed order: shuffles, then the warps ascending)
template <int TEAM> __device__ __forceinline__ float team_sum(float v, float *smem /* [2][32] */, int &flip) {
  constexpr int W = TEAM < 32 ? TEAM : 32;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  if (TEAM > 32) {
    // two buffers in turn: a warp that is already at the next row's sum cannot overwrite this one's
    float *b = smem + 32 * flip;
    flip ^= 1;
    if ((threadIdx.x & 31) == 0) b[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < (TEAM + 31) / 32; ++w) v += b[w];
  }
  return v;
}

// largest magnitude over the lanes that hold one 128-column block
template <int LANES> __device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  return v;
}

// 16 bytes that are read once: not kept in L1
__device__ __forceinline__ uint4 load_stream(const uint4 *p) {
  uint4 v;
  asm("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// columns from F on are written as zero, also where the row's statistics are infinite or NaN
template <int V> __device__ __forceinline__ void clear_padding(float (&f)[V], int c, int F) {
  if ((c + 1) * V > F) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (c * V + i >= F) f[i] = 0.f;
  }
}

// Entry-point checks: a matrix of `rows` x F elements of `es` bytes under the library's rule for activations.
inline bool matrix_ok(const void *p, int64_t ld, int64_t F, int es) {
  return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld >= F && (ld * es) % 16 == 0;
}
inline bool dtype_ok(int dt) { return dt == VARCO_F32 || dt == VARCO_BF16; }
inline int elem_size(int dt) { return dt == VARCO_F32 ? 4 : 2; }

// Workspace of the operators: [256 bytes status | scratch]; base rounded up to 256 bytes.
constexpr size_t kStatusBytes = 256;
inline char *ws_align(void *ws) {
  char *p = static_cast<char *>(ws);
  return p + ((256 - (reinterpret_cast<uintptr_t>(p) & 255u)) & 255u);
}
// SMs of the current device (a host call of about 20 ns once the context is there)
inline int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return n;
}
size_t norm_scratch_bytes(int F);         // of rows up to F wide
size_t clip_scratch_bytes();

}  // namespace vops

#endif  // VARCO_OPS_COMMON_CUH_
