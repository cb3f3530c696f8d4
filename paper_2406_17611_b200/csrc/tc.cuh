// Inline-PTX wrappers of the 5th-generation tensor-core path: mbarriers with bounded waits, TMA tile copies, TMEM allocation
// and loads, tcgen05.mma of kinds f16 and f8f6f4, descriptors, tensor maps.
#ifndef VARCO_TC_CUH_
#define VARCO_TC_CUH_

#include <cuda.h>

#include "device_common.cuh"

namespace vtc {

constexpr uint32_t kIdleNs = 1000000u;            // hint of a role with time to spare
constexpr uint32_t kSpinLimit = 1u << 24;
constexpr long long kSpinClocks = 2000000000ll;   // about one second of SM clocks

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint64_t *bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t *bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t *bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// HINT: how long the thread may sleep in the instruction, in ns (0: the hardware's own short limit, which wakes sooner)
template <uint32_t HINT = 0> __device__ __forceinline__ bool mbar_try_wait(uint64_t *bar, uint32_t parity) {
  uint32_t ok;
  if (HINT)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity), "r"(HINT)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
  return ok != 0;
}
// Bounded wait.  Returns false (and raises the flags) when the limit is hit or another role gave up.  A role with time to
// spare waits with a hint: one that asks again and again takes issue slots from the warps that work.
template <uint32_t HINT = 0>
__device__ __forceinline__ bool mbar_wait(uint64_t *bar, uint32_t parity, volatile int *abort_smem, int *err, int code) {
  if (mbar_try_wait<HINT>(bar, parity)) return true;
  const long long t0 = clock64();
  for (uint32_t it = 0; it < kSpinLimit; ++it) {
    if (mbar_try_wait<HINT>(bar, parity)) return true;
    if (HINT || (it & 255u) == 255u) {
      if (*abort_smem) return false;
      if (clock64() - t0 > kSpinClocks) break;
    }
  }
  *abort_smem = 1;
  atomicCAS(err, 0, code);
  return false;
}

// Wait of a role that is about to leave: bounded too, but raises nothing (who gave up has said so).
__device__ __forceinline__ void mbar_wait_quietly(uint64_t *bar, uint32_t parity) {
  const long long t0 = clock64();
  while (!mbar_try_wait<kIdleNs>(bar, parity) && clock64() - t0 <= kSpinClocks) {
  }
}
// Parity of the phase that stage s's last fill completes, for a loader that would fill `stage` next with parity `phase`.  A stage
// that was never filled gives the phase before the first, which every wait takes as complete.
__host__ __device__ constexpr uint32_t last_fill(int s, int stage, uint32_t phase) { return s < stage ? phase : phase ^ 1u; }
// Every load that the loader has issued has landed: before that its CTA must not retire, whoever gave up.
template <int STAGES> __device__ __forceinline__ void drain_loads(uint64_t *full, int stage, uint32_t phase) {
  for (int s = 0; s < STAGES; ++s) mbar_wait_quietly(&full[s], last_fill(s, stage, phase));
}

__device__ __forceinline__ void tma_load_2d(void *smem_dst, const CUtensorMap *tmap, int x, int y, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          smem_u32(smem_dst)),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t *slot_smem, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot_smem)), "r"(cols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ void umma_bf16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// arrives on the mbarrier once every tcgen05.mma issued so far by this thread has completed
__device__ __forceinline__ void umma_commit(uint64_t *bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
               : "memory");
}
// Every tcgen05.mma that this thread has issued has completed, whoever gave up: before that TMEM must not be freed and the
// operands' shared memory not left.  `drained`: a barrier of its own with a count of one.
__device__ __forceinline__ void drain_umma(uint64_t *drained) {
  umma_commit(drained);
  mbar_wait_quietly(drained, 0);
}
// 16 or 32 accumulator columns of this thread's TMEM lane
__device__ __forceinline__ void tmem_ld(uint32_t taddr, float2 (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(r[0].x), "=f"(r[0].y), "=f"(r[1].x), "=f"(r[1].y), "=f"(r[2].x), "=f"(r[2].y), "=f"(r[3].x), "=f"(r[3].y), "=f"(r[4].x),
        "=f"(r[4].y), "=f"(r[5].x), "=f"(r[5].y), "=f"(r[6].x), "=f"(r[6].y), "=f"(r[7].x), "=f"(r[7].y)
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld(uint32_t taddr, float2 (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(r[0].x), "=f"(r[0].y), "=f"(r[1].x), "=f"(r[1].y), "=f"(r[2].x), "=f"(r[2].y), "=f"(r[3].x), "=f"(r[3].y), "=f"(r[4].x),
        "=f"(r[4].y), "=f"(r[5].x), "=f"(r[5].y), "=f"(r[6].x), "=f"(r[6].y), "=f"(r[7].x), "=f"(r[7].y), "=f"(r[8].x),
        "=f"(r[8].y), "=f"(r[9].x), "=f"(r[9].y), "=f"(r[10].x), "=f"(r[10].y), "=f"(r[11].x), "=f"(r[11].y), "=f"(r[12].x),
        "=f"(r[12].y), "=f"(r[13].x), "=f"(r[13].y), "=f"(r[14].x), "=f"(r[14].y), "=f"(r[15].x), "=f"(r[15].y)
      : "r"(taddr)
      : "memory");
}
// register budget of the warpgroup: the shares of all warpgroups add up to what the block was launched with
template <int N> __device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared-memory matrix descriptor, 128-byte swizzle, Blackwell descriptor version 1.
//   K-major operand : rows of 128 bytes, 8-row groups 1024 B apart (SBO); LBO unused (1).
//   MN-major operand: rows are K indices holding 64 contiguous MN elements of 2 bytes; 8-row K groups 1024 B apart (SBO);
//                     successive 64-element MN chunks `lbo_bytes` apart (LBO).
__device__ __forceinline__ uint64_t smem_desc(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((lbo_bytes >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)((sbo_bytes >> 4) & 0x3FFFu) << 32;
  d |= 1ull << 46;   // descriptor version
  d |= 2ull << 61;   // SWIZZLE_128B
  return d;
}
__device__ __forceinline__ uint64_t smem_desc_kmajor(uint32_t saddr) { return smem_desc(saddr, 16, 1024); }
// Instruction descriptor of kind f16: bf16 inputs, 32-bit accumulation.
__host__ __device__ constexpr uint32_t instr_desc_bf16(int M, int N, int a_mn_major, int b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn_major << 15) | ((uint32_t)b_mn_major << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// Instruction descriptor of kind f8f6f4: e4m3 inputs, 32-bit accumulation, both operands K-major.
__host__ __device__ constexpr uint32_t instr_desc_e4m3(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// ------------------------------------------------------------------------------------------ host
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = [] {
    void *ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      return reinterpret_cast<EncodeTiledFn>(ptr);
    return (EncodeTiledFn) nullptr;
  }();
  return fn;
}

// 2-D tensor map over a row-major matrix: `cols` valid columns (reads beyond are zero filled, writes beyond dropped),
// `rows` rows, leading dimension ld elements, box {box_cols, box_rows}.
inline int make_map(CUtensorMap *m, const void *ptr, CUtensorMapDataType type, int es, int64_t rows, int64_t cols, int64_t ld,
                    int box_cols, int box_rows, CUtensorMapSwizzle swizzle) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return VARCO_CUDA;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * es};
  cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1u, 1u};
  CUresult r = fn(m, type, 2, const_cast<void *>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? VARCO_OK : VARCO_CUDA;
}

}  // namespace vtc

#endif  // VARCO_TC_CUH_
