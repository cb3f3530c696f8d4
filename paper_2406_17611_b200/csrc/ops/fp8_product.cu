// Product of two e4m3 matrices with a scale for each block of 128, on the 5th-generation tensor cores.
//
//   Y[m][n] = act( sum_kb sA[kb][m] sB[n / 128][kb] sum_{k in block kb} A8[m][k] B8[n][k] + bias[n] )
//   act: nothing, ReLU, or the product with 1[mask[m][n] > 0] (the ReLU's backward);
//   outputs: Y in bf16 or fp32 and, if asked, its 8-bit form with one scale per row and 128 columns -- the operand of
//   the next product, written from the 32-bit accumulators instead of by a pass of its own.
//
// The scales change along the contraction, so the tensor cores add one block of 128 (four instructions of K = 32) into
// a fresh TMEM accumulator, and the epilogue warps add acc += scale x partial in 32-bit registers while the next block
// is multiplied into the other accumulator.
//
// Persistent CTAs work through output tiles of 128 rows and 256, 128 or 64 columns.  Warps by role:
//   0 .. EPI-1   accumulators and outputs: warp w reads TMEM lanes 32 (w % 4) .. + 31 (one row a thread) and part w / 4
//                of the columns
//   EPI          TMA loads of the operands (128-byte swizzle)
//   EPI + 1      tcgen05.mma, one thread
//   EPI + 2, 3   scales: half of the rows each, loaded four blocks ahead in registers, handed over with the accumulator
// Bound: the SM's own work, not memory: times follow the SM clock (2.45M x 1024 x 256 with both outputs: 1640 us at 1965 MHz, 1955
// back to back under the power cap at 1575 to 1665 MHz, while the norm, which HBM bounds, keeps its time).  A tile of two blocks
// takes 6200 clocks at either clock; its epilogue warps add, take the maximum, pack, stage and store one after the other.
// Long contractions (16,384 x 4096 x 4096: 295 us = 1.86 PFLOP/s in a burst, 342 us sustained): 1250 to 1310 clocks a block.
// Known parts, none of which is that long: instructions 512; the round of an accumulator 1230 (instructions, commit and wake 170,
// add 450, hand back 100), 615 a block with two; operands 800 with 64 CTAs at work (48 KB at 61 bytes a clock of an SM; with all 148
// not measured).
// Every mbarrier wait is bounded: on expiry the status word is set, every role runs to its end without waiting (the
// outputs are then invalid), loads and instructions in flight are waited for (bounded as well), TMEM is released and the
// kernel returns.
#include <cstring>

#include "fp8_product.h"
#include "ops_common.cuh"
#include "tc.cuh"

namespace {

using namespace vops;
using namespace vtc;

constexpr int kTileM = 128, kTileK = 128, kUmmaK = 32;
constexpr int kAhead = 4;                 // blocks whose scales are on their way

struct ProductParams {
  CUtensorMap tmA, tmB;             // e4m3, boxes {128, 128} and {128, NT}
  int64_t M, work;                  // work: output tiles
  int N, kblocks, m_tiles, n_tiles;
  int step_m, step_n;               // gridDim.x = step_m * n_tiles + step_n
  const float *sa, *sb, *bias;
  int64_t ld_sa, sb_n, sb_k;
  const void *mask;
  void *y;
  uint8_t *y8;
  float *sy;
  int64_t ldmask, ldy, ldy8, ld_sy;
  int *err;
};

// NT: output columns of a tile; EPI: epilogue warps; STAGES: operand stages; REGS: registers of an epilogue thread (the
// launch's share of all threads is split again between the epilogue and the other warps; 0: not split); LINE: bytes
// of a row in a staging piece (32 rows); PIECES: of them for an epilogue warp; CH: accumulator columns of one load; CTAS: of one SM
template <int NT_, int EPI_, int STAGES_, int REGS_, int PIECES_, int CH_, int CTAS_, int LINE_> struct Config {
  static constexpr int NT = NT_, EPI = EPI_, STAGES = STAGES_, REGS = REGS_, PIECES = PIECES_, CH = CH_, CTAS = CTAS_, LINE = LINE_;
  static constexpr int ACCS = 512 / NT / CTAS;                 // accumulators in TMEM: a power of two
  static constexpr int NB = (NT + kBlock - 1) / kBlock;   // column blocks of a tile
  static constexpr int kThreads = EPI * 32 + 128;         // setmaxnreg works on whole warpgroups
  static constexpr int kCols = NT * 4 / EPI;              // columns of one thread
  static constexpr uint32_t kABytes = kTileM * kTileK, kBBytes = NT * kTileK;
  static constexpr uint32_t kStaging = STAGES * (kABytes + kBBytes);
  static constexpr uint32_t kScales = kStaging + EPI * PIECES * 32 * LINE;      // [accumulators][column blocks][128]
  static constexpr uint32_t kBias = kScales + ACCS * NB * kTileM * 4;
  static constexpr uint32_t kExch = kBias + EPI * kCols * 4;
  static constexpr uint32_t kBars = kExch + (kCols < kBlock && NT >= kBlock ? 2 * EPI * 32 * 4 : 0);
  static constexpr uint32_t kTotal = kBars + (2 * STAGES + 2 * ACCS + 1) * 8 + 16;
  static constexpr int kLaunchRegs = 65536 / (CTAS * kThreads) / 8 * 8;
  static constexpr int kOtherRegs = (kLaunchRegs * kThreads - REGS * EPI * 32) / 128 / 8 * 8;
  static_assert(REGS == 0 || (kOtherRegs >= 24 && kOtherRegs * 128 + REGS * EPI * 32 <= kLaunchRegs * kThreads), "register split");
};

// Output tiles of one CTA: every gridDim.x-th, columns fastest (neighbouring CTAs share rows of A in L2).
struct TileWalk {
  int mt, nt;
  __device__ __forceinline__ explicit TileWalk(const ProductParams &p) : mt(blockIdx.x / p.n_tiles), nt(blockIdx.x % p.n_tiles) {}
  __device__ __forceinline__ void next(const ProductParams &p) {
    mt += p.step_m;
    nt += p.step_n;
    if (nt >= p.n_tiles) {
      nt -= p.n_tiles;
      ++mt;
    }
  }
};

// acc += s * (accumulator columns [taddr, taddr + COLS)), CH columns at a time.  Longer or overlapping loads are no faster
// here (the other warps of the scheduler fill the gap) and cost registers that the epilogue then spills.
template <int COLS, int CH>
__device__ __forceinline__ void add_scaled(uint32_t taddr, const float *scale, float2 (&acc)[COLS / 2]) {
  const float s = *scale;
#pragma unroll
  for (int c = 0; c < COLS; c += CH) {
    float2 r[CH / 2];
    tmem_ld(taddr + c, r);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) acc[c / 2 + i] = __ffma2_rn(r[i], make_float2(s, s), acc[c / 2 + i]);
  }
}

// 16 bytes of output from registers; RELU: negative values become zero in the conversion, a NaN stays
template <bool RELU> __device__ __forceinline__ uint32_t bf16x2(float2 f) {
  uint32_t r;
  if (RELU) asm("cvt.rn.relu.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(f.y), "f"(f.x));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(f.y), "f"(f.x));
  return r;
}
template <bool RELU> __device__ __forceinline__ uint4 pack_row(const float2 *f, __nv_bfloat16) {
  return make_uint4(bf16x2<RELU>(f[0]), bf16x2<RELU>(f[1]), bf16x2<RELU>(f[2]), bf16x2<RELU>(f[3]));
}
template <bool RELU> __device__ __forceinline__ uint4 pack_row(const float2 *f, float) {
  if (RELU) return make_uint4(__float_as_uint(relu(f[0].x)), __float_as_uint(relu(f[0].y)), __float_as_uint(relu(f[1].x)), __float_as_uint(relu(f[1].y)));
  return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
}
template <bool RELU> __device__ __forceinline__ uint32_t e4m3x4(float2 a, float2 b, float inv) {
  uint32_t r;
  a = __fmul2_rn(a, make_float2(inv, inv));
  b = __fmul2_rn(b, make_float2(inv, inv));
  if (RELU)
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.relu.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.relu.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(r) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  else
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(r) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
template <bool RELU> __device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  if (RELU) asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  else asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// a 16-byte part whose last columns lie past N: those become zero (ES: bytes of an element, `n`: columns that stay)
template <int ES> __device__ __forceinline__ uint4 keep_first(uint4 v, int n) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int bytes = n * ES - i * 4;
    if (bytes < 4) w[i] = bytes <= 0 ? 0u : w[i] & ((1u << bytes * 8) - 1u);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Place of 16-byte part j of row r in a staged piece of PARTS parts a row: a thread that holds a row and lanes that share a
// line both meet every bank once.
template <int PARTS> __device__ __forceinline__ int place(int r, int j) {
  return r * PARTS + (PARTS == 8 ? (j ^ r) & 7 : (j ^ (r >> 1)) & 3);
}
// A staged piece of 32 rows to memory: PARTS lanes write a row's line, 32 / PARTS rows at a time.
template <int PARTS, int ES>
__device__ __forceinline__ void store_lines(const uint4 *stg, char *base, int64_t stride, int row0, int col, int M, int N, int lane) {
  constexpr int R = 32 / PARTS, V = 16 / ES;
  const int r0 = lane / PARTS, j = lane % PARTS;
  char *out = base + (int64_t)(row0 + r0) * stride + (int64_t)(col + j * V) * ES;   // bytes: past 2^31 for wide outputs
  if (row0 + 32 <= M && col + PARTS * V <= N) {
    uint4 v[PARTS];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) v[k] = stg[place<PARTS>(k * R + r0, j)];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      *reinterpret_cast<uint4 *>(out) = v[k];
      out += R * stride;
    }
  } else if (col + j * V < N) {
#pragma unroll 1
    for (int r = r0; r < 32 && row0 + r < M; r += R) {
      *reinterpret_cast<uint4 *>(out) = keep_first<ES>(stg[place<PARTS>(r, j)], N - col - j * V);
      out += R * stride;
    }
  }
}
// 16 bytes to shared memory in the background (`bytes` of them from memory, the rest zero)
__device__ __forceinline__ void copy16_async(void *smem, const void *g, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(smem)), "l"(g), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

template <typename T, typename CFG, bool RELU>
__global__ void __launch_bounds__(CFG::kThreads, CFG::CTAS) fp8_product_kernel(const __grid_constant__ ProductParams p) {
  constexpr int NT = CFG::NT, EPI = CFG::EPI, STAGES = CFG::STAGES, COLS = CFG::kCols, ACCS = CFG::ACCS, NB = CFG::NB;
  extern __shared__ uint8_t smem_raw[];
  // aligned by an offset, not by a cast of the address: the compiler keeps knowing that it is shared memory
  uint8_t *base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t *sA = base, *sB = base + STAGES * CFG::kABytes;
  float *scales = reinterpret_cast<float *>(base + CFG::kScales);
  uint64_t *full = reinterpret_cast<uint64_t *>(base + CFG::kBars), *empty = full + STAGES, *tfull = empty + STAGES, *tempty = tfull + ACCS, *drained = tempty + ACCS;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(drained + 1);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < ACCS; ++a) {
      mbar_init(&tfull[a], 3);          // the tensor cores' commit and the two scale warps
      mbar_init(&tempty[a], EPI);
    }
    mbar_init(drained, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == EPI + 1) tmem_alloc(tmem_slot, ACCS * NT);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp >= EPI) {
    if constexpr (CFG::REGS != 0) regs_dec<CFG::kOtherRegs>();
    if (warp == EPI && lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t tx = CFG::kABytes + CFG::kBBytes;
      for (TileWalk w(p); ok && w.mt < p.m_tiles; w.next(p)) {
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (!mbar_wait<kIdleNs>(&empty[stage], phase ^ 1u, abort_flag, p.err, 21)) {
            ok = false;
            break;
          }
          mbar_expect_tx(&full[stage], tx);
          tma_load_2d(sA + stage * CFG::kABytes, &p.tmA, kb * kTileK, w.mt * kTileM, &full[stage]);
          tma_load_2d(sB + stage * CFG::kBBytes, &p.tmB, kb * kTileK, w.nt * NT, &full[stage]);
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      drain_loads<STAGES>(full, stage, phase);
    } else if (warp == EPI + 1 && lane == 0) {
      const uint32_t idesc = instr_desc_e4m3(kTileM, NT);
      int stage = 0;
      uint32_t phase = 0, it = 0;
      bool ok = true;
      for (TileWalk w(p); ok && w.mt < p.m_tiles; w.next(p)) {
        for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
          const uint32_t acc = it % ACCS;
          if (!mbar_wait(&full[stage], phase, abort_flag, p.err, 23) ||
              !mbar_wait(&tempty[acc], ((it / ACCS) & 1u) ^ 1u, abort_flag, p.err, 22)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a = smem_u32(sA + stage * CFG::kABytes), b = smem_u32(sB + stage * CFG::kBBytes);
#pragma unroll
          for (int kk = 0; kk < kTileK / kUmmaK; ++kk)
            umma_f8(tmem_base + acc * NT, smem_desc_kmajor(a + kk * kUmmaK), smem_desc_kmajor(b + kk * kUmmaK), idesc, kk != 0);
          umma_commit(&tfull[acc]);
          umma_commit(&empty[stage]);
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      drain_umma(drained);
    } else if (warp >= EPI + 2) {
      // rows r0 and r0 + 32 of the tile: sA of the row times sB of each 128-column block
      const int r0 = (warp - EPI - 2) * 64 + lane, M = (int)p.M;
      const int64_t total = (p.work - blockIdx.x + gridDim.x - 1) / gridDim.x * p.kblocks;
      float sa[kAhead][2], sb[kAhead][NB];
      TileWalk w(p);
      int kb = 0;
      const float *pa0 = p.sa, *pa1 = p.sa, *pb = p.sb;
      auto load = [&](float (&a)[2], float (&b)[NB]) {
        if (kb == 0) {
          const int m = w.mt * kTileM + r0;
          pa0 = p.sa + (m < M ? m : 0);
          pa1 = p.sa + (m + 32 < M ? m + 32 : 0);
          pb = p.sb + (int64_t)(w.nt * NT / kBlock) * p.sb_n;
        }
        a[0] = __ldg(pa0);
        a[1] = __ldg(pa1);
#pragma unroll
        for (int j = 0; j < NB; ++j) b[j] = w.nt * NT + j * kBlock < p.N ? __ldg(pb + j * p.sb_n) : 0.f;
        pa0 += p.ld_sa;
        pa1 += p.ld_sa;
        pb += p.sb_k;
        if (++kb == p.kblocks) {
          kb = 0;
          w.next(p);
        }
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i < total) load(sa[i], sb[i]);
      bool ok = true;
      for (int64_t n = 0; ok && n < total; n += kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (ok && n + i < total) {
            const uint32_t acc = (uint32_t)(n + i) % ACCS, use = (uint32_t)((n + i) / ACCS);
            ok = mbar_wait<kIdleNs>(&tempty[acc], (use & 1u) ^ 1u, abort_flag, p.err, 26);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
              scales[(acc * NB + j) * kTileM + r0] = sa[i][0] * sb[i][j];
              scales[(acc * NB + j) * kTileM + r0 + 32] = sa[i][1] * sb[i][j];
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&tfull[acc]);
            if (n + i + kAhead < total) load(sa[i], sb[i]);
          }
        }
      }
    }
  } else {
    if constexpr (CFG::REGS != 0) regs_inc<CFG::REGS>();
    // Pieces of 32 rows x LINE bytes of Y go through the warp's staging tile: written by rows, read by lines.
    constexpr int ES = (int)sizeof(T), V = 16 / ES, LINE = CFG::LINE, SLAB = LINE / ES, PARTS = LINE / 16, NY = COLS / SLAB, NE = COLS / 64,
                  PIECES = CFG::PIECES;
    const int quarter = warp & 3, part = warp >> 2;
    uint4 *stg = reinterpret_cast<uint4 *>(base + CFG::kStaging + warp * (PIECES * 32 * LINE));
    float *bias = reinterpret_cast<float *>(base + CFG::kBias) + warp * COLS;
    uint32_t *exch = reinterpret_cast<uint32_t *>(base + CFG::kExch);
    const float *my_scale = scales + part * COLS / kBlock * kTileM + quarter * 32 + lane;
    uint32_t it = 0, flip = 0;
    int bias_tile = -1;
    bool ok = true;
    const int M = (int)p.M;
    const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(part * COLS);
    for (TileWalk w(p); w.mt < p.m_tiles; w.next(p)) {
      const int row0 = w.mt * kTileM + quarter * 32, nt = w.nt;
      const int col0 = nt * NT + part * COLS;
      const bool here = row0 < M && col0 < p.N;            // this warp has outputs in the tile
      // The mask's pieces travel while the blocks are multiplied.  Columns past N are copied as zeros: their sums are scale x 0,
      // NaN where the scale is not finite, and must not reach the block's magnitude (a row whose mask leaves nothing is zero
      // whatever its operand holds; without a mask such a row's block is NaN all the same).
      auto load_mask = [&](int i0) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const int j = lane % PARTS, c = col0 + (i0 + i) * SLAB + j * V;
          if (i0 + i < NY) {
            const int bytes = min(V, max(p.N - c, 0)) * ES;
            const T *from = (const T *)p.mask + (bytes ? c : 0);
#pragma unroll
            for (int k = 0; k < PARTS; ++k) {
              const int r = k * (32 / PARTS) + lane / PARTS;
              const bool in = row0 + r < M;
              copy16_async(stg + i * (32 * PARTS) + place<PARTS>(r, j), from + (int64_t)(in ? row0 + r : 0) * p.ldmask, in ? bytes : 0);
            }
          }
        }
        copy_commit();
      };
      if (p.mask && here) load_mask(0);
      float2 acc[COLS / 2];
      if (p.bias) {
        if (bias_tile != nt) {
          bias_tile = nt;
          __syncwarp();
          for (int i = lane; i < COLS; i += 32) bias[i] = col0 + i < p.N ? p.bias[col0 + i] : 0.f;
          __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < COLS; i += 4) {
          const float4 b = *reinterpret_cast<const float4 *>(bias + i);
          acc[i / 2] = make_float2(b.x, b.y);
          acc[i / 2 + 1] = make_float2(b.z, b.w);
        }
      } else {
#pragma unroll
        for (int i = 0; i < COLS / 2; ++i) acc[i] = make_float2(0.f, 0.f);
      }
      for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
        const uint32_t buf = it % ACCS;
        ok = ok && mbar_wait(&tfull[buf], (it / ACCS) & 1u, abort_flag, p.err, 24);
        tc_fence_after();
        add_scaled<COLS, CFG::CH>(taddr + buf * NT, my_scale + buf * (NB * kTileM), acc);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&tempty[buf]);
      }
      if (p.mask && here) {
#pragma unroll
        for (int i = 0; i < NY; ++i) {
          if (i % PIECES == 0) {
            if (i > 0) {
              __syncwarp();
              load_mask(i);
            }
            copy_wait();
            __syncwarp();
          }
#pragma unroll
          for (int j = 0; j < PARTS; ++j) {
            float f[V];
            unpack16(stg[(i % PIECES) * (32 * PARTS) + place<PARTS>(lane, j)], f, T());
#pragma unroll
            for (int k = 0; k < V; k += 2) {
              float2 &a = acc[(i * SLAB + j * V + k) / 2];
              a = make_float2(f[k] > 0.f ? a.x : 0.f, f[k + 1] > 0.f ? a.y : 0.f);
            }
          }
        }
        __syncwarp();
      }
      float inv = 0.f;
      if (p.y8) {
        float t0 = 0.f, t1 = 0.f, t2 = 0.f, t3 = 0.f;
#pragma unroll
        for (int i = 0; i < COLS / 2; i += 4) {
          t0 = max3<RELU>(acc[i].x, acc[i].y, t0);
          t1 = max3<RELU>(acc[i + 1].x, acc[i + 1].y, t1);
          t2 = max3<RELU>(acc[i + 2].x, acc[i + 2].y, t2);
          t3 = max3<RELU>(acc[i + 3].x, acc[i + 3].y, t3);
        }
        uint32_t bits = here ? abs_bits(max3<RELU>(t0, t1, max3<RELU>(t2, t3, 0.f))) : 0u;
        if (COLS < kBlock && NT >= kBlock) {   // the block's other half is in the warp four further: a named barrier for each pair
          uint32_t *e = exch + flip * (EPI * 32);
          flip ^= 1u;
          e[warp * 32 + lane] = bits;
          asm volatile("bar.sync %0, 64;" ::"r"(1 + quarter + (part >> 1) * 4) : "memory");
          bits = max(bits, e[(warp ^ 4) * 32 + lane]);
        }
        const Scale s = block_scale(bits);
        inv = s.inv;
        if (here && row0 + lane < M && (COLS * part % kBlock == 0)) p.sy[(int64_t)(col0 / kBlock) * p.ld_sy + row0 + lane] = s.s;
      }
      if (here && p.y) {
#pragma unroll
        for (int i = 0; i < NY; ++i) {
          if (col0 + i * SLAB < p.N) {
#pragma unroll
            for (int j = 0; j < PARTS; ++j) stg[place<PARTS>(lane, j)] = pack_row<RELU>(acc + (i * SLAB + j * V) / 2, T());
            __syncwarp();
            store_lines<PARTS, ES>(stg, (char *)p.y, p.ldy * ES, row0, col0 + i * SLAB, M, p.N, lane);
            __syncwarp();
          }
        }
      }
      if (here && p.y8) {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          if (col0 + i * 64 < p.N) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 *f = acc + (i * 64 + j * 16) / 2;
              stg[place<4>(lane, j)] =
                  make_uint4(e4m3x4<RELU>(f[0], f[1], inv), e4m3x4<RELU>(f[2], f[3], inv), e4m3x4<RELU>(f[4], f[5], inv), e4m3x4<RELU>(f[6], f[7], inv));
            }
            __syncwarp();
            store_lines<4, 1>(stg, (char *)p.y8, p.ldy8, row0, col0 + i * 64, M, p.N, lane);
            __syncwarp();
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == EPI + 1) tmem_dealloc(tmem_base, ACCS * NT);
}

template <typename T, typename CFG, bool RELU> int launch_as(ProductParams &p, const varco_fp8_desc_t *d, const void *A8, const void *B8, cudaStream_t st) {
  constexpr int smem = 1024 + (int)CFG::kTotal;
  static_assert(smem <= (CFG::CTAS == 1 ? 232448 : 233472 / CFG::CTAS - 1024), "shared memory of the SM");
  VARCO_CUDA_CHECK(cudaFuncSetAttribute(fp8_product_kernel<T, CFG, RELU>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  p.n_tiles = (p.N + CFG::NT - 1) / CFG::NT;
  p.m_tiles = (int)((p.M + kTileM - 1) / kTileM);
  if (make_map(&p.tmA, A8, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.M, d->K, d->lda, kTileK, kTileM, CU_TENSOR_MAP_SWIZZLE_128B) ||
      make_map(&p.tmB, B8, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.N, d->K, d->ldb, kTileK, CFG::NT, CU_TENSOR_MAP_SWIZZLE_128B))
    return VARCO_CUDA;
  const int sms = sm_count();
  if (sms <= 0) return VARCO_CUDA;
  p.work = (int64_t)p.m_tiles * p.n_tiles;
  const int most = sms * CFG::CTAS, grid = (int)(p.work < most ? p.work : most);
  p.step_m = grid / p.n_tiles, p.step_n = grid % p.n_tiles;
  fp8_product_kernel<T, CFG, RELU><<<grid, CFG::kThreads, smem, st>>>(p);
  VARCO_KERNEL_LAUNCHED();
  return VARCO_OK;
}
template <typename T, typename CFG> int launch(ProductParams &p, const varco_fp8_desc_t *d, const void *A8, const void *B8, cudaStream_t st) {
  return d->relu ? launch_as<T, CFG, true>(p, d, A8, B8, st) : launch_as<T, CFG, false>(p, d, A8, B8, st);
}

typedef Config<256, 8, 3, 232, 2, 16, 1, 128> Wide;
typedef Config<128, 4, 3, 208, 1, 16, 2, 64> Duo;
typedef Config<128, 8, 5, 0, 1, 32, 1, 128> Mid;
typedef Config<64, 4, 3, 0, 2, 32, 2, 128> Slim;

// The tile by the output's width.  A wide tile reads A least often (1M x 1024 x 256 with both outputs: 686 us with 256 columns,
// 796 with two CTAs of 128 an SM); columns past N are multiplied for nothing (1M x 128 x 1024: 329 us with 256 columns, 291 with
// 128, 230 with two CTAs of 128; 233,000 x 41 x 602: 94, 51, 57 and with two CTAs of 64 columns 39).  Where 256 columns leave
// over half of the SMs without a tile, or 128 all but one round of them, one CTA of 128 columns with all eight epilogue warps
// spreads better (1000 x 1024 x 1024: 9.2 against 7.4 us; 4000 rows, 128 tiles of 148: 9.8 against 11.5).
template <typename T> int dispatch(ProductParams &p, const varco_fp8_desc_t *d, const void *A8, const void *B8, cudaStream_t st) {
  const int64_t rows = (d->M + kTileM - 1) / kTileM;
  const int sms = sm_count();
  if (d->N <= 64) return launch<T, Slim>(p, d, A8, B8, st);
  if (d->N <= 128) return rows > sms ? launch<T, Duo>(p, d, A8, B8, st) : launch<T, Mid>(p, d, A8, B8, st);
  return rows * ((d->N + 255) / 256) > sms / 2 ? launch<T, Wide>(p, d, A8, B8, st) : launch<T, Mid>(p, d, A8, B8, st);
}

}  // namespace

extern "C" int varco_fp8_product(const varco_fp8_desc_t *d, const void *A8, const float *sA, const void *B8, const float *sB, const float *bias,
                                 const void *mask, void *Y, void *Y8, float *sY, void *workspace, size_t ws_bytes, void *stream) {
  if (!d || d->M < 0 || d->N < 1 || d->K < 1 || !dtype_ok(d->dtype) || !workspace) return VARCO_INVALID_ARG;
  if (ws_bytes < 256 + kStatusBytes) return VARCO_WORKSPACE_TOO_SMALL;
  if (d->M > INT32_MAX - 256 || d->N > INT32_MAX - 512 || d->K > INT32_MAX - 256) return VARCO_UNSUPPORTED;
  if (d->M == 0) return VARCO_OK;
  const int es = elem_size(d->dtype);
  if (!matrix_ok(A8, d->lda, d->K, 1) || !matrix_ok(B8, d->ldb, d->K, 1) || !sA || !sB || d->ld_sa < d->M || d->sb_n < 0 || d->sb_k < 0 ||
      (!Y && !Y8) || (Y && !matrix_ok(Y, d->ldy, d->N, es)) || (mask && !matrix_ok(mask, d->ldmask, d->N, es)) ||
      (Y8 && (!matrix_ok(Y8, d->ldy8, d->N, 1) || !sY || d->ld_sy < d->M)))
    return VARCO_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  const int sms = sm_count();
  if (sms <= 0) return VARCO_CUDA;
  if (few_rows_pay(d->M, d->N, d->K, Y8 != nullptr, sms)) return varco_launch_fp8_few_rows(d, A8, sA, B8, sB, bias, mask, Y, Y8, sY, st);
  ProductParams p;
  memset(&p, 0, sizeof(p));
  p.M = d->M, p.N = d->N, p.kblocks = (d->K + kTileK - 1) / kTileK;
  p.sa = sA, p.sb = sB, p.bias = bias, p.ld_sa = d->ld_sa, p.sb_n = d->sb_n, p.sb_k = d->sb_k;
  p.mask = mask, p.ldmask = d->ldmask, p.y = Y, p.ldy = d->ldy, p.y8 = (uint8_t *)Y8, p.ldy8 = d->ldy8, p.sy = sY, p.ld_sy = d->ld_sy;
  p.err = reinterpret_cast<int *>(ws_align(workspace));
  return es == 4 ? dispatch<float>(p, d, A8, B8, st) : dispatch<__nv_bfloat16>(p, d, A8, B8, st);
}
