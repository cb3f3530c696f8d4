// Root-mean-square norm of the residual stream, forward and backward.
//
//   forward    h = x + r;  rstd = 1 / sqrt(mean(h^2) + eps);  y = gain . h . rstd
//   backward   t = gain . dy;  dh = dres + rstd (t - h rstd^2 mean(t . h));  dgain = sum over rows of dy . h . rstd
//              (dh is the gradient of both addends: of x and of r)
//
// Everything is computed in 32 bits from the loaded values and rounded once per output; y, and the 8-bit form of it,
// come from the unrounded sum h.  The 8-bit form (e4m3, one scale per row and 128 columns) is what the 8-bit product
// reads: writing it here saves that operator's own pass over the rows.
//
// Bound: HBM.  Each row is read once and stays in registers between the statistics and the outputs: a team of 2 to 32
// lanes holds a row of up to 160 chunks of 16 bytes, a whole CTA a longer one, and the next row's loads are on their way
// meanwhile.  2.45M x 256 bf16 with residual and 8-bit output: forward 935 us, backward 931 us (6.1 TB/s of the 6.5
// that a copy reaches); 233,000 x 602 fp32: 193 us (5.8).
#include "ops_common.cuh"

namespace {

using namespace vops;

struct NormParams {
  int64_t rows;
  int F;
  float eps;
  const void *x, *r;       // forward: the addends; backward: h, dres
  const void *dy;          // backward only
  const float *gain, *rstd_in;
  void *h, *y;             // forward: sum and normalised rows; backward: y = dh
  uint8_t *y8;
  float *scales, *rstd;
  float *dgain_part;       // backward: [gridDim.x][F] (or dgain itself when there is one CTA), or nullptr
  float *dgain;            // backward: where the last CTA adds the lines (nullptr: another kernel does, or nobody)
  unsigned *arrived;       // CTAs that have written their lines; zero between calls
  int64_t ldx, ldr, ldh, ldy, ld8, lds, lddy;
};

// The 8-bit form of a team's row.  A 128-column block lies in neighbouring lanes of one chunk column, or, for teams
// narrower than a block, in JB chunk columns of all lanes.
template <typename T, int TEAM, int NCH, int V>
__device__ __forceinline__ void quantize_row(const NormParams &p, int64_t row, int lane, const float (&f)[NCH][V]) {
  const int nchunks = chunks_of_eight<V>(p.F);
  constexpr int PER = kBlock / V, LANES = TEAM < PER ? TEAM : PER, JB = PER / LANES;
#pragma unroll
  for (int j0 = 0; j0 < NCH; j0 += JB) {
    uint32_t m = 0;
#pragma unroll
    for (int j = j0; j < j0 + JB && j < NCH; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) m = max(m, abs_bits(f[j][i]));
    m = lanes_max<LANES>(m);
    const Scale s = block_scale(m);
#pragma unroll
    for (int j = j0; j < j0 + JB && j < NCH; ++j) {
      const int c = lane + j * TEAM;
      if (row < p.rows && c < nchunks) {
        store_e4m3(p.y8 + row * p.ld8 + (int64_t)c * V, f[j], s.inv);
        if (c % PER == 0) p.scales[(int64_t)(c / PER) * p.lds + row] = s.s;
      }
    }
  }
}

// The gain of a lane's chunks: in registers while they are few, else in shared memory (ones where there is none).
template <int TEAM, int NCH, int V, bool REGS> struct Gain;
template <int TEAM, int NCH, int V> struct Gain<TEAM, NCH, V, true> {
  float g[NCH][V];
  __device__ __forceinline__ void load(const float *gain, int F, int lane, float *) {
#pragma unroll
    for (int j = 0; j < NCH; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int col = (lane + j * TEAM) * V + i;
        g[j][i] = gain && col < F ? gain[col] : 1.f;
      }
  }
  __device__ __forceinline__ void get(int j, int, float (&w)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = g[j][i];
  }
};
template <int TEAM, int NCH, int V> struct Gain<TEAM, NCH, V, false> {
  const float *s;
  __device__ __forceinline__ void load(const float *gain, int F, int, float *smem) {
    for (int col = threadIdx.x; col < TEAM * NCH * V; col += blockDim.x) smem[col] = gain && col < F ? gain[col] : 1.f;
    __syncthreads();
    s = smem;
  }
  __device__ __forceinline__ void get(int j, int lane, float (&w)[V]) const {
    const float4 *q = reinterpret_cast<const float4 *>(s + (lane + j * TEAM) * V);
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 x = q[i / 4];
      w[i] = x.x, w[i + 1] = x.y, w[i + 2] = x.z, w[i + 3] = x.w;
    }
  }
};
template <int NCH, int V> constexpr bool gain_in_regs() { return NCH * V <= 16; }

// Rows that a team of the forward takes in one trip: two where a lane has one chunk of one matrix to load (2.45M x 256 bf16
// without a residual: 545 against 452 us; with one, two rows cost registers: 948 against 992 us).
template <int TEAM, int NCH, bool RES> constexpr int rows_a_trip() { return TEAM <= 32 && NCH == 1 && !RES ? 2 : 1; }

// 16-byte chunks of a row as they come from memory, one row ahead of the arithmetic: with a row's worth of loads always on
// its way the kernels need half of the resident warps to keep HBM busy
template <int NCH> struct Chunks {
  uint4 v[NCH];
  template <typename T> __device__ __forceinline__ void load(const void *base, int64_t ld, int64_t row, int lane, int team, int nchunks, bool live) {
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = lane + j * team;
      v[j] = make_uint4(0u, 0u, 0u, 0u);
      if (live && c < nchunks) v[j] = load_stream(reinterpret_cast<const uint4 *>((const T *)base + row * ld) + c);
    }
  }
};

template <typename T, int TEAM, int NCH, bool RES>
__global__ void __launch_bounds__(threads_per_cta<TEAM>()) norm_fwd_kernel(const NormParams p) {
  constexpr int V = ElemTraits<T>::kVec;
  __shared__ float red[64];
  int flip = 0;
  const int lane = threadIdx.x % TEAM;
  const int nchunks = (p.F + V - 1) / V;
  __shared__ __align__(16) float sgain[gain_in_regs<NCH, V>() ? 4 : TEAM * NCH * V];
  Gain<TEAM, NCH, V, gain_in_regs<NCH, V>()> gain;
  gain.load(p.gain, p.F, lane, sgain);
  const float inv_f = 1.f / (float)p.F;
  constexpr int R = rows_a_trip<TEAM, NCH, RES>();
  const int64_t step = (int64_t)gridDim.x * rows_per_cta<TEAM>() * R;
  int64_t row0 = (int64_t)blockIdx.x * rows_per_cta<TEAM>() * R;
  const int64_t rows = p.rows;
  auto row_of = [&](int64_t first, int q) { return first + q * rows_per_cta<TEAM>() + threadIdx.x / TEAM; };
  Chunks<NCH> x[R], r[R];
#pragma unroll
  for (int q = 0; q < R; ++q) {
    x[q].template load<T>(p.x, p.ldx, row_of(row0, q), lane, TEAM, nchunks, row_of(row0, q) < rows);
    if (RES) r[q].template load<T>(p.r, p.ldr, row_of(row0, q), lane, TEAM, nchunks, row_of(row0, q) < rows);
  }
  // teams of one CTA take the same number of trips: those past the last row stay for the shuffles and barriers
  for (; row0 < rows; row0 += step) {
    float h[R][NCH][V];
#pragma unroll
    for (int q = 0; q < R; ++q) {
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
        unpack16(x[q].v[j], h[q][j], T());
        if (RES) {
          float f[V];
          unpack16(r[q].v[j], f, T());
#pragma unroll
          for (int i = 0; i < V; ++i) h[q][j][i] += f[i];
        }
        clear_padding<V>(h[q][j], lane + j * TEAM, p.F);
      }
      const int64_t next = row_of(row0 + step, q);
      x[q].template load<T>(p.x, p.ldx, next, lane, TEAM, nchunks, next < rows);
      if (RES) r[q].template load<T>(p.r, p.ldr, next, lane, TEAM, nchunks, next < rows);
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int64_t row = row_of(row0, q);
      const bool live = row < rows;
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < NCH; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) ss = fmaf(h[q][j][i], h[q][j][i], ss);
      ss = team_sum<TEAM>(ss, red, flip);
      const float rstd = rsqrtf(ss * inv_f + p.eps);
      if (live && lane == 0 && p.rstd) p.rstd[row] = rstd;
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
        const int c = lane + j * TEAM;
        const bool here = live && c < nchunks;
        if (here && p.h) *reinterpret_cast<uint4 *>((T *)p.h + row * p.ldh + (int64_t)c * V) = pack16(h[q][j], T());
        float w[V];
        gain.get(j, lane, w);
#pragma unroll
        for (int i = 0; i < V; ++i) h[q][j][i] = h[q][j][i] * rstd * w[i];
        clear_padding<V>(h[q][j], c, p.F);
        if (here && p.y) *reinterpret_cast<uint4 *>((T *)p.y + row * p.ldy + (int64_t)c * V) = pack16(h[q][j], T());
      }
      if (p.y8) quantize_row<T, TEAM, NCH, V>(p, row, lane, h[q]);
    }
  }
}

constexpr int kLines = 16;   // of the gain gradient that a thread of the last CTA loads at once

template <typename T, int TEAM, int NCH, bool RES>
__global__ void __launch_bounds__(threads_per_cta<TEAM>()) norm_bwd_kernel(const NormParams p) {
  constexpr int V = ElemTraits<T>::kVec;
  __shared__ float red[64];
  extern __shared__ float gsum[];   // [chunks * V] gain gradient of this CTA
  int flip = 0;
  const int lane = threadIdx.x % TEAM;
  const int nchunks = (p.F + V - 1) / V;
  __shared__ __align__(16) float sgain[gain_in_regs<NCH, V>() ? 4 : TEAM * NCH * V];
  Gain<TEAM, NCH, V, gain_in_regs<NCH, V>()> gain;
  gain.load(p.gain, p.F, lane, sgain);
  float dg[NCH][V];
#pragma unroll
  for (int j = 0; j < NCH; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) dg[j][i] = 0.f;
  const float inv_f = 1.f / (float)p.F;
  const int64_t step = (int64_t)gridDim.x * rows_per_cta<TEAM>();
  int64_t row = (int64_t)blockIdx.x * rows_per_cta<TEAM>() + threadIdx.x / TEAM;
  Chunks<NCH> hc, yc, rc;
  float rstd_next = row < p.rows ? p.rstd_in[row] : 0.f;
  hc.template load<T>(p.x, p.ldx, row, lane, TEAM, nchunks, row < p.rows);
  yc.template load<T>(p.dy, p.lddy, row, lane, TEAM, nchunks, row < p.rows);
  if (RES) rc.template load<T>(p.r, p.ldr, row, lane, TEAM, nchunks, row < p.rows);
  for (int64_t row0 = (int64_t)blockIdx.x * rows_per_cta<TEAM>(); row0 < p.rows; row0 += step, row += step) {
    const bool live = row < p.rows, more = row + step < p.rows;
    float h[NCH][V], t[NCH][V];
    const float rstd = rstd_next;
    float dot = 0.f;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      unpack16(hc.v[j], h[j], T());
      unpack16(yc.v[j], t[j], T());
      clear_padding<V>(h[j], lane + j * TEAM, p.F);
      clear_padding<V>(t[j], lane + j * TEAM, p.F);
    }
    hc.template load<T>(p.x, p.ldx, row + step, lane, TEAM, nchunks, more);
    yc.template load<T>(p.dy, p.lddy, row + step, lane, TEAM, nchunks, more);
    rstd_next = more ? p.rstd_in[row + step] : 0.f;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      float w[V];
      gain.get(j, lane, w);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        dg[j][i] = fmaf(t[j][i], h[j][i] * rstd, dg[j][i]);
        t[j][i] *= w[i];
        dot = fmaf(t[j][i], h[j][i], dot);
      }
    }
    dot = team_sum<TEAM>(dot, red, flip);
    const float k = rstd * rstd * dot * inv_f;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = lane + j * TEAM;
      const bool here = live && c < nchunks;
      float res[V];
      if (RES) {
        unpack16(rc.v[j], res, T());
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) res[i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) t[j][i] = fmaf(rstd, t[j][i] - h[j][i] * k, res[i]);
      clear_padding<V>(t[j], c, p.F);
      if (here && p.y) *reinterpret_cast<uint4 *>((T *)p.y + row * p.ldy + (int64_t)c * V) = pack16(t[j], T());
    }
    if (p.y8) quantize_row<T, TEAM, NCH, V>(p, row, lane, t);
    if (RES) rc.template load<T>(p.r, p.ldr, row + step, lane, TEAM, nchunks, more);
  }
  if (!p.dgain_part) return;
  // the teams of a warp add their columns by shuffles, the warps of the CTA one after the other (a fixed order), then the
  // CTA writes its line
  if (TEAM < 32) {
#pragma unroll
    for (int j = 0; j < NCH; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int o = TEAM; o < 32; o <<= 1) dg[j][i] += __shfl_xor_sync(0xFFFFFFFFu, dg[j][i], o);
  }
  constexpr int TURN = TEAM < 32 ? 32 : TEAM;      // threads that write at once
  for (int turn = 0; turn < threads_per_cta<TEAM>() / TURN; ++turn) {
    if ((int)threadIdx.x / TURN == turn && (int)threadIdx.x % TURN < TEAM) {
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
        const int c = lane + j * TEAM;
        if (c < nchunks) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int col = c * V + i;
            gsum[col] = (turn ? gsum[col] : 0.f) + dg[j][i];
          }
        }
      }
    }
    __syncthreads();
  }
  for (int col = threadIdx.x; col < p.F; col += blockDim.x) p.dgain_part[(int64_t)blockIdx.x * p.F + col] = gsum[col];
  if (!p.dgain) return;
  // the CTA that comes last adds all lines: in slices of every so many lines, slices ascending, whichever CTA it is
  __shared__ int last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.arrived, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  const int wide = min((p.F + 31) / 32 * 32, threads_per_cta<TEAM>()), slices = threads_per_cta<TEAM>() / wide, slice = (int)threadIdx.x / wide;
  for (int col = (int)threadIdx.x % wide; col - (int)threadIdx.x % wide < p.F; col += wide) {
    float v = 0.f;
    if (slice < slices && col < p.F) {
      for (int i = slice; i < (int)gridDim.x; i += slices * kLines) {
        float x[kLines];
#pragma unroll
        for (int u = 0; u < kLines; ++u) x[u] = i + u * slices < (int)gridDim.x ? __ldcg(p.dgain_part + (int64_t)(i + u * slices) * p.F + col) : 0.f;
#pragma unroll
        for (int u = 0; u < kLines; ++u) v += x[u];
      }
    }
    __syncthreads();
    gsum[threadIdx.x] = v;
    __syncthreads();
    if (slice == 0 && col < p.F) {
      for (int i = 1; i < slices; ++i) v += gsum[i * wide + threadIdx.x];
      p.dgain[col] = v;
    }
  }
  if (threadIdx.x == 0) *p.arrived = 0;
}

// dgain[c] = sum over the CTAs of the backward kernel, in their order within each of the 32 slices, slices ascending
__global__ void __launch_bounds__(1024) dgain_reduce_kernel(const float *__restrict__ part, int parts, int F,
                                                            float *__restrict__ dgain) {
  __shared__ float s[32][33];
  const int col = blockIdx.x * 32 + threadIdx.x;
  float v = 0.f;
  if (col < F)
    for (int i = threadIdx.y; i < parts; i += 32) v += part[(int64_t)i * F + col];
  s[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  v = s[threadIdx.x][threadIdx.y];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  if (threadIdx.x == 0 && blockIdx.x * 32 + threadIdx.y < F) dgain[blockIdx.x * 32 + threadIdx.y] = v;
}

constexpr int kMaxF = 16384;
// Lines of gain-gradient partials that the workspace has room for: enough for every resident CTA of narrow rows, two an SM
// of the widest.
int max_parts(int F) {
  const int64_t lines = ((int64_t)8 << 20) / ((int64_t)F * 4);
  return (int)(lines < 148 * 2 ? 148 * 2 : lines > 148 * 32 ? 148 * 32 : lines);
}

// CTAs of a kernel that one SM holds
template <typename K> int resident(K kernel, int threads, size_t smem) {
  int n = 0;
  return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) == cudaSuccess && n > 0 ? n : 1;
}

template <typename T, int TEAM, int NCH, bool RES> int launch_fwd_as(const NormParams &p, int sms, cudaStream_t st) {
  constexpr int threads = threads_per_cta<TEAM>(), rows = rows_per_cta<TEAM>() * rows_a_trip<TEAM, NCH, RES>();
  static const int most = resident(norm_fwd_kernel<T, TEAM, NCH, RES>, threads, 0);
  const int64_t ctas = (p.rows + rows - 1) / rows, all = (int64_t)sms * most;
  norm_fwd_kernel<T, TEAM, NCH, RES><<<(unsigned)(ctas < all ? ctas : all), threads, 0, st>>>(p);
  VARCO_KERNEL_LAUNCHED();
  return VARCO_OK;
}
template <typename T, int TEAM, int NCH> int launch_fwd(const NormParams &p, int sms, cudaStream_t st) {
  return p.r ? launch_fwd_as<T, TEAM, NCH, true>(p, sms, st) : launch_fwd_as<T, TEAM, NCH, false>(p, sms, st);
}
// TEAM lanes with as many chunks each as the row needs, at most MAX
template <typename T, int TEAM, int MAX> int launch_fwd_lanes(const NormParams &p, int nc, int sms, cudaStream_t st) {
  if constexpr (MAX >= 2) {
    if (nc <= TEAM * (MAX - 1)) return launch_fwd_lanes<T, TEAM, MAX - 1>(p, nc, sms, st);
  }
  return launch_fwd<T, TEAM, MAX>(p, sms, st);
}

struct GainGrad {
  float *out, *part;         // dgain (or nullptr) and the workspace's lines
  unsigned *arrived;         // in the workspace's status block, zeroed with it
};
// Whether the backward's last CTA adds the gain gradient's lines itself: while that takes it two rounds of loads.  It costs the GPU
// up to 1 us and saves the host a launch, which is what a small call waits for.  Last CTA against a second kernel: 2000 x 64, one
// round: calls 6.2 and 8.2 us (GPU 5.0 and 4.7); 1000 x 100, two: 7.2 and 8.2 (6.0 and 5.0); 8000 x 64, four: 9.2 and 9.2 (7.7 and
// 5.8).
bool last_adds(int64_t lines, int F, int threads) {
  const int cols = (F + 31) / 32 * 32, wide = cols < threads ? cols : threads, slices = threads / wide;
  return lines > 1 && (cols + wide - 1) / wide * ((lines + slices * kLines - 1) / (slices * kLines)) <= 2;
}
template <typename T, int TEAM, int NCH, bool RES> int launch_bwd_as(const NormParams &p, const GainGrad &d, int sms, cudaStream_t st) {
  constexpr int threads = threads_per_cta<TEAM>(), rows = rows_per_cta<TEAM>();
  const int64_t row = round_up64(p.F, ElemTraits<T>::kVec);
  const size_t smem = d.out ? (size_t)(row > threads ? row : threads) * 4 : 0;
  if (smem > 40 * 1024)
    VARCO_CUDA_CHECK(cudaFuncSetAttribute(norm_bwd_kernel<T, TEAM, NCH, RES>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  static const int most = resident(norm_bwd_kernel<T, TEAM, NCH, RES>, threads, TEAM * NCH * 16);
  int64_t all = (int64_t)sms * most;
  if (d.out && all > max_parts(p.F)) all = max_parts(p.F);
  const int64_t ctas = (p.rows + rows - 1) / rows;
  const unsigned grid = (unsigned)(ctas < all ? ctas : all);
  NormParams q = p;
  q.dgain_part = !d.out ? nullptr : grid == 1 ? d.out : d.part;
  const bool last = last_adds(grid, p.F, threads);
  if (d.out && last) q.dgain = d.out, q.arrived = d.arrived;
  norm_bwd_kernel<T, TEAM, NCH, RES><<<grid, threads, smem, st>>>(q);
  VARCO_KERNEL_LAUNCHED();
  if (d.out && grid > 1 && !last) {
    dgain_reduce_kernel<<<(p.F + 31) / 32, dim3(32, 32), 0, st>>>(d.part, (int)grid, p.F, d.out);
    VARCO_KERNEL_LAUNCHED();
  }
  return VARCO_OK;
}
template <typename T, int TEAM, int NCH> int launch_bwd(const NormParams &p, const GainGrad &d, int sms, cudaStream_t st) {
  return p.r ? launch_bwd_as<T, TEAM, NCH, true>(p, d, sms, st) : launch_bwd_as<T, TEAM, NCH, false>(p, d, sms, st);
}

// Rows longer than lanes of a warp hold take a CTA that is just wide enough; F(TEAM, NCH) launches.
#define VARCO_NORM_CTA(F, nc)                                   \
  if (nc <= 64) return F(64, 1);                                \
  if (nc <= 96) return F(96, 1);                                \
  if (nc <= 128) return F(128, 1);                              \
  if (nc <= 192) return F(96, 2);                               \
  if (nc <= 256) return F(128, 2);                              \
  if (nc <= 384) return F(192, 2);                              \
  if (nc <= 512) return F(256, 2);                              \
  if (nc <= 768) return F(384, 2);                              \
  if (nc <= 1024) return F(512, 2);                             \
  if (nc <= 2048) return F(1024, 2);                            \
  if constexpr (sizeof(T) == 4) return F(1024, 4);              \
  return VARCO_UNSUPPORTED;

// Team and chunks a lane by the number of chunks of a row (GB/s of rows with residual and 8-bit output unless said).  Several
// chunks a lane fill the team better where the row is ragged (bf16 300 wide: 16 x 3 5450, 32 x 2 3899; 602: 16 x 5 5467, a CTA
// of 96 4600) and keep more loads on their way where there is no residual (602: 16 x 5 5696, a CTA of 96 3980; 1024: 32 x 4
// 6091, a CTA of 128 4897); where the row fits, one or two are better (256: 16 x 2 6137, 8 x 4 5947; 512: 32 x 2 6131, 16 x 4
// 5804; 1024: a CTA of 128 6160, 32 x 4 5816).  The borders, with a residual:
//   bf16 58 chunks: 16 x 4 5265, 32 x 2 5191;  60: 5385, 5408;  62: 5322, 5389.  fp32 58: 5577, 5231;  64: 5966, 5911
//   bf16 104 chunks: 32 x 4 5435, a CTA of 128 5305;  112: 5491, 5835;  120: 5429, 5684;  past 128, a CTA of 192: 130: 32 x 5 5225,
//   4926;  144: 5513, 5424.  fp32 104: 5677, 5424;  112: 5738, 5781;  119: 5455, 5782;  130: 5424, 5768;  160: 5757, 6133
template <typename T> int forward(const NormParams &p, int sms, cudaStream_t st) {
#define F(TEAM, NCH) launch_fwd<T, TEAM, NCH>(p, sms, st)
  constexpr int V = ElemTraits<T>::kVec;
  const int nc = (p.F + V - 1) / V;
  if (nc <= 2 && !(sizeof(T) == 4 && p.y8)) return F(2, 1);   // 16 bytes of an 8-bit row are four fp32 chunks: four lanes
  if (nc <= 4) return F(4, 1);
  if (p.r && nc <= 16) return launch_fwd_lanes<T, 8, 2>(p, nc, sms, st);
  if (p.r && nc <= 32) return launch_fwd_lanes<T, 16, 2>(p, nc, sms, st);
  if (sizeof(T) == 2 && p.r && nc >= 60 && nc <= 64) return F(32, 2);
  if (!p.r || nc < 112 || (sizeof(T) == 2 && nc > 128)) {
    if (nc <= 40) return launch_fwd_lanes<T, 8, 5>(p, nc, sms, st);
    if (nc <= 80) return launch_fwd_lanes<T, 16, 5>(p, nc, sms, st);
    if (nc <= 160) return launch_fwd_lanes<T, 32, 5>(p, nc, sms, st);
  }
  VARCO_NORM_CTA(F, nc)
#undef F
}

// The backward holds a row three times (row, gradient, gain gradient): lanes take few values.  bf16 with a residual: one chunk
// (256 wide: 32 x 1 5927, 16 x 2 4000; 512: a CTA of 64 5934, 32 x 2 3495); without one, and fp32, two (bf16 256: 16 x 2 5759,
// 32 x 1 5097; fp32 128: 16 x 2 6271, 32 x 1 6026).  CTAs of bf16 rows up to 4096 wide are faster with one chunk a thread than with
// two (2048: 348 against 463 us).  CTAs of 1024 threads have 64 registers a thread: rows past 8192
// columns spill (16,384 wide: bf16 4.2, fp32 3.5 TB/s).
template <typename T> int backward(const NormParams &p, const GainGrad &d, int sms, cudaStream_t st) {
#define F(TEAM, NCH) launch_bwd<T, TEAM, NCH>(p, d, sms, st)
  constexpr int V = ElemTraits<T>::kVec;
  const int nc = (p.F + V - 1) / V;
  if (nc <= 4) return F(4, 1);
  if (nc <= 8) return F(8, 1);
  if constexpr (sizeof(T) == 2) {
    if (p.r) {
      if (nc <= 16) return F(16, 1);
      if (nc <= 32) return F(32, 1);
    }
  }
  if (nc <= 16) return F(8, 2);
  if (nc <= 32) return F(16, 2);
  if constexpr (sizeof(T) == 2) {
    if (nc > 128 && nc <= 192) return F(192, 1);
    if (nc > 192 && nc <= 256) return F(256, 1);
    if (nc > 256 && nc <= 384) return F(384, 1);
    if (nc > 384 && nc <= 512) return F(512, 1);
  }
  VARCO_NORM_CTA(F, nc)
#undef F
}

int check(const varco_norm_desc_t *d) {
  if (!d || d->rows < 0 || d->F < 1 || !dtype_ok(d->dtype) || !(d->eps > 0.f)) return VARCO_INVALID_ARG;
  return d->F > kMaxF ? VARCO_UNSUPPORTED : VARCO_OK;
}
bool eight_ok(const varco_norm_desc_t *d, const void *y8, const float *scales) {
  if (!y8) return !scales;
  return scales && (reinterpret_cast<uintptr_t>(scales) & 3u) == 0 && matrix_ok(y8, d->ld8, d->F, 1) && d->lds >= d->rows;
}

}  // namespace

// Lines for every width up to F: max_parts rounds down, so a narrower row can need some bytes more than F itself does (512
// wide: 8 MB, 1000 wide: 8 MB - 608 bytes).
size_t vops::norm_scratch_bytes(int F) {
  const size_t most = (size_t)148 * 32 * F * 4, all = (size_t)8 << 20, least = (size_t)148 * 2 * F * 4;
  return most < all ? most : least > all ? least : all;
}

extern "C" {

int varco_norm_fwd(const varco_norm_desc_t *d, const void *X, const void *R, const float *gain, void *H, void *Y,
                   void *Y8, float *scales, float *rstd, void *stream) {
  if (int rc = check(d)) return rc;
  if (d->rows == 0) return VARCO_OK;
  const int es = elem_size(d->dtype);
  if (!matrix_ok(X, d->ldx, d->F, es) || (R && !matrix_ok(R, d->ldr, d->F, es)) || (H && !matrix_ok(H, d->ldh, d->F, es)) ||
      (Y && !matrix_ok(Y, d->ldy, d->F, es)) || !eight_ok(d, Y8, scales) || (!Y && !Y8 && !H && !rstd))
    return VARCO_INVALID_ARG;
  NormParams p = {};
  p.rows = d->rows, p.F = d->F, p.eps = d->eps;
  p.x = X, p.r = R, p.gain = gain, p.h = H, p.y = Y, p.y8 = (uint8_t *)Y8, p.scales = scales, p.rstd = rstd;
  p.ldx = d->ldx, p.ldr = d->ldr, p.ldh = d->ldh, p.ldy = d->ldy, p.ld8 = d->ld8, p.lds = d->lds;
  const int sms = sm_count();
  if (sms <= 0) return VARCO_CUDA;
  return d->dtype == VARCO_F32 ? forward<float>(p, sms, (cudaStream_t)stream) : forward<__nv_bfloat16>(p, sms, (cudaStream_t)stream);
}

int varco_norm_bwd(const varco_norm_desc_t *d, const void *dY, const void *H, const float *rstd, const float *gain,
                   const void *dRes, void *dX, void *dX8, float *scales, float *dgain, void *workspace, size_t ws_bytes,
                   void *stream) {
  if (int rc = check(d)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (d->rows == 0) {
    if (dgain) VARCO_CUDA_CHECK(cudaMemsetAsync(dgain, 0, (size_t)d->F * 4, st));
    return VARCO_OK;
  }
  const int es = elem_size(d->dtype);
  if (!matrix_ok(dY, d->ldy, d->F, es) || !matrix_ok(H, d->ldh, d->F, es) || !rstd || (dRes && !matrix_ok(dRes, d->ldr, d->F, es)) ||
      (dX && !matrix_ok(dX, d->ldx, d->F, es)) || !eight_ok(d, dX8, scales) || (!dX && !dX8 && !dgain))
    return VARCO_INVALID_ARG;
  float *part = nullptr;
  unsigned *arrived = nullptr;
  if (dgain) {
    if (!workspace) return VARCO_INVALID_ARG;
    if (ws_bytes < 256 + kStatusBytes + (size_t)max_parts(d->F) * d->F * 4) return VARCO_WORKSPACE_TOO_SMALL;
    arrived = reinterpret_cast<unsigned *>(ws_align(workspace) + 160);
    part = reinterpret_cast<float *>(ws_align(workspace) + kStatusBytes);
  }
  NormParams p = {};
  p.rows = d->rows, p.F = d->F;
  p.x = H, p.dy = dY, p.r = dRes, p.rstd_in = rstd, p.gain = gain, p.y = dX, p.y8 = (uint8_t *)dX8, p.scales = scales;
  p.ldx = d->ldh, p.lddy = d->ldy, p.ldr = d->ldr, p.ldy = d->ldx, p.ld8 = d->ld8, p.lds = d->lds;
  const int sms = sm_count();
  if (sms <= 0) return VARCO_CUDA;
  const GainGrad g = {dgain, part, arrived};
  return d->dtype == VARCO_F32 ? backward<float>(p, g, sms, st) : backward<__nv_bfloat16>(p, g, sms, st);
}

}  // extern "C"
