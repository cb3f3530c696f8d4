// The norm over all gradients and the clipped step.
//
//   norm = sqrt(sum over all tensors of g^2);  c = min(1, max_norm / (norm + eps))
//   grad_clip   g <- c g                 clip_step   w <- w - lr c g, and the bf16 copy of w that the layers read
//
// One cooperative launch: every CTA adds the squares of its chunks and leaves one 64-bit partial; behind a barrier over
// the grid every CTA adds all partials in the same order -- no atomics on values, the same bits in every run -- and goes
// over its chunks again, last ones first, since those are still in L2.  The tensors' table travels in the kernel's
// parameters: no copy to the device, nothing to keep between calls.  More tensors than a table holds take the two
// passes as separate launches.
//
// Squares leave the 32-bit range below 1e-19 and above 1.8e19.  Sixteen squares are added in 32 bits; where that sum is
// not well inside the range, the same sixteen are added again in 64 bits.  So the norm is right whenever it is itself a
// 32-bit number, at one comparison per sixteen elements.
//
// Bound: HBM (gradients twice, unless they stay in L2), or the launch when the model is small.  302M weights with bf16 copies
// in 216 tensors: 760 us (18 bytes a weight at 7.1 TB/s, some of them from L2; two launches forwards took 777); nine tensors
// of 0.2M weights: 6.0 us.  The norm alone: 176 us (6.8 TB/s, some from L2) and 4.8; scaling in place 628 and 6.6.
#include <algorithm>

#include "ops_common.cuh"

namespace {

using namespace vops;

constexpr int kThreads = 256;
constexpr int kMaxCtas = 148 * 8;          // partials of one group of tensors
constexpr int kGroup = 800;                // tensors of the largest table: 32,000 bytes of parameters
constexpr int kMaxGroups = 21;             // 16,800 tensors
constexpr long long kSpinClocks = 2000000000ll;   // about one second of SM clocks

enum Mode { kNorm = 0, kClip = 1, kStep = 2 };
enum Pass { kBoth = 0, kPartials = 1, kApply = 2 };

struct Entry {
  void *g;
  float *w;
  __nv_bfloat16 *copy;
  int64_t count;
  int first_chunk;                         // of the launch's chunks
  int bf16;                                // type of g
};
template <int CAP> struct Table {
  Entry e[CAP];
};
struct Args {
  int num, chunks;                         // entries of the table, chunks of all of them
  int chunk;                               // elements of one chunk, a multiple of kThreads * 8
  int pass, parts;                         // partials in all (pass kApply), where this launch's begin (kPartials)
  float max_norm, eps, lr;
  float *norm;
  double *part;
  unsigned *barrier;                       // [arrived, generation]
  int *err;
};

__device__ __forceinline__ int find(const Entry *e, int num, int chunk) {
  int lo = 0, hi = num - 1;                // last entry with first_chunk <= chunk
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (e[mid].first_chunk <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double s[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
  __syncthreads();
  double r = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) r += s[w];
  return r;
}

template <int N> __device__ __forceinline__ double squares(const float (&f)[N]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s = fmaf(f[i], f[i], s);
  if (s > 1e-25f && s < 1e30f) return (double)s;   // false for NaN and for an overflow too
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < N; ++i) d = fma((double)f[i], (double)f[i], d);
  return d;
}

// elements before the first 16-byte boundary
__device__ __forceinline__ int to_boundary(const void *p, int es) { return (int)((16u - ((uint32_t)(uintptr_t)p & 15u)) & 15u) / es; }

// `n` elements of one chunk from `src`
template <typename T> __device__ double chunk_squares(const T *src, int n) {
  constexpr int V = ElemTraits<T>::kVec, U = 16 / V;      // 16 elements a thread and trip
  double acc = 0.0;
  float f[16];
  const int head = min(n, to_boundary(src, sizeof(T)));
#pragma unroll
  for (int u = 0; u < 16; ++u) f[u] = 0.f;
  if ((int)threadIdx.x < head) f[0] = ElemTraits<T>::to_f(src[threadIdx.x]);
  const int nv = (n - head) / V, tail = head + nv * V + (int)threadIdx.x;
  if (tail < n) f[1] = ElemTraits<T>::to_f(src[tail]);   // fewer than V at either end
  acc += squares(f);
  const uint4 *v4 = reinterpret_cast<const uint4 *>(src + head);
  for (int i = threadIdx.x; i < nv; i += kThreads * U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (i + u * kThreads < nv) v = __ldg(v4 + i + u * kThreads);
      float x[V];
      unpack16(v, x, T());
#pragma unroll
      for (int j = 0; j < V; ++j) f[u * V + j] = x[j];
    }
    acc += squares(f);
  }
  return acc;
}

// All CTAs of the grid have written what they wrote before it.  Bounded: false (and the status word set) when the others do
// not come within a second, which a cooperative launch rules out as long as the counters are what the last call left: a
// workspace that was not zeroed, or whose call gave up, has to be zeroed (again).
__device__ bool grid_barrier(unsigned *bar, int *err) {
  __shared__ int ok;
  __syncthreads();
  if (threadIdx.x == 0) {
    volatile unsigned *gen = bar + 1;
    const unsigned g = *gen;
    __threadfence();
    ok = 1;
    if (atomicAdd(bar, 1u) == gridDim.x - 1) {
      *bar = 0;
      __threadfence();
      *gen = g + 1;
    } else {
      const long long t0 = clock64();
      while (*gen == g) {
        if (clock64() - t0 > kSpinClocks) {
          ok = 0;
          atomicCAS(err, 0, 31);
          break;
        }
        __nanosleep(32);
      }
    }
    __threadfence();
  }
  __syncthreads();
  return ok != 0;
}

// a NaN norm gives a NaN factor, an infinite one zero
__device__ __forceinline__ float clip_factor(float norm, float max_norm, float eps) {
  const float c = max_norm / (norm + eps);
  return c > 1.f ? 1.f : c;
}

template <typename T> __device__ void scale_chunk(T *g, int n, float c) {
  constexpr int V = ElemTraits<T>::kVec;
  const int head = min(n, to_boundary(g, sizeof(T)));
  const int nv = (n - head) / V, tail = head + nv * V + (int)threadIdx.x;
  if ((int)threadIdx.x < head) g[threadIdx.x] = ElemTraits<T>::from_f(ElemTraits<T>::to_f(g[threadIdx.x]) * c);
  if (tail < n) g[tail] = ElemTraits<T>::from_f(ElemTraits<T>::to_f(g[tail]) * c);
  uint4 *v4 = reinterpret_cast<uint4 *>(g + head);
  for (int i = threadIdx.x; i < nv; i += kThreads * 4) {
    uint4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u * kThreads < nv) v[u] = v4[i + u * kThreads];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i + u * kThreads < nv) {
        float f[V];
        unpack16(v[u], f, T());
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] *= c;
        v4[i + u * kThreads] = pack16(f, T());
      }
    }
  }
}

template <typename T> __device__ __forceinline__ void step_one(const T *g, float *w, __nv_bfloat16 *copy, int i, float k) {
  const float x = fmaf(-k, ElemTraits<T>::to_f(g[i]), w[i]);
  w[i] = x;
  if (copy) copy[i] = __float2bfloat16_rn(x);
}
template <typename T> __device__ __forceinline__ void load8(const T *g, float (&f)[8]) {
  if (sizeof(T) == 4) {
    float a[4], b[4];
    unpack16(reinterpret_cast<const uint4 *>(g)[0], a, 0.f);
    unpack16(reinterpret_cast<const uint4 *>(g)[1], b, 0.f);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = a[j], f[4 + j] = b[j];
  } else {
    unpack16(*reinterpret_cast<const uint4 *>(g), f, __nv_bfloat16());
  }
}

template <typename T> __device__ void step_chunk(const T *g, float *w, __nv_bfloat16 *copy, int n, float k) {
  // elements in front of the place where all three are on a 16-byte boundary, if there is one
  int head = copy ? to_boundary(copy, 2) : sizeof(T) == 2 ? to_boundary(g, 2) : to_boundary(w, 4);
  head = min(head, n);
  const bool together = ((reinterpret_cast<uintptr_t>(g + head) | reinterpret_cast<uintptr_t>(w + head)) & 15u) == 0 &&
                        (!copy || (reinterpret_cast<uintptr_t>(copy + head) & 15u) == 0);
  if (together) {
    const int nv = (n - head) / 8, tail = head + nv * 8 + (int)threadIdx.x;
    if ((int)threadIdx.x < head) step_one(g, w, copy, threadIdx.x, k);
    if (tail < n) step_one(g, w, copy, tail, k);
    for (int i = threadIdx.x; i < nv; i += kThreads) {
      const int at = head + i * 8;
      float f[8], x[8];
      load8(g + at, f);
      load8(w + at, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = fmaf(-k, f[j], x[j]);
      float4 *wp = reinterpret_cast<float4 *>(w + at);
      wp[0] = make_float4(x[0], x[1], x[2], x[3]);
      wp[1] = make_float4(x[4], x[5], x[6], x[7]);
      if (copy) *reinterpret_cast<uint4 *>(copy + at) = pack16(x, __nv_bfloat16());
    }
  } else {
    for (int i = threadIdx.x; i < n; i += kThreads * 8) {
      float f[8], x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i + u * kThreads < n) f[u] = ElemTraits<T>::to_f(g[i + u * kThreads]), x[u] = w[i + u * kThreads];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i + u * kThreads < n) {
          x[u] = fmaf(-k, f[u], x[u]);
          w[i + u * kThreads] = x[u];
          if (copy) copy[i + u * kThreads] = __float2bfloat16_rn(x[u]);
        }
    }
  }
}

template <int CAP, int MODE>
__global__ void __launch_bounds__(kThreads) clip_kernel(const __grid_constant__ Table<CAP> t, const __grid_constant__ Args a) {
  int parts = a.parts;
  if (a.pass != kApply) {
    double acc = 0.0;
    for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
      const Entry &e = t.e[find(t.e, a.num, c)];
      const int64_t at = (int64_t)(c - e.first_chunk) * a.chunk;
      const int n = (int)min((int64_t)a.chunk, e.count - at);
      acc += e.bf16 ? chunk_squares((const __nv_bfloat16 *)e.g + at, n) : chunk_squares((const float *)e.g + at, n);
    }
    acc = block_sum(acc);
    if (threadIdx.x == 0) a.part[(a.pass == kPartials ? parts : 0) + blockIdx.x] = acc;
    if (a.pass == kPartials) return;
    if (!grid_barrier(a.barrier, a.err)) return;
    parts = gridDim.x;
  }
  if (MODE == kNorm && blockIdx.x > 0) return;
  double v = 0.0;
  for (int i = threadIdx.x; i < parts; i += kThreads) v += __ldcg(a.part + i);
  const float total = (float)sqrt(block_sum(v));
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.norm) *a.norm = total;
  if (MODE == kNorm) return;
  const float c = clip_factor(total, a.max_norm, a.eps);
  if (MODE == kClip && c == 1.f) return;   // nothing to scale: the gradients stay as they are, bit for bit
  for (int b = blockIdx.x; b < a.chunks; b += gridDim.x) {
    const int k = a.chunks - 1 - b;
    const Entry &e = t.e[find(t.e, a.num, k)];
    const int64_t at = (int64_t)(k - e.first_chunk) * a.chunk;
    const int n = (int)min((int64_t)a.chunk, e.count - at);
    if (MODE == kClip) {
      if (e.bf16) scale_chunk((__nv_bfloat16 *)e.g + at, n, c);
      else scale_chunk((float *)e.g + at, n, c);
    } else {
      __nv_bfloat16 *copy = e.copy ? e.copy + at : nullptr;
      if (e.bf16) step_chunk((const __nv_bfloat16 *)e.g + at, e.w + at, copy, n, c * a.lr);
      else step_chunk((const float *)e.g + at, e.w + at, copy, n, c * a.lr);
    }
  }
}

struct Lists {
  void *const *g;
  const int64_t *count;
  const int32_t *dtype;
  float *const *w;
  void *const *copies;
  int32_t num;
};

// Chunk size: small enough that a small model still spreads over the SMs, large enough that finding a chunk's tensor
// costs little.
int chunk_size(int64_t elements) {
  if (elements <= (int64_t)148 * 8 * 2048) return 2048;
  return elements <= (int64_t)148 * 8 * 16384 ? 8192 : 32768;
}

// tensors [first, last) as a launch table
template <int CAP> int make_table(Table<CAP> &t, Args &a, const Lists &l, int32_t first, int32_t last) {
  int64_t elements = 0, chunks = 0;
  for (int32_t i = first; i < last; ++i) elements += l.count[i];
  a.chunk = chunk_size(elements);
  a.num = 0;
  for (int32_t i = first; i < last; ++i) {
    if (l.count[i] == 0) continue;
    Entry &e = t.e[a.num++];
    e.g = l.g[i];
    e.count = l.count[i];
    e.bf16 = l.dtype[i] == VARCO_BF16;
    e.w = l.w ? l.w[i] : nullptr;
    e.copy = l.copies ? (__nv_bfloat16 *)l.copies[i] : nullptr;
    e.first_chunk = (int)chunks;
    chunks += (l.count[i] + a.chunk - 1) / a.chunk;
  }
  if (chunks > INT32_MAX) return VARCO_UNSUPPORTED;
  a.chunks = (int)chunks;
  return VARCO_OK;
}

// one launch over tensors [first, last); *parts grows by the partials that it leaves
template <int CAP, int MODE> int launch(const Lists &l, Args &a, int32_t first, int32_t last, int *parts, int sms, cudaStream_t st) {
  Table<CAP> t;
  if (int rc = make_table(t, a, l, first, last)) return rc;
  static const int resident = [] {
    int n = 0;
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, clip_kernel<CAP, MODE>, kThreads, 0) == cudaSuccess ? n : 0;
  }();
  if (resident <= 0) return VARCO_CUDA;
  const int most = std::min(sms * std::min(resident, 8), kMaxCtas);
  int grid = std::max(1, std::min(a.chunks, most));
  if (a.pass == kApply && MODE == kNorm) grid = 1;
  a.parts = *parts;
  void *args[] = {&t, &a};
  if (a.pass == kBoth)
    VARCO_CUDA_CHECK(cudaLaunchCooperativeKernel((const void *)clip_kernel<CAP, MODE>, dim3(grid), dim3(kThreads), args, 0, st));
  else
    VARCO_CUDA_CHECK(cudaLaunchKernel((const void *)clip_kernel<CAP, MODE>, dim3(grid), dim3(kThreads), args, 0, st));
  VARCO_KERNEL_LAUNCHED();
  if (a.pass == kPartials) *parts += grid;
  return VARCO_OK;
}

bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <int MODE> int run(const Lists &l, float lr, float max_norm, float eps, float *norm, void *ws, size_t ws_bytes, cudaStream_t st) {
  if (l.num < 0 || (l.num > 0 && (!l.g || !l.count || !l.dtype || (MODE == kStep && !l.w))) || !ws || !aligned_to(norm, 4)) return VARCO_INVALID_ARG;
  if (MODE != kNorm && (!(max_norm >= 0.f) || !(eps > 0.f) || !(lr == lr))) return VARCO_INVALID_ARG;
  if (l.num > kGroup * kMaxGroups) return VARCO_UNSUPPORTED;
  if (ws_bytes < 256 + kStatusBytes + vops::clip_scratch_bytes()) return VARCO_WORKSPACE_TOO_SMALL;
  for (int32_t i = 0; i < l.num; ++i) {
    if (l.count[i] < 0 || !dtype_ok(l.dtype[i])) return VARCO_INVALID_ARG;
    if (l.count[i] == 0) continue;
    if (!l.g[i] || !aligned_to(l.g[i], l.dtype[i] == VARCO_F32 ? 4 : 2)) return VARCO_INVALID_ARG;
    if (MODE == kStep && (!l.w[i] || !aligned_to(l.w[i], 4) || (l.copies && !aligned_to(l.copies[i], 2)))) return VARCO_INVALID_ARG;
  }
  const int sms = sm_count();
  if (sms <= 0) return VARCO_CUDA;
  char *base = ws_align(ws);
  Args a = {};
  a.max_norm = max_norm, a.eps = eps, a.lr = lr, a.norm = norm;
  a.err = reinterpret_cast<int *>(base);
  a.barrier = reinterpret_cast<unsigned *>(base + 128);           // in the status block, zeroed with it
  a.part = reinterpret_cast<double *>(base + kStatusBytes);
  int parts = 0;
  // the table's size is what a launch copies: a small model takes the small one
  if (l.num <= 32) return launch<32, MODE>(l, a, 0, l.num, &parts, sms, st);
  if (l.num <= 256) return launch<256, MODE>(l, a, 0, l.num, &parts, sms, st);
  if (l.num <= kGroup) return launch<kGroup, MODE>(l, a, 0, l.num, &parts, sms, st);
  for (int pass = kPartials; pass <= kApply; ++pass) {
    a.pass = pass;
    for (int32_t first = 0; first < l.num; first += kGroup) {
      if (int rc = launch<kGroup, MODE>(l, a, first, std::min(l.num, first + kGroup), &parts, sms, st)) return rc;
      if (MODE == kNorm && pass == kApply) break;
    }
  }
  return VARCO_OK;
}

}  // namespace

size_t vops::clip_scratch_bytes() { return (size_t)kMaxCtas * kMaxGroups * sizeof(double); }

extern "C" {

int varco_grad_norm(void *const *grads, const int64_t *counts, const int32_t *dtypes, int32_t num, float *norm, void *workspace,
                    size_t ws_bytes, void *stream) {
  if (!norm) return VARCO_INVALID_ARG;
  return run<kNorm>({grads, counts, dtypes, nullptr, nullptr, num}, 0.f, 0.f, 1.f, norm, workspace, ws_bytes, (cudaStream_t)stream);
}

int varco_grad_clip(void *const *grads, const int64_t *counts, const int32_t *dtypes, int32_t num, float max_norm, float eps,
                    float *norm, void *workspace, size_t ws_bytes, void *stream) {
  return run<kClip>({grads, counts, dtypes, nullptr, nullptr, num}, 0.f, max_norm, eps, norm, workspace, ws_bytes, (cudaStream_t)stream);
}

int varco_clip_step(void *const *grads, const int64_t *counts, const int32_t *dtypes, float *const *weights, void *const *copies,
                    int32_t num, float lr, float max_norm, float eps, float *norm, void *workspace, size_t ws_bytes, void *stream) {
  return run<kStep>({grads, counts, dtypes, weights, copies, num}, lr, max_norm, eps, norm, workspace, ws_bytes, (cudaStream_t)stream);
}

}  // extern "C"
