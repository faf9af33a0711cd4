// Global L2 norm over a list of tensors and clipping by it, the clip of an aggregated gradient:
//   s = sum over tensors and elements of x^2,   f = min(1, max_norm / sqrt(s)) (1 where s = 0),   y = f x.
// Both kernels are bound by memory: one element is one multiply-add.  The list travels in the kernel's parameters, so a
// call copies nothing to the device beforehand.  The bf16 gradients of BERT-Large (289 tensors, 667 MB): norm 99 us
// (6.7 TB/s), scaling 211 us (6.3 TB/s).
//
// Work is cut into chunks of 32 KB that never cross a tensor, and block b takes the chunks b, b + grid, ...; every
// block's sum is written to its own word and the words are added in one order, so a sum does not depend on timing.
#include "dp_chain.cuh"
#include "dp_clip.cuh"
#include "dp_internal.h"

namespace dpk {

constexpr int kNormThreads = 256;
// 16-byte loads in flight per thread, and blocks per SM.  Measured on the bf16 gradients of BERT-Large (667 MB read twice and
// written once, the three kernels together): 4 x 8 357 us, 4 x 16 337, 8 x 8 327, 8 x 12 321, 16 x 8 369 (registers).
constexpr int kNormVecs = 8, kNormBlocks = 12;
constexpr int kGroup = 32;                                          // squares at most that are summed in fp32
constexpr int kNormMaxBlocks = 8192;                                // partial sums that the workspace holds
constexpr size_t kNormWorkspace = kNormMaxBlocks * sizeof(double);

// Up to N tensors of one launch.  chunk0[k] = index of tensor k's first chunk.
template <int N>
struct TensorSet {
  const void* in[N];
  void* out[N];
  long long size[N];
  unsigned int chunk0[N + 1];
  int n;
};

template <typename T> struct Vec16;
template <> struct Vec16<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void unpack(const uint4& u, float* x) {
    x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ void store(float* p, float x) { *p = x; }
};
template <> struct Vec16<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void unpack(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(w[k] << 16);
      x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
      w[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
};

// sum of x[0..n)^2, in fp32 where that is safe: a sum that overflowed, or is so small that squares may have been lost
// below fp32's range, is formed again in fp64.  (All-zero groups, the rows of ids that a batch did not use, stay fast.)
template <int N>
__device__ __forceinline__ double group_sqsum(const float (&x)[N]) {
  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k) s = fmaf(x[k], x[k], s);
  if (s > 1e-30f && s < 1e38f) return (double)s;
  double d = 0.0;
  float top = 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k) top = fmaxf(top, fabsf(x[k]));
  if (s == 0.0f && top == 0.0f) return 0.0;
#pragma unroll
  for (int k = 0; k < N; ++k) d = fma((double)x[k], (double)x[k], d);
  return d;
}

// The tensor that holds chunk c: its index, found by halving (chunk0 is ascending; empty tensors own no chunk).
template <int N>
__device__ __forceinline__ int tensor_of(const TensorSet<N>& S, unsigned int c) {
  int lo = 0, hi = S.n;            // chunk0[lo] <= c < chunk0[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (S.chunk0[mid] <= c) lo = mid; else hi = mid;
  }
  return lo;
}

// A tensor is read as [head: elements before the first 16-byte boundary][vectors][tail].  Chunk j covers the vectors
// [j * 2048, (j + 1) * 2048); the first chunk also takes the head, the last one the tail.
template <typename T>
struct Cut {
  long long head, vecs, tail0;     // tail0: first element behind the vectors
  __device__ __forceinline__ Cut(const T* p, long long n) {
    constexpr int V = Vec16<T>::kN;
    const long long off = (long long)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
    head = off ? V - off : 0;
    if (head > n) head = n;
    vecs = (n - head) / V;
    tail0 = head + vecs * V;
  }
};

__device__ __forceinline__ double block_sum(double a, double* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_down_sync(0xffffffffu, a, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = a;
  __syncthreads();
  double t = 0.0;
  if (threadIdx.x == 0)
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) t += red[w];
  return t;                        // valid in thread 0
}

// partial[block] (+)= sum of squares of the block's chunks.  add: partial holds an earlier launch's sum.  A block is one or
// more teams of kNormThreads, each with chunks of its own.
template <typename T, int N, int TEAMS>
__global__ void __launch_bounds__(kNormThreads * TEAMS)
k_list_sqsum(const __grid_constant__ TensorSet<N> S, double* partial, int add) {
  constexpr int V = Vec16<T>::kN;
  __shared__ double red[kNormThreads * TEAMS / 32];
  wait_for_predecessor();
  let_successor_in();
  const unsigned int chunks = S.chunk0[S.n];
  const int tid = threadIdx.x % kNormThreads;
  double sum = 0.0;
  for (unsigned int c = blockIdx.x * TEAMS + threadIdx.x / kNormThreads; c < chunks; c += gridDim.x * TEAMS) {
    const int k = tensor_of(S, c);
    const T* p = static_cast<const T*>(S.in[k]);
    const long long n = S.size[k];
    const Cut<T> cut(p, n);
    const long long j = c - S.chunk0[k];
    const uint4* q = reinterpret_cast<const uint4*>(p + cut.head);
    constexpr int A = TEAMS == 1 ? kNormVecs : kNormVecs / 2;      // in flight; a block of four teams has half the registers
#pragma unroll 1
    for (int part = 0; part < kNormVecs / A; ++part) {
      const long long v0 = (j * kNormVecs + part * A) * kNormThreads + tid;
      uint4 u[A];
#pragma unroll
      for (int i = 0; i < A; ++i) {
        const long long v = v0 + i * kNormThreads;
        u[i] = v < cut.vecs ? q[v] : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int i0 = 0; i0 < A; i0 += kGroup / 8) {
        float x[kGroup / 8 * V];
#pragma unroll
        for (int i = 0; i < kGroup / 8; ++i) Vec16<T>::unpack(u[i0 + i], x + i * V);
        sum += group_sqsum(x);
      }
    }
    if (j == 0 && (long long)tid < cut.head) {
      const double y = Vec16<T>::load(p + tid);
      sum = fma(y, y, sum);
    }
    if (c + 1 == S.chunk0[k + 1] && cut.tail0 + tid < n) {
      const double y = Vec16<T>::load(p + cut.tail0 + tid);
      sum = fma(y, y, sum);
    }
  }
  const double t = block_sum(sum, red);
  if (threadIdx.x == 0) partial[blockIdx.x] = add ? partial[blockIdx.x] + t : t;
}

// sqsum (+)= sum of the partial sums, in index order per thread and then by a fixed tree.
__global__ void __launch_bounds__(1024)
k_partials_sum(const double* partial, int n, double* sqsum, int add) {
  __shared__ double red[32];
  wait_for_predecessor();
  let_successor_in();
  double a = 0.0;
  for (int i = threadIdx.x; i < n; i += blockDim.x) a += partial[i];
  const double t = block_sum(a, red);
  if (threadIdx.x == 0) *sqsum = add ? *sqsum + t : t;
}

// out = f * in.  Chunks are taken from the last to the first: the norm pass, which read them the other way, left the
// last ones in L2.  With f = 1 and out = in a tensor is left alone.
template <typename T, int N>
__global__ void __launch_bounds__(kNormThreads)
k_list_scale(const __grid_constant__ TensorSet<N> S, const double* sqsum, double max_norm,
             float* told) {
  constexpr int V = Vec16<T>::kN;
  __shared__ float f_shared;
  wait_for_predecessor();
  if (threadIdx.x == 0) {
    float norm;
    f_shared = clip_factor(*sqsum, max_norm, &norm);
    if (told && blockIdx.x == 0) { told[0] = norm; told[1] = f_shared; }
  }
  __syncthreads();
  const float f = f_shared;
  const unsigned int chunks = S.chunk0[S.n];
  for (unsigned int b = blockIdx.x; b < chunks; b += gridDim.x) {
    const unsigned int c = chunks - 1 - b;
    const int k = tensor_of(S, c);
    const T* p = static_cast<const T*>(S.in[k]);
    T* o = static_cast<T*>(S.out[k]);
    if (f == 1.0f && o == p) continue;
    const long long n = S.size[k];
    const Cut<T> cut(p, n);
    const long long j = c - S.chunk0[k];
    const bool first = j == 0, last = c + 1 == S.chunk0[k + 1];
    if (((reinterpret_cast<uintptr_t>(o) ^ reinterpret_cast<uintptr_t>(p)) & 15u) == 0) {
      const uint4* q = reinterpret_cast<const uint4*>(p + cut.head);
      uint4* w = reinterpret_cast<uint4*>(o + cut.head);
      const long long v0 = j * (kNormThreads * kNormVecs) + threadIdx.x;
      uint4 u[kNormVecs];
#pragma unroll
      for (int i = 0; i < kNormVecs; ++i) {
        const long long v = v0 + i * kNormThreads;
        if (v < cut.vecs) u[i] = q[v];
      }
#pragma unroll
      for (int i = 0; i < kNormVecs; ++i) {
        const long long v = v0 + i * kNormThreads;
        float x[V];
        if (v < cut.vecs) {
          Vec16<T>::unpack(u[i], x);
#pragma unroll
          for (int e = 0; e < V; ++e) x[e] *= f;
          __stcs(w + v, Vec16<T>::pack(x));      // not read again here: leaves the inputs their place in L2
        }
      }
    } else {                       // differently aligned: the same elements one by one, neighbours by neighbouring threads
      const long long e0 = cut.head + j * (kNormThreads * kNormVecs) * V;
      long long e1 = e0 + (long long)kNormThreads * kNormVecs * V;
      if (e1 > cut.tail0) e1 = cut.tail0;
      for (long long e = e0 + threadIdx.x; e < e1; e += kNormThreads) Vec16<T>::store(o + e, Vec16<T>::load(p + e) * f);
    }
    if (first && (long long)threadIdx.x < cut.head)
      Vec16<T>::store(o + threadIdx.x, Vec16<T>::load(p + threadIdx.x) * f);
    if (last && cut.tail0 + threadIdx.x < n)
      Vec16<T>::store(o + cut.tail0 + threadIdx.x, Vec16<T>::load(p + cut.tail0 + threadIdx.x) * f);
  }
}

static int chained(cudaError_t e) {
  note_launch(1);
  return e == cudaSuccess ? DP_OK : DP_ERR_CUDA;
}

static int norm_grid(unsigned long long chunks) {
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  unsigned int cap = (unsigned int)sms * kNormBlocks;
  if (cap > (unsigned int)kNormMaxBlocks) cap = kNormMaxBlocks;
  return (int)(chunks < (unsigned long long)cap ? (chunks ? chunks : 1) : cap);
}

// Chunks of a tensor of n elements whose first 16-byte boundary lies `head` elements in: at least one, so that the
// head and tail of a short tensor have an owner; none for an empty tensor.
static long long chunk_count(const void* p, long long n, size_t es) {
  if (n <= 0) return 0;
  const long long V = 16 / (long long)es;
  const long long off = (long long)((reinterpret_cast<uintptr_t>(p) & 15u) / es);
  long long head = off ? V - off : 0;
  if (head > n) head = n;
  const long long vecs = (n - head) / V, per = kNormThreads * kNormVecs;
  const long long c = (vecs + per - 1) / per;
  return c ? c : 1;
}

// Fills S from tensor k on, as many as fit; returns the index behind the last one taken.
template <int N>
static int fill_set(TensorSet<N>& S, const void* const* in, void* const* out, const int64_t* sizes, int k, int n, size_t es) {
  S.n = 0;
  unsigned long long chunks = 0;
  for (; k < n && S.n < N; ++k) {
    if (sizes[k] == 0) continue;
    const unsigned long long c = (unsigned long long)chunk_count(in[k], sizes[k], es);
    if (chunks + c > 0xf0000000ull) break;       // 2^32 chunks of 32 KB: never reached by a tensor that fits the device
    S.in[S.n] = in[k];
    S.out[S.n] = out ? out[k] : nullptr;
    S.size[S.n] = sizes[k];
    S.chunk0[S.n++] = (unsigned int)chunks;
    chunks += c;
  }
  S.chunk0[S.n] = (unsigned int)chunks;
  return k;
}

// Up to this many chunks one block sums a list, in one launch: the host's second launch costs more than the time that more
// blocks would save.  One block of 64 x 64 with its FFN and norms (13 chunks): 15.7 -> 12.9 us a pass; one layer of 64 x 64
// (1 chunk) with its AdamW step: 12.3 -> 8.6.  Norm and scaling of one fp32 tensor in a bare loop of calls, many blocks against one: 1
// chunk 6.5, 4.5 us; 8 6.4, 5.6; 12 6.4, 6.7; 16 6.4, 7.5; 24 6.4, 9.1 -- the fewer other calls the host makes, the lower they
// cross.  Replayed from a graph, where the host does not count: 1 chunk 4.5, 3.9; 4 4.3, 4.4; 8 4.4, 5.3; 16 5.4, 7.1.
constexpr unsigned long long kOneBlockChunks = 16;

template <typename T, int N>
static int list_sqsum(const void* const* in, const int64_t* sizes, int n, double* partial, double* sqsum, int add,
                      cudaStream_t s) {
  // every launch of the call uses the same blocks, as many as all its chunks ask for, so each partial sum is written
  unsigned long long total = 0;
  for (int j = 0; j < n; ++j) total += (unsigned long long)chunk_count(in[j], sizes[j], sizeof(T));
  int k = 0, add_partial = 0;
  if (n <= N && total <= kOneBlockChunks) {      // little work: one block, whose sum is the answer
    TensorSet<N> S;
    fill_set<N>(S, in, nullptr, sizes, 0, n, sizeof(T));
    return chained(launch_chained(k_list_sqsum<T, N, 4>, 1, 4 * kNormThreads, 0, s, S, sqsum, add));
  }
  const int grid = norm_grid(total);
  do {
    TensorSet<N> S;
    k = fill_set<N>(S, in, nullptr, sizes, k, n, sizeof(T));
    if (const int rc = chained(launch_chained(k_list_sqsum<T, N, 1>, grid, kNormThreads, 0, s, S, partial, add_partial))) return rc;
    add_partial = 1;
  } while (k < n);
  return chained(launch_chained(k_partials_sum, 1, 1024, 0, s, partial, grid, sqsum, add));
}

template <typename T, int N>
static int list_scale(const void* const* in, void* const* out, const int64_t* sizes, int n, const double* sqsum,
                      double max_norm, float* told, cudaStream_t s) {
  int k = 0;
  do {
    TensorSet<N> S;
    k = fill_set<N>(S, in, out, sizes, k, n, sizeof(T));
    if (const int rc = chained(launch_chained(k_list_scale<T, N>, norm_grid(S.chunk0[S.n]), kNormThreads, 0, s, S, sqsum, max_norm, told))) return rc;
  } while (k < n);
  return DP_OK;
}

static bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

static int check_list(const void* const* in, void* const* out, bool want_out, const int64_t* sizes, int n, int dtype) {
  if (n < 0 || (n > 0 && (!in || !sizes || (want_out && !out)))) return DP_ERR_ARG;
  if (dtype != DP_F32 && dtype != DP_BF16) return DP_ERR_ARG;
  const size_t es = dtype == DP_F32 ? 4 : 2;
  for (int k = 0; k < n; ++k) {
    if (sizes[k] < 0 || sizes[k] > (int64_t)1 << 44) return DP_ERR_ARG;
    if (sizes[k] == 0) continue;
    if (!in[k] || (want_out && !out[k])) return DP_ERR_ARG;
    if (misaligned(in[k], es) || (want_out && misaligned(out[k], es))) return DP_ERR_ALIGN;
  }
  return DP_OK;
}

// A short list travels in 2 KB of parameters, a long one in 29 KB.
constexpr int kShortList = 64, kLongList = 1024;

}  // namespace dpk

using namespace dpk;

extern "C" {

size_t dp_global_norm_workspace_bytes(void) { return kNormWorkspace; }

int dp_global_sqnorm(const void* const* tensors, const int64_t* sizes, int n_tensors, int dtype, int accumulate_into,
                     double* sqsum, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const int rc = check_list(tensors, nullptr, false, sizes, n_tensors, dtype);
  if (rc != DP_OK) return rc;
  if (!sqsum) return DP_ERR_ARG;
  if (misaligned(sqsum, 8)) return DP_ERR_ALIGN;
  if (!workspace || misaligned(workspace, 256) || workspace_bytes < kNormWorkspace) return DP_ERR_WORKSPACE;
  double* partial = static_cast<double*>(workspace);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == DP_F32)
    return n_tensors <= kShortList ? list_sqsum<float, kShortList>(tensors, sizes, n_tensors, partial, sqsum, accumulate_into, s)
                                   : list_sqsum<float, kLongList>(tensors, sizes, n_tensors, partial, sqsum, accumulate_into, s);
  return n_tensors <= kShortList
             ? list_sqsum<__nv_bfloat16, kShortList>(tensors, sizes, n_tensors, partial, sqsum, accumulate_into, s)
             : list_sqsum<__nv_bfloat16, kLongList>(tensors, sizes, n_tensors, partial, sqsum, accumulate_into, s);
}

int dp_clip_by_global_norm(const void* const* tensors, void* const* outs, const int64_t* sizes, int n_tensors, int dtype,
                           const double* sqsum, double max_norm, float* norm_and_factor, void* cuda_stream) {
  const int rc = check_list(tensors, outs, true, sizes, n_tensors, dtype);
  if (rc != DP_OK) return rc;
  if (!sqsum || !(max_norm > 0.0) || !std::isfinite(max_norm)) return DP_ERR_ARG;
  if (misaligned(sqsum, 8) || misaligned(norm_and_factor, 4)) return DP_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == DP_F32)
    return n_tensors <= kShortList
               ? list_scale<float, kShortList>(tensors, outs, sizes, n_tensors, sqsum, max_norm, norm_and_factor, s)
               : list_scale<float, kLongList>(tensors, outs, sizes, n_tensors, sqsum, max_norm, norm_and_factor, s);
  return n_tensors <= kShortList
             ? list_scale<__nv_bfloat16, kShortList>(tensors, outs, sizes, n_tensors, sqsum, max_norm, norm_and_factor, s)
             : list_scale<__nv_bfloat16, kLongList>(tensors, outs, sizes, n_tensors, sqsum, max_norm, norm_and_factor, s);
}

int dp_clip_adamw_step(float* theta, float* m, float* v, float* g, int zero_g, int64_t n, const double* sqsum,
                       double max_norm, double lr, double beta1, double beta2, double xi, double weight_decay, int64_t t,
                       void* cuda_stream) {
  AdamArgs aa;
  if (n < 0 || !(max_norm > 0.0) || !std::isfinite(max_norm)) return DP_ERR_ARG;
  const int rc = make_adam_args(lr, beta1, beta2, xi, weight_decay, t, &aa);
  if (rc != DP_OK) return rc;
  if (n == 0) return DP_OK;
  if (!theta || !m || !v || !g || !sqsum) return DP_ERR_ARG;
  if (misaligned(theta, 4) || misaligned(m, 4) || misaligned(v, 4) || misaligned(g, 4) || misaligned(sqsum, 8))
    return DP_ERR_ALIGN;
  return launch_clip_adamw(theta, m, v, g, zero_g, n, sqsum, max_norm, aa, static_cast<cudaStream_t>(cuda_stream)) ==
                 cudaSuccess ? DP_OK : DP_ERR_CUDA;
}

}  // extern "C"
