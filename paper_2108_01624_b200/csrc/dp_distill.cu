// Distillation of logits z [N, V] from a teacher's top K logits t [N, K] over the words ids [N, K]:
//   q = softmax(t / tau) over the K words,  p = softmax(z / tau) over the vocabulary,
//   loss = w tau^2 sum_k q_k (log q_k - log p_ids_k),   dz = w tau (p - q at its words).
//
// Bound by memory: a row is read once and its gradient written once.  It stays in registers between the three things that
// need it (its maximum, the sum of its exponentials, the gradient): up to 8 vectors of 16 bytes a thread, 512 threads a
// row, so 32768 bf16 or 16384 fp32 words; longer rows are read again, from L2.  Rows of at most 8 vectors a lane have a
// warp of their own.  Rows start anywhere: vectors lie on 16-byte boundaries of memory, and the two that reach beyond
// the row are moved element by element.
// Sums and statistics are fp32; a gradient is rounded once.
#include <cmath>

#include "dp_chain.cuh"
#include "dp_internal.h"

namespace dpk {

constexpr int kDistillThreads = 512;
constexpr int kDistillWords = 1024;              // most words of a teacher
constexpr float kLog2ePerE = 1.4426950408889634f;

struct DistillArgs {
  const void* z;
  const int32_t* ids;
  const void* t;
  const float* weights;
  float* loss;
  void* dz;
  long long ld, ld_out;
  int N, V, K, t_bf16;
  float scale2;                                  // log2(e) / tau
  float tau, inv_tau;
  int* status;
};

template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float(float x) { return x; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Element u of a 16-byte vector, and the vector of E floats.
template <typename T> __device__ __forceinline__ float lane_of(const uint4& v, int u) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if constexpr (sizeof(T) == 4) return __uint_as_float(w[u]);
  else return __uint_as_float(u & 1 ? w[u >> 1] & 0xffff0000u : w[u >> 1] << 16);
}
template <typename T> __device__ __forceinline__ uint4 packed(const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (sizeof(T) == 4) {
      w[k] = __float_as_uint(x[k]);
    } else {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
      w[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Reductions over the threads of a row: a warp, or the block through `red` (every call ends with all threads past it).
template <bool WARP, int N, typename F>
__device__ __forceinline__ void over_row(float (&x)[N], float (*red)[N], F f) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = f(k, x[k], __shfl_xor_sync(0xffffffffu, x[k], o));
  }
  if constexpr (!WARP) {
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) red[threadIdx.x >> 5][k] = x[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = red[0][k];
    for (int w = 1; w < warps; ++w) {
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = f(k, x[k], red[w][k]);
    }
    __syncthreads();
  }
}

// NV: vectors a thread keeps; 0: rows of any length, read three times.  WARP: a warp per row, several rows a block.
template <typename T, int NV, bool WARP>
__global__ void __launch_bounds__(kDistillThreads, NV == 8 && !WARP ? 2 : 1) k_distill(const __grid_constant__ DistillArgs a) {
  constexpr int E = 16 / sizeof(T);              // elements of a vector
  constexpr int KEEP = NV ? NV : 1;
  extern __shared__ float smem[];
  __shared__ float red_max[16][2];
  __shared__ float red_sum[16][3];
  wait_for_predecessor();
  let_successor_in();
  const int threads = WARP ? 32 : (int)blockDim.x, tid = WARP ? (int)threadIdx.x & 31 : (int)threadIdx.x;
  const int rows = WARP ? (int)blockDim.x >> 5 : 1, mine = WARP ? (int)threadIdx.x >> 5 : 0;
  float* s_t = smem + (size_t)mine * 4 * a.K;    // the teacher's logits and words; the student's logits, then gradients, there
  int* s_id = reinterpret_cast<int*>(s_t + a.K);
  float* s_z = s_t + 2 * a.K;
  int* s_to = s_id + 2 * a.K;                    // where the gradient goes, or -1
  const auto barrier = [] {
    if constexpr (WARP) __syncwarp();
    else __syncthreads();
  };
  for (long long n = (long long)blockIdx.x * rows + mine; n < a.N; n += (long long)gridDim.x * rows) {
    const T* z = static_cast<const T*>(a.z) + n * a.ld;
    T* out = a.dz ? static_cast<T*>(a.dz) + n * a.ld_out : nullptr;
    const int off = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));   // elements of the first vector before the row
    const bool same = out && (reinterpret_cast<uintptr_t>(out) & 15) / sizeof(T) == (unsigned)off;
    const int nv = (off + a.V + E - 1) / E;
    // the teacher's words
    float top[2] = {-INFINITY, -INFINITY};       // of the student, of the teacher
    for (int k = tid; k < a.K; k += threads) {
      int id = a.ids[n * a.K + k];
      if (id >= a.V) {
        atomicCAS(a.status, 0, (int)STATUS_BAD_ID);
        id = -1;
      }
      float t = a.t_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(a.t)[n * a.K + k]) : static_cast<const float*>(a.t)[n * a.K + k];
      if (id < 0 || t == -INFINITY) {
        id = -1;
        t = -INFINITY;
      }
      s_id[k] = id;
      s_t[k] = t;
      top[1] = fmaxf(top[1], t == t ? t : INFINITY);   // a NaN makes the differences to the maximum NaN
    }
    const auto load = [&](int v) -> uint4 {      // vector v of the row, -inf outside
      const int e0 = v * E - off;
      if (e0 >= 0 && e0 + E <= a.V) return *reinterpret_cast<const uint4*>(z + e0);
      float x[E];
#pragma unroll
      for (int u = 0; u < E; ++u) x[u] = e0 + u >= 0 && e0 + u < a.V ? to_float(z[e0 + u]) : -INFINITY;
      return packed<T>(x);
    };
    uint4 keep[KEEP];
    if constexpr (NV > 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int v = tid + j * threads;
        keep[j] = v < nv ? load(v) : make_uint4(0, 0, 0, 0);
      }
    }
    const auto each = [&](auto f) {              // f(vector, its data)
      if constexpr (NV > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int v = tid + j * threads;
          if (v < nv) f(v, keep[j]);
        }
      } else {
        for (int v = tid; v < nv; v += threads) f(v, load(v));
      }
    };
    each([&](int, const uint4& x) {
#pragma unroll
      for (int u = 0; u < E; ++u) top[0] = fmaxf(top[0], lane_of<T>(x, u));
    });
    over_row<WARP, 2>(top, red_max, [](int, float x, float y) { return fmaxf(x, y); });
    barrier();                                   // s_id and s_t are complete
    const bool live = top[1] != -INFINITY;       // uniform over the row
    const float base = top[0] == -INFINITY ? 0.0f : top[0];
    const float w = live ? (a.weights ? a.weights[n] : 1.0f) : 0.0f;
    // sums: of the student's exponentials, the teacher's, and the teacher's weight times the gap of the two logits
    float sum[3] = {0.0f, 0.0f, 0.0f};
    if (live) {
      each([&](int, const uint4& x) {
#pragma unroll
        for (int u = 0; u < E; ++u) sum[0] += exp2_fast((lane_of<T>(x, u) - base) * a.scale2);
      });
      for (int k = tid; k < a.K; k += threads) {
        if (s_id[k] < 0) continue;
        const float x = to_float(z[s_id[k]]) - base, t = s_t[k] - top[1], e = exp2_fast(t * a.scale2);
        s_z[k] = x;
        sum[1] += e;
        if (e != 0.0f) sum[2] += e * ((t - x) * a.inv_tau);
      }
    }
    over_row<WARP, 3>(sum, red_sum, [](int, float x, float y) { return x + y; });
    if (tid == 0) a.loss[n] = live ? w * a.tau * a.tau * (sum[2] / sum[1] + (logf(sum[0]) - logf(sum[1]))) : 0.0f;
    if (out) {
      const float c = w * a.tau, cp = c / sum[0], cq = c / sum[1];
      for (int k = tid; k < a.K; k += threads) {
        const int id = s_id[k];
        float q = 0.0f;
        bool first = live && id >= 0;            // the same word again adds to its first place
        if (first) {
          for (int o = 0; o < a.K; ++o) {
            if (s_id[o] != id) continue;
            first = first && o >= k;
            q += exp2_fast((s_t[o] - top[1]) * a.scale2);
          }
        }
        s_to[k] = first ? id : -1;
        if (first) s_z[k] = cp * exp2_fast(s_z[k] * a.scale2) - cq * q;
      }
      each([&](int v, const uint4& x) {
        float g[E];
#pragma unroll
        for (int u = 0; u < E; ++u) g[u] = live ? cp * exp2_fast((lane_of<T>(x, u) - base) * a.scale2) : 0.0f;
        const int e0 = v * E - off;
        if (same && e0 >= 0 && e0 + E <= a.V) {
          *reinterpret_cast<uint4*>(out + e0) = packed<T>(g);
        } else {
#pragma unroll
          for (int u = 0; u < E; ++u)
            if (e0 + u >= 0 && e0 + u < a.V) out[e0 + u] = from_float<T>(g[u]);
        }
      });
      barrier();                                 // the words' own values come last
      for (int k = tid; k < a.K; k += threads)
        if (s_to[k] >= 0) out[s_to[k]] = from_float<T>(s_z[k]);
    }
    barrier();                                   // the words' arrays are free again
  }
}

// The form for rows of `nv` vectors at most: a warp a row up to 8 vectors a lane, then blocks of up to 512 threads.
template <typename T>
static cudaError_t launch_distill(const DistillArgs& a, cudaStream_t s) {
  const long long nv = (a.V + 16 / (int)sizeof(T) - 1) / (16 / (int)sizeof(T)) + 1;
  const size_t words = (size_t)4 * a.K * sizeof(float);
  if (nv <= 8 * 32) {
    int rows = 8;
    while (rows > 1 && rows * words > 32768) rows >>= 1;
    const unsigned grid = (unsigned)((a.N + rows - 1) / rows);
    return launch_chained(nv <= 2 * 32 ? k_distill<T, 2, true> : k_distill<T, 8, true>, grid, 32 * rows, rows * words, s, a);
  }
  const int per = nv <= 4 * kDistillThreads ? 4 : 8;
  const int threads = nv > 8 * kDistillThreads ? kDistillThreads : (int)((nv + 32 * per - 1) / (32 * per)) * 32;
  return launch_chained(nv > 8 * kDistillThreads ? k_distill<T, 0, false> : per == 4 ? k_distill<T, 4, false> : k_distill<T, 8, false>,
                        (unsigned)a.N, threads, words, s, a);
}

}  // namespace dpk

using namespace dpk;

extern "C" int dp_distill_loss(const dp_distill* p, float* loss, void* dlogits, int64_t ld_out, void* cuda_stream) {
  if (!p || !p->logits || !p->top_ids || !p->top_logits || !loss) return DP_ERR_ARG;
  if ((p->dtype != DP_F32 && p->dtype != DP_BF16) || (p->teacher_dtype != DP_F32 && p->teacher_dtype != DP_BF16)) return DP_ERR_ARG;
  if (p->N <= 0 || p->V <= 0 || p->K <= 0) return DP_ERR_ARG;
  // the temperature and its inverse as fp32 numbers
  if (!(p->temperature >= 1e-30 && p->temperature <= 1e30)) return DP_ERR_ARG;
  const long long ld = p->N > 1 ? p->ld : p->V, ldo = p->N > 1 ? ld_out : p->V;
  if (ld < p->V || (dlogits && ldo < p->V) || (dlogits == p->logits && ldo != ld)) return DP_ERR_ARG;
  if (p->K > kDistillWords || p->V > (1 << 30)) return DP_ERR_UNSUPPORTED;
  const size_t e = p->dtype == DP_F32 ? 4 : 2;
  if (misaligned(p->logits, e) || misaligned(dlogits, e) || misaligned(p->top_ids, 4) || misaligned(loss, 4) ||
      misaligned(p->weights, 4) || misaligned(p->top_logits, p->teacher_dtype == DP_F32 ? 4 : 2)) return DP_ERR_ALIGN;
  int* status = status_ptr();
  if (!status) return DP_ERR_CUDA;
  const DistillArgs a = {p->logits, p->top_ids, p->top_logits, p->weights, loss, dlogits, ld, ldo, p->N, p->V, p->K,
                         p->teacher_dtype == DP_BF16, (float)(kLog2ePerE / p->temperature), (float)p->temperature,
                         (float)(1.0 / p->temperature), status};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  note_launch(1);
  const cudaError_t rc = p->dtype == DP_F32 ? launch_distill<float>(a, s) : launch_distill<__nv_bfloat16>(a, s);
  return rc == cudaSuccess ? DP_OK : DP_ERR_CUDA;
}
