// Distillation of logits z [N, V] from a teacher's top K logits t [N, K] over the words ids [N, K]:
//   q = softmax(t / tau) over the K words,  p = softmax(z / tau) over the vocabulary,
//   loss = w tau^2 sum_k q_k (log q_k - log p_ids_k),   dz = w tau (p - q at its words).
//
// Bound by memory: a row is read once and its gradient written once.  A block of up to 512 threads walks over its rows; a row
// lies in shared memory while it is needed three times (maximum, sum of exponentials, gradient), every thread fetching and
// reading its own vectors, so that the next row's are on their way as soon as this row's have been read for the last
// time; several blocks an SM (three at 30522 bf16 words) fill one another's pauses.  Short rows have a warp of their own and stay in
// registers; rows beyond shared memory (some 110 thousand bf16 words) are read three times, 2.7 of them from memory: up to three blocks an
// SM keep more of them in flight than L2 holds (8192 rows of 128256 bf16 words: 1590 us; of 110000, which fit, 787).
// Rows start anywhere: vectors of 16 bytes lie on 16-byte boundaries of memory, the two that reach beyond the row are masked,
// and those that reach beyond the first or last row are read element by element.
// Sums and statistics are fp32; a gradient is rounded once.
#include <algorithm>
#include <cmath>

#include "dp_chain.cuh"
#include "dp_internal.h"
#include "dp_ptx.cuh"

namespace dpk {

constexpr int kDistillThreads = 512;
constexpr size_t kRowsMost = 225 * 1024;         // dynamic shared memory of a block of k_distill_rows, at most
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
__global__ void __launch_bounds__(kDistillThreads) k_distill(const __grid_constant__ DistillArgs a) {
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
    if (tid == 0) a.loss[n] = live ? w * a.tau * (a.tau * (sum[2] / sum[1] + (logf(sum[0]) - logf(sum[1])))) : 0.0f;
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

__device__ __forceinline__ float warp_max(float x) {       // NaN are passed over
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}

// The larger of the elements of a vector so far.
template <typename T> __device__ __forceinline__ float vector_max(const uint4& d) {
  if constexpr (sizeof(T) == 4) {
    return fmaxf(fmaxf(__uint_as_float(d.x), __uint_as_float(d.y)), fmaxf(__uint_as_float(d.z), __uint_as_float(d.w)));
  } else {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&d);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
}

// 2^((x + less) scale) of the elements of a vector, two at a time.
template <typename T>
__device__ __forceinline__ void vector_powers(const uint4& d, ptx::f32x2 less, ptx::f32x2 scale, ptx::f32x2 (&e)[8 / sizeof(T)]) {
#pragma unroll
  for (int u = 0; u < (int)(8 / sizeof(T)); ++u) {
    const float2 y = ptx::unpack2(ptx::mul2(ptx::add2(ptx::pack2(lane_of<T>(d, 2 * u), lane_of<T>(d, 2 * u + 1)), less), scale));
    e[u] = ptx::pack2(exp2_fast(y.x), exp2_fast(y.y));
  }
}

// Rows in shared memory.  Dynamic shared memory: a row, then the teacher's words, those of two rows.
// Three barriers a row: the maximum (the row and its words are complete in shared memory), the sums (what the words need of the
// row has been read), the gradient (the words' own values come last).
template <typename T>
__global__ void __launch_bounds__(kDistillThreads, 3) k_distill_rows(const __grid_constant__ DistillArgs a, int row_bytes) {
  constexpr int E = 16 / sizeof(T);              // elements of a vector
  extern __shared__ __align__(16) uint8_t rows[];
  __shared__ float red_max[16][2];
  __shared__ float red_sum[16][4];
  wait_for_predecessor();
  let_successor_in();
  const int threads = (int)blockDim.x, tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = threads >> 5;
  float* words = reinterpret_cast<float*>(rows + row_bytes);
  const uintptr_t begin = reinterpret_cast<uintptr_t>(a.z), end = begin + ((a.N - 1) * a.ld + a.V) * sizeof(T);
  const uint32_t rows32 = (uint32_t)__cvta_generic_to_shared(rows);
  // A row: its first byte, its vectors, whether they all lie inside the tensor (of those of the first and the last row one may
  // reach beyond it: they are then read element by element).
  struct Row { uintptr_t at; int nv; bool inside; };
  const auto row_of = [&](long long n) -> Row {
    Row r;
    r.at = begin + (uintptr_t)(n * a.ld) * sizeof(T);
    r.nv = n < a.N ? (int)(((r.at & 15) + (uintptr_t)a.V * sizeof(T) + 15) >> 4) : 0;
    const uintptr_t first = r.at & ~(uintptr_t)15;
    r.inside = first >= begin && first + (uintptr_t)r.nv * 16 <= end;
    return r;
  };
  const auto copy = [&](int v, const uint8_t* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(rows32 + v * 16), "l"(from) : "memory");
  };
  const auto fetch = [&](const Row& r, int v) {              // this thread's vectors from v on
    const uintptr_t first = r.at & ~(uintptr_t)15;
    for (; v < r.nv; v += threads) {
      const uintptr_t at = first + (uintptr_t)v * 16;
      if (r.inside || (at >= begin && at + 16 <= end)) {
        copy(v, reinterpret_cast<const uint8_t*>(at));
      } else {
#pragma unroll
        for (int u = 0; u < E; ++u)
          if (at + u * sizeof(T) >= begin && at + (u + 1) * sizeof(T) <= end)
            reinterpret_cast<T*>(rows + v * 16)[u] = *reinterpret_cast<const T*>(at + u * sizeof(T));
      }
    }
  };
  struct Word { int id; float t; };
  const auto word = [&](long long n, int k) -> Word {        // of the teacher; id -1: an empty place
    Word w = {-1, -INFINITY};
    if (n < a.N && k < a.K) {
      w.id = a.ids[n * a.K + k];
      w.t = a.t_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(a.t)[n * a.K + k]) : static_cast<const float*>(a.t)[n * a.K + k];
      if (w.id >= a.V) {
        atomicCAS(a.status, 0, (int)STATUS_BAD_ID);
        w.id = -1;
      }
      if (w.id < 0 || w.t == -INFINITY) w = {-1, -INFINITY};
    }
    return w;
  };
  long long n = blockIdx.x;
  Row row = row_of(n);
  fetch(row, tid);
  Word next = word(n, tid);
  for (int i = 0; n < a.N; n += gridDim.x, ++i) {
    float* s_t = words + (size_t)(i & 1) * 4 * a.K;          // the teacher's logits, the student's exponents, the teacher's powers
    float *s_y = s_t + a.K, *s_q = s_y + a.K;
    int* s_id = reinterpret_cast<int*>(s_q + a.K);           // the words
    const T* z = reinterpret_cast<const T*>(rows + (row.at & 15));
    const int off = (int)(row.at & 15) / (int)sizeof(T), nv = row.nv, last = nv - 1;
    float top_t = -INFINITY, top = -INFINITY;
    for (int k = tid; k < a.K; k += threads) {
      const Word w = k == tid ? next : word(n, k);
      s_id[k] = w.id;
      s_t[k] = w.t;
      top_t = fmaxf(top_t, w.t == w.t ? w.t : INFINITY);     // a NaN makes the differences to the maximum NaN
    }
    next = word(n + gridDim.x, tid);
    asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
    const auto trim = [&](int v) {               // the elements beside the row become -inf
#pragma unroll
      for (int u = 0; u < E; ++u)
        if (v * E - off + u < 0 || v * E - off + u >= a.V) reinterpret_cast<T*>(rows + v * 16)[u] = from_float<T>(-INFINITY);
    };
    if (tid == 0) trim(0);
    if (tid == (last & (threads - 1))) trim(last);      // threads: a power of two
#pragma unroll 4
    for (int v = tid; v < nv; v += threads) top = fmaxf(top, vector_max<T>(*reinterpret_cast<const uint4*>(rows + v * 16)));
    top = warp_max(top);
    if (32 * warp < a.K) top_t = warp_max(top_t);
    if (lane == 0) red_max[warp][0] = top, red_max[warp][1] = top_t;
    __syncthreads();
    top = warp_max(lane < warps ? red_max[lane][0] : -INFINITY);
    top_t = warp_max(lane < warps ? red_max[lane][1] : -INFINITY);
    const bool live = top_t != -INFINITY;
    // powers of two of (x - the maximum) log2(e) / tau: the difference first, since the exponents of small temperatures are
    // large numbers, whose own rounding would be more than fp32 holds as a power
    const float base = top == -INFINITY ? 0.0f : top;
    const auto exponent = [&](float x) { return (x - base) * a.scale2; };
    const ptx::f32x2 less = ptx::pack2(-base, -base), scale = ptx::pack2(a.scale2, a.scale2);
    const auto exponent_t = [&](float t) { return (t - top_t) * a.scale2; };
    const float w = live ? (a.weights ? a.weights[n] : 1.0f) : 0.0f;
    // sums: of the student's powers, the teacher's, and the teacher's weight times the gap of the two exponents
    float sum_t = 0.0f, gap = 0.0f;
    for (int k = tid; k < a.K; k += threads) {
      const int id = s_id[k];
      if (id < 0) continue;
      const float y = exponent(to_float(z[id])), t = exponent_t(s_t[k]), e = exp2_fast(t);
      sum_t += e;
      if (e != 0.0f) gap += e * (t - y);
      // the same word again adds to its first place (s_q < 0: not the first)
      int again = 0;
#pragma unroll 4
      for (int o = 0; o < a.K; ++o) again += s_id[o] == id;
      float q = e;
      if (again > 1) {
        q = 0.0f;
        bool first = true;
        for (int o = 0; o < a.K; ++o) {
          if (s_id[o] != id) continue;
          first = first && o >= k;
          q += exp2_fast(exponent_t(s_t[o]));
        }
        if (!first) q = -1.0f;
      }
      s_y[k] = y;
      s_q[k] = q;
    }
    ptx::f32x2 part[2] = {0ull, 0ull};
#pragma unroll 2
    for (int v = tid; v < nv; v += threads) {
      const uint4 d = *reinterpret_cast<const uint4*>(rows + v * 16);
      ptx::f32x2 e[E / 2];
      vector_powers<T>(d, less, scale, e);
#pragma unroll
      for (int u = 0; u < E / 2; ++u) part[u & 1] = ptx::add2(part[u & 1], e[u]);
    }
    const float2 halves = ptx::unpack2(ptx::add2(part[0], part[1]));
    float sum = halves.x + halves.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (32 * warp < a.K) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        sum_t += __shfl_xor_sync(0xffffffffu, sum_t, o);
        gap += __shfl_xor_sync(0xffffffffu, gap, o);
      }
    }
    if (lane == 0) *reinterpret_cast<float4*>(red_sum[warp]) = make_float4(sum, sum_t, gap, 0.0f);
    __syncthreads();
    const float4 r = lane < warps ? *reinterpret_cast<const float4*>(red_sum[lane]) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    sum = r.x, sum_t = r.y, gap = r.z;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {            // at most 16 warps
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
      sum_t += __shfl_xor_sync(0xffffffffu, sum_t, o);
    }
    if (warp == 0) {
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) gap += __shfl_xor_sync(0xffffffffu, gap, o);
      if (lane == 0) a.loss[n] = live ? w * a.tau * (a.tau * (0.693147181f * (gap / sum_t + (log2f(sum) - log2f(sum_t))))) : 0.0f;
    }
    const Row after = row_of(n + gridDim.x);
    const int nv2 = after.inside ? after.nv : 0;
    const uint8_t* from = reinterpret_cast<const uint8_t*>(after.at & ~(uintptr_t)15);
    T* out = a.dz ? static_cast<T*>(a.dz) + n * a.ld_out : nullptr;
    sum = __shfl_sync(0xffffffffu, sum, 0);      // lanes 16 and up have summed nothing
    sum_t = __shfl_sync(0xffffffffu, sum_t, 0);
    const float c = w * a.tau, cp = __fdividef(c, sum), cq = __fdividef(c, sum_t);
    const bool same = (reinterpret_cast<uintptr_t>(out) & 15) == (row.at & 15);
    // whole vectors of the result: [lo, hi)
    const int lo = off ? 1 : 0, hi = out && same ? (off + a.V) / E : lo;
    if (out) {
      const auto single = [&](int v) {           // element by element
#pragma unroll
        for (int u = 0; u < E; ++u) {
          const int e = v * E - off + u;
          if (e >= 0 && e < a.V) out[e] = from_float<T>(live ? cp * exp2_fast(exponent(to_float(reinterpret_cast<const T*>(rows + v * 16)[u]))) : 0.0f);
        }
      };
      if (!same) {
        for (int v = tid; v < nv; v += threads) single(v);
      } else {
        if (tid == 0 && lo) single(0);
        if (tid == (last & (threads - 1)) && last >= hi && last >= lo) single(last);
      }
    }
    const uint8_t* there = rows;
    int v = tid;
    if (live) {
      uint4* to = reinterpret_cast<uint4*>(out - off);
      const ptx::f32x2 cp2 = ptx::pack2(cp, cp);
#pragma unroll 2
      for (; v < nv; v += threads) {
        const uint4 d = *reinterpret_cast<const uint4*>(there + v * 16);
        if (v < nv2) copy(v, from + (size_t)v * 16);   // its place is free: the words have been read, and this was its last time
        if (v >= lo && v < hi) {
          ptx::f32x2 e[E / 2];
          float g[E];
          vector_powers<T>(d, less, scale, e);
#pragma unroll
          for (int u = 0; u < E / 2; ++u) {
            const float2 x = ptx::unpack2(ptx::mul2(e[u], cp2));
            g[2 * u] = x.x;
            g[2 * u + 1] = x.y;
          }
          to[v] = packed<T>(g);
        }
      }
    } else {                                     // a row without a teacher may hold anything
      uint4* to = reinterpret_cast<uint4*>(out - off);
      for (; v < nv; v += threads) {
        if (v < nv2) copy(v, from + (size_t)v * 16);
        if (v >= lo && v < hi) to[v] = make_uint4(0, 0, 0, 0);
      }
    }
    fetch(after, after.inside ? v : tid);        // a row may begin one vector further on
    row = after;
    __syncthreads();
    if (out && live) {
      for (int k = tid; k < a.K; k += threads) {
        const float q = s_q[k];
        if (s_id[k] >= 0 && !(q < 0.0f)) out[s_id[k]] = from_float<T>(cp * exp2_fast(s_y[k]) - cq * q);
      }
    }
  }
}

// The form for rows of `nv` vectors at most: a warp a row up to 8 vectors a lane, then a block a row.
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
  const size_t row_bytes = (size_t)nv * 16, list = (size_t)8 * a.K * sizeof(float), smem = row_bytes + list;
  if (smem > kRowsMost) return launch_chained(k_distill<T, 0, false>, (unsigned)a.N, kDistillThreads, words, s, a);
  // A power of two of threads, at least four vectors each, and as many blocks an SM as threads and shared memory allow.  256 threads
  // where three rows fit (30522 bf16 words: 182 us for 6144 rows; 384 threads 188, 512 197), more where fewer do.
  const int rows = std::max(1, (int)(kRowsMost / (smem + 1536)));
  int threads = 64;
  while (threads < (rows >= 3 && a.N > sm_count() ? 256 : kDistillThreads) && threads * 8 <= nv) threads *= 2;
  const int resident = std::min(rows, 3 * kDistillThreads / threads);
  const unsigned grid = (unsigned)std::min<long long>(a.N, (long long)resident * sm_count());
  static signed char ready[kMaxDevices] = {};    // 0 unknown, 1 ready, -1 failed (one flag per form and device)
  const int dev = current_device();
  if (dev < 0) return cudaErrorInvalidDevice;
  if (!ready[dev])
    ready[dev] = cudaFuncSetAttribute(k_distill_rows<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRowsMost) == cudaSuccess ? 1 : -1;
  if (ready[dev] < 0) return cudaErrorInvalidValue;
  return launch_chained(k_distill_rows<T>, grid, threads, smem, s, a, (int)row_bytes);
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
  if (dlogits && dlogits != p->logits && rows_meet(p->logits, ld, dlogits, ldo, p->N, p->V, (int)e)) return DP_ERR_ARG;
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
