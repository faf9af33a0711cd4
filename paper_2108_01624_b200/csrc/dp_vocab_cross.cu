// The cross term of a table that a vocabulary head shares with the token embedding: example i's gradient of the table is
// sum_u e_u at row ids_u (the embedding's part) plus G_i^T X_i (the head's), and the norm of the sum needs
//   2 sum over inputs u, tokens t of G[t][ids_u] <x_t, e_u>,   G[t][v] = w_t (exp(<x_t, W_v> + bias_v - lse_t) - [v = label_t]).
// Only the columns of G that the ids name are formed: two products of [inputs, d] x [d, tokens] an example, of the named
// rows of W and of e.
//
// Bound by memory (e and the named rows of W are read once): a warp takes 16 inputs against up to 32 tokens by m16n8k16
// products.  A dot product does not mind the order of its terms, so a lane
// gives 8 neighbouring elements of a row (16 bytes) to the places that two products ask of it, the same for both operands.
// Aligned bf16 rows of whole 128-byte lines come through shared memory, each warp's own three lines ahead (256 x 128 inputs, 20
// tokens, d = 1024: 61 us straight into registers, four rows' halves of a line a load); others straight from memory into the operands.
// fp32 rows are split into three bf16 numbers in registers: six products, the smallest first.
// fp32 sums; the products drop low bits at every step, so each run of kCrossSeg elements is summed apart.  G is not rounded.
#include <algorithm>

#include "dp_chain.cuh"
#include "dp_internal.h"

namespace dpk {

constexpr int kCrossSeg = 256;

struct CrossArgs {
  const void* x;
  const void* w;
  const void* e;
  const float* bias;
  const int32_t* labels;
  const float* weights;
  const float* lse;
  const int32_t* ids;
  float* out;                    // sqnorm, or partial sums [B][chunks]
  long long ldx, ldw, lde;
  int B, T, Tu, d, V;
  unsigned chunks, t_chunks, all;   // all: (128-input x 8 NT-token) tasks of an example, shared by `chunks` blocks
  int vec;
  int* status;
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Elements [k, k + 8) of a row as PLANES times four words of two bf16 numbers, zeros beyond d.
template <typename T> struct CrossRow;
template <> struct CrossRow<__nv_bfloat16> {
  static constexpr int PLANES = 1;
  uint32_t r[1][4];
  __device__ __forceinline__ void load(const void* base, long long row, int k, int d, bool vec) {
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(base) + row + k;
    if (vec && k + 8 <= d) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      r[0][0] = v.x, r[0][1] = v.y, r[0][2] = v.z, r[0][3] = v.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = k + 2 * j < d ? __bfloat16_as_ushort(p[2 * j]) : 0u, hi = k + 2 * j + 1 < d ? __bfloat16_as_ushort(p[2 * j + 1]) : 0u;
        r[0][j] = lo | hi << 16;
      }
    }
  }
};
template <> struct CrossRow<float> {
  static constexpr int PLANES = 3;
  uint32_t r[3][4];
  __device__ __forceinline__ void load(const void* base, long long row, int k, int d, bool vec) {
    const float* p = static_cast<const float*>(base) + row + k;
    float x[8];
    if (vec && k + 8 <= d) {
      const float4 u = *reinterpret_cast<const float4*>(p), v = *reinterpret_cast<const float4*>(p + 4);
      x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = k + j < d ? p[j] : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
        r[q][j] = *reinterpret_cast<const uint32_t*>(&h);
        x[2 * j] -= __uint_as_float(r[q][j] << 16);
        x[2 * j + 1] -= __uint_as_float(r[q][j] & 0xffff0000u);
      }
    }
  }
};

// c += rows (a of lane/4, b of lane/4 + 8) x tokens over 32 elements.
template <typename R>
__device__ __forceinline__ void cross_step(float (&c)[4], const R& a, const R& b, const R& x) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if constexpr (R::PLANES == 1) {
      mma_bf16(c, a.r[0][2 * s], b.r[0][2 * s], a.r[0][2 * s + 1], b.r[0][2 * s + 1], x.r[0][2 * s], x.r[0][2 * s + 1]);
    } else {
      constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
      for (int q = 0; q < 6; ++q)
        mma_bf16(c, a.r[pa[q]][2 * s], b.r[pa[q]][2 * s], a.r[pa[q]][2 * s + 1], b.r[pa[q]][2 * s + 1], x.r[pb[q]][2 * s], x.r[pb[q]][2 * s + 1]);
    }
  }
}

// The words of the inputs that this lane's products belong to, u and u + 8: -1 where there is none.
__device__ __forceinline__ int2 cross_words(const CrossArgs& a, long long i, int u) {
  int id[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    id[h] = u + 8 * h < a.Tu ? a.ids[i * a.Tu + u + 8 * h] : -1;
    if (u + 8 * h < a.Tu && (id[h] < 0 || id[h] >= a.V)) {
      atomicCAS(a.status, 0, (int)STATUS_BAD_ID);
      id[h] = -1;
    }
  }
  return make_int2(id[0], id[1]);
}

// Sum of G times <x, e> over a lane's products: words of rows g and g + 8, tokens t0 + 8 j + 2 q and the next.
template <int NT>
__device__ __forceinline__ float cross_finish(const CrossArgs& a, long long i, int2 id, int t0, int q, const float (&cz)[NT][4], const float (&ck)[NT][4]) {
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int t = t0 + 8 * j + 2 * q + (k & 1), v = k >> 1 ? id.y : id.x;
      if (t >= a.T || v < 0) continue;
      const long long n = i * a.T + t;
      const int y = a.labels[n];
      if (y < 0 || y >= a.V) continue;
      const float z = cz[j][k] + (a.bias ? a.bias[v] : 0.0f) - a.lse[n];
      const float G = v == y ? expm1f(z) : expf(z);
      sum = fmaf((a.weights ? a.weights[n] : 1.0f) * G, ck[j][k], sum);
    }
  }
  return sum;
}

// The block's sum into its place.
__device__ __forceinline__ void cross_store(const CrossArgs& a, long long i, float sum, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_down_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += red[w];
    if (a.chunks > 1) a.out[i * a.chunks + blockIdx.x] = 2.0f * s;
    else a.out[i] += 2.0f * s;
  }
  __syncthreads();
}

// Block (chunk, example, and every 65535th after it): eight warps, 16 inputs each, against NT groups of 8 tokens.
template <typename T, int NT>
__global__ void __launch_bounds__(256) k_vocab_cross(const __grid_constant__ CrossArgs a) {
  __shared__ float red[8];
  wait_for_predecessor();
  let_successor_in();
  using R = CrossRow<T>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  for (long long i = blockIdx.y; i < a.B; i += gridDim.y) {
    float sum = 0.0f;
    for (unsigned task = blockIdx.x; task < a.all; task += a.chunks) {
      const int u0 = (int)(task / a.t_chunks) * 128 + warp * 16, t0 = (int)(task % a.t_chunks) * (NT * 8);
      if (u0 >= a.Tu) continue;
      const int2 id = cross_words(a, i, u0 + g);
      // rows that do not count are read from a place that exists; their columns or rows of the products are left out below
      const long long w0 = (long long)max(id.x, 0) * a.ldw, w1 = (long long)max(id.y, 0) * a.ldw;
      const long long e0 = (i * a.Tu + min(u0 + g, a.Tu - 1)) * a.lde, e1 = (i * a.Tu + min(u0 + g + 8, a.Tu - 1)) * a.lde;
      float cz[NT][4] = {}, ck[NT][4] = {};
      for (int k0 = 0; k0 < a.d; k0 += kCrossSeg) {
        float sz[NT][4] = {}, sk[NT][4] = {};
        const int k1 = min(k0 + kCrossSeg, (a.d + 31) / 32 * 32);
#pragma unroll 2
        for (int k = k0 + 8 * q; k < k1; k += 32) {
          R wa, wb, ea, eb;
          wa.load(a.w, w0, k, a.d, a.vec);
          wb.load(a.w, w1, k, a.d, a.vec);
          ea.load(a.e, e0, k, a.d, a.vec);
          eb.load(a.e, e1, k, a.d, a.vec);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            R x;
            x.load(a.x, (i * a.T + min(t0 + 8 * j + g, a.T - 1)) * a.ldx, k, a.d, a.vec);
            cross_step(sz[j], wa, wb, x);
            cross_step(sk[j], ea, eb, x);
          }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            cz[j][k] += sz[j][k];
            ck[j][k] += sk[j][k];
          }
      }
      sum += cross_finish<NT>(a, i, id, t0, q, cz, ck);
    }
    cross_store(a, i, sum, red);
  }
}

// The same for bf16 rows of whole 128-byte lines (64 elements).  Shared memory: the tokens' rows [8 NT][d], and of every warp
// kCrossStages times one line of its 16 rows of W and of e.  16-byte chunks of odd rows change places with those 64 bytes on, so
// that the eight lanes of a phase (two rows, four chunks) meet eight different ones.
constexpr int kCrossStages = 4, kCrossStageBytes = 2 * 16 * 128;

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

template <int NT>
__global__ void __launch_bounds__(256) k_vocab_cross_lines(const __grid_constant__ CrossArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[8];
  wait_for_predecessor();
  let_successor_in();
  using R = CrossRow<__nv_bfloat16>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int lines = a.d / 64, row_bytes = a.d * 2;
  uint8_t* mine = smem + (size_t)8 * NT * row_bytes + (size_t)warp * (kCrossStages * kCrossStageBytes);
  const uint32_t smem32 = (uint32_t)__cvta_generic_to_shared(smem), mine32 = (uint32_t)__cvta_generic_to_shared(mine);
  const auto place = [](int row, int chunk) { return (uint32_t)((chunk ^ ((row & 1) << 2)) << 4); };
  const auto chunk_of = [&](const uint8_t* rows, int stride, int row, int line, int chunk, R& r) {
    const uint4 v = *reinterpret_cast<const uint4*>(rows + row * stride + line * 128 + place(row, chunk));
    r.r[0][0] = v.x, r.r[0][1] = v.y, r.r[0][2] = v.z, r.r[0][3] = v.w;
  };
  for (long long i = blockIdx.y; i < a.B; i += gridDim.y) {
    float sum = 0.0f;
    for (unsigned task = blockIdx.x; task < a.all; task += a.chunks) {
      const int u0 = (int)(task / a.t_chunks) * 128 + warp * 16, t0 = (int)(task % a.t_chunks) * (NT * 8);
      const bool busy = u0 < a.Tu;
      __syncthreads();                             // the tokens' rows of the task before have been read
      for (int c = threadIdx.x; c < 8 * NT * lines * 8; c += 256) {
        const int row = c / (lines * 8), chunk = c - row * (lines * 8);
        copy16(smem32 + row * row_bytes + (chunk >> 3) * 128 + place(row, chunk & 7),
               static_cast<const __nv_bfloat16*>(a.x) + (i * a.T + min(t0 + row, a.T - 1)) * a.ldx + chunk * 8);
      }
      const int2 id = busy ? cross_words(a, i, u0 + g) : make_int2(-1, -1);
      // copies: 4 rows of a line a time, 8 lanes each; rows that do not count from a place that exists
      const __nv_bfloat16 *from_w[4], *from_e[4];
      uint32_t to[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int row = 4 * k + (lane >> 3);       // k < 2: rows 0 .. 7, whose words are id.x of lanes 4 row
        const int word = __shfl_sync(0xffffffffu, k < 2 ? id.x : id.y, (row & 7) * 4);
        from_w[k] = static_cast<const __nv_bfloat16*>(a.w) + (long long)max(word, 0) * a.ldw + (lane & 7) * 8;
        from_e[k] = static_cast<const __nv_bfloat16*>(a.e) + (i * a.Tu + min(u0 + row, a.Tu - 1)) * a.lde + (lane & 7) * 8;
        to[k] = mine32 + row * 128 + place(row, lane & 7);
      }
      const auto fetch = [&](int line) {
        if (busy && line < lines) {
          const uint32_t st = (line % kCrossStages) * kCrossStageBytes;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            copy16(to[k] + st, from_w[k] + line * 64);
            copy16(to[k] + st + 2048, from_e[k] + line * 64);
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
#pragma unroll
      for (int s = 0; s < kCrossStages - 1; ++s) fetch(s);
      asm volatile("cp.async.wait_group %0;" ::"n"(kCrossStages - 2) : "memory");   // the tokens' rows came with the first line
      __syncthreads();
      if (!busy) continue;
      float cz[NT][4] = {}, ck[NT][4] = {};
      for (int l0 = 0; l0 < lines; l0 += kCrossSeg / 64) {
        float sz[NT][4] = {}, sk[NT][4] = {};
        for (int line = l0; line < lines && line < l0 + kCrossSeg / 64; ++line) {
          asm volatile("cp.async.wait_group %0;" ::"n"(kCrossStages - 2) : "memory");
          __syncwarp();
          fetch(line + kCrossStages - 1);          // into the stage that was read last time round
          const uint8_t* st = mine + (line % kCrossStages) * kCrossStageBytes;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            R wa, wb, ea, eb;
            chunk_of(st, 128, g, 0, 4 * h + q, wa);
            chunk_of(st, 128, g + 8, 0, 4 * h + q, wb);
            chunk_of(st + 2048, 128, g, 0, 4 * h + q, ea);
            chunk_of(st + 2048, 128, g + 8, 0, 4 * h + q, eb);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              R x;
              chunk_of(smem, row_bytes, 8 * j + g, line, 4 * h + q, x);
              cross_step(sz[j], wa, wb, x);
              cross_step(sk[j], ea, eb, x);
            }
          }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            cz[j][k] += sz[j][k];
            ck[j][k] += sk[j][k];
          }
      }
      sum += cross_finish<NT>(a, i, id, t0, q, cz, ck);
    }
    cross_store(a, i, sum, red);
  }
}

// sqnorm[i] += the partial sums of example i, in order.
__global__ void __launch_bounds__(256) k_vocab_cross_sum(const float* part, int B, int chunks, float* sqnorm) {
  wait_for_predecessor();
  let_successor_in();
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= B) return;
  float s = 0.0f;
  for (int k = 0; k < chunks; ++k) s += part[(long long)i * chunks + k];
  sqnorm[i] += s;
}

// Blocks of an example: enough that the device is full, as long as each has a task.
static int cross_chunks(int B, long long all) {
  const long long want = (4ll * sm_count() + B - 1) / B;
  return (int)std::max<long long>(1, std::min<long long>(std::min<long long>(all, want), kCrossChunks));
}

template <typename T>
static cudaError_t launch_cross(const CrossArgs& a, int nt, cudaStream_t s) {
  const dim3 grid(a.chunks, (unsigned)std::min(a.B, 65535));
  return nt == 1 ? launch_chained(k_vocab_cross<T, 1>, grid, 256, 0, s, a)
       : nt == 3 ? launch_chained(k_vocab_cross<T, 3>, grid, 256, 0, s, a)
                 : launch_chained(k_vocab_cross<T, 4>, grid, 256, 0, s, a);
}

constexpr int kCrossLinesMost = 225 * 1024;      // shared memory of a block of k_vocab_cross_lines, at most
static size_t lines_smem(int nt, int d) { return (size_t)8 * nt * d * 2 + 8 * kCrossStages * kCrossStageBytes; }
static cudaError_t launch_lines(const CrossArgs& a, int nt, cudaStream_t s) {
  static signed char ready[kMaxDevices] = {};    // 0 unknown, 1 ready, -1 failed
  const int dev = current_device();
  if (dev < 0) return cudaErrorInvalidDevice;
  if (!ready[dev]) {
    bool ok = true;
    for (const void* k : {(const void*)k_vocab_cross_lines<1>, (const void*)k_vocab_cross_lines<3>, (const void*)k_vocab_cross_lines<4>})
      ok = ok && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kCrossLinesMost) == cudaSuccess;
    ready[dev] = ok ? 1 : -1;
  }
  if (ready[dev] < 0) return cudaErrorInvalidValue;
  const dim3 grid(a.chunks, (unsigned)std::min(a.B, 65535));
  const size_t smem = lines_smem(nt, a.d);
  return nt == 1 ? launch_chained(k_vocab_cross_lines<1>, grid, 256, smem, s, a)
       : nt == 3 ? launch_chained(k_vocab_cross_lines<3>, grid, 256, smem, s, a)
                 : launch_chained(k_vocab_cross_lines<4>, grid, 256, smem, s, a);
}

int launch_vocab_cross(const dp_vocab_head& h, const float* lse, const int32_t* ids, const void* G_emb, long long ld_emb, int Tu,
                       float* sqnorm, float* partial, int* status, cudaStream_t s) {
  const bool f32 = h.dtype == DP_F32;
  // 8, 24 or 32 tokens a pass over the inputs' rows: as few passes as registers allow, no more columns than they need.  256 x 128 inputs,
  // width 1024, bf16, us with 8 / 24 / 32 a pass, replayed: 8 tokens 22 / 25 / 32, 9 tokens 41 / 26 / 32, 24 tokens 62 / 30 / 35, 25 tokens
  // 80 / 54 / 36, 64 tokens 142 / 84 / 73; from 33 to 48 twice 24 would be better than twice 32 (57 for 69).  In fp32 8 a pass would also be
  // where blocks are few (64 x 128 inputs, width 256: 9 tokens 16 / 21 / 23, 32 tokens 17 / 24 / 27).
  const int nt = h.T <= 8 ? 1 : h.T <= 24 ? 3 : 4;
  CrossArgs a = {h.X, h.W, G_emb, h.bias, h.labels, h.weights, lse, ids, sqnorm, h.ldx, h.ldw, ld_emb, h.B, h.T, Tu, h.d, h.V};
  a.t_chunks = (unsigned)ceil_div(h.T, 8 * nt);
  const long long all = (long long)ceil_div(Tu, 128) * a.t_chunks;
  if (all > 0x7fffffffll) return DP_ERR_UNSUPPORTED;
  a.all = (unsigned)all;
  a.chunks = (unsigned)cross_chunks(h.B, all);
  if (a.chunks > 1) a.out = partial;
  const int e = f32 ? 4 : 8;
  a.vec = !misaligned(h.X, 16) && !misaligned(h.W, 16) && !misaligned(G_emb, 16) && h.ldx % e == 0 && h.ldw % e == 0 && ld_emb % e == 0;
  a.status = status;
  note_launch(1);
  const bool whole = !f32 && a.vec && h.d % 64 == 0 && lines_smem(nt, h.d) <= kCrossLinesMost;
  const cudaError_t rc = f32 ? launch_cross<float>(a, nt, s) : whole ? launch_lines(a, nt, s) : launch_cross<__nv_bfloat16>(a, nt, s);
  if (rc != cudaSuccess) return DP_ERR_CUDA;
  if (a.chunks > 1) {
    note_launch(1);
    if (launch_chained(k_vocab_cross_sum, (unsigned)ceil_div(h.B, 256), 256, 0, s, partial, h.B, a.chunks, sqnorm) != cudaSuccess)
      return DP_ERR_CUDA;
  }
  return DP_OK;
}

}  // namespace dpk
