// Tensors whose per-example gradients are given as rows, [B][width] fp32: small parameters (a position-bias table, the
// gain of a head norm) for which a layer's own kernel has already formed every example's gradient.  The two steps that
// the whole-model clip needs of them: the squared norm of every example's row, and the clipped sum over the examples.
// One tensor's rows are read once, a few MB at most, so that both are bound by latency; many tensors are walked one after
// another by the norms (every one costs a trip to memory, and a row narrower than 256 leaves threads idle).  Sums run in a
// fixed order.
#include "dp_chain.cuh"
#include "dp_internal.h"

namespace dpk {

constexpr int kMaxRows = 128;
struct RowSet {
  const float* grad[kMaxRows];
  float* acc[kMaxRows];
  long long width[kMaxRows];
  int col0[kMaxRows + 1];        // first 32-column block of the tensor (accumulate)
  int n;
};

// One block per example: all tensors' rows, squared and summed in fp64 per thread, then by a fixed tree, rounded once at the
// end.  A thread's run is width / 256 long: in fp32 a row of 2^24 equal values came out wrong by 9e-4, and a squared norm that is
// too small lets its example add more than C.  In a graph, against fp32 sums: 256 rows of 512 2.0 us (1.9), with 48 more
// tensors of width 64 14.6 (14.4), 8 rows of 2^20 196 (182); with 8 loads in flight in place of 4 these take 2.0, 15.1 and 117.
__global__ void __launch_bounds__(256)
k_rows_sqnorm(const __grid_constant__ RowSet R, float* sqnorm, int add) {
  __shared__ double red[8];
  wait_for_predecessor();
  let_successor_in();
  const long long i = blockIdx.x;
  double s = 0.0;
  for (int k = 0; k < R.n; ++k) {
    const float* row = R.grad[k] + i * R.width[k];
#pragma unroll 4
    for (long long j = threadIdx.x; j < R.width[k]; j += 256) {
      const double x = row[j];
      s = fma(x, x, s);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += red[w];
    sqnorm[i] = (float)(add ? sqnorm[i] + t : t);
  }
}

// acc[j] += sum_i clip[i] * grad[i][j].  A block owns 32 columns of one tensor; its 32 warps take every 32nd example
// each (8 loads in flight) and their sums are added in warp order.
constexpr int kAccWarps = 32;
__global__ void __launch_bounds__(32 * kAccWarps)
k_rows_accum(const __grid_constant__ RowSet R, int B, const float* clip) {
  __shared__ float part[kAccWarps][32];
  wait_for_predecessor();
  let_successor_in();
  int k = 0;
  while (R.col0[k + 1] <= (int)blockIdx.x) ++k;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long width = R.width[k], col = (long long)((int)blockIdx.x - R.col0[k]) * 32 + lane;
  float s = 0.0f;
  if (col < width) {
    const float* g = R.grad[k] + col;
#pragma unroll 8
    for (int i = warp; i < B; i += kAccWarps) s = fmaf(clip[i], g[(long long)i * width], s);
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && col < width) {
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < kAccWarps; ++w) t += part[w][lane];
    R.acc[k][col] += t;
  }
}

static bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

static int check_rows(const dp_rows* rows, int n, int B, bool need_acc) {
  if (!rows || n <= 0 || B <= 0) return DP_ERR_ARG;
  for (int k = 0; k < n; ++k) {
    if (!rows[k].grad || rows[k].width <= 0 || rows[k].width > (int64_t)1 << 30 || (need_acc && !rows[k].acc)) return DP_ERR_ARG;
    if (misaligned(rows[k].grad, 4) || (need_acc && misaligned(rows[k].acc, 4))) return DP_ERR_ALIGN;
  }
  return DP_OK;
}

// Tensors [k, ...) of the list, as many as one launch takes; returns the index behind the last.
static int fill_rows(RowSet& R, const dp_rows* rows, int k, int n) {
  R.n = 0;
  R.col0[0] = 0;
  for (; k < n && R.n < kMaxRows; ++k) {
    const long long blocks = (rows[k].width + 31) / 32;
    if (R.n && R.col0[R.n] + blocks > (1 << 30)) break;
    R.grad[R.n] = rows[k].grad;
    R.acc[R.n] = rows[k].acc;
    R.width[R.n] = rows[k].width;
    R.col0[R.n + 1] = R.col0[R.n] + (int)blocks;
    ++R.n;
  }
  return k;
}

}  // namespace dpk

using namespace dpk;

extern "C" {

int dp_rows_sqnorms(const dp_rows* rows, int n_rows, int B, float* sqnorm, int accumulate_into, void* cuda_stream) {
  const int rc = check_rows(rows, n_rows, B, false);
  if (rc != DP_OK) return rc;
  if (!sqnorm) return DP_ERR_ARG;
  if (misaligned(sqnorm, 4)) return DP_ERR_ALIGN;
  for (int k = 0; k < n_rows;) {
    RowSet R;
    const int add = accumulate_into || k > 0;
    k = fill_rows(R, rows, k, n_rows);
    const cudaError_t e = launch_chained(k_rows_sqnorm, B, 256, 0, static_cast<cudaStream_t>(cuda_stream), R, sqnorm, add);
    note_launch(1);
    if (e != cudaSuccess) return DP_ERR_CUDA;
  }
  return DP_OK;
}

int dp_rows_clipped_accumulate(const dp_rows* rows, int n_rows, int B, const float* clip, void* cuda_stream) {
  const int rc = check_rows(rows, n_rows, B, true);
  if (rc != DP_OK) return rc;
  if (!clip) return DP_ERR_ARG;
  if (misaligned(clip, 4)) return DP_ERR_ALIGN;
  for (int k = 0; k < n_rows;) {
    RowSet R;
    k = fill_rows(R, rows, k, n_rows);
    const cudaError_t e = launch_chained(k_rows_accum, R.col0[R.n], 32 * kAccWarps, 0, static_cast<cudaStream_t>(cuda_stream), R, B, clip);
    note_launch(1);
    if (e != cudaSuccess) return DP_ERR_CUDA;
  }
  return DP_OK;
}

}  // extern "C"
