// A learned relative position bias by buckets: table[num_buckets][n_heads], score bias
//   bias[h][q][k] = table[bucket(k - q - offset)][h]
// and every example's gradient of the table from the gradient G[b][h][q][k] of the scores,
//   rows[b][n][h] = sum over (q, k) with bucket(k - q - offset) = n of G[b][h][q][k].
//
// The bucket depends on k - q alone, so both are Toeplitz: the bias is one line of Tq + Tk - 1 values per head that
// every query reads at another place, and the gradient is a sum along diagonals first, over buckets last.  Both kernels
// are bound by memory: the bias by writing [H][Tq][Tk], the gradient by reading G once.
#include <cstring>

#include "dp_internal.h"

namespace dpk {

constexpr int kMaxBuckets = 256;
constexpr int kMaxTokens = 1 << 24;              // relative positions stay far inside 32 bits

// Buckets of one side by distance n >= 0: bucket j covers [start[j], start[j + 1]), start[0] = 0, the last one all beyond.
// With both sides, a key behind its query (rel > 0) has half added; with one side it counts as distance 0.
struct Buckets {
  int half;                                      // buckets per side
  int both;
  int start[kMaxBuckets + 1];
  __device__ __forceinline__ int of(int rel) const {
    const int n = rel > 0 ? (both ? rel : 0) : -rel;
    int lo = 0, hi = half;                       // start[lo] <= n < start[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= n) lo = mid; else hi = mid;
    }
    return lo + ((both && rel > 0) ? half : 0);
  }
  // Relative positions of bucket b, both ends included; false where the bucket is empty.
  __device__ __forceinline__ bool range(int b, int& lo, int& hi) const {
    const int far = 1 << 30;
    if (b < half) {
      lo = b + 1 < half ? 1 - start[b + 1] : -far;
      hi = b == 0 ? (both ? 0 : far) : -start[b];
      return lo <= hi;
    }
    const int j = b - half;
    lo = j == 0 ? 1 : start[j];
    hi = j + 1 < half ? start[j + 1] - 1 : far;
    return lo <= hi;
  }
};

// ---------------------------------------------------------------------------------------------
// Forward.  A block of 8 warps writes a tile of columns x rows of one head; the line of bias values that the tile
// needs is looked up once into shared memory (in the output's type).  VEC: a lane owns 16 bytes of neighbouring columns
// and walks down the rows: from one row to the next its window of the line moves by one value, so it shifts its
// registers and reads a single new value.  Otherwise a lane owns every 32nd column, one element per store.
// ---------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ T to_type(float x);
template <> __device__ __forceinline__ float to_type<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 to_type<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

constexpr int kBiasCols = 256, kBiasRowsPerWarp = 16;

template <typename T, typename TT, bool VEC>
__global__ void __launch_bounds__(256)
k_relpos_bias(const TT* __restrict__ table, const __grid_constant__ Buckets bk, int n_heads, int Tq, int Tk, int offset,
              T* __restrict__ out, long long stride_h, long long stride_q, int warps_x) {
  constexpr int V = 16 / sizeof(T);
  extern __shared__ __align__(16) unsigned char bias_smem[];
  T* line = reinterpret_cast<T*>(bias_smem);
  const int warps_y = 8 / warps_x;
  const int cols = kBiasCols * warps_x, rows = kBiasRowsPerWarp * warps_y;
  const int c0 = blockIdx.x * cols, q0 = blockIdx.y * rows, h = blockIdx.z;
  const int n_line = cols + rows - 1;
  // line[i]: relative position (c0 - q0 - offset) + i - (rows - 1)
  const int rel0 = c0 - q0 - offset - (rows - 1);
  for (int i = threadIdx.x; i < n_line; i += 256)
    line[i] = to_type<T>(to_float(table[(long long)bk.of(rel0 + i) * n_heads + h]));
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int wx = warp % warps_x, wy = warp / warps_x;
  const int r0 = wy * kBiasRowsPerWarp;
  const int r1 = min(r0 + kBiasRowsPerWarp, Tq - q0);
  T* o = out + (long long)h * stride_h + (long long)q0 * stride_q + c0;
  if (VEC) {
    for (int cc = wx * kBiasCols + lane * V; cc < (wx + 1) * kBiasCols; cc += 32 * V) {
      if (c0 + cc >= Tk) break;
      T w[V];
#pragma unroll
      for (int j = 0; j < V; ++j) w[j] = line[cc + j - r0 + rows - 1];
      for (int r = r0; r < r1; ++r) {
        uint4 u;
        memcpy(&u, w, 16);
        *reinterpret_cast<uint4*>(o + (long long)r * stride_q + cc) = u;
#pragma unroll
        for (int j = V - 1; j > 0; --j) w[j] = w[j - 1];
        if (r + 1 < r1) w[0] = line[cc - (r + 1) + rows - 1];
      }
    }
  } else {
    for (int r = r0; r < r1; ++r)
#pragma unroll 4
      for (int cc = wx * kBiasCols + lane; cc < (wx + 1) * kBiasCols; cc += 32)
        if (c0 + cc < Tk) o[(long long)r * stride_q + cc] = line[cc - r + rows - 1];
  }
}

// ---------------------------------------------------------------------------------------------
// Per-example gradient.  A group of LG lanes (a warp or a part of one) takes a unit: up to R rows of one (example, head)
// times LG * V neighbouring columns, V columns a lane.  Walking down the rows, a diagonal moves one column to the right
// per row: inside a lane that is another register of its V sums (renamed by unrolling the rows V at a time), at the
// lane's right edge the sum is handed to the next lane, and the one that leaves the last lane is complete and goes to
// shared memory.  That costs one add per element and one shuffle per V of them, with no atomic.  After the rows the
// group sums its line of diagonals by buckets, in a fixed order.
// ---------------------------------------------------------------------------------------------
template <typename T, int V> struct Strip;
template <> struct Strip<__nv_bfloat16, 8> {
  uint4 u;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { u = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void clear() { u = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ float get(int j) const {
    const uint32_t w = j < 2 ? u.x : j < 4 ? u.y : j < 6 ? u.z : u.w;
    return __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
  }
};
template <> struct Strip<__nv_bfloat16, 2> {
  uint32_t u;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { u = __ldcs(reinterpret_cast<const unsigned int*>(p)); }
  __device__ __forceinline__ void clear() { u = 0u; }
  __device__ __forceinline__ float get(int j) const { return __uint_as_float(j & 1 ? u & 0xffff0000u : u << 16); }
};
template <> struct Strip<__nv_bfloat16, 1> {
  unsigned short u;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { u = __ldcs(reinterpret_cast<const unsigned short*>(p)); }
  __device__ __forceinline__ void clear() { u = 0; }
  __device__ __forceinline__ float get(int) const { return __uint_as_float((uint32_t)u << 16); }
};
template <> struct Strip<float, 4> {
  float4 u;
  __device__ __forceinline__ void load(const float* p) { u = __ldcs(reinterpret_cast<const float4*>(p)); }
  __device__ __forceinline__ void clear() { u = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ float get(int j) const { return j == 0 ? u.x : j == 1 ? u.y : j == 2 ? u.z : u.w; }
};
template <> struct Strip<float, 1> {
  float u;
  __device__ __forceinline__ void load(const float* p) { u = __ldcs(p); }
  __device__ __forceinline__ void clear() { u = 0.f; }
  __device__ __forceinline__ float get(int) const { return u; }
};

constexpr int kGradWarps = 8;
constexpr int kGradRowBlock = 8;                 // rows whose loads are issued together

struct GradArgs {
  long long stride_b, stride_h, stride_q;
  int B, H, Tq, Tk, offset, causal;
  int lg_log, R, n_ct, n_rt;                     // log2 of lanes per group, rows per unit, column and row units
  long long units;
  int accumulate;
};

template <typename T, int V>
__global__ void __launch_bounds__(32 * kGradWarps)
k_relpos_grad(const T* __restrict__ G, const __grid_constant__ Buckets bk, const __grid_constant__ GradArgs a,
              const int32_t* __restrict__ q_len, const int32_t* __restrict__ k_len, float* __restrict__ partial,
              float* __restrict__ rows) {
  extern __shared__ float diag_smem[];
  const int LG = 1 << a.lg_log, CW = LG * V;
  const int lane = threadIdx.x & 31, li = lane & (LG - 1);
  const int group = threadIdx.x >> a.lg_log;     // within the block
  const int groups = (32 * kGradWarps) >> a.lg_log;
  float* buf = diag_smem + (long long)group * (a.R + CW);
  const long long unit = (long long)blockIdx.x * groups + group;
  const bool live = unit < a.units;
  const int per_bh = a.n_ct * a.n_rt;
  const long long bh = live ? unit / per_bh : 0;
  const int u_in = live ? (int)(unit - bh * per_bh) : 0;
  const int rt = u_in / a.n_ct, ct = u_in - rt * a.n_ct;
  const int b = (int)(bh / a.H), h = (int)(bh - (long long)b * a.H);
  const int q_end = q_len ? min(max(q_len[b], 0), a.Tq) : a.Tq;
  const int k_end = k_len ? min(max(k_len[b], 0), a.Tk) : a.Tk;
  const int c0 = ct * CW, c = c0 + li * V;
  int q0 = rt * a.R;
  const int r_hi = min(q0 + a.R, q_end);
  // a causal unit starts at the first row that sees its first column
  if (a.causal) q0 = max(q0, c0 - a.offset);
  int n = live && c0 < k_end ? max(r_hi - q0, 0) : 0;
  const int valid = min(max(k_end - c, 0), V);   // of this lane's columns
  const T* p = G + (long long)b * a.stride_b + (long long)h * a.stride_h + (long long)q0 * a.stride_q + c;

  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.0f;
  // the groups of a warp walk together: as many rounds as the longest of them
  int rounds = (n + kGradRowBlock - 1) / kGradRowBlock;
  rounds = __reduce_max_sync(0xffffffffu, rounds);
  for (int t = 0; t < rounds; ++t) {
    const int r0 = t * kGradRowBlock;
    Strip<T, V> x[kGradRowBlock];
#pragma unroll
    for (int r = 0; r < kGradRowBlock; ++r) {
      x[r].clear();
      const bool seen = r0 + r < n && valid > 0 && (!a.causal || c <= q0 + r0 + r + a.offset);
      if (seen) x[r].load(p + (long long)(r0 + r) * a.stride_q);
    }
#pragma unroll
    for (int r = 0; r < kGradRowBlock; ++r) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int s = (j + kGradRowBlock * V - r) % V;       // the register that holds column j's diagonal in row r
        acc[s] += j < valid ? x[r].get(j) : 0.0f;            // selected, never multiplied: a masked place may hold NaN
      }
      const int s = (V - 1 + kGradRowBlock * V - r) % V;
      const float out = acc[s];
      const float in = __shfl_up_sync(0xffffffffu, out, 1, LG);
      if (li == LG - 1 && r0 + r < a.R) buf[CW - 1 - (r0 + r) + a.R] = out;
      acc[s] = li == 0 ? 0.0f : in;
    }
  }
  // buf[d + R]: diagonal d = (column - c0) - (row - q0), -walked <= d < CW.  (kGradRowBlock is a multiple of V.)
  const int walked = rounds * kGradRowBlock;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int d = li * V + j - walked;
    if (d + a.R >= 0) buf[d + a.R] = acc[j];
  }
  __syncwarp();
  const int rel = c0 - q0 - a.offset;            // relative position of diagonal 0
  const int d_lo = max(-walked, -a.R), d_hi = a.causal ? min(CW - 1, -rel) : CW - 1;
  const int nb = bk.both ? 2 * bk.half : bk.half;
  for (int k = 0; k < nb; ++k) {
    int lo, hi;
    const bool some = bk.range(k, lo, hi);
    lo = max(lo - rel, d_lo);
    hi = min(hi - rel, d_hi);
    float s = 0.0f;
    if (some && n > 0)
      for (int d = lo + li; d <= hi; d += LG) s += buf[d + a.R];
    for (int o = LG >> 1; o > 0; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o, LG);
    if (live && li == 0) {
      if (partial) {
        partial[unit * nb + k] = s;
      } else {
        float* w = rows + ((long long)b * nb + k) * a.H + h;
        *w = a.accumulate ? *w + s : s;
      }
    }
  }
}

// rows[b][n][h] (+)= sum over the units of (b, h), in order.
__global__ void __launch_bounds__(256)
k_relpos_units(const float* __restrict__ partial, int B, int H, int nb, int units, float* __restrict__ rows, int add) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long long)B * H * nb) return;
  const int n = (int)(i % nb);                   // neighbours read neighbouring words
  const long long bh = i / nb;
  const float* p = partial + bh * units * nb + n;
  float s = 0.0f;
#pragma unroll 4
  for (int u = 0; u < units; ++u) s += p[(long long)u * nb];
  const long long b = bh / H, h = bh - b * H;
  float* w = rows + (b * nb + n) * H + h;
  *w = add ? *w + s : s;
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
// a <- a * m for a little-endian number of `len` 32-bit words; returns the new length.
static int mul_small(uint32_t* a, int len, uint32_t m) {
  uint64_t carry = 0;
  for (int i = 0; i < len; ++i) {
    carry += (uint64_t)a[i] * m;
    a[i] = (uint32_t)carry;
    carry >>= 32;
  }
  if (carry) a[len++] = (uint32_t)carry;
  return len;
}
static int power_product(uint32_t* a, uint32_t x, int px, uint32_t y, int py) {
  int len = 1;
  a[0] = 1;
  for (int i = 0; i < px; ++i) len = mul_small(a, len, x);
  for (int i = 0; i < py; ++i) len = mul_small(a, len, y);
  return len;
}
// (n / exact)^rest >= (far / exact)^j, i.e. n^rest * exact^j >= far^j * exact^rest, in whole numbers of any length.
static bool border_reached(uint32_t n, uint32_t exact, uint32_t far, int rest, int j) {
  uint32_t a[2 * kMaxBuckets + 2], b[2 * kMaxBuckets + 2];
  const int la = power_product(a, n, rest, exact, j), lb = power_product(b, far, j, exact, rest);
  if (la != lb) return la > lb;
  for (int i = la - 1; i >= 0; --i)
    if (a[i] != b[i]) return a[i] > b[i];
  return true;
}

static int make_buckets(int num_buckets, int max_distance, int both, Buckets* bk) {
  if (num_buckets < 2 || num_buckets > kMaxBuckets || max_distance < 1 || max_distance > kMaxTokens) return DP_ERR_ARG;
  if (both && (num_buckets & 1)) return DP_ERR_ARG;
  const int half = both ? num_buckets / 2 : num_buckets, exact = half / 2, rest = half - exact;
  if (exact < 1 || max_distance <= exact) return DP_ERR_ARG;
  bk->half = half;
  bk->both = both ? 1 : 0;
  for (int j = 0; j <= exact; ++j) bk->start[j] = j;
  for (int j = 1; j < rest; ++j) {
    // the border lies at exact * (max_distance / exact)^(j / rest); where fp64 cannot tell on which side of a whole
    // number that is, it is decided in whole numbers
    const double t = exact * std::pow((double)max_distance / exact, (double)j / rest);
    double n = std::ceil(t);
    const double near = std::floor(t + 0.5);
    if (std::fabs(t - near) < 1e-9 * t) n = border_reached((uint32_t)near, exact, max_distance, rest, j) ? near : near + 1.0;
    bk->start[exact + j] = (int)n;
  }
  bk->start[half] = 0x7fffffff;
  return DP_OK;
}

static bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

static int check_relpos(const dp_relpos* p, Buckets* bk) {
  if (!p || p->n_heads <= 0 || p->Tq <= 0 || p->Tk <= 0) return DP_ERR_ARG;
  if (p->Tq > kMaxTokens || p->Tk > kMaxTokens || p->offset > 4 * (int64_t)kMaxTokens || p->offset < -4 * (int64_t)kMaxTokens)
    return DP_ERR_ARG;
  return make_buckets(p->num_buckets, p->max_distance, p->bidirectional, bk);
}

template <typename T, typename TT>
static cudaError_t launch_bias(const dp_relpos& p, const Buckets& bk, const void* table, void* out, long long sh,
                               long long sq, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  // few queries: all eight warps side by side along the keys; otherwise below one another, which shares more of the line
  const int wx = p.Tq <= kBiasRowsPerWarp ? 8 : 1, wy = 8 / wx;
  const int cols = kBiasCols * wx, rows = kBiasRowsPerWarp * wy;
  const dim3 grid(ceil_div(p.Tk, cols), ceil_div(p.Tq, rows), p.n_heads);
  const size_t smem = (size_t)(cols + rows) * sizeof(T);
  const bool vec = !misaligned(out, 16) && p.Tk % V == 0 && sh % V == 0 && sq % V == 0;
  if (vec)
    k_relpos_bias<T, TT, true><<<grid, 256, smem, s>>>(static_cast<const TT*>(table), bk, p.n_heads, p.Tq, p.Tk,
                                                       (int)p.offset, static_cast<T*>(out), sh, sq, wx);
  else
    k_relpos_bias<T, TT, false><<<grid, 256, smem, s>>>(static_cast<const TT*>(table), bk, p.n_heads, p.Tq, p.Tk,
                                                        (int)p.offset, static_cast<T*>(out), sh, sq, wx);
  return counted(1);
}

// How G is cut: V columns a lane, LG lanes a group, R rows a unit.  Many rows per unit amortise the sum over buckets;
// few give every warp slot of the GPU a unit.
struct GradPlan { int V, lg_log, R, n_ct, n_rt; long long units; };
static GradPlan plan_grad(int B, const dp_relpos& p, int V) {
  GradPlan g;
  g.V = V;
  int lanes = ceil_div(p.Tk, V);
  g.lg_log = 2;
  while (g.lg_log < 5 && (1 << g.lg_log) < lanes) ++g.lg_log;
  const int CW = V << g.lg_log;
  g.n_ct = ceil_div(p.Tk, CW);
  g.R = (512 << g.lg_log) >> 5;                  // bounds the shared memory of a warp's groups
  const long long want = 148ll * 32 * (32 >> g.lg_log);
  while (g.R > 32 && (long long)B * p.n_heads * g.n_ct * ceil_div(p.Tq, g.R) < want) g.R >>= 1;
  g.n_rt = ceil_div(p.Tq, g.R);
  g.units = (long long)B * p.n_heads * g.n_ct * g.n_rt;
  return g;
}

// Columns per lane: 16 bytes of them where every row starts on a 16-byte boundary and ends on one, else 4, else one.
static int grad_vec(const void* G, int dtype, int Tk, long long sb, long long sh, long long sq) {
  const int es = dtype == DP_F32 ? 4 : 2;
  for (int bytes : {16, 4}) {
    const int V = bytes / es;
    if (!misaligned(G, bytes) && Tk % V == 0 && sb % V == 0 && sh % V == 0 && sq % V == 0) return V;
  }
  return 1;
}

template <typename T, int V>
static cudaError_t launch_grad(const void* G, const Buckets& bk, const GradArgs& a, const int32_t* q_len,
                               const int32_t* k_len, float* partial, float* rows, cudaStream_t s) {
  const int groups = (32 * kGradWarps) >> a.lg_log;
  const size_t smem = (size_t)groups * (a.R + (V << a.lg_log)) * sizeof(float);
  const long long blocks = (a.units + groups - 1) / groups;
  if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  k_relpos_grad<T, V><<<(unsigned)blocks, 32 * kGradWarps, smem, s>>>(static_cast<const T*>(G), bk, a, q_len, k_len,
                                                                      partial, rows);
  return counted(1);
}

}  // namespace dpk

using namespace dpk;

extern "C" {

int dp_relpos_bucket_starts(int num_buckets, int max_distance, int bidirectional, int32_t* starts) {
  Buckets bk;
  const int rc = make_buckets(num_buckets, max_distance, bidirectional, &bk);
  if (rc != DP_OK) return rc;
  if (!starts) return DP_ERR_ARG;
  memcpy(starts, bk.start, bk.half * sizeof(int32_t));
  return DP_OK;
}

int dp_relpos_bias(const dp_relpos* p, const void* table, int table_dtype, void* out, int out_dtype, int64_t stride_h,
                   int64_t stride_q, void* cuda_stream) {
  Buckets bk;
  const int rc = check_relpos(p, &bk);
  if (rc != DP_OK) return rc;
  if (!table || !out || stride_h < 0 || stride_q < p->Tk) return DP_ERR_ARG;
  if ((table_dtype != DP_F32 && table_dtype != DP_BF16) || (out_dtype != DP_F32 && out_dtype != DP_BF16)) return DP_ERR_ARG;
  if (p->n_heads > 65535 || ceil_div(p->Tq, kBiasRowsPerWarp * 8) > 65535) return DP_ERR_UNSUPPORTED;
  if (misaligned(table, table_dtype == DP_F32 ? 4 : 2) || misaligned(out, out_dtype == DP_F32 ? 4 : 2)) return DP_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (out_dtype == DP_F32)
    e = table_dtype == DP_F32 ? launch_bias<float, float>(*p, bk, table, out, stride_h, stride_q, s)
                              : launch_bias<float, __nv_bfloat16>(*p, bk, table, out, stride_h, stride_q, s);
  else
    e = table_dtype == DP_F32 ? launch_bias<__nv_bfloat16, float>(*p, bk, table, out, stride_h, stride_q, s)
                              : launch_bias<__nv_bfloat16, __nv_bfloat16>(*p, bk, table, out, stride_h, stride_q, s);
  return e == cudaSuccess ? DP_OK : DP_ERR_CUDA;
}

size_t dp_relpos_workspace_bytes(const dp_relpos* p, int B) {
  Buckets bk;
  if (check_relpos(p, &bk) != DP_OK || B <= 0) return 0;
  long long most = 0;                            // over the ways to cut G, which depend on its alignment
  for (int V : {8, 4, 2, 1}) {
    const GradPlan g = plan_grad(B, *p, V);
    if (g.units > most) most = g.units;
  }
  return (size_t)most * p->num_buckets * sizeof(float);
}

int dp_relpos_bias_grad(const dp_relpos* p, int B, int causal, const void* G, int dtype, int64_t stride_b,
                        int64_t stride_h, int64_t stride_q, const int32_t* q_len, const int32_t* k_len, float* rows,
                        int accumulate_into, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  Buckets bk;
  const int rc = check_relpos(p, &bk);
  if (rc != DP_OK) return rc;
  if (B <= 0 || !G || !rows || stride_b < 0 || stride_h < 0 || stride_q < 0) return DP_ERR_ARG;
  if (dtype != DP_F32 && dtype != DP_BF16) return DP_ERR_ARG;
  if (misaligned(G, dtype == DP_F32 ? 4 : 2) || misaligned(rows, 4) || misaligned(q_len, 4) || misaligned(k_len, 4))
    return DP_ERR_ALIGN;
  const int V = grad_vec(G, dtype, p->Tk, stride_b, stride_h, stride_q);
  const GradPlan g = plan_grad(B, *p, V);
  const int nb = p->num_buckets, per_bh = g.n_ct * g.n_rt;
  if (g.units > 0x7fffffffll || (long long)B * p->n_heads * nb > 0x7fffffffll * 128) return DP_ERR_UNSUPPORTED;
  float* partial = nullptr;
  if (per_bh > 1) {
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < (size_t)g.units * nb * sizeof(float))
      return DP_ERR_WORKSPACE;
    partial = static_cast<float*>(workspace);
  }
  GradArgs a = {stride_b, stride_h, stride_q, B, p->n_heads, p->Tq, p->Tk, (int)p->offset, causal ? 1 : 0,
                g.lg_log, g.R, g.n_ct, g.n_rt, g.units, accumulate_into ? 1 : 0};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (dtype == DP_F32)
    e = V == 4 ? launch_grad<float, 4>(G, bk, a, q_len, k_len, partial, rows, s)
               : launch_grad<float, 1>(G, bk, a, q_len, k_len, partial, rows, s);
  else
    e = V == 8   ? launch_grad<__nv_bfloat16, 8>(G, bk, a, q_len, k_len, partial, rows, s)
        : V == 2 ? launch_grad<__nv_bfloat16, 2>(G, bk, a, q_len, k_len, partial, rows, s)
                 : launch_grad<__nv_bfloat16, 1>(G, bk, a, q_len, k_len, partial, rows, s);
  if (e != cudaSuccess) return DP_ERR_CUDA;
  if (partial) {
    const long long n = (long long)B * p->n_heads * nb;
    k_relpos_units<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(partial, B, p->n_heads, nb, per_bh, rows, a.accumulate);
    if (counted(1) != cudaSuccess) return DP_ERR_CUDA;
  }
  return DP_OK;
}

}  // extern "C"
