// RMS norm of every query and key head with a learned gain, and the position rotation, in one pass; and the backward
// pass, which also yields every example's gradients of the two gains.  With x one head of one token, D wide:
//   r = 1 / sqrt(mean(x^2) + eps),  xhat = r x,  y = R(p) (gain * xhat)
// where R(p) turns the pair (a, b) number j by the angle p * inv_freq[j]: (a cos - b sin, b cos + a sin).  Backward, with
// u = R(-p) dy and w = gain * u:
//   dx = r (w - xhat mean(w xhat)),     d gain of example i = sum over its tokens and heads of u * xhat.
// Bound by memory: forward reads x and writes y, backward reads x and dy and writes dx.  A group of lanes holds a whole
// head in registers, so nothing is read twice; the gains' gradients stay in registers over all heads a lane meets.
//
// The angle.  p * inv_freq loses its fractional turns in fp32 at far positions.  The host turns inv_freq[j] / (2 pi) into
// a 64-bit binary fraction of a turn; p times that, modulo 2^64, is an ordinary wrapping integer product, and its upper
// 32 bits are the angle in turns to 2^-32, at any 32-bit position, for the price of one multiplication.
#include "dp_internal.h"

namespace dpk {

constexpr int kMaxPairs = 256;                   // D <= 512

struct View {                                    // [B, T, H, D], D contiguous; strides in elements
  const void* in;
  const void* dout;                              // backward: gradient of the output
  void* out;                                     // forward: the output; backward: gradient of the input
  const float* gain;                             // [D] or null (ones)
  float* rows;                                   // backward: [B][D] gain gradients, or null
  long long in_b, in_t, in_h, dout_b, dout_t, dout_h, out_b, out_t, out_h;
  int heads, slices;                             // heads, and groups' shares of them per token
};

struct QkArgs {
  View v[2];                                     // queries, keys
  const int32_t* positions;                      // [B, T] or null: 0 .. T-1
  const int32_t* lengths;                        // [B] or null
  float eps, inv_dim;
  int B, T, pairs, rot_pairs, heads_per_item, group_log;
  int chunk, n_chunks;                           // backward: tokens per block, blocks per example and kind
  int accumulate;
  float* partial;                                // backward: [B][n_chunks][2][D], or null
  unsigned long long turn[kMaxPairs];            // fraction of a turn per position, 2^-64 units
};

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// How a lane holds its share of a head: NP pairs (a[i], b[i]).
// VEC: NP neighbouring pairs fetched as two 16-byte vectors.  In the `halves` layout (pair j = elements j and
//   j + rot/2) these are the vectors at j0 and j0 + rot/2; in the `neighbours` layout (elements 2j, 2j + 1), and beyond the
//   rotated part, the two vectors at 2 j0 (beyond the rotated part any pairing serves: the angle is 0).
// Otherwise: pairs lane, lane + group, ...; elements one by one.
template <typename T, int NP, bool VEC, bool INTER>
struct Lane {
  int o1, o2;                                    // VEC: the two vectors' first elements
  int p0, step, pairs, rot_pairs;                // otherwise
  bool on;
  __device__ __forceinline__ Lane(int li, int group, const QkArgs& a) : step(group), pairs(a.pairs), rot_pairs(a.rot_pairs) {
    if (VEC) {
      p0 = li * NP;
      on = p0 < a.pairs;
      const bool split = !INTER && p0 < a.rot_pairs;
      o1 = split ? p0 : 2 * p0;
      o2 = split ? p0 + a.rot_pairs : 2 * p0 + NP;
    } else {
      p0 = li;
      on = true;
      o1 = o2 = 0;
    }
  }
  __device__ __forceinline__ int pair(int i) const { return VEC ? p0 + i : p0 + i * step; }
  __device__ __forceinline__ bool has(int i) const { return VEC ? on : pair(i) < pairs; }
  __device__ __forceinline__ void places(int i, int& e1, int& e2) const {    // of pair(i)
    const int p = pair(i);
    if (!INTER && p < rot_pairs) { e1 = p; e2 = p + rot_pairs; }
    else { e1 = 2 * p; e2 = 2 * p + 1; }
  }
  struct Raw { uint4 u1, u2; };
  template <typename P>
  __device__ __forceinline__ void read(const P* x, float (&f)[2 * NP]) const {     // f[i] = a, f[NP + i] = b
    if constexpr (VEC) {
      const uint4* q1 = reinterpret_cast<const uint4*>(x + o1);
      const uint4* q2 = reinterpret_cast<const uint4*>(x + o2);
      Raw r;
      r.u1 = r.u2 = make_uint4(0u, 0u, 0u, 0u);
      if (on) { r.u1 = *q1; r.u2 = *q2; }
      float t[2 * NP];
      const uint32_t w[8] = {r.u1.x, r.u1.y, r.u1.z, r.u1.w, r.u2.x, r.u2.y, r.u2.z, r.u2.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if constexpr (sizeof(P) == 4) {
          t[k] = __uint_as_float(w[k]);
        } else {
          t[2 * k] = __uint_as_float(w[k] << 16);
          t[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        f[i] = INTER ? t[2 * i] : t[i];
        f[NP + i] = INTER ? t[2 * i + 1] : t[NP + i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        f[i] = f[NP + i] = 0.0f;
        if (has(i)) {
          int e1, e2;
          places(i, e1, e2);
          f[i] = load1(x + e1);
          f[NP + i] = load1(x + e2);
        }
      }
    }
  }
  template <typename P>
  __device__ __forceinline__ void write(P* x, const float (&f)[2 * NP]) const {
    if constexpr (VEC) {
      if (!on) return;
      float t[2 * NP];
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        t[INTER ? 2 * i : i] = f[i];
        t[INTER ? 2 * i + 1 : NP + i] = f[NP + i];
      }
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if constexpr (sizeof(P) == 4) {
          w[k] = __float_as_uint(t[k]);
        } else {
          const __nv_bfloat162 h = __floats2bfloat162_rn(t[2 * k], t[2 * k + 1]);
          w[k] = *reinterpret_cast<const uint32_t*>(&h);
        }
      }
      *reinterpret_cast<uint4*>(x + o1) = make_uint4(w[0], w[1], w[2], w[3]);
      *reinterpret_cast<uint4*>(x + o2) = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        if (has(i)) {
          int e1, e2;
          places(i, e1, e2);
          store1(x + e1, f[i]);
          store1(x + e2, f[NP + i]);
        }
      }
    }
  }
  // fp32 per-element parameters (gains) in the same order; 1 where there are none
  __device__ __forceinline__ void gains(const float* g, float (&f)[2 * NP]) const {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      f[i] = f[NP + i] = 1.0f;
      if (g && has(i)) {
        int e1, e2;
        element(i, e1, e2);
        f[i] = g[e1];
        f[NP + i] = g[e2];
      }
    }
  }
  // Elements that f[i] and f[NP + i] of read() hold.
  __device__ __forceinline__ void element(int i, int& e1, int& e2) const {
    if (VEC) {
      e1 = INTER ? o1 + 2 * i : o1 + i;
      e2 = INTER ? o1 + 2 * i + 1 : o2 + i;
    } else {
      places(i, e1, e2);
    }
  }
};

template <int NP>
__device__ __forceinline__ void angles(const unsigned long long* turn, int pos, const int (&pair)[NP], const bool (&turns)[NP],
                                       float (&cs)[NP], float (&sn)[NP]) {
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    cs[i] = 1.0f;
    sn[i] = 0.0f;
    if (turns[i]) {
      const unsigned long long t = turn[pair[i]] * (unsigned long long)(long long)pos;
      // signed, so that angles just below a whole turn are small negative ones; in units of pi
      sincospif((float)(int)(unsigned int)(t >> 32) * 0x1p-31f, &sn[i], &cs[i]);
    }
  }
}

__device__ __forceinline__ float group_sum(float s, int group) {
  for (int o = group >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

constexpr int kQkThreads = 256;

// Forward.  A group of lanes takes one item: a share of the query (or key) heads of one token, whose angles it forms once.
template <typename T, int NP, bool VEC, bool INTER>
__global__ void __launch_bounds__(kQkThreads)
k_qknorm(const __grid_constant__ QkArgs a) {
  const int group = 1 << a.group_log;
  const int li = threadIdx.x & (group - 1);
  const Lane<T, NP, VEC, INTER> L(li, group, a);
  const int slices = a.v[0].slices + a.v[1].slices;
  const long long item = ((long long)blockIdx.x * kQkThreads + threadIdx.x) >> a.group_log;
  const long long tok = item / slices;
  int sl = (int)(item - tok * slices);
  bool live = tok < (long long)a.B * a.T;
  const int b = live ? (int)(tok / a.T) : 0, t = live ? (int)(tok - (long long)b * a.T) : 0;
  if (live && a.lengths && t >= a.lengths[b]) live = false;
  const int kind = sl >= a.v[0].slices;
  if (kind) sl -= a.v[0].slices;
  const View& v = a.v[kind];
  const int h0 = sl * a.heads_per_item;
  const int nh = live ? min(a.heads_per_item, v.heads - h0) : 0;
  const int pos = !live ? 0 : a.positions ? a.positions[tok] : t;
  int pair[NP];
  bool turns[NP];
  float cs[NP], sn[NP], gain[2 * NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    pair[i] = L.pair(i);
    turns[i] = live && L.has(i) && pair[i] < a.rot_pairs;
  }
  angles<NP>(a.turn, pos, pair, turns, cs, sn);
  L.gains(v.gain, gain);
  const T* x = static_cast<const T*>(v.in) + b * v.in_b + t * v.in_t + h0 * v.in_h;
  T* y = static_cast<T*>(v.out) + b * v.out_b + t * v.out_t + h0 * v.out_h;
  const int rounds = __reduce_max_sync(0xffffffffu, nh);
#pragma unroll 2
  for (int h = 0; h < rounds; ++h) {
    const bool act = h < nh;
    float f[2 * NP];
#pragma unroll
    for (int i = 0; i < 2 * NP; ++i) f[i] = 0.0f;
    if (act) L.read(x + h * v.in_h, f);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * NP; ++i) s = fmaf(f[i], f[i], s);
    s = group_sum(s, group);
    const float r = act ? rsqrtf(s * a.inv_dim + a.eps) : 0.0f;   // 0: idle heads add nothing, even with eps = 0
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const float p = f[i] * r * gain[i], q = f[NP + i] * r * gain[NP + i];
      f[i] = p * cs[i] - q * sn[i];
      f[NP + i] = q * cs[i] + p * sn[i];
    }
    if (act) L.write(y + h * v.out_h, f);
  }
}

// Backward.  A block takes a run of one example's tokens for the queries or for the keys; its groups share the
// (token, head share) items.  Every lane adds u * xhat of its elements over all heads it meets; at the end the block's
// sums go, in a fixed order, to the example's row or, where an example has several blocks, to a partial row.
template <typename T, int NP, bool VEC, bool INTER>
__global__ void __launch_bounds__(kQkThreads)
k_qknorm_grad(const __grid_constant__ QkArgs a) {
  extern __shared__ float gsum[];                // [warps][D]
  const int group = 1 << a.group_log;
  const int li = threadIdx.x & (group - 1);
  const Lane<T, NP, VEC, INTER> L(li, group, a);
  const int kind = blockIdx.z;
  const View& v = a.v[kind];
  const int b = blockIdx.y, D = 2 * a.pairs;
  const int t0 = blockIdx.x * a.chunk;
  int t1 = min(t0 + a.chunk, a.T);
  if (a.lengths) t1 = min(t1, a.lengths[b]);
  const int n_items = max(t1 - t0, 0) * v.slices;
  const int groups = kQkThreads >> a.group_log, mine = threadIdx.x >> a.group_log;
  float gain[2 * NP], sum[2 * NP];
  L.gains(v.gain, gain);
#pragma unroll
  for (int i = 0; i < 2 * NP; ++i) sum[i] = 0.0f;
  int pair[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) pair[i] = L.pair(i);
  // the groups of a warp walk together
  const int walks = (n_items + groups - 1) / groups;
  for (int w = 0; w < walks; ++w) {
    const int item = w * groups + mine;
    const bool live = item < n_items;
    const int t = t0 + (live ? item / v.slices : 0), sl = live ? item % v.slices : 0;
    const int h0 = sl * a.heads_per_item;
    const int nh = live ? min(a.heads_per_item, v.heads - h0) : 0;
    const int pos = !live ? 0 : a.positions ? a.positions[(long long)b * a.T + t] : t;
    bool turns[NP];
    float cs[NP], sn[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) turns[i] = live && L.has(i) && pair[i] < a.rot_pairs;
    angles<NP>(a.turn, pos, pair, turns, cs, sn);
    const T* x = static_cast<const T*>(v.in) + b * v.in_b + t * v.in_t + h0 * v.in_h;
    const T* g = static_cast<const T*>(v.dout) + b * v.dout_b + t * v.dout_t + h0 * v.dout_h;
    T* y = static_cast<T*>(v.out) + b * v.out_b + t * v.out_t + h0 * v.out_h;
    const int rounds = __reduce_max_sync(0xffffffffu, nh);
#pragma unroll 2
    for (int h = 0; h < rounds; ++h) {
      const bool act = h < nh;
      float f[2 * NP], u[2 * NP];
#pragma unroll
      for (int i = 0; i < 2 * NP; ++i) f[i] = u[i] = 0.0f;
      if (act) { L.read(x + h * v.in_h, f); L.read(g + h * v.dout_h, u); }
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < 2 * NP; ++i) s = fmaf(f[i], f[i], s);
      s = group_sum(s, group);
      const float r = act ? rsqrtf(s * a.inv_dim + a.eps) : 0.0f;   // 0: idle heads add nothing, even with eps = 0
      float m = 0.0f;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const float p = u[i] * cs[i] + u[NP + i] * sn[i], q = u[NP + i] * cs[i] - u[i] * sn[i];
        f[i] *= r;
        f[NP + i] *= r;                          // xhat
        sum[i] = fmaf(p, f[i], sum[i]);
        sum[NP + i] = fmaf(q, f[NP + i], sum[NP + i]);
        u[i] = p * gain[i];
        u[NP + i] = q * gain[NP + i];            // w
        m = fmaf(u[i], f[i], m);
        m = fmaf(u[NP + i], f[NP + i], m);
      }
      m = group_sum(m, group) * a.inv_dim;
#pragma unroll
      for (int i = 0; i < 2 * NP; ++i) u[i] = r * (u[i] - f[i] * m);
      if (act) L.write(y + h * v.out_h, u);
    }
  }
  if (!v.rows) return;                           // uniform over the block
  // lanes with the same elements: first inside the warp, then over the warps
#pragma unroll
  for (int i = 0; i < 2 * NP; ++i)
    for (int o = 16; o >= group; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) < group) {
#pragma unroll
    for (int i = 0; i < NP; ++i)
      if (L.has(i)) {
        int e1, e2;
        L.element(i, e1, e2);
        gsum[warp * D + e1] = sum[i];
        gsum[warp * D + e2] = sum[NP + i];
      }
  }
  __syncthreads();
  for (int d = threadIdx.x; d < D; d += kQkThreads) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kQkThreads / 32; ++w) s += gsum[w * D + d];
    if (a.partial) {
      a.partial[(((long long)b * a.n_chunks + blockIdx.x) * 2 + kind) * D + d] = s;
    } else {
      float* o = v.rows + (long long)b * D + d;
      *o = a.accumulate ? *o + s : s;
    }
  }
}

// rows[b][d] (+)= sum over the chunks, in order.  One block per (example, kind); 256 / 32 chunk strands per 32 columns.
__global__ void __launch_bounds__(256)
k_qknorm_rows(const float* __restrict__ partial, int n_chunks, int D, float* __restrict__ rows_q, float* __restrict__ rows_k,
              int add) {
  __shared__ float part[8][32];
  const int b = blockIdx.x, kind = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* rows = kind ? rows_k : rows_q;
  if (!rows) return;
  const int d = blockIdx.y * 32 + lane;
  float s = 0.0f;
  if (d < D) {
#pragma unroll 4
    for (int c = warp; c < n_chunks; c += 8) s += partial[(((long long)b * n_chunks + c) * 2 + kind) * D + d];
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && d < D) {
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += part[w][lane];
    float* o = rows + (long long)b * D + d;
    *o = add ? *o + t : t;
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
static bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

static int check_qk(const dp_qknorm* p) {
  if (!p || p->B <= 0 || p->T <= 0 || p->dim <= 0 || p->n_q < 0 || p->n_k < 0 || p->n_q + (int64_t)p->n_k <= 0) return DP_ERR_ARG;
  if (p->dtype != DP_F32 && p->dtype != DP_BF16) return DP_ERR_ARG;
  if ((p->dim & 1) || p->rot < 0 || (p->rot & 1) || p->rot > p->dim) return DP_ERR_ARG;
  if (!(p->eps >= 0.0) || !std::isfinite(p->eps)) return DP_ERR_ARG;
  if (p->n_q > 65535 || p->n_k > 65535 || p->B > 65535 * 32 || p->T > 1 << 24) return DP_ERR_UNSUPPORTED;
  if (p->dim > 2 * kMaxPairs) return DP_ERR_UNSUPPORTED;
  if (p->rot > 0 && !p->inv_freq) return DP_ERR_ARG;
  for (int j = 0; j < p->rot / 2; ++j)
    if (!std::isfinite(p->inv_freq[j])) return DP_ERR_ARG;
  if (misaligned(p->gain_q, 4) || misaligned(p->gain_k, 4) || misaligned(p->positions, 4) || misaligned(p->lengths, 4))
    return DP_ERR_ALIGN;
  return DP_OK;
}

static int check_heads(const dp_heads* x, size_t es) {
  if (!x || !x->data || x->stride_b < 0 || x->stride_t < 0 || x->stride_h < 0) return DP_ERR_ARG;
  return misaligned(x->data, es) ? DP_ERR_ALIGN : DP_OK;
}

// Vectors: a lane's V pairs lie whole inside or whole outside the rotated part, one warp holds the head, and (vec_heads)
// every head starts on a 16-byte boundary.
static bool vec_dims(const dp_qknorm* p, int V) {
  return p->dim % (2 * V) == 0 && p->rot % (2 * V) == 0 && p->dim <= 2 * V * 32;
}
static bool vec_heads(const dp_heads& x, int V) {
  return !misaligned(x.data, 16) && x.stride_b % V == 0 && x.stride_t % V == 0 && x.stride_h % V == 0;
}

// Tokens per block of the backward pass: enough blocks to fill the GPU several times over, so that the last round of
// blocks costs little, but no more than 512 partial rows per example.
static int grad_chunk(const dp_qknorm* p) {
  const long long kinds = (p->n_q > 0) + (p->n_k > 0);
  long long chunks = (148ll * 2 * 8 + (long long)p->B * kinds - 1) / ((long long)p->B * kinds);
  if (chunks > 512) chunks = 512;
  if (chunks > p->T) chunks = p->T;
  return (int)((p->T + chunks - 1) / chunks);
}

static void fill_args(const dp_qknorm* p, QkArgs* a, bool backward) {
  a->positions = p->positions;
  a->lengths = p->lengths;
  a->eps = (float)p->eps;
  a->inv_dim = (float)(1.0 / p->dim);
  a->B = p->B;
  a->T = p->T;
  a->pairs = p->dim / 2;
  a->rot_pairs = p->rot / 2;
  a->v[0].heads = p->n_q;
  a->v[1].heads = p->n_k;
  a->v[0].gain = p->gain_q;
  a->v[1].gain = p->gain_k;
  // Heads that share one set of angles: up to 8, fewer while there are too few items to fill the GPU.
  const long long rows = (long long)p->B * p->T * (p->n_q + p->n_k);
  int hp = 8;
  while (hp > 1 && rows / hp < 148ll * 256) hp >>= 1;
  a->heads_per_item = hp;
  for (int k = 0; k < 2; ++k) a->v[k].slices = ceil_div(a->v[k].heads, hp);
  a->chunk = backward ? grad_chunk(p) : 0;
  a->n_chunks = backward ? ceil_div(p->T, a->chunk) : 0;
  // inv_freq / (2 pi) modulo one turn, as a 64-bit fraction (x87 arithmetic: 64 bits of mantissa)
  const long double two_pi = 6.283185307179586476925286766559005768L;
  for (int j = 0; j < p->rot / 2; ++j) {
    long double f = (long double)p->inv_freq[j] / two_pi;
    f -= std::floor(f);
    const long double scaled = f * 18446744073709551616.0L;
    a->turn[j] = scaled >= 18446744073709551615.0L ? ~0ull : (unsigned long long)(scaled + 0.5L);
  }
}

// Calls fn.template run<T, NP, VEC, INTER>() for the form that the sizes and alignments allow.
template <typename T, typename F>
static cudaError_t pick(const QkArgs& a, bool vec, bool inter, F fn) {
  constexpr int V = 16 / sizeof(T);
  if (vec) return inter ? fn.template run<T, V, true, true>() : fn.template run<T, V, true, false>();
  const int np = ceil_div(a.pairs, 32);
  if (np <= 1) return inter ? fn.template run<T, 1, false, true>() : fn.template run<T, 1, false, false>();
  if (np <= 2) return inter ? fn.template run<T, 2, false, true>() : fn.template run<T, 2, false, false>();
  if (np <= 4) return inter ? fn.template run<T, 4, false, true>() : fn.template run<T, 4, false, false>();
  return inter ? fn.template run<T, 8, false, true>() : fn.template run<T, 8, false, false>();
}

struct Forward {
  const QkArgs& a;
  cudaStream_t s;
  template <typename T, int NP, bool VEC, bool INTER>
  cudaError_t run() const {
    const long long items = (long long)a.B * a.T * (a.v[0].slices + a.v[1].slices);
    const int per = kQkThreads >> a.group_log;
    const long long blocks = (items + per - 1) / per;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    k_qknorm<T, NP, VEC, INTER><<<(unsigned)blocks, kQkThreads, 0, s>>>(a);
    return counted(1);
  }
};

struct Backward {
  const QkArgs& a;
  cudaStream_t s;
  template <typename T, int NP, bool VEC, bool INTER>
  cudaError_t run() const {
    const size_t smem = (size_t)(kQkThreads / 32) * 2 * a.pairs * sizeof(float);
    const dim3 grid(a.n_chunks, a.B, 2);
    k_qknorm_grad<T, NP, VEC, INTER><<<grid, kQkThreads, smem, s>>>(a);
    return counted(1);
  }
};

// Lanes per head.
static int group_log(int pairs, bool vec, int V) {
  if (!vec) return 5;
  int g = 0;
  while ((V << g) < pairs) ++g;
  return g;
}

}  // namespace dpk

using namespace dpk;

extern "C" {

int dp_qknorm_rope(const dp_qknorm* p, const dp_heads* q, const dp_heads* k, const dp_heads* out_q, const dp_heads* out_k,
                   void* cuda_stream) {
  int rc = check_qk(p);
  if (rc != DP_OK) return rc;
  const size_t es = p->dtype == DP_F32 ? 4 : 2;
  const int V = (int)(16 / es);
  const dp_heads* in[2] = {q, k};
  const dp_heads* out[2] = {out_q, out_k};
  const int heads[2] = {p->n_q, p->n_k};
  QkArgs a = {};
  bool vec = vec_dims(p, V);
  for (int i = 0; i < 2; ++i) {
    if (heads[i] == 0) continue;
    if ((rc = check_heads(in[i], es)) != DP_OK || (rc = check_heads(out[i], es)) != DP_OK) return rc;
    vec = vec && vec_heads(*in[i], V) && vec_heads(*out[i], V);
    a.v[i].in = in[i]->data;
    a.v[i].in_b = in[i]->stride_b; a.v[i].in_t = in[i]->stride_t; a.v[i].in_h = in[i]->stride_h;
    a.v[i].out = out[i]->data;
    a.v[i].out_b = out[i]->stride_b; a.v[i].out_t = out[i]->stride_t; a.v[i].out_h = out[i]->stride_h;
  }
  fill_args(p, &a, false);
  a.group_log = group_log(a.pairs, vec, V);
  const Forward f{a, static_cast<cudaStream_t>(cuda_stream)};
  const bool inter = p->interleaved != 0;
  const cudaError_t e = p->dtype == DP_F32 ? pick<float>(a, vec, inter, f) : pick<__nv_bfloat16>(a, vec, inter, f);
  return e == cudaSuccess ? DP_OK : DP_ERR_CUDA;
}

size_t dp_qknorm_workspace_bytes(const dp_qknorm* p) {
  if (check_qk(p) != DP_OK) return 0;
  const size_t chunks = (size_t)ceil_div(p->T, grad_chunk(p));
  return chunks > 1 ? chunks * (size_t)p->B * 2 * (size_t)p->dim * sizeof(float) : 0;
}

int dp_qknorm_rope_backward(const dp_qknorm* p, const dp_heads* q, const dp_heads* k, const dp_heads* dout_q,
                            const dp_heads* dout_k, const dp_heads* dq, const dp_heads* dk, float* rows_q, float* rows_k,
                            int accumulate_into, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_qk(p);
  if (rc != DP_OK) return rc;
  if (p->B > 65535) return DP_ERR_UNSUPPORTED;
  const size_t es = p->dtype == DP_F32 ? 4 : 2;
  const int V = (int)(16 / es);
  const dp_heads* in[2] = {q, k};
  const dp_heads* dout[2] = {dout_q, dout_k};
  const dp_heads* out[2] = {dq, dk};
  float* rows[2] = {rows_q, rows_k};
  const int heads[2] = {p->n_q, p->n_k};
  QkArgs a = {};
  bool vec = vec_dims(p, V);
  for (int i = 0; i < 2; ++i) {
    if (heads[i] == 0) continue;
    if ((rc = check_heads(in[i], es)) != DP_OK || (rc = check_heads(dout[i], es)) != DP_OK ||
        (rc = check_heads(out[i], es)) != DP_OK)
      return rc;
    if (misaligned(rows[i], 4)) return DP_ERR_ALIGN;
    vec = vec && vec_heads(*in[i], V) && vec_heads(*dout[i], V) && vec_heads(*out[i], V);
    a.v[i].in = in[i]->data;
    a.v[i].in_b = in[i]->stride_b; a.v[i].in_t = in[i]->stride_t; a.v[i].in_h = in[i]->stride_h;
    a.v[i].dout = dout[i]->data;
    a.v[i].dout_b = dout[i]->stride_b; a.v[i].dout_t = dout[i]->stride_t; a.v[i].dout_h = dout[i]->stride_h;
    a.v[i].out = out[i]->data;
    a.v[i].out_b = out[i]->stride_b; a.v[i].out_t = out[i]->stride_t; a.v[i].out_h = out[i]->stride_h;
    a.v[i].rows = rows[i];
  }
  fill_args(p, &a, true);
  a.group_log = group_log(a.pairs, vec, V);
  a.accumulate = accumulate_into ? 1 : 0;
  const bool want_rows = a.v[0].rows || a.v[1].rows;
  if (a.n_chunks > 1 && want_rows) {
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < dp_qknorm_workspace_bytes(p)) return DP_ERR_WORKSPACE;
    a.partial = static_cast<float*>(workspace);
  }
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const Backward f{a, s};
  const bool inter = p->interleaved != 0;
  const cudaError_t e = p->dtype == DP_F32 ? pick<float>(a, vec, inter, f) : pick<__nv_bfloat16>(a, vec, inter, f);
  if (e != cudaSuccess) return DP_ERR_CUDA;
  if (a.partial) {
    k_qknorm_rows<<<dim3(p->B, ceil_div(p->dim, 32), 2), 256, 0, s>>>(a.partial, a.n_chunks, p->dim, a.v[0].rows,
                                                                      a.v[1].rows, a.accumulate);
    if (counted(1) != cudaSuccess) return DP_ERR_CUDA;
  }
  return DP_OK;
}

}  // extern "C"
