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
#include <type_traits>

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
__device__ __forceinline__ float zero1(const float*) { return 0.0f; }
__device__ __forceinline__ __nv_bfloat16 zero1(const __nv_bfloat16*) { return __float2bfloat16_rn(0.0f); }
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
  // A head in flight: fetch() issues the loads, unpack() makes fp32 of them (f[i] = a, f[NP + i] = b; 0 where nothing was
  // fetched).
  struct VecRaw { uint4 u1, u2; };
  struct OneRaw { T x[2 * NP]; };
  using Raw = std::conditional_t<VEC, VecRaw, OneRaw>;
  __device__ __forceinline__ Raw fetch(const T* x, bool act) const {
    Raw r;
    if constexpr (VEC) {
      r.u1 = r.u2 = make_uint4(0u, 0u, 0u, 0u);
      if (on && act) {
        r.u1 = *reinterpret_cast<const uint4*>(x + o1);
        r.u2 = *reinterpret_cast<const uint4*>(x + o2);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        r.x[i] = r.x[NP + i] = zero1(x);
        if (act && has(i)) {
          int e1, e2;
          places(i, e1, e2);
          r.x[i] = x[e1];
          r.x[NP + i] = x[e2];
        }
      }
    }
    return r;
  }
  __device__ __forceinline__ void unpack(const Raw& r, float (&f)[2 * NP]) const {
    if constexpr (VEC) {
      float t[2 * NP];
      const uint32_t w[8] = {r.u1.x, r.u1.y, r.u1.z, r.u1.w, r.u2.x, r.u2.y, r.u2.z, r.u2.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if constexpr (sizeof(T) == 4) {
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
      for (int i = 0; i < 2 * NP; ++i) f[i] = load1(&r.x[i]);
    }
  }
  __device__ __forceinline__ void write(T* x, const float (&f)[2 * NP]) const {
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
        if constexpr (sizeof(T) == 4) {
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

// Sine and cosine of the angle of each pair.  EXACT (fp32 data): within 2 ulp.  Otherwise the hardware approximations on
// [-pi, pi], off by at most 2^-21 of the pair's length: the data's own bf16 rounding is 2^12 times that, and the accurate
// pair costs about ten times the instructions of the two.
template <int NP, bool EXACT>
__device__ __forceinline__ void angles(const unsigned long long* turn, int pos, const int (&pair)[NP], const bool (&turns)[NP],
                                       float (&cs)[NP], float (&sn)[NP]) {
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    cs[i] = 1.0f;
    sn[i] = 0.0f;
    if (turns[i]) {
      const unsigned long long t = turn[pair[i]] * (unsigned long long)(long long)pos;
      // signed, so that angles just below a whole turn are small negative ones; in units of pi
      const float half_turns = (float)(int)(unsigned int)(t >> 32) * 0x1p-31f;
      if (EXACT) {
        sincospif(half_turns, &sn[i], &cs[i]);
      } else {
        sn[i] = __sinf(half_turns * 3.14159265f);
        cs[i] = __cosf(half_turns * 3.14159265f);
      }
    }
  }
}

// Two fp32 operations per instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "mul.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
template <int N> __device__ __forceinline__ float2 at2(const float (&f)[N], int i) { return make_float2(f[i], f[i + 1]); }
template <int N> __device__ __forceinline__ void put2(float (&f)[N], int i, float2 v) { f[i] = v.x; f[i + 1] = v.y; }

template <int N>
__device__ __forceinline__ float dot(const float (&a)[N], const float (&b)[N]) {      // N even
  float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < N; i += 2) s = fma2(at2(a, i), at2(b, i), s);
  return s.x + s.y;
}
template <int N>
__device__ __forceinline__ void scale(float (&a)[N], float r) {
#pragma unroll
  for (int i = 0; i < N; i += 2) put2(a, i, mul2(at2(a, i), make_float2(r, r)));
}
// (a, b) <- (a c1 - b s1, b c2 + a s2) for each pair; f[i] = a, f[NP + i] = b.  s1n = -s1.
template <int NP>
__device__ __forceinline__ void turn_pairs(float (&f)[2 * NP], const float (&c1)[NP], const float (&s1n)[NP],
                                           const float (&c2)[NP], const float (&s2)[NP]) {
  if constexpr (NP % 2 == 0) {
#pragma unroll
    for (int i = 0; i < NP; i += 2) {
      const float2 a = at2(f, i), b = at2(f, NP + i);
      put2(f, i, fma2(a, at2(c1, i), mul2(b, at2(s1n, i))));
      put2(f, NP + i, fma2(b, at2(c2, i), mul2(a, at2(s2, i))));
    }
  } else {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const float a = f[i], b = f[NP + i];
      f[i] = fmaf(a, c1[i], b * s1n[i]);
      f[NP + i] = fmaf(b, c2[i], a * s2[i]);
    }
  }
}

__device__ __forceinline__ float group_sum(float s, int group) {
  for (int o = group >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

constexpr int kQkThreads = 256;
#ifndef DP_QK_FWD_AHEAD
#define DP_QK_FWD_AHEAD 2
#endif
#ifndef DP_QK_FWD_BLOCKS
#define DP_QK_FWD_BLOCKS 2
#endif
#ifndef DP_QK_BWD_BLOCKS
#define DP_QK_BWD_BLOCKS 2
#endif
#ifndef DP_QK_BWD_AHEAD
#define DP_QK_BWD_AHEAD 1
#endif
#ifndef DP_QK_HP
#define DP_QK_HP 8
#endif
#ifndef DP_QK_CHUNK
#define DP_QK_CHUNK 128
#endif
constexpr int kHeadsPerItem = DP_QK_HP, kMaxChunk = DP_QK_CHUNK;
constexpr int kFwdAhead = DP_QK_FWD_AHEAD, kBwdAhead = DP_QK_BWD_AHEAD;

// Forward.  A group of lanes takes one item: a share of the query (or key) heads of one token, whose angles it forms once.
template <typename T, int NP, bool VEC, bool INTER>
__global__ void __launch_bounds__(kQkThreads, VEC ? DP_QK_FWD_BLOCKS : 1)
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
  angles<NP, sizeof(T) == 4>(a.turn, pos, pair, turns, cs, sn);
  L.gains(v.gain, gain);
  // the gain is folded into the rotation: y_a = r (a g_a cos - b g_b sin), y_b = r (b g_b cos + a g_a sin)
  float c1[NP], s1n[NP], c2[NP], s2[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    c1[i] = gain[i] * cs[i];
    s1n[i] = -gain[NP + i] * sn[i];
    c2[i] = gain[NP + i] * cs[i];
    s2[i] = gain[i] * sn[i];
  }
  const T* x = static_cast<const T*>(v.in) + b * v.in_b + t * v.in_t + h0 * v.in_h;
  T* y = static_cast<T*>(v.out) + b * v.out_b + t * v.out_t + h0 * v.out_h;
  const int rounds = __reduce_max_sync(0xffffffffu, nh);
  // kFwdAhead heads' loads are in flight while one is worked on
  typename Lane<T, NP, VEC, INTER>::Raw raw[kFwdAhead];
#pragma unroll
  for (int k = 0; k < kFwdAhead; ++k) raw[k] = L.fetch(x + k * v.in_h, k < nh);
  for (int h = 0; h < rounds; h += kFwdAhead) {
#pragma unroll
    for (int k = 0; k < kFwdAhead; ++k) {
      const bool act = h + k < nh;
      float f[2 * NP];
      L.unpack(raw[k], f);
      raw[k] = L.fetch(x + (h + k + kFwdAhead) * v.in_h, h + k + kFwdAhead < nh);
      const float s = group_sum(dot(f, f), group);
      scale(f, rsqrtf(s * a.inv_dim + a.eps));
      turn_pairs<NP>(f, c1, s1n, c2, s2);
      if (act) L.write(y + (h + k) * v.out_h, f);
    }
  }
}

// Backward.  A block takes a run of one example's tokens for the queries or for the keys; its groups share the
// (token, head share) items.  Every lane adds u * xhat of its elements over all heads it meets; at the end the block's
// sums go, in a fixed order, to the example's row or, where an example has several blocks, to a partial row.
template <typename T, int NP, bool VEC, bool INTER>
__global__ void __launch_bounds__(kQkThreads, VEC ? DP_QK_BWD_BLOCKS : 1)
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
    angles<NP, sizeof(T) == 4>(a.turn, pos, pair, turns, cs, sn);
    float snn[NP];                               // R(-p): the sine with the other sign
#pragma unroll
    for (int i = 0; i < NP; ++i) snn[i] = -sn[i];
    const T* x = static_cast<const T*>(v.in) + b * v.in_b + t * v.in_t + h0 * v.in_h;
    const T* g = static_cast<const T*>(v.dout) + b * v.dout_b + t * v.dout_t + h0 * v.dout_h;
    T* y = static_cast<T*>(v.out) + b * v.out_b + t * v.out_t + h0 * v.out_h;
    const int rounds = __reduce_max_sync(0xffffffffu, nh);
    typename Lane<T, NP, VEC, INTER>::Raw rx[kBwdAhead], rg[kBwdAhead];
#pragma unroll
    for (int k = 0; k < kBwdAhead; ++k) {
      rx[k] = L.fetch(x + k * v.in_h, k < nh);
      rg[k] = L.fetch(g + k * v.dout_h, k < nh);
    }
    for (int h = 0; h < rounds; h += kBwdAhead) {
#pragma unroll
      for (int k = 0; k < kBwdAhead; ++k) {
        const bool act = h + k < nh;
        float f[2 * NP], u[2 * NP];
        L.unpack(rx[k], f);
        L.unpack(rg[k], u);
        rx[k] = L.fetch(x + (h + k + kBwdAhead) * v.in_h, h + k + kBwdAhead < nh);
        rg[k] = L.fetch(g + (h + k + kBwdAhead) * v.dout_h, h + k + kBwdAhead < nh);
        turn_pairs<NP>(u, cs, sn, cs, snn);
        const float s = group_sum(dot(f, f), group);
        // 0 for idle heads, which then add nothing even with eps = 0
        const float r = act ? rsqrtf(s * a.inv_dim + a.eps) : 0.0f;
        // with u' = r u: sum += u' x (= u xhat), w' = gain u', dx = w' - x r^2 mean(w' x)
        scale(u, r);
#pragma unroll
        for (int i = 0; i < 2 * NP; i += 2) {
          put2(sum, i, fma2(at2(u, i), at2(f, i), at2(sum, i)));
          put2(u, i, mul2(at2(u, i), at2(gain, i)));
        }
        const float m = -(group_sum(dot(u, f), group) * a.inv_dim) * r * r;
#pragma unroll
        for (int i = 0; i < 2 * NP; i += 2) put2(u, i, fma2(at2(f, i), make_float2(m, m), at2(u, i)));
        if (act) L.write(y + (h + k) * v.out_h, u);
      }
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

// Tokens per block of the backward pass: a power of two, so that a block's items divide evenly among its groups, as large
// as still gives enough blocks to fill the GPU several times over (the last round of blocks then costs little); at most 512
// partial rows per example.
static int grad_chunk(const dp_qknorm* p) {
  const long long kinds = (p->n_q > 0) + (p->n_k > 0), per_token = (long long)p->B * kinds;
  int chunk = kMaxChunk;
  while (chunk > 1 && per_token * ceil_div(p->T, chunk) < 148ll * 2 * 6) chunk >>= 1;
  while (ceil_div(p->T, chunk) > 512) chunk <<= 1;
  return chunk;
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
  // Heads that share one set of angles: up to kHeadsPerItem, fewer while the items would not fill the GPU's groups.
  const long long rows = (long long)p->B * p->T * (p->n_q + p->n_k), fill = 148ll * 512 >> a->group_log;
  int hp = kHeadsPerItem;
  while (hp > 1 && rows < fill * hp) hp >>= 1;
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
  a.group_log = group_log(p->dim / 2, vec, V);
  fill_args(p, &a, false);
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
  a.group_log = group_log(p->dim / 2, vec, V);
  fill_args(p, &a, true);
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
