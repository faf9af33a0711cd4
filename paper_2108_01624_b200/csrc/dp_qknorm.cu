// RMS norm of every query and key head with a learned gain, and the position rotation, in one pass; and the backward
// pass, which also yields every example's gradients of the two gains.  With x one head of one token, D wide:
//   r = 1 / sqrt(mean(x^2) + eps),  xhat = r x,  y = R(p) (gain * xhat)
// where R(p) turns the pair (a, b) number j by the angle p * inv_freq[j]: (a cos - b sin, b cos + a sin).  Backward, with
// u = R(-p) dy and w = gain * u:
//   dx = r (w - xhat mean(w xhat)),     d gain of example i = sum over its tokens and heads of u * xhat.
// Bound by memory: forward reads x and writes y, backward reads x and dy and writes dx.  A group of lanes holds a whole
// head in registers, so nothing is read twice; the gains' gradients stay in registers over all heads a lane meets.
// 256 x 128 tokens of 16 + 16 bf16 heads of 64: forward 46 us (5.8 TB/s, 0.89 of the copy bandwidth), backward 66 us
// (6.1 TB/s, 0.93).
//
// The angle.  p * inv_freq loses its fractional turns in fp32 at far positions.  The host turns inv_freq[j] / (2 pi) into
// a 64-bit binary fraction of a turn; p times that, modulo 2^64, is an ordinary wrapping integer product, and its upper
// 32 bits are the angle in units of 2^-32 turns, at any 32-bit position, for the price of one multiplication.
#include <cfloat>
#include <type_traits>

#include "dp_chain.cuh"
#include "dp_internal.h"

namespace dpk {

constexpr int kMaxPairs = 256;                   // D <= 512

// How the heads of one kind (queries or keys) are shared out.  A warp takes a unit: tokens_per_unit neighbouring tokens times
// `heads_per_unit` heads.  Its groups of lanes stand as (tokens x heads) = 2^gt x 2^gh, and each walks down the tokens
// with heads_per_group heads of every token, whose angles it forms once.
struct Share {
  int heads, heads_per_group, gh, gt, heads_per_unit, head_blocks, tokens_per_unit, chunks;
  long long units;
};

struct View {                                    // [B, T, H, D], D contiguous; strides in elements
  const void* in;
  const void* dout;                              // backward: gradient of the output
  void* out;                                     // forward: the output; backward: gradient of the input
  const float* gain;                             // [D] or null (ones)
  float* rows;                                   // backward: [B][D] gain gradients, or null
  float* partial;                                // backward: [B][chunks * head_blocks][D], or null (one unit per example)
  long long in_b, in_t, in_h, dout_b, dout_t, dout_h, out_b, out_t, out_h;
  Share share;
};

struct QkArgs {
  View v[2];                                     // queries, keys
  const int32_t* positions;                      // [B, T] or null: 0 .. T-1
  const int32_t* lengths;                        // [B] or null
  float eps, inv_dim;
  int B, T, pairs, rot_pairs, group_log;
  int accumulate;
  unsigned long long turn[kMaxPairs];            // fraction of a turn per position, 2^-64 units
};

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float zero1(const float*) { return 0.0f; }
__device__ __forceinline__ __nv_bfloat16 zero1(const __nv_bfloat16*) { return __float2bfloat16_rn(0.0f); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// 16 bytes to shared memory, asynchronously; with get = false the source is not read and zeros are written.
__device__ __forceinline__ void copy16(uint4* slot, const void* src, bool get) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((unsigned)__cvta_generic_to_shared(slot)), "l"(src),
               "r"(get ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_mark() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

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
  // A head in flight.  VEC: copied asynchronously into the lane's own 32 bytes of shared memory (slot[0], slot[32]: the
  // 16-byte words of a warp side by side), so that deep prefetch costs no registers; only the lane itself reads them, so its
  // own wait is all the synchronisation there is.  Otherwise fetched into registers, one head ahead.  0 without `act`.
  struct VecRaw { uint4 u1, u2; };
  struct OneRaw { T x[2 * NP]; };
  using Raw = std::conditional_t<VEC, VecRaw, OneRaw>;
  __device__ __forceinline__ void issue(const T* x, bool act, uint4* slot) const {
    const bool get = act && on;
    copy16(slot, x + o1, get);
    copy16(slot + 32, x + o2, get);
  }
  __device__ __forceinline__ Raw take(const uint4* slot) const { return {slot[0], slot[32]}; }
  __device__ __forceinline__ Raw fetch(const T* x, bool act) const {
    Raw r;
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
  // Fractions of a turn per position of the lane's pairs; 0 where nothing turns.
  __device__ __forceinline__ void turns(const QkArgs& a, uint2 (&f)[NP]) const {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const unsigned long long x = has(i) && pair(i) < rot_pairs ? a.turn[pair(i)] : 0ull;
      f[i] = make_uint2((unsigned)x, (unsigned)(x >> 32));
    }
  }
  // Elements that f[i] and f[NP + i] of unpack() hold.
  __device__ __forceinline__ void element(int i, int& e1, int& e2) const {
    if (VEC) {
      e1 = INTER ? o1 + 2 * i : o1 + i;
      e2 = INTER ? o1 + 2 * i + 1 : o2 + i;
    } else {
      places(i, e1, e2);
    }
  }
};

// Sine and cosine of pos * turn (a 64-bit fraction of a turn per position; 0 for what does not turn, which gives exactly 0
// and 1).  A float holds 24 of the angle's 32 bits.
// EXACT (fp32 data): the nearest quarter turn is taken off in whole numbers first, so that those 24 bits count from the nearest
// zero of the sine or cosine: each is off by 2^-24 and the function's 2 ulp of itself, and by 1.6 units of 2^-32 turns.
// Otherwise the hardware approximations on [-pi, pi]: the angle in 24 bits and its product with pi are off by up to 3.0e-7, the sine
// by 2^-21.4 and the cosine by 2^-21.2, together below 2^-20 of the pair's length.  The data's own bf16 rounding is 2^12 times
// that, and the accurate pair costs about ten times the instructions of the two.
template <bool EXACT>
__device__ __forceinline__ void angle(uint2 turn, int pos, float& cs, float& sn) {
  // bits 32..63 of turn * pos modulo 2^64, pos signed
  unsigned h = turn.y * (unsigned)pos + __umulhi(turn.x, (unsigned)pos);
  if (pos < 0) h -= turn.x;
  if (EXACT) {
    const unsigned quarter = (h + 0x20000000u) >> 30;
    float s, c;
    sincospif((float)(int)(h - (quarter << 30)) * 0x1p-31f, &s, &c);
    sn = quarter & 1u ? c : s;
    cs = quarter & 1u ? s : c;
    if (quarter & 2u) sn = -sn;
    if ((quarter + 1u) & 2u) cs = -cs;
  } else {
    // as a signed number, so that angles just below a whole turn are small negative ones
    const float half_turns = (float)(int)h * 0x1p-31f;
    sn = __sinf(half_turns * 3.14159265f);
    cs = __cosf(half_turns * 3.14159265f);
  }
}

// Sum over a group of 2^GL lanes (GL < 0: of `group` lanes, known at run time only).
template <int GL>
__device__ __forceinline__ float group_sum(float s, int group) {
  if constexpr (GL >= 0) {
#pragma unroll
    for (int o = (1 << GL) >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  } else {
    for (int o = group >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
  return s;
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
  static_assert(NP % 2 == 0, "pairs are turned two at a time");
#pragma unroll
  for (int i = 0; i < NP; i += 2) {
    const float2 a = at2(f, i), b = at2(f, NP + i);
    put2(f, i, fma2(a, at2(c1, i), mul2(b, at2(s1n, i))));
    put2(f, NP + i, fma2(b, at2(c2, i), mul2(a, at2(s2, i))));
  }
}

// Measured on the BERT-Large microbatch (forward 268 MB, backward 403 MB; device time of the main kernel):
//   heads in flight per group   forward  2: 55 us, 4: 51, 8: 53        backward  2: 84, 4: 76
//   warps resident per SM       forward 12: 51 us, 16: 51, 20: 55      backward  8: 82, 12: 76, 16: 100 (registers spill)
//   warps per block             forward  1, 2, 4: 50 to 51 us; one token for each of 64 sequences 4.2, 4.8, 5.4 us
// One warp a block, then: warps never wait for one another, and a finished one makes room at once.
// Units: two waves of them (one: 51 / 75 us and 18.0 on few examples in fp32; two: 50 / 76 and 16.7; three: 53 / 80).
constexpr int kFwdStages = 4, kBwdStages = 4;    // heads in flight per group (powers of two)
constexpr int kFwdWarps = 16, kBwdWarps = 12;    // resident per SM
constexpr int kWaves = 2, kHeadsPerGroup = 8;

// Where one group of lanes is on its walk over its unit: heads_per_group heads of a token, then its next token.  Two of
// these run over a unit, one that issues copies some heads ahead and one that computes.
template <bool FLAT>
struct Walk {
  int token, tstep, end, b, t;
  bool live;                                     // this group's token exists
  // tokens [first, end) of the unit: of example b, or, FLAT, of all examples one behind another
  __device__ __forceinline__ Walk(const Share& s, int gi, int first, int end_, int b_)
      : token(first + (gi >> s.gh) - (1 << s.gt)), tstep(1 << s.gt), end(end_), b(b_), t(0), live(false) {}
  __device__ __forceinline__ void next(const QkArgs& a) {
    token += tstep;
    live = token < end;
    t = live ? token : 0;
    if (FLAT && live) {
      b = token / a.T;
      t = token - b * a.T;
      if (a.lengths && t >= a.lengths[b]) live = false;
    }
  }
};

// Which unit of which kind a block (one warp) has.
__device__ __forceinline__ void unit_of(const QkArgs& a, int& kind, long long& unit) {
  unit = blockIdx.x;
  kind = unit >= a.v[0].share.units;
  if (kind) unit -= a.v[0].share.units;
}

// Forward.
template <typename T, int NP, bool VEC, bool INTER, int GL>
__global__ void __launch_bounds__(32, VEC ? kFwdWarps : 1)
k_qknorm(const __grid_constant__ QkArgs a) {
  __shared__ uint4 ring_all[VEC ? kFwdStages * 64 : 1];            // [stages][2][32]
  wait_for_predecessor();
  let_successor_in();
  int kind;
  long long unit;
  unit_of(a, kind, unit);
  const View& v = a.v[kind];
  const Share& s = v.share;
  const int glog = GL >= 0 ? GL : a.group_log, group = 1 << glog;
  const int lane = threadIdx.x, li = lane & (group - 1), gi = lane >> glog;
  const Lane<T, NP, VEC, INTER> L(li, group, a);
  uint4* ring = ring_all + lane;
  const int per = s.heads_per_group, hstep = 1 << s.gh;
  const int h0 = (int)(unit % s.head_blocks) * s.heads_per_unit + (gi & (hstep - 1));
  const int mine = h0 < s.heads ? min(per, (s.heads - h0 + hstep - 1) >> s.gh) : 0;      // heads of a token
  const long long first = unit / s.head_blocks * s.tokens_per_unit;
  const int end = (int)min((long long)a.B * a.T, first + s.tokens_per_unit);
  const int walks = (int)((end - first + (1 << s.gt) - 1) >> s.gt), steps = walks * per;
  Walk<true> ahead(s, gi, (int)first, end, 0), at = ahead;
  const T* in = static_cast<const T*>(v.in) + h0 * v.in_h;
  T* out = static_cast<T*>(v.out) + h0 * v.out_h;
  const long long in_step = hstep * v.in_h, out_step = hstep * v.out_h;
  const T* src = in;
  int aj = per, an = 0;                          // ahead: head of the token, step
  typename Lane<T, NP, VEC, INTER>::Raw pending;
  auto issue = [&]() {
    if (an < steps) {
      if (aj == per) {
        ahead.next(a);
        src = in + ahead.b * v.in_b + ahead.t * v.in_t;
        aj = 0;
      }
      if constexpr (VEC) L.issue(src, ahead.live && aj < mine, ring + (an & (kFwdStages - 1)) * 64);
      else pending = L.fetch(src, ahead.live && aj < mine);
      src += in_step;
      ++aj;
      ++an;
    }
    if (VEC) copies_mark();
  };
#pragma unroll 1
  for (int n = 0; n < (VEC ? kFwdStages - 1 : 1); ++n) issue();
  float gain[2 * NP];
  L.gains(v.gain, gain);
  uint2 turn[NP];
  L.turns(a, turn);
  int n = 0;
  for (int w = 0; w < walks; ++w) {
    at.next(a);
    const int pos = !at.live ? 0 : a.positions ? a.positions[at.token] : at.t;
    // the gain is folded into the rotation: y_a = r (a g_a cos - b g_b sin), y_b = r (b g_b cos + a g_a sin)
    float c1[NP], s1n[NP], c2[NP], s2[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      float cs, sn;
      angle<sizeof(T) == 4>(turn[i], pos, cs, sn);
      c1[i] = gain[i] * cs;
      s1n[i] = -gain[NP + i] * sn;
      c2[i] = gain[NP + i] * cs;
      s2[i] = gain[i] * sn;
    }
    T* y = out + at.b * v.out_b + at.t * v.out_t;
#pragma unroll 1
    for (int j = 0; j < per; ++j, ++n) {
      const bool act = at.live && j < mine;
      float f[2 * NP];
      if constexpr (VEC) {
        issue();
        copies_wait<kFwdStages - 1>();
        L.unpack(L.take(ring + (n & (kFwdStages - 1)) * 64), f);
      } else {
        L.unpack(pending, f);
        issue();
      }
      scale(f, rsqrtf(group_sum<GL>(dot(f, f), group) * a.inv_dim + a.eps));
      turn_pairs<NP>(f, c1, s1n, c2, s2);
      if (act) L.write(y, f);
      y += out_step;
    }
  }
}

// Backward.  Every lane adds u * xhat of its elements over all heads it meets; at the unit's end the groups' sums go, in a
// fixed order, to the example's row or, where an example has several units, to a partial row.
template <typename T, int NP, bool VEC, bool INTER, int GL>
__global__ void __launch_bounds__(32, VEC ? kBwdWarps : 1)
k_qknorm_grad(const __grid_constant__ QkArgs a) {
  __shared__ uint4 ring_all[VEC ? kBwdStages * 128 : 1];           // [stages][x, dy][2][32]
  wait_for_predecessor();
  let_successor_in();
  int kind;
  long long unit;
  unit_of(a, kind, unit);
  const View& v = a.v[kind];
  const Share& s = v.share;
  const int glog = GL >= 0 ? GL : a.group_log, group = 1 << glog;
  const int lane = threadIdx.x, li = lane & (group - 1), gi = lane >> glog;
  const Lane<T, NP, VEC, INTER> L(li, group, a);
  uint4* ring = ring_all + lane;
  const int parts = s.chunks * s.head_blocks, b = (int)(unit / parts), part = (int)(unit - (long long)b * parts);
  const int chunk = part / s.head_blocks;
  const int per = s.heads_per_group, hstep = 1 << s.gh;
  const int h0 = (part - chunk * s.head_blocks) * s.heads_per_unit + (gi & (hstep - 1));
  const int mine = h0 < s.heads ? min(per, (s.heads - h0 + hstep - 1) >> s.gh) : 0;      // heads of a token
  const int first = chunk * s.tokens_per_unit;
  int end = min(a.T, first + s.tokens_per_unit);
  if (a.lengths) end = min(end, a.lengths[b]);
  const int walks = (max(end - first, 0) + (1 << s.gt) - 1) >> s.gt, steps = walks * per;
  Walk<false> ahead(s, gi, first, end, b), at = ahead;
  const T* in = static_cast<const T*>(v.in) + b * v.in_b + h0 * v.in_h;
  const T* dout = static_cast<const T*>(v.dout) + b * v.dout_b + h0 * v.dout_h;
  T* out = static_cast<T*>(v.out) + b * v.out_b + h0 * v.out_h;
  const long long in_step = hstep * v.in_h, dout_step = hstep * v.dout_h, out_step = hstep * v.out_h;
  const T* src = in;
  const T* gsrc = dout;
  int aj = per, an = 0;
  typename Lane<T, NP, VEC, INTER>::Raw pending, gpending;
  auto issue = [&]() {
    if (an < steps) {
      if (aj == per) {
        ahead.next(a);
        src = in + ahead.t * v.in_t;
        gsrc = dout + ahead.t * v.dout_t;
        aj = 0;
      }
      const bool act = ahead.live && aj < mine;
      if constexpr (VEC) {
        uint4* slot = ring + (an & (kBwdStages - 1)) * 128;
        L.issue(src, act, slot);
        L.issue(gsrc, act, slot + 64);
      } else {
        pending = L.fetch(src, act);
        gpending = L.fetch(gsrc, act);
      }
      src += in_step;
      gsrc += dout_step;
      ++aj;
      ++an;
    }
    if (VEC) copies_mark();
  };
#pragma unroll 1
  for (int n = 0; n < (VEC ? kBwdStages - 1 : 1); ++n) issue();
  float gain[2 * NP], sum[2 * NP];
  L.gains(v.gain, gain);
#pragma unroll
  for (int i = 0; i < 2 * NP; ++i) sum[i] = 0.0f;
  uint2 turn[NP];
  L.turns(a, turn);
  int n = 0;
  for (int w = 0; w < walks; ++w) {
    at.next(a);
    const int pos = !at.live ? 0 : a.positions ? a.positions[(long long)b * a.T + at.t] : at.t;
    float cs[NP], sn[NP], snn[NP];               // R(-p): the sine with the other sign
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      angle<sizeof(T) == 4>(turn[i], pos, cs[i], sn[i]);
      snn[i] = -sn[i];
    }
    T* y = out + at.t * v.out_t;
#pragma unroll 1
    for (int j = 0; j < per; ++j, ++n) {
      const bool act = at.live && j < mine;
      float f[2 * NP], u[2 * NP];
      if constexpr (VEC) {
        issue();
        copies_wait<kBwdStages - 1>();
        const uint4* slot = ring + (n & (kBwdStages - 1)) * 128;
        L.unpack(L.take(slot), f);
        L.unpack(L.take(slot + 64), u);
      } else {
        L.unpack(pending, f);
        L.unpack(gpending, u);
        issue();
      }
      turn_pairs<NP>(u, cs, sn, cs, snn);
      const float square = group_sum<GL>(dot(f, f), group);
      // 0 for idle groups, which then add nothing even with eps = 0
      const float r = act ? rsqrtf(square * a.inv_dim + a.eps) : 0.0f;
      // with u' = r u: sum += u' x (= u xhat), w' = gain u', dx = w' - x r^2 mean(w' x)
      scale(u, r);
#pragma unroll
      for (int i = 0; i < 2 * NP; i += 2) {
        put2(sum, i, fma2(at2(u, i), at2(f, i), at2(sum, i)));
        put2(u, i, mul2(at2(u, i), at2(gain, i)));
      }
      const float m = -(group_sum<GL>(dot(u, f), group) * a.inv_dim) * r * r;
#pragma unroll
      for (int i = 0; i < 2 * NP; i += 2) put2(u, i, fma2(at2(f, i), make_float2(m, m), at2(u, i)));
      if (act) L.write(y, u);
      y += out_step;
    }
  }
  if (!v.rows) return;                           // uniform over the warp
#pragma unroll
  for (int i = 0; i < 2 * NP; ++i)
    for (int o = 16; o >= group; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
  if (gi == 0) {
    const int D = 2 * a.pairs;
    float* row = v.partial ? v.partial + unit * D : v.rows + (long long)b * D;
    const bool add = !v.partial && a.accumulate;
#pragma unroll
    for (int i = 0; i < NP; ++i)
      if (L.has(i)) {
        int e1, e2;
        L.element(i, e1, e2);
        row[e1] = add ? row[e1] + sum[i] : sum[i];
        row[e2] = add ? row[e2] + sum[NP + i] : sum[NP + i];
      }
  }
}

// rows[b][d] (+)= sum over an example's partial rows.  A block owns COLS columns of one example; its threads stand as strands
// x columns, a strand takes every (number of strands)-th partial row, and the strands are added in a fixed order.  Many
// partial rows get more strands on fewer columns.
struct RowSums { const float* partial[2]; float* rows[2]; int parts[2]; };
template <int COLS>
__global__ void __launch_bounds__(1024)
k_qknorm_rows(const RowSums R, int D, int add) {
  __shared__ float part[32][COLS];
  wait_for_predecessor();
  const int b = blockIdx.x, kind = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if (!R.partial[kind]) return;
  const int d = blockIdx.y * COLS + (lane & (COLS - 1)), n = R.parts[kind];
  const float* p = R.partial[kind] + (long long)b * n * D + d;
  float s = 0.0f;
  if (d < D) {
#pragma unroll 8
    for (int c = threadIdx.x / COLS; c < n; c += blockDim.x / COLS) s += p[(long long)c * D];
  }
#pragma unroll
  for (int o = 16; o >= COLS; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane < COLS) part[warp][lane] = s;
  __syncthreads();
  if (warp) return;
  float t = 0.0f;
  for (int w = lane / COLS; w < warps; w += 32 / COLS) t += part[w][lane & (COLS - 1)];
#pragma unroll
  for (int o = 16; o >= COLS; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if (lane < COLS && d < D) {
    float* o = R.rows[kind] + (long long)b * D + d;
    *o = add ? *o + t : t;
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------

static int check_qk(const dp_qknorm* p) {
  if (!p || p->B <= 0 || p->T <= 0 || p->dim <= 0 || p->n_q < 0 || p->n_k < 0 || p->n_q + (int64_t)p->n_k <= 0) return DP_ERR_ARG;
  if (p->dtype != DP_F32 && p->dtype != DP_BF16) return DP_ERR_ARG;
  if ((p->dim & 1) || p->rot < 0 || (p->rot & 1) || p->rot > p->dim) return DP_ERR_ARG;
  // eps is added in fp32: 0, or a normal number there
  if (!(p->eps == 0.0 || (p->eps >= FLT_MIN && p->eps <= FLT_MAX))) return DP_ERR_ARG;
  if (p->n_q > 65535 || p->n_k > 65535 || p->T > 1 << 24 || (int64_t)p->B * p->T > 1 << 30)
    return DP_ERR_UNSUPPORTED;
  if (p->dim > 2 * kMaxPairs) return DP_ERR_UNSUPPORTED;
  if (p->rot > 0 && !p->inv_freq) return DP_ERR_ARG;
  for (int j = 0; j < p->rot / 2; ++j)
    if (!std::isfinite(p->inv_freq[j])) return DP_ERR_ARG;
  if (misaligned(p->gain_q, 4) || misaligned(p->gain_k, 4) || misaligned(p->positions, 4) || misaligned(p->lengths, 4))
    return DP_ERR_ALIGN;
  return DP_OK;
}

// Copies x to *h after the checks; the stride of an extent of one, which nothing depends on, becomes 0.  Heads that are written
// do not overlap one another.
static int take_heads(const dp_qknorm* p, int heads, const dp_heads* x, size_t es, bool written, dp_heads* h) {
  if (!x || !x->data || x->stride_b < 0 || x->stride_t < 0 || x->stride_h < 0) return DP_ERR_ARG;
  const long long extent[3] = {p->B, p->T, heads}, stride[3] = {x->stride_b, x->stride_t, x->stride_h};
  if (written && !lies_apart(p->dim, 3, extent, stride)) return DP_ERR_ARG;
  *h = {x->data, p->B > 1 ? x->stride_b : 0, p->T > 1 ? x->stride_t : 0, heads > 1 ? x->stride_h : 0};
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

// Shares the heads out (see Share).  `warps` is about what the GPU holds at once.  While there is less than a head for each
// of their groups, heads are spread as widely as they go; with more, a group takes up to kHeadsPerGroup heads of a token,
// and tokens_per_unit grows until kWaves waves of units cover everything.
static Share share_heads(const dp_qknorm* p, int heads, int group_log, long long warps, bool flat) {
  Share s = {};
  s.heads = heads;
  if (heads == 0) return s;
  const int groups_log = 5 - group_log;
  const long long tokens = flat ? (long long)p->B * p->T : p->T, rows = (long long)p->B * p->T * (p->n_q + p->n_k);
  s.heads_per_group = kHeadsPerGroup;
  while (s.heads_per_group > 1 && (rows < ((warps * s.heads_per_group) << groups_log) || s.heads_per_group > heads)) s.heads_per_group >>= 1;
  // neighbouring groups take neighbouring heads, as long as a token has them; the rest of the warp takes further tokens,
  // as long as there are such
  while (s.gh < groups_log && (s.heads_per_group << (s.gh + 1)) <= heads) ++s.gh;
  s.gt = groups_log - s.gh;
  while (s.gt > 0 && (1ll << (s.gt - 1)) >= tokens) { --s.gt; ++s.gh; }
  s.heads_per_unit = s.heads_per_group << s.gh;
  s.head_blocks = ceil_div(heads, s.heads_per_unit);
  const long long strands = (flat ? 1 : p->B) * (long long)s.head_blocks;      // units per run of tokens
  const long long share = warps * kWaves * heads / (p->n_q + p->n_k) + 1;
  long long chunks = (share + strands / 2) / strands;
  const long long most = (tokens + (1 << s.gt) - 1) >> s.gt;
  chunks = chunks < 1 ? 1 : chunks > most ? most : chunks;
  s.tokens_per_unit = (int)(((most + chunks - 1) / chunks) << s.gt);
  s.chunks = (int)((tokens + s.tokens_per_unit - 1) / s.tokens_per_unit);
  s.units = strands * s.chunks;
  return s;
}

// Warps that an SM holds at once, as many as the registers of the kernels allow.
constexpr long long kSms = 148;
static Share backward_share(const dp_qknorm* p, int heads, int group_log) {
  return share_heads(p, heads, group_log, kSms * kBwdWarps, false);
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
  a->v[0].gain = p->gain_q;
  a->v[1].gain = p->gain_k;
  for (int k = 0; k < 2; ++k) {
    const int heads = k ? p->n_k : p->n_q;
    a->v[k].share = backward ? backward_share(p, heads, a->group_log)
                             : share_heads(p, heads, a->group_log, kSms * kFwdWarps, true);
  }
  // inv_freq / (2 pi) modulo one turn, as a 64-bit fraction (x87 arithmetic: 64 bits of mantissa)
  const long double two_pi = 6.283185307179586476925286766559005768L;
  for (int j = 0; j < p->rot / 2; ++j) {
    long double f = (long double)p->inv_freq[j] / two_pi;
    f -= std::floor(f);
    const long double scaled = f * 18446744073709551616.0L;
    a->turn[j] = scaled >= 18446744073709551615.0L ? ~0ull : (unsigned long long)(scaled + 0.5L);
  }
}

// Calls fn.template run<T, NP, VEC, INTER, GL>() for the form that the sizes and alignments allow.  The lanes per head are a
// constant of the kernel at the usual widths (64 to 256 in bf16, 32 to 128 in fp32), where the sums over them unroll.
template <typename T, bool INTER, typename F>
static cudaError_t pick_form(const QkArgs& a, bool vec, F fn) {
  constexpr int V = 16 / sizeof(T);
  if (vec) {
    if (a.group_log == 2) return fn.template run<T, V, true, INTER, 2>();
    if (a.group_log == 3) return fn.template run<T, V, true, INTER, 3>();
    if (a.group_log == 4) return fn.template run<T, V, true, INTER, 4>();
    return fn.template run<T, V, true, INTER, -1>();
  }
  return a.pairs <= 4 * 32 ? fn.template run<T, 4, false, INTER, -1>() : fn.template run<T, 8, false, INTER, 5>();
}
template <typename T, typename F>
static cudaError_t pick(const QkArgs& a, bool vec, bool inter, F fn) {
  return inter ? pick_form<T, true>(a, vec, fn) : pick_form<T, false>(a, vec, fn);
}

template <bool BACKWARD>
struct Launch {
  const QkArgs& a;
  cudaStream_t s;
  template <typename T, int NP, bool VEC, bool INTER, int GL>
  cudaError_t run() const {
    const long long units = a.v[0].share.units + a.v[1].share.units;
    if (units > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    note_launch(1);
    if constexpr (BACKWARD) return launch_chained(k_qknorm_grad<T, NP, VEC, INTER, GL>, (unsigned)units, 32, 0, s, a);
    else return launch_chained(k_qknorm<T, NP, VEC, INTER, GL>, (unsigned)units, 32, 0, s, a);
  }
};

// Lanes per head: V pairs a lane in vectors, else 4, or 8 where 32 lanes of 4 do not hold a head.
static int group_log(int pairs, bool vec, int V) {
  const int per = vec ? V : pairs <= 4 * 32 ? 4 : 8;
  int g = 0;
  while ((per << g) < pairs) ++g;
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
    dp_heads x, y;
    if ((rc = take_heads(p, heads[i], in[i], es, false, &x)) != DP_OK || (rc = take_heads(p, heads[i], out[i], es, true, &y)) != DP_OK)
      return rc;
    vec = vec && vec_heads(x, V) && vec_heads(y, V);
    View& v = a.v[i];
    v.in = x.data; v.in_b = x.stride_b; v.in_t = x.stride_t; v.in_h = x.stride_h;
    v.out = y.data; v.out_b = y.stride_b; v.out_t = y.stride_t; v.out_h = y.stride_h;
  }
  a.group_log = group_log(p->dim / 2, vec, V);
  fill_args(p, &a, false);
  const Launch<false> f{a, static_cast<cudaStream_t>(cuda_stream)};
  const bool inter = p->interleaved != 0;
  const cudaError_t e = p->dtype == DP_F32 ? pick<float>(a, vec, inter, f) : pick<__nv_bfloat16>(a, vec, inter, f);
  return e == cudaSuccess ? DP_OK : DP_ERR_CUDA;
}

// Partial rows of both kinds, for a given lane grouping.
static size_t partial_bytes(const dp_qknorm* p, int glog, size_t* of_queries) {
  size_t n[2];
  for (int k = 0; k < 2; ++k) {
    const Share s = backward_share(p, k ? p->n_k : p->n_q, glog);
    n[k] = s.units > p->B ? (size_t)s.units * p->dim * sizeof(float) : 0;
  }
  if (of_queries) *of_queries = n[0];
  return n[0] + n[1];
}

size_t dp_qknorm_workspace_bytes(const dp_qknorm* p) {
  if (check_qk(p) != DP_OK) return 0;
  // the grouping depends on the tensors' alignment, which is not known here: the larger of the two
  const int V = p->dtype == DP_F32 ? 4 : 8;
  const size_t one = partial_bytes(p, group_log(p->dim / 2, false, V), nullptr);
  const size_t vec = vec_dims(p, V) ? partial_bytes(p, group_log(p->dim / 2, true, V), nullptr) : 0;
  return one > vec ? one : vec;
}

int dp_qknorm_rope_backward(const dp_qknorm* p, const dp_heads* q, const dp_heads* k, const dp_heads* dout_q,
                            const dp_heads* dout_k, const dp_heads* dq, const dp_heads* dk, float* rows_q, float* rows_k,
                            int accumulate_into, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_qk(p);
  if (rc != DP_OK) return rc;
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
    dp_heads x, g, y;
    if ((rc = take_heads(p, heads[i], in[i], es, false, &x)) != DP_OK || (rc = take_heads(p, heads[i], dout[i], es, false, &g)) != DP_OK ||
        (rc = take_heads(p, heads[i], out[i], es, true, &y)) != DP_OK)
      return rc;
    if (misaligned(rows[i], 4)) return DP_ERR_ALIGN;
    vec = vec && vec_heads(x, V) && vec_heads(g, V) && vec_heads(y, V);
    View& v = a.v[i];
    v.in = x.data; v.in_b = x.stride_b; v.in_t = x.stride_t; v.in_h = x.stride_h;
    v.dout = g.data; v.dout_b = g.stride_b; v.dout_t = g.stride_t; v.dout_h = g.stride_h;
    v.out = y.data; v.out_b = y.stride_b; v.out_t = y.stride_t; v.out_h = y.stride_h;
    v.rows = rows[i];
  }
  a.group_log = group_log(p->dim / 2, vec, V);
  fill_args(p, &a, true);
  a.accumulate = accumulate_into ? 1 : 0;
  const bool want_rows = a.v[0].rows || a.v[1].rows;
  size_t of_queries = 0;
  const size_t need = want_rows ? partial_bytes(p, a.group_log, &of_queries) : 0;
  if (need) {
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < dp_qknorm_workspace_bytes(p)) return DP_ERR_WORKSPACE;
    for (int k = 0; k < 2; ++k)
      if (a.v[k].share.units > p->B) a.v[k].partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + (k ? of_queries : 0));
  }
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const Launch<true> f{a, s};
  const bool inter = p->interleaved != 0;
  const cudaError_t e = p->dtype == DP_F32 ? pick<float>(a, vec, inter, f) : pick<__nv_bfloat16>(a, vec, inter, f);
  if (e != cudaSuccess) return DP_ERR_CUDA;
  if (need) {
    RowSums R = {};
    int most = 1;
    for (int k = 0; k < 2; ++k) {
      if (!a.v[k].partial || !a.v[k].rows) continue;
      R.partial[k] = a.v[k].partial;
      R.rows[k] = a.v[k].rows;
      R.parts[k] = a.v[k].share.chunks * a.v[k].share.head_blocks;
      if (R.parts[k] > most) most = R.parts[k];
    }
    // a handful of partial rows per strand, whose loads are all in flight.  The call with 4, 8, 32 warps on 32 columns, 32 warps on 8
    // columns: 13 partial rows an example 34.1, 34.4, 38.3, 56.5 us; 32 rows 14.3, 13.3, 13.2, 17.8; 128 rows 21.4, 16.8, 13.6, 13.2;
    // 512 rows 42, 26, 13.1, 9.9; 2048 rows 137, 72, 23.9, 11.5 (bf16 heads of 64)
    const int warps = most <= 8 ? 4 : most <= 64 ? 8 : 32;
    const bool narrow = most > 256;
    const cudaError_t er = launch_chained(narrow ? k_qknorm_rows<8> : k_qknorm_rows<32>,
                                          dim3(p->B, ceil_div(p->dim, narrow ? 8 : 32), 2), 32 * warps, 0, s, R, p->dim,
                                          a.accumulate);
    note_launch(1);
    if (er != cudaSuccess) return DP_ERR_CUDA;
  }
  return DP_OK;
}

}  // extern "C"
