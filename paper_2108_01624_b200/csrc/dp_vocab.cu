// Softmax cross entropy of tokens X [N, d] against a vocabulary table W [V, d] and a bias, without keeping the logits:
//   z = X W^T + bias,  lse_n = log sum_v exp z_nv,  loss_n = w_n (lse_n - z_n,label)
//   G_nv = w_n (exp(z_nv - lse_n) - [v = label_n])
//   dX = G W,   |G_i^T X_i|^2 (+ |sum_t G_i|^2) of every example i,   acc += sum_i clip_i G_i^T X_i.
//
// k_vocab_gemm is one tensor-core kernel in four forms:
//   LSE    z tile by tile; the epilogue keeps a row's maximum and its sum of exponentials over the tile's columns
//   GRAD   z again; the epilogue turns it into G and stores it, for a piece of the vocabulary at a time
//   DX     dX = G W over the piece
//   DW     acc += G^T X over the piece
// All are bound by the tensor cores where there are enough tokens (256 x 20 tokens of width 1024 and 30522 words are 0.32
// TFLOP a product), and by reading the table where there are few.  There, alone: LSE 204 us (1.57 PFLOP/s, tensor pipe 86 % of the
// time), GRAD 272 (it writes 625 MB of G besides: without its stores 221), DX 210 (1.52 PFLOP/s), DW 417 (both planes of G: 1.53), the norms
// 113 (6.1 TB/s); back to back under the power cap 10 to 25 % longer.  Copies of 128 columns: stages of 64 with twice as many in
// flight took 230 us in LSE, and a forwarding warp in the odd CTA instead of one barrier for the pair's copies 10 more.
//
// Exactness.  A product of bf16 numbers is exact in fp32 and the tensor cores sum in fp32, but drop low bits at every
// step of 16: a sum of 64 steps comes out 7e-7 too small.  So
//   - a sum longer than `seg` blocks is taken over by the epilogue, which adds its parts in registers (norms: every 32 steps);
//   - the label's own logit is formed by itself, in fp64: loss = w log1p(exp(lse of the others - z_label)) keeps its relative error
//     where the model is sure of the label.  G_label = w expm1(z_label - lse) does so for the lse that it is given, an fp32 number:
//     with one that dp_vocab_loss has rounded, every G is off by up to ulp(lse) / 2 of its exponential, G_label by that times w;
//   - G is held as two bf16 numbers, hi + lo, to 2^-16 of it: rows (token, plane) of G meet rows (token, plane) of X in the
//     sums over tokens, whose results are fp32.  dX in bf16 reads hi alone: its own rounding is as large.
//   - fp32 X and W are split into three bf16 numbers each for the logits (24 bits; six products, the smallest first) and
//     into two for the products with G (2^-16 again, four products).
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "dp_chain.cuh"
#include "dp_internal.h"
#include "dp_ptx.cuh"
#include "dp_tma.h"

namespace dpk {
using namespace ptx;

enum : int { V_LSE = 0, V_GRAD = 1, V_DX = 2, V_DW = 3 };

constexpr int V_THREADS = 320;                  // warp 0 TMA, warp 1 UMMA issue (even CTA), warps 2..9 epilogue
constexpr int V_TILE = 256;                     // rows and columns of a pair's tile; a CTA holds 128 rows of it
constexpr int V_BOX_BYTES = 128 * 128;          // one copy: 64 bf16 columns of 128 rows, 128-byte swizzle
constexpr int V_STAGE_COLS = 32;                // GRAD: columns that a warp turns at a time
constexpr int V_WARP_STAGE = 32 * 2 * V_STAGE_COLS * 2;   // 32 tokens x 2 planes, 64-byte rows; DX, DW: 32 x 32 fp32
constexpr float kLog2e = 1.4426950408889634f;

// K columns (or rows) of a stage and stages in flight.
template <int MODE> struct VForm {
  static constexpr bool KMAJOR_A = MODE != V_DW;               // rows of A are tokens with K contiguous
  static constexpr bool KMAJOR_B = MODE == V_LSE || MODE == V_GRAD;
  static constexpr int BK = 128;
  static constexpr int STAGES = 3;
  static constexpr int HALF_BYTES = BK / 64 * V_BOX_BYTES;     // 128 rows (columns) of one operand
  static constexpr int STAGE_BYTES = 2 * HALF_BYTES;
  // an epilogue warp's own: 128 bias values, or what it turns
  static constexpr int WARP_BYTES = MODE == V_LSE ? 128 * 4 : V_WARP_STAGE;
};

struct VCtl {
  uint64_t full[3], empty[3], tmem_full[2], tmem_empty[2], drain;   // full, tmem_empty: the even CTA's count for the pair
  uint32_t tmem_base;
  int abort;
};

template <int MODE> constexpr int v_smem() {
  return 1024 + VForm<MODE>::STAGES * VForm<MODE>::STAGE_BYTES + 8 * VForm<MODE>::WARP_BYTES + (int)sizeof(VCtl);
}
static_assert(v_smem<V_LSE>() <= 232448 && v_smem<V_GRAD>() <= 232448 && v_smem<V_DX>() <= 232448, "over a CTA's shared memory");

struct alignas(64) VParams {
  CUtensorMap a[3], b[3];        // operand planes
  CUtensorMap st;                // GRAD: G
  int n_pairs;
  unsigned char pa[8], pb[8];    // planes of each product, smallest product first
  int kb;                        // K blocks of one product
  int seg;                       // K blocks that are summed before the epilogue takes over
  int tiles_m, tiles_n, nt;      // nt: columns of a tile, 256 or 128
  int units;                     // CTA pairs
  int sharers;                   // DX, DW: the pairs that share what whole tiles leave over, at least one K block each
  int M, N;                      // rows and columns that exist
  int sub;                       // columns of one block of G (GRAD, DX, DW)
  int v0, V;                     // first vocabulary entry of the piece, entries in all
  int planes2;                   // GRAD: store rows 2, 3 of a token too (fp32 X: two planes)
  int stride_c;                  // leading dimension of the output is stride_c (DX, DW)
  const float* bias;             // LSE: [V] or null; GRAD: [columns of all blocks], -inf beyond V
  const int32_t* labels;         // LSE
  const float4* meta;            // GRAD: of every token lse log2e, rounded, and scale over what it was rounded by; G at the label; label (bits)
  float2* part;                  // LSE: [2 tiles_n][M] maximum times log2e, and sum
  float* bias_part;              // GRAD: [rows of 32 tokens][columns of the piece] column sums, or null
  float4* slots;                 // DX, DW: tiles that several pairs share, [2 units][64 groups of four columns][256 rows]
  float* sum;                    // DX: fp32 sums over the pieces [M, N]; DW: the accumulator
  void* out;                     // DX: the result
  int out_bf16, first, last, vec;
  int* status;
};

struct VWork { int tile, j0, j1; };

// What the pair does next.  LSE, GRAD: whole tiles in turn.  DX, DW: whole tiles in turn while there is one for every pair;
// the K blocks of the tiles that are left, laid end to end, are shared evenly.
struct VShare {
  long long lo, hi, pos;         // this pair's part of that line
  int tile, whole;               // next whole tile, and how many of them there are
};
__host__ __device__ __forceinline__ long long share_begin(long long total, int units, int u) { return total * u / units; }
__host__ __device__ __forceinline__ int whole_tiles(int mode, int tiles, int units) {
  return mode == V_LSE || mode == V_GRAD ? tiles : tiles / units * units;
}
template <int MODE>
__device__ __forceinline__ VShare share_of(const VParams& P, int unit) {
  const int tiles = P.tiles_m * P.tiles_n;
  VShare s;
  s.whole = whole_tiles(MODE, tiles, P.units);
  s.tile = unit;
  const long long line = (long long)(tiles - s.whole) * P.n_pairs * P.kb;
  s.lo = s.pos = unit < P.sharers ? share_begin(line, P.sharers, unit) : line;
  s.hi = unit < P.sharers ? share_begin(line, P.sharers, unit + 1) : line;
  return s;
}
template <int MODE>
__device__ __forceinline__ bool next_work(const VParams& P, VShare& s, VWork& w) {
  const int nkb = P.n_pairs * P.kb;
  if (s.tile < s.whole) {
    w = {s.tile, 0, nkb};
    s.tile += P.units;
    return true;
  }
  if (MODE == V_LSE || MODE == V_GRAD || s.pos >= s.hi) return false;
  const long long t = s.pos / nkb, end = (t + 1) * nkb < s.hi ? (t + 1) * nkb : s.hi;
  w.tile = s.whole + (int)t;
  w.j0 = (int)(s.pos - t * nkb);
  w.j1 = w.j0 + (int)(end - s.pos);
  s.pos = end;
  return true;
}

template <int MODE>
__device__ __forceinline__ void tile_origin(const VParams& P, int tile, int& m0, int& n0) {
  if (MODE == V_LSE || MODE == V_GRAD) {        // the tiles of a column block of W follow one another
    n0 = tile / P.tiles_m;
    m0 = tile - n0 * P.tiles_m;
  } else {                                      // the tiles of a row block of G follow one another
    m0 = tile / P.tiles_n;
    n0 = tile - m0 * P.tiles_n;
  }
  m0 *= V_TILE;
  n0 *= P.nt;
}

// What a token without a loss has for `meta`: powers 2^-inf.
#define kNoToken make_float4(INFINITY, 0.0f, 0.0f, __int_as_float(-1))

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Copies of a CTA pair: the data go to this CTA's shared memory, the completion to a barrier of the even CTA (its address in
// the cluster's window).
__device__ __forceinline__ uint32_t in_even_cta(uint64_t* bar) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(bar)));
  return a;
}
__device__ __forceinline__ void pair_load2(uint8_t* dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void pair_load3(uint8_t* dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void load2(uint8_t* dst, const CUtensorMap* map, uint64_t* bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void store4(const CUtensorMap* map, const void* src, int x, int y, int z, int w) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// Copies of K block j of a tile into a stage: this CTA's 128 rows of A and its half of the columns of B.
template <int MODE>
__device__ __forceinline__ void load_block(const VParams& P, uint8_t* st, uint32_t bar, int j, int m0, int n0, int rank) {
  using F = VForm<MODE>;
  const int pair = j / P.kb, k = (j - pair * P.kb) * F::BK;
  const CUtensorMap *a = &P.a[P.pa[pair]], *b = &P.b[P.pb[pair]];
  const int m = m0 + 128 * rank, n = n0 + (P.nt >> 1) * rank;
  uint8_t* sb = st + F::HALF_BYTES;
  if (MODE == V_LSE || MODE == V_GRAD) {
    pair_load2(st, a, bar, k, m);
    pair_load2(st + V_BOX_BYTES, a, bar, k + 64, m);
    pair_load2(sb, b, bar, k, n);
    pair_load2(sb + V_BOX_BYTES, b, bar, k + 64, n);
  } else if (MODE == V_DX) {                    // A: columns of G, block by block; B: rows of W
    const int z = k / P.sub, x = k - z * P.sub;
    pair_load3(st, a, bar, x, m, z);
    pair_load3(st + V_BOX_BYTES, a, bar, x + 64, m, z);
    pair_load2(sb, b, bar, n, P.v0 + k);
    if (P.nt == 256) pair_load2(sb + V_BOX_BYTES, b, bar, n + 64, P.v0 + k);
  } else {                                      // A: rows of G; B: rows of X
    const int z = m / P.sub, x = m - z * P.sub;
    pair_load3(st, a, bar, x, k, z);
    pair_load3(st + V_BOX_BYTES, a, bar, x + 64, k, z);
    pair_load2(sb, b, bar, n, k);
    if (P.nt == 256) pair_load2(sb + V_BOX_BYTES, b, bar, n + 64, k);
  }
}

// Exponentials are powers of two: exp(z - m) = 2^(z log2e - top) with top = m log2e rounded to fp32, one fma and one
// rounding an element, and what top was rounded by in a factor of the row.

// Maximum (as `top`) and sum of powers over this thread's 128 columns of logits, the label's left out.
__device__ __forceinline__ void finish_lse(const VParams& P, f32x2 (&z)[64], int m, int n0, int col, int label) {
  const int rel = label - (P.v0 + n0 + col);
  if (__any_sync(0xffffffffu, (unsigned)rel < 128u)) {
#pragma unroll
    for (int j = 0; j < 64; ++j) {
      const float2 v = unpack2(z[j]);
      z[j] = pack2(rel == 2 * j ? -INFINITY : v.x, rel == 2 * j + 1 ? -INFINITY : v.y);
    }
  }
  float high[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int j = 0; j < 64; ++j) {
    const float2 v = unpack2(z[j]);
    high[j & 3] = fmaxf(high[j & 3], fmaxf(v.x, v.y));
  }
  const float top = fmaxf(fmaxf(high[0], high[1]), fmaxf(high[2], high[3])) * kLog2e;
  const float base = top == -INFINITY ? 0.0f : -top;        // a row of -inf keeps powers of -inf: 0
  const f32x2 k2 = pack2(kLog2e, kLog2e), base2 = pack2(base, base);
  f32x2 s[2] = {0ull, 0ull};
#pragma unroll
  for (int j = 0; j < 64; ++j) {
    const float2 e = unpack2(fma2(z[j], k2, base2));
    s[j & 1] = add2(s[j & 1], pack2(ex2(e.x), ex2(e.y)));
  }
  const float2 sum = unpack2(add2(s[0], s[1]));
  if (m < P.M) P.part[(size_t)((n0 + col) >> 7) * P.M + m] = make_float2(top, sum.x + sum.y);
}

// G of this thread's 128 columns: two planes through shared memory, 32 columns at a time, and the warp's column sums.  (Measured
// instead, GRAD at 272 us: plain stores of the turned chunk 327; 64 columns of half the tokens at a time 336; column sums by
// m16n8k16 products of the staged rows, at 297 with shuffles then, 378.)
__device__ __forceinline__ void finish_grad(const VParams& P, f32x2 (&z)[64], uint8_t* stage, float4 meta, int m0w, int n0, int col,
                                            int lane) {
  const int rel = __float_as_int(meta.w) - (P.v0 + n0 + col);     // no label: -1, never in range
  const bool labelled = __float_as_int(meta.w) >= 0;
  const int at = n0 + col, z4 = at / P.sub, x4 = at - z4 * P.sub;
  const f32x2 k2 = pack2(kLog2e, kLog2e), base2 = pack2(-meta.x, -meta.x), scale2 = pack2(meta.y, meta.y), minus2 = pack2(-1.0f, -1.0f);
#pragma unroll
  for (int ch = 0; ch < 4; ++ch) {
    f32x2 g[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float2 e = unpack2(fma2(z[ch * 16 + j], k2, base2));
      g[j] = mul2(pack2(ex2(e.x), ex2(e.y)), scale2);
    }
    if (__any_sync(0xffffffffu, labelled && (unsigned)(rel - ch * 32) < 32u)) {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float2 v = unpack2(g[j]);
        const int r = labelled ? rel - ch * 32 - 2 * j : -1;
        g[j] = pack2(r == 0 ? meta.z : v.x, r == 1 ? meta.z : v.y);
      }
    }
    if (lane == 0) store_wait_read();           // the copy of the chunk before has left the staging rows
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) {               // 16 bytes = 8 columns
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float2 v = unpack2(g[c * 4 + u]);
        const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
        hi[u] = *reinterpret_cast<const uint32_t*>(&h);
        const f32x2 back = pack2(__uint_as_float(hi[u] << 16), __uint_as_float(hi[u] & 0xffff0000u));
        const float2 left = unpack2(fma2(back, minus2, g[c * 4 + u]));
        const __nv_bfloat162 l = __floats2bfloat162_rn(left.x, left.y);
        lo[u] = *reinterpret_cast<const uint32_t*>(&l);
      }
      uint8_t* p = stage + lane * 128 + ((c ^ (lane & 3)) << 4);       // 64-byte swizzle: rows 2 lane and 2 lane + 1
      *reinterpret_cast<uint4*>(p) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(p + 64) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0 && m0w < P.M) {
      store4(&P.st, stage, x4 + ch * 32, 0, m0w, z4);
      if (P.planes2) store4(&P.st, stage, x4 + ch * 32, 2, m0w, z4);
    }
    if (lane == 0) store_commit();
    if (P.bias_part) {
      // sum over the warp's 32 tokens: at every step a lane keeps half of its columns and hands the others over, so
      // that lane l ends with column l
      float s[32];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float2 v = unpack2(g[j]);
        s[2 * j] = v.x;
        s[2 * j + 1] = v.y;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int j = 0; j < o; ++j) {
          const float keep = up ? s[j + o] : s[j], give = up ? s[j] : s[j + o];
          s[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      }
      P.bias_part[(size_t)(m0w >> 5) * P.N + at + ch * 32 + lane] = s[0];
    }
  }
}

// Four neighbouring columns from c on of a row of dX: summed over the pieces so far, rounded after the last.
__device__ __forceinline__ void put_dx(const VParams& P, int m, int c, float4 v) {
  if (m >= P.M || c >= P.N) return;
  const size_t at = (size_t)m * P.N + c, to = (size_t)m * P.stride_c + c;
  if (P.vec && c + 4 <= P.N) {                  // rows of dX and of the sums start on 16-byte boundaries
    if (!P.first) {
      const float4 s = *reinterpret_cast<const float4*>(P.sum + at);
      v = make_float4(v.x + s.x, v.y + s.y, v.z + s.z, v.w + s.w);
    }
    if (!P.last) {
      *reinterpret_cast<float4*>(P.sum + at) = v;
    } else if (P.out_bf16) {
      const __nv_bfloat162 h[2] = {__floats2bfloat162_rn(v.x, v.y), __floats2bfloat162_rn(v.z, v.w)};
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(P.out) + to) = *reinterpret_cast<const uint2*>(h);
    } else {
      *reinterpret_cast<float4*>(static_cast<float*>(P.out) + to) = v;
    }
    return;
  }
  const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (c + j >= P.N) break;
    const float y = P.first ? x[j] : x[j] + P.sum[at + j];
    if (!P.last) P.sum[at + j] = y;
    else if (P.out_bf16) static_cast<__nv_bfloat16*>(P.out)[to + j] = __float2bfloat16_rn(y);
    else static_cast<float*>(P.out)[to + j] = y;
  }
}

// acc += for four neighbouring columns from c on of a row.  An element has one writer per launch.
__device__ __forceinline__ void put_dw(const VParams& P, int m, int c, float4 v) {
  const int row = P.v0 + m;
  if (row >= P.V || c >= P.N) return;
  float* o = P.sum + (size_t)row * P.stride_c + c;
  if (P.vec && c + 4 <= P.N) {
    asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(o), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
  } else {
    const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < P.N) atomicAdd(o + j, x[j]);
  }
}

template <int MODE>
__global__ void __launch_bounds__(V_THREADS, 1) k_vocab_gemm(const __grid_constant__ VParams P) {
  extern __shared__ uint8_t smem_raw[];
  wait_for_predecessor();
  let_successor_in();
  using F = VForm<MODE>;
  constexpr int STAGES = F::STAGES;
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staging = tiles + STAGES * F::STAGE_BYTES;
  VCtl* S = reinterpret_cast<VCtl*>(staging + 8 * F::WARP_BYTES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &S->abort;
  const int rank = (int)cluster_ctarank(), unit = (int)cluster_id_x();

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&S->full[s], 1); mbar_init(&S->empty[s], 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(&S->tmem_full[b], 1); mbar_init(&S->tmem_empty[b], 16); }
    mbar_init(&S->drain, 1);
    S->abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) { tmem_alloc_pair(&S->tmem_base, 512); tmem_relinquish_pair(); }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();           // the peer's barriers are initialised before anyone signals them
  tc_fence_after();
  const uint32_t tmem_base = S->tmem_base;
  constexpr bool whole = MODE == V_LSE || MODE == V_GRAD;
  VShare share = share_of<MODE>(P, unit);
  VWork w;

  if (warp == 0) {
    if (lane == 0) {   // ---------------- TMA producer (each CTA, its own halves) ----------------
      uint32_t it = 0;
      bool alive = true;
      const uint32_t tx = 2u * (uint32_t)(F::HALF_BYTES + (!F::KMAJOR_B && P.nt == 128 ? V_BOX_BYTES : F::HALF_BYTES));   // of both CTAs
      while (alive && next_work<MODE>(P, share, w)) {
        int m0, n0;
        tile_origin<MODE>(P, w.tile, m0, n0);
        for (int j = w.j0; j < w.j1; ++j, ++it) {
          const uint32_t slot = it % STAGES, ph = (it / STAGES) & 1u;
          if (!mbar_wait(&S->empty[slot], ph ^ 1u, abort_flag, P.status, 61, (int)it)) { alive = false; break; }
          if (rank == 0) mbar_arrive_expect_tx(&S->full[slot], tx);
          load_block<MODE>(P, tiles + slot * F::STAGE_BYTES, in_even_cta(&S->full[slot]), j, m0, n0, rank);
        }
      }
      // Every copy of the pair has landed before either CTA's shared memory is released (the odd CTA waits for the even one
      // at the end).
      const uint32_t pending = it < (uint32_t)STAGES ? it : (uint32_t)STAGES;
      for (uint32_t k = 0; rank == 0 && k < pending; ++k) {
        const uint32_t j = it - 1 - k;
        mbar_wait_drain(&S->full[j % STAGES], (j / STAGES) & 1u, P.status);
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {   // ---------------- UMMA issuer (even CTA only) ----------------
      const uint32_t idesc = idesc_bf16_f32(256, P.nt, !F::KMAJOR_A, !F::KMAJOR_B);
      uint32_t it = 0, part = 0;
      bool alive = true;
      while (alive && next_work<MODE>(P, share, w)) {
        for (int j0 = w.j0; j0 < w.j1 && alive; j0 += P.seg, ++part) {
          const int j1 = j0 + P.seg < w.j1 ? j0 + P.seg : w.j1;
          const uint32_t buf = part & 1u, tph = (part >> 1) & 1u;
          if (!mbar_wait(&S->tmem_empty[buf], tph ^ 1u, abort_flag, P.status, 63, (int)part)) { alive = false; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + buf * 256u;
          for (int j = j0; j < j1; ++j, ++it) {
            const uint32_t slot = it % STAGES, ph = (it / STAGES) & 1u;
            if (!mbar_wait(&S->full[slot], ph, abort_flag, P.status, 64, (int)it)) { alive = false; break; }
            tc_fence_after();
            const uint32_t am = smem_u32(tiles + slot * F::STAGE_BYTES), an = am + F::HALF_BYTES;
#pragma unroll
            for (int k = 0; k < F::BK / 16; ++k) {
              const uint64_t ad = F::KMAJOR_A ? smem_desc_sw128(am + (k >> 2) * V_BOX_BYTES + (k & 3) * 32, 16, 1024)
                                              : smem_desc_sw128(am + k * 2048, V_BOX_BYTES, 1024);
              const uint64_t bd = F::KMAJOR_B ? smem_desc_sw128(an + (k >> 2) * V_BOX_BYTES + (k & 3) * 32, 16, 1024)
                                              : smem_desc_sw128(an + k * 2048, V_BOX_BYTES, 1024);
              umma_bf16_pair(d_tmem, ad, bd, idesc, (j > j0 || k > 0) ? 1u : 0u);
            }
            umma_commit_pair(&S->empty[slot], (uint16_t)3);
          }
          if (alive) umma_commit_pair(&S->tmem_full[buf], (uint16_t)3);
        }
      }
      umma_commit_pair(&S->drain, (uint16_t)1);
      mbar_wait_drain(&S->drain, 0u, P.status);
    }
  } else {   // ---------------- epilogue warps 2..9: lanes [32 q, +32), columns [h nt/2, +nt/2) ----------------
    const int q = warp & 3, h = warp >= 6 ? 1 : 0;
    const int half = P.nt >> 1;
    uint8_t* stage = staging + (warp - 2) * F::WARP_BYTES;
    uint32_t part = 0;
    bool alive = true;
    while (next_work<MODE>(P, share, w)) {
      int m0, n0;
      tile_origin<MODE>(P, w.tile, m0, n0);
      const int m0w = m0 + 128 * rank + 32 * q, m = m0w + lane, col = h * half;
      float4 meta = kNoToken;
      int label = -1;
      if (MODE == V_LSE && m < P.M) label = P.labels[m];
      if (MODE == V_GRAD && m < P.M) meta = P.meta[m];
      // The sums start from the bias: -inf beyond the vocabulary, which has no weight in a sum and is zero in G.
      const float* bias_w = nullptr;
      if (MODE == V_LSE) {
        float* own = reinterpret_cast<float*>(stage);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int v = P.v0 + n0 + col + 32 * k + lane;
          own[32 * k + lane] = v >= P.V ? -INFINITY : P.bias ? P.bias[v] : 0.0f;
        }
        __syncwarp();
        bias_w = own;
      } else if (MODE == V_GRAD) {
        bias_w = P.bias + P.v0 + n0 + col;      // padded
      }
      f32x2 acc[64];
#pragma unroll
      for (int j = 0; j < 64; j += 2) {
        if constexpr (whole) {
          const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(bias_w + 2 * j);
          acc[j] = b.x;
          acc[j + 1] = b.y;
        } else {
          acc[j] = acc[j + 1] = 0ull;
        }
      }
      if (MODE == V_LSE) __syncwarp();          // everyone has read the bias values
      for (int j0 = w.j0; j0 < w.j1; j0 += P.seg, ++part) {
        const uint32_t buf = part & 1u, tph = (part >> 1) & 1u;
        if (alive) alive = __all_sync(0xffffffffu, mbar_wait(&S->tmem_full[buf], tph, abort_flag, P.status, 66, (int)part));
        if (!alive) continue;
        tc_fence_after();
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) {
          if (whole || ch * 32 < half) {
            uint32_t v[32];
            tmem_ld_32x32(tmem_base + ((uint32_t)(q * 32) << 16) + buf * 256u + (uint32_t)(col + ch * 32), v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j)
              acc[ch * 16 + j] = add2(acc[ch * 16 + j], pack2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])));
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(&S->tmem_empty[buf], 0u);
      }
      if (!alive) continue;
      if constexpr (MODE == V_LSE) {
        finish_lse(P, acc, m, n0, col, label);
      } else if constexpr (MODE == V_GRAD) {
        finish_grad(P, acc, stage, meta, m0w, n0, col, lane);
      } else {
        const bool shared_tile = w.j0 != 0 || w.j1 != P.n_pairs * P.kb;
        const int slot = 2 * unit + ((long long)(w.tile - share.whole) * (P.n_pairs * P.kb) > share.lo ? 1 : 0);
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) {
          if (ch * 32 >= half) continue;
          const int c = n0 + col + ch * 32;
          if (shared_tile) {
            float4* to = P.slots + ((size_t)slot * (V_TILE / 4) + (col + ch * 32) / 4) * V_TILE + (m - m0);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              *reinterpret_cast<ulonglong2*>(to + j * V_TILE) = make_ulonglong2(acc[ch * 16 + 2 * j], acc[ch * 16 + 2 * j + 1]);
          } else {                              // turned in shared memory: a warp writes 128 bytes of 4 rows at a time
            ulonglong2* mine = reinterpret_cast<ulonglong2*>(stage + lane * 128);
#pragma unroll
            for (int j = 0; j < 8; ++j) mine[j ^ (lane & 7)] = make_ulonglong2(acc[ch * 16 + 2 * j], acc[ch * 16 + 2 * j + 1]);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int r = 4 * j + (lane >> 3), g = lane & 7;
              const float4 v = reinterpret_cast<const float4*>(stage + r * 128)[g ^ (r & 7)];
              if constexpr (MODE == V_DX) put_dx(P, m0w + r, c + 4 * g, v);
              else put_dw(P, m0w + r, c + 4 * g, v);
            }
            __syncwarp();
          }
        }
      }
    }
    if (MODE == V_GRAD && lane == 0) store_wait_all();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();           // neither CTA leaves while the other may still read its memory or signal it
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

// The tiles of a DX or DW launch that several pairs shared: their parts are added, in an order that the sizes decide.  Block (t, r):
// tile t of those that were shared, 16 / STRANDS rows from (r / 4) of them on, columns [64 (r % 4), +64).  Strands of threads take a run
// of the parts each; a warp reads 4 rows, 8 groups of four columns (64 bytes of a slot, 128 of a result at a time).  One strand where
// a tile has up to eight parts (four strands are four times the blocks, most of whose threads idle), four where more: gradients of width
// 1024, 10000 words with one / four strands, replayed: 256 tokens (18 parts a tile) 51 / 44 us, 512 (9 parts) 55.5 / 55.3, 768 (6 parts) 60.4 /
// 61.1, 2048 (2 parts) 104 / 112.
template <int MODE, int STRANDS>
__global__ void __launch_bounds__(256) k_vocab_join(const __grid_constant__ VParams P) {
  constexpr int OUTPUTS = 256 / STRANDS, ROWS = 16 / STRANDS;
  __shared__ float4 strands[STRANDS][OUTPUTS];
  wait_for_predecessor();
  let_successor_in();
  const int nkb = P.n_pairs * P.kb, tiles = P.tiles_m * P.tiles_n, whole = whole_tiles(MODE, tiles, P.units);
  const long long line = (long long)(tiles - whole) * nkb, begin = (long long)blockIdx.x * nkb;
  // block x of the line is in the share of unit ((x + 1) * sharers - 1) / line: units u0 .. last have a part of the tile
  const int u0 = (int)(((begin + 1) * P.sharers - 1) / line), last = (int)(((begin + nkb) * P.sharers - 1) / line);
  if (last == u0) return;                                         // one unit had it all, and has written it
  int m0, n0;
  tile_origin<MODE>(P, whole + (int)blockIdx.x, m0, n0);
  const int strand = threadIdx.x / OUTPUTS, one = threadIdx.x % OUTPUTS, lane = one & 31, warp = one >> 5;
  const int r0 = (blockIdx.y >> 2) * ROWS, r = r0 + (warp >> 1) * 4 + (lane & 3), g = (blockIdx.y & 3) * 16 + (warp & 1) * 8 + (lane >> 2);
  if ((blockIdx.y & 3) * 64 >= P.nt || m0 + r0 >= P.M) return;
  const int parts = last - u0 + 1, k0 = parts * strand / STRANDS, k1 = parts * (strand + 1) / STRANDS;
  const size_t slot_size = (size_t)(V_TILE / 4) * V_TILE;
  const float4* from = P.slots + (size_t)g * V_TILE + r;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int k = k0; k < k1; ++k) {                                 // the tile is the first of a unit's share but, perhaps, unit u0's
    const float4 x = from[(2 * (u0 + k) + (k == 0 && begin > share_begin(line, P.sharers, u0) ? 1 : 0)) * slot_size];
    v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
  }
  if constexpr (STRANDS > 1) {
    strands[strand][one] = v;
    __syncthreads();
    if (strand) return;
#pragma unroll
    for (int k = 1; k < STRANDS; ++k) {
      const float4 x = strands[k][one];
      v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
    }
  }
  if constexpr (MODE == V_DX) put_dx(P, m0 + r, n0 + 4 * g, v);
  else put_dw(P, m0 + r, n0 + 4 * g, v);
}

// =================================================================================================
// Squared norms of short examples (at most 128 rows of planes): |G_i^T X_i|^2 = sum over rows r, s of the example of
// (<x_r, x_s> + bias) <g_r, g_s>.  A CTA takes as many whole examples as 128 rows hold and some blocks of G; both Grams are
// 128 x 128 x 16 UMMAs of a tile with itself, of which the epilogue uses each row's own example.  Both are taken over by
// the epilogue every kNormSeg stages: the parts of G's are added in registers (its squares are one large, the label's, and a
// vocabulary of small ones, which a longer sum on the tensor core would lose), then those of X's are multiplied by it as they come, so
// that no width makes a sum longer (one sum of X's: 2.8e-4 of a squared norm lost at width 65536, 4e-6 now).  What the tensor core
// drops makes norms too small: at 256 x 20 tokens of width 1024 and 30522 words by 3.2e-6 in the mean with 8 stages, 1.6e-6 with 4, 0.8e-6 with
// 2, 0.4e-6 with 1 (in fp32 throughout 2e-7 to either side), and the norms with GRAD take 416, 418, 423 and 431 us replayed.
// Bound by reading G: 113 us for 625 MB, where the layers' kernel with one example at a time took 318.
// =================================================================================================
constexpr int N_STAGES = 6, N_STAGE_BYTES = 2 * V_BOX_BYTES;    // 128 rows x 128 columns
constexpr int N_THREADS = 192;                                  // warp 0 TMA, warp 1 UMMA, warps 2..5 epilogue
constexpr int kNormSeg = 4;                                     // stages of 128 columns
struct NCtl {
  uint64_t full[N_STAGES], empty[N_STAGES], tmem_full[2], tmem_empty[2], drain;
  uint32_t tmem_base;
  int abort;
  float row[128];
};
constexpr int N_SMEM = 1024 + N_STAGES * N_STAGE_BYTES + (int)sizeof(NCtl);
struct alignas(64) NParams {
  CUtensorMap x, g;
  int rows;                      // of an example
  int examples;                  // of a CTA's 128 rows
  int B, groups, splits, subs, sub, dp, bias;
  float* partial;                // [B][splits]
  int* status;
};

__global__ void __launch_bounds__(N_THREADS, 1) k_vocab_norms(const __grid_constant__ NParams P) {
  extern __shared__ uint8_t smem_raw[];
  wait_for_predecessor();
  let_successor_in();
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  NCtl* S = reinterpret_cast<NCtl*>(tiles + N_STAGES * N_STAGE_BYTES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &S->abort;
  if (threadIdx.x == 0) {
    for (int s = 0; s < N_STAGES; ++s) { mbar_init(&S->full[s], 1); mbar_init(&S->empty[s], 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(&S->tmem_full[b], 1); mbar_init(&S->tmem_empty[b], 4); }
    mbar_init(&S->drain, 1);
    S->abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) { tmem_alloc(&S->tmem_base, 256); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = S->tmem_base;        // columns 0, 128: the parts in turn
  const int px = (P.dp + 127) / 128;              // stages of X
  const int items = P.groups * P.splits;

  if (warp == 0) {
    if (lane == 0) {   // ---------------- TMA producer ----------------
      uint32_t it = 0;
      bool alive = true;
      for (int item = blockIdx.x; item < items && alive; item += gridDim.x) {
        const int grp = item % P.groups, split = item / P.groups;
        const int y = grp * P.examples * P.rows;
        const int s0 = (int)((long long)P.subs * split / P.splits), s1 = (int)((long long)P.subs * (split + 1) / P.splits);
        const int sub_stages = P.sub / 128, pg = (s1 - s0) * sub_stages, all = pg + px;
        for (int j = 0; j < all; ++j, ++it) {
          const uint32_t slot = it % N_STAGES, ph = (it / N_STAGES) & 1u;
          if (!mbar_wait(&S->empty[slot], ph ^ 1u, abort_flag, P.status, 71, (int)it)) { alive = false; break; }
          uint8_t* st = tiles + slot * N_STAGE_BYTES;
          mbar_arrive_expect_tx(&S->full[slot], (uint32_t)N_STAGE_BYTES);
          if (j < pg) {
            const int z = s0 + j / sub_stages, x = j % sub_stages * 128;
            tma_load_3d(st, &P.g, &S->full[slot], x, y, z);
            tma_load_3d(st + V_BOX_BYTES, &P.g, &S->full[slot], x + 64, y, z);
          } else {                                // columns beyond X's arrive as zeros
            load2(st, &P.x, &S->full[slot], 128 * (j - pg), y);
            load2(st + V_BOX_BYTES, &P.x, &S->full[slot], 128 * (j - pg) + 64, y);
          }
        }
      }
      const uint32_t pending = it < (uint32_t)N_STAGES ? it : (uint32_t)N_STAGES;
      for (uint32_t k = 0; k < pending; ++k) {
        const uint32_t j = it - 1 - k;
        mbar_wait_drain(&S->full[j % N_STAGES], (j / N_STAGES) & 1u, P.status);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {   // ---------------- UMMA issuer ----------------
      const int n = (P.examples * P.rows + 15) / 16 * 16;
      const uint32_t idesc = idesc_bf16_f32(128, n, false, false);
      uint32_t it = 0, part = 0;
      bool alive = true;
      for (int item = blockIdx.x; item < items && alive; item += gridDim.x) {
        const int split = item / P.groups;
        const int s0 = (int)((long long)P.subs * split / P.splits), s1 = (int)((long long)P.subs * (split + 1) / P.splits);
        const int pg = (s1 - s0) * (P.sub / 128), all = pg + px;
        for (int j0 = 0; j0 < all && alive; ++part) {
          const int end = j0 < pg ? pg : all, j1 = j0 + kNormSeg < end ? j0 + kNormSeg : end;
          const uint32_t buf = part & 1u, tph = (part >> 1) & 1u;
          if (!mbar_wait(&S->tmem_empty[buf], tph ^ 1u, abort_flag, P.status, 72, (int)part)) { alive = false; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + buf * 128u;
          for (int j = j0; j < j1; ++j, ++it) {
            const uint32_t slot = it % N_STAGES, ph = (it / N_STAGES) & 1u;
            if (!mbar_wait(&S->full[slot], ph, abort_flag, P.status, 74, (int)it)) { alive = false; break; }
            tc_fence_after();
            const uint32_t a = smem_u32(tiles + slot * N_STAGE_BYTES);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const uint64_t desc = smem_desc_sw128(a + (k >> 2) * V_BOX_BYTES + (k & 3) * 32, 16, 1024);
              umma_bf16(d_tmem, desc, desc, idesc, (j > j0 || k > 0) ? 1u : 0u);
            }
            umma_commit(&S->empty[slot]);
          }
          if (alive) umma_commit(&S->tmem_full[buf]);
          j0 = j1;
        }
      }
      umma_commit(&S->drain);
      mbar_wait_drain(&S->drain, 0u, P.status);
    }
  } else {   // ---------------- epilogue warps 2..5: a row each ----------------
    const int q = warp & 3, r = q * 32 + lane;
    const uint32_t lane_base = tmem_base + ((uint32_t)(q * 32) << 16);
    uint32_t part = 0;
    bool alive = true;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
      const int grp = item % P.groups, split = item / P.groups;
      const int s0 = (int)((long long)P.subs * split / P.splits), s1 = (int)((long long)P.subs * (split + 1) / P.splits);
      const int parts_g = ((s1 - s0) * (P.sub / 128) + kNormSeg - 1) / kNormSeg, parts_x = (px + kNormSeg - 1) / kNormSeg;
      float acc[128];
#pragma unroll
      for (int j = 0; j < 128; ++j) acc[j] = 0.0f;
      float sum = 0.0f, one = P.bias ? 1.0f : 0.0f;
      const int c0 = r / P.rows * P.rows, c1 = c0 + P.rows;       // this row's example
      for (int k = 0; k < parts_g + parts_x; ++k, ++part) {
        const uint32_t buf = part & 1u, tph = (part >> 1) & 1u;
        if (alive) alive = __all_sync(0xffffffffu, mbar_wait(&S->tmem_full[buf], tph, abort_flag, P.status, 76, (int)part));
        if (!alive) continue;
        tc_fence_after();
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) {
          uint32_t v[32];
          tmem_ld_32x32(lane_base + buf * 128u + (uint32_t)ch * 32u, v);
          tmem_ld_wait();
          if (k < parts_g) {
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[ch * 32 + j] += __uint_as_float(v[j]);
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              const bool own = ch * 32 + j >= c0 && ch * 32 + j < c1;
              sum += own ? (__uint_as_float(v[j]) + one) * acc[ch * 32 + j] : 0.0f;
            }
          }
        }
        if (k == parts_g) one = 0.0f;             // the bias' part has come with the first of X's
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S->tmem_empty[buf]);
      }
      S->row[r] = sum;
      asm volatile("bar.sync 1, 128;" ::: "memory");
      const int e = threadIdx.x - 64, i = grp * P.examples + e;
      if (alive && e < P.examples && i < P.B) {
        float s = 0.0f;
        for (int k = 0; k < P.rows; ++k) s += S->row[e * P.rows + k];
        P.partial[(size_t)i * P.splits + split] = s;
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem_base, 256);
  }
}

// ---- what surrounds the products ------------------------------------------------------------------------------------
struct VHead {                   // dp_vocab_head with its sizes worked out
  const void* x;
  const void* w;
  const float* bias;
  const int32_t* labels;
  const float* weights;
  long long ldx, ldw;
  int N, T, d, V, f32, vec;      // vec: rows of X and W start on 16-byte boundaries
};

// A label that takes part: -1 for none, and for one beyond the vocabulary, which is reported.
__device__ __forceinline__ int label_of(const VHead& H, int n, int* status) {
  const int y = H.labels[n];
  if (y >= H.V) {
    atomicCAS(status, 0, (int)STATUS_BAD_ID);
    return -1;
  }
  return y < 0 ? -1 : y;
}
// Elements [c, c + 8) of a row, zeros beyond d.
__device__ __forceinline__ void eight(const VHead& H, const void* p, long long row, int c, float (&x)[8]) {
  if (H.vec && c + 8 <= H.d) {
    if (H.f32) {
      const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + row + c);
      const float4 u = q[0], v = q[1];
      x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
    } else {
      const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + row + c);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      x[j] = c + j >= H.d ? 0.0f : H.f32 ? static_cast<const float*>(p)[row + c + j] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[row + c + j]);
  }
}
__device__ __forceinline__ double warp_sum(double s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

// A bf16 number and what it leaves of x.
__device__ __forceinline__ __nv_bfloat16 split_off(float& x) {
  const __nv_bfloat16 h = __float2bfloat16_rn(x);
  x -= __bfloat162float(h);
  return h;
}

// The bf16 parts of eight numbers, which keep what is left.
__device__ __forceinline__ uint4 split_eight(float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = __bfloat16_as_ushort(split_off(x[2 * j])), hi = __bfloat16_as_ushort(split_off(x[2 * j + 1]));
    w[j] = lo | hi << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Planes of W and (from row H.V on) X: out[plane][row][dp], zeros beyond d; a warp a row.  (fp32: three, bf16: one, where the
// tensors' own rows cannot be copied by TMA.)
__global__ void __launch_bounds__(256)
k_vocab_planes(const __grid_constant__ VHead H, int rows_x, int dp, int planes, __nv_bfloat16* out_w, __nv_bfloat16* out_x) {
  wait_for_predecessor();
  let_successor_in();
  const int lane = threadIdx.x & 31;
  for (long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); r < (long long)H.V + rows_x; r += (long long)gridDim.x * 8) {
    const bool isx = r >= H.V;
    const long long row = isx ? r - H.V : r, rows = isx ? rows_x : H.V;
    __nv_bfloat16* out = (isx ? out_x : out_w) + row * dp;
    for (int c = 8 * lane; c < dp; c += 256) {
      float x[8];
      eight(H, isx ? H.x : H.w, row * (isx ? H.ldx : H.ldw), c, x);
      for (int p = 0; p < planes; ++p) *reinterpret_cast<uint4*>(out + p * rows * dp + c) = split_eight(x);
    }
  }
}

// A warp per token: its row of X as R rows of planes (zeros where it has no label: what such a row holds may be
// anything), the third plane of fp32 apart, and its `meta`; all threads: the bias, padded.  Column `one` (-1: none) beyond X's is a
// one: with it as X's last column the norm of G^T X holds the bias' part (as that of W, whose column d is zero, it leaves
// the logits alone).
__global__ void __launch_bounds__(256)
k_vocab_tokens(const __grid_constant__ VHead H, const float* lse, const float* clip, int R, int dp, int one, __nv_bfloat16* xe,
               __nv_bfloat16* x2, float4* meta, float* bias, int columns, int* status) {
  wait_for_predecessor();
  let_successor_in();
  const int n = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  // without sign: of 2^26 tokens a step is 2^31
  for (unsigned v = blockIdx.x * 256 + threadIdx.x; v < (unsigned)columns; v += gridDim.x * 256)
    bias[v] = v >= H.V ? -INFINITY : H.bias ? H.bias[v] : 0.0f;
  if (n >= H.N) return;
  const int y = label_of(H, n, status);
  double s = 0.0;
#pragma unroll 4
  for (int c = 8 * lane; c < dp; c += 256) {
    float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (y >= 0) {
      float w[8];
      eight(H, H.x, (long long)n * H.ldx, c, x);
      eight(H, H.w, (long long)y * H.ldw, c, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fma((double)x[j], (double)w[j], s);
    }
    if ((unsigned)(one - c) < 8u) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = c + j == one ? 1.0f : x[j];
    }
    uint4* row = reinterpret_cast<uint4*>(xe + (size_t)n * R * dp + c);
    row[0] = row[dp / 8] = split_eight(x);
    if (R == 4) {
      row[2 * (dp / 8)] = row[3 * (dp / 8)] = split_eight(x);
      *reinterpret_cast<uint4*>(x2 + (size_t)n * dp + c) = split_eight(x);
    }
  }
  float4 m = kNoToken;
  if (y >= 0) {
    const double z = warp_sum(s) + (H.bias ? (double)H.bias[y] : 0.0);
    float scale = H.weights ? H.weights[n] : 1.0f;
    if (clip) scale *= clip[n / H.T];
    const float top = lse[n] * kLog2e, left = fmaf(lse[n], kLog2e, -top);
    m = make_float4(top, scale * ex2(-left), scale * expm1f((float)(z - (double)lse[n])), __int_as_float(y));
  }
  if (lane == 0) meta[n] = m;
}

// lse and loss of a token from the parts over the column blocks, which leave the label out: a warp per token (eight
// neighbours a block, whose parts share sectors), its label's logit in fp64.  With `carry`, more columns are to come: the
// parts become one, kept there.
__global__ void __launch_bounds__(256, 5)
k_vocab_loss(const __grid_constant__ VHead H, const float2* part, int parts, float2* carry, float* loss, float* lse, int* status) {
  wait_for_predecessor();
  let_successor_in();
  const int lane = threadIdx.x & 31, n = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (n >= H.N) return;
  const int y = label_of(H, n, status);
  if (y < 0) {
    if (lane == 0 && !carry) loss[n] = lse[n] = 0.0f;
    return;
  }
  float2 ahead[4];                              // the first 128 parts are on their way while the logit is formed
#pragma unroll
  for (int j = 0; j < 4; ++j) ahead[j] = lane + 32 * j < parts ? part[(size_t)(lane + 32 * j) * H.N + n] : make_float2(-INFINITY, 0.0f);
  double s = 0.0;
#pragma unroll 4
  for (int c = 8 * lane; c < H.d && !carry; c += 256) {
    float x[8], w[8];
    eight(H, H.x, (long long)n * H.ldx, c, x);
    eight(H, H.w, (long long)y * H.ldw, c, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fma((double)x[j], (double)w[j], s);
  }
  float most = -INFINITY, sum = 0.0f;
  const auto join = [&](float2 v) {
    const float top = fmaxf(most, v.x);
    if (top != -INFINITY) {
      sum = sum * ex2(most - top) + v.y * ex2(v.x - top);
      most = top;
    } else {
      sum += v.y;                               // 0, or NaN
    }
  };
#pragma unroll
  for (int j = 0; j < 4; ++j) join(ahead[j]);
#pragma unroll 4
  for (int p = lane + 128; p < parts; p += 32) join(part[(size_t)p * H.N + n]);
  float top = most;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  float all = top == -INFINITY ? sum : sum * ex2(most - top);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
  const double z = warp_sum(s) + (H.bias ? (double)H.bias[y] : 0.0);
  if (carry) {
    if (lane == 0) carry[n] = make_float2(top, all);
  } else if (lane == 0) {
    const double others = ((double)top + (double)log2f(all)) * 0.69314718055994530942;   // -inf where there are none
    const float gap = (float)(others - z);
    float l = gap > 0.0f ? gap + log1pf(expf(-gap)) : log1pf(expf(gap));
    if (z == INFINITY) l = NAN;                 // as any other infinite logit
    loss[n] = (H.weights ? H.weights[n] : 1.0f) * l;
    lse[n] = (float)(z == -INFINITY ? others : z + (double)l);
  }
}

// acc_b[v] += the sum over rows of part[row][v]: 32 columns a block, eight strands of rows, added in order.
__global__ void __launch_bounds__(256) k_vocab_bias(const float* part, int rows, int cols, int n, float* acc_b) {
  __shared__ float s[8][33];
  wait_for_predecessor();
  let_successor_in();
  const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float sum = 0.0f;
#pragma unroll 8
  for (int r = strand; r < rows; r += 8) sum += part[(size_t)r * cols + c];
  s[strand][lane] = sum;
  __syncthreads();
  if (strand == 0 && c < n) {
#pragma unroll
    for (int k = 1; k < 8; ++k) sum += s[k][lane];
    acc_b[c] += sum;
  }
}

// sqnorm[i] = or += the parts of example i, in order: a warp an example, its lanes every 32nd part each, then a fixed tree.
__global__ void __launch_bounds__(256) k_vocab_norm_sum(const float* part, int B, int parts, float* sqnorm, int add) {
  wait_for_predecessor();
  let_successor_in();
  const int i = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (i >= B) return;
  float s = 0.0f;
  for (int k = lane; k < parts; k += 32) s += part[(long long)i * parts + k];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o);
  if (lane == 0) sqnorm[i] = add ? sqnorm[i] + s : s;
}

// ---- host side --------------------------------------------------------------------------------------------------------
int set_vocab_wait_limit(long long cycles) {
  return cudaMemcpyToSymbol(g_wait_limit_cycles, &cycles, sizeof(cycles)) == cudaSuccess ? DP_OK : DP_ERR_CUDA;
}

static bool vocab_kernels_ready() {
  static signed char state[kMaxDevices] = {};     // 0 unknown, 1 ready, -1 failed
  const int dev = current_device();
  if (dev < 0) return false;
  if (!state[dev]) {
    const auto opt = [](const void* k, int bytes) {
      return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
    };
    state[dev] = (opt((const void*)k_vocab_gemm<V_LSE>, v_smem<V_LSE>()) && opt((const void*)k_vocab_gemm<V_GRAD>, v_smem<V_GRAD>()) &&
                  opt((const void*)k_vocab_gemm<V_DX>, v_smem<V_DX>()) && opt((const void*)k_vocab_gemm<V_DW>, v_smem<V_DW>()) && opt((const void*)k_vocab_norms, N_SMEM)) ? 1 : -1;
  }
  return state[dev] > 0;
}

// A bf16 tensor of up to four dimensions, innermost first; strides (bytes) of dimensions 1.. .
static bool encode(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
                   const cuuint32_t* box, CUtensorMapSwizzle swizzle) {
  EncodeTiledFn fn = encode_fn();
  const cuuint32_t ones[4] = {1u, 1u, 1u, 1u};
  return fn && fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, ones,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Boxes of 64 columns x 128 rows of [rows, cols] with a row stride in elements.
static bool encode_rows(CUtensorMap* map, const void* base, long long rows, int cols, long long ld) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64u, 128u};
  return encode(map, base, 2, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// The same of every block of G [blocks][rows, ld][sub].
static bool encode_blocks(CUtensorMap* map, const void* base, long long rows, int sub, long long ld, int blocks, long long block) {
  const cuuint64_t dims[3] = {(cuuint64_t)sub, (cuuint64_t)rows, (cuuint64_t)blocks};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)block * 2};
  const cuuint32_t box[3] = {64u, 128u, 1u};
  return encode(map, base, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

// Maxima and sums of the column blocks that are joined at a time.  Beyond it a product ends and begins, and its tail waits for the join:
// the loss of 2000 x 100 tokens of width 64, 30522 words (all of it 765 MB) takes 3909 us with 64 MiB, 3728 with 128, 3658 with 256, 3594 with
// 512, 3598 in one.
constexpr size_t kPartBytes = (size_t)256 << 20;
constexpr int kSubColumns = 2048;               // columns of one block of G, at most
// G of one piece, unless one block alone is larger.  Every piece costs the start and the end of three kernels and another pass
// over the sums of dX: 256 x 20 tokens of width 1024, 30522 words, gradient / clipped sum with pieces of 128 MiB 1048 / 987 us, 256 MiB
// 875 / 932, 384 MiB 781 / 908, all of G (640 MiB) 686 / 863.
constexpr size_t kPieceBytes = (size_t)1 << 30;

// How many CTAs share a group's blocks of G: each forms the Gram of X again, so as few as fill the device well, by the
// columns that the longest-working CTA sums.
static int norm_splits(int groups, int subs, int sub, int dp) {
  int best = 1;
  long long least = 0;
  for (int s = 1; s <= subs; ++s) {
    const long long rounds = ((long long)groups * s + sm_count() - 1) / sm_count(), cost = rounds * (dp + (long long)ceil_div(subs, s) * sub);
    if (s == 1 || cost < least) best = s, least = cost;
  }
  return best;
}

// Sizes and the workspace of a call.
struct VPlan {
  int R;                         // rows of X and G per token: 2, or 4 for fp32
  int dp;                        // width of packed rows
  bool direct;                   // X and W can be copied by TMA as they are
  int sub, n_sub, piece_subs, pieces;
  int mt;                        // 256-token tiles
  int loss_columns;              // vocabulary entries whose parts are joined at a time
  size_t part, xe, x2, xp, wp, meta, padded, G, slots, dx, gram, cols, bias, total;
  int gram_count;                // partial sums per example of one piece
  bool gram_way;
  int short_examples;            // examples that 128 rows of planes hold; 0: longer ones, for the layers' norm kernels
};

static bool direct_rows(const void* p, long long ld) { return !misaligned(p, 16) && ld % 8 == 0; }

static dp_layer piece_layer(const dp_vocab_head& h, const VPlan& p, const void* xe, const void* G) {
  dp_layer L = {};
  L.kind = DP_LINEAR;
  L.dtype = DP_BF16;
  L.path = DP_PATH_AUTO;
  L.has_bias = h.bias && p.R == 2;     // a column of ones stands for it where tokens have rows of several planes of X
  L.B = h.B;
  L.T = h.T * p.R;
  L.d_in = p.dp;
  L.d_out = p.sub;
  L.A = xe;
  L.G = G;
  return L;
}

// op: 0 loss, 1 backward, 2 clipped sum
static VPlan plan_vocab(const dp_vocab_head& h, int op) {
  VPlan p = {};
  const long long N = (long long)h.B * h.T;
  const bool f32 = h.dtype == DP_F32;
  p.R = f32 ? 4 : 2;
  p.dp = (h.d + (f32 && h.bias && op == 1 ? 1 : 0) + 63) / 64 * 64;
  p.direct = !f32 && direct_rows(h.W, h.ldw) && (op != 0 || direct_rows(h.X, h.ldx));
  p.n_sub = ceil_div(h.V, kSubColumns);
  p.sub = (ceil_div(h.V, p.n_sub) + 255) / 256 * 256;
  p.n_sub = ceil_div(h.V, p.sub);
  p.mt = (int)((N + V_TILE - 1) / V_TILE);
  size_t at = 0;
  const auto take = [&](size_t& off, size_t bytes) {
    off = at;
    at = align_up(at + bytes, 256);
  };
  const int planes = f32 ? 3 : 1;
  if (!p.direct) take(p.wp, (size_t)planes * h.V * p.dp * 2);
  if (op == 0) {
    if (!p.direct) take(p.xp, (size_t)planes * N * p.dp * 2);
    const long long tiles = std::max<long long>(1, (long long)(kPartBytes / (2 * N * sizeof(float2))));
    p.loss_columns = (int)std::min<long long>(ceil_div(h.V, V_TILE), tiles) * V_TILE;
    take(p.part, (size_t)(1 + 2 * (p.loss_columns / V_TILE)) * N * sizeof(float2));
    p.total = at;
    return p;
  }
  const size_t block = (size_t)N * p.R * p.sub * 2;
  int subs = (int)std::min<size_t>(std::max<size_t>(kPieceBytes / block, 1), (size_t)p.n_sub);
  p.pieces = ceil_div(p.n_sub, subs);
  p.piece_subs = ceil_div(p.n_sub, p.pieces);
  p.pieces = ceil_div(p.n_sub, p.piece_subs);
  take(p.xe, (size_t)N * p.R * p.dp * 2);
  if (f32) take(p.x2, (size_t)N * p.dp * 2);
  take(p.meta, (size_t)N * sizeof(float4));
  take(p.padded, (size_t)p.n_sub * p.sub * sizeof(float));
  take(p.G, block * p.piece_subs);
  take(p.slots, (size_t)2 * (sm_count() / 2) * V_TILE * V_TILE * sizeof(float));
  if (op == 1) {
    if (p.pieces > 1) take(p.dx, (size_t)N * h.d * sizeof(float));
    p.short_examples = 128 / (p.R * h.T);
    const dp_layer L = piece_layer(h, p, nullptr, nullptr);
    p.gram_way = use_gram(L);
    const int first = 0, way = p.gram_way ? 1 : 0;
    p.gram_count = p.piece_subs * (p.short_examples ? 1 : (int)umma_sqnorm_partials_per_example(&L, &first, 1, &way));
    take(p.gram, (size_t)h.B * p.gram_count * sizeof(float));
    if (!p.gram_way && h.bias && p.R == 2) take(p.cols, (size_t)p.piece_subs * h.B * p.sub * sizeof(float));
  } else if (h.bias) {
    take(p.bias, (size_t)p.mt * 8 * p.piece_subs * p.sub * sizeof(float));
  }
  p.total = at;
  return p;
}

static int check_head(const dp_vocab_head* h) {
  if (!h || !h->X || !h->W || !h->labels) return DP_ERR_ARG;
  if (h->dtype != DP_F32 && h->dtype != DP_BF16) return DP_ERR_ARG;
  if (h->B <= 0 || h->T <= 0 || h->d <= 0 || h->V <= 0) return DP_ERR_ARG;
  if (h->ldx < h->d || h->ldw < h->d) return DP_ERR_ARG;
  if ((long long)h->B * h->T > (1 << 26) || h->V > (1 << 26) || h->d > (1 << 16) || h->ldx > (1ll << 36) || h->ldw > (1ll << 36))
    return DP_ERR_UNSUPPORTED;
  const size_t e = h->dtype == DP_F32 ? 4 : 2;
  if (misaligned(h->X, e) || misaligned(h->W, e) || misaligned(h->labels, 4) || misaligned(h->bias, 4) || misaligned(h->weights, 4))
    return DP_ERR_ALIGN;
  return DP_OK;
}

static VHead head_of(const dp_vocab_head& h) {
  const int f32 = h.dtype == DP_F32, e = f32 ? 4 : 8;
  const int vec = !misaligned(h.X, 16) && !misaligned(h.W, 16) && h.ldx % e == 0 && h.ldw % e == 0;
  return {h.X, h.W, h.bias, h.labels, h.weights, h.ldx, h.ldw, h.B * h.T, h.T, h.d, h.V, f32, vec};
}

struct VRun {                    // a call under way
  const dp_vocab_head& h;
  const VPlan& p;
  char* ws;
  cudaStream_t s;
  int* status;
  template <typename T> T* at(size_t off) const { return reinterpret_cast<T*>(ws + off); }
};

#define VOCAB_CUDA(expr) do { note_launch(1); if ((expr) != cudaSuccess) return DP_ERR_CUDA; } while (0)

static int pack_rows(const VRun& r, int rows_x, size_t off_x) {
  const bool f32 = r.h.dtype == DP_F32;
  const unsigned grid = (unsigned)std::min<long long>(((long long)r.h.V + rows_x + 7) / 8, (long long)sm_count() * 8);
  VOCAB_CUDA(launch_chained(k_vocab_planes, grid, 256, 0, r.s, head_of(r.h), rows_x, r.p.dp, f32 ? 3 : 1, r.at<__nv_bfloat16>(r.p.wp),
                            r.at<__nv_bfloat16>(off_x)));
  return DP_OK;
}

// Rows [v0, v0 + rows) of W in planes, and the products of a logit.
static int logits_operands(const VRun& r, VParams& P, int v0, int rows) {
  const dp_vocab_head& h = r.h;
  const bool f32 = h.dtype == DP_F32;
  for (int k = 0; k < (f32 ? 3 : 1); ++k) {
    const bool ok = r.p.direct ? encode_rows(&P.b[k], static_cast<const __nv_bfloat16*>(h.W) + v0 * h.ldw, rows, h.d, h.ldw)
                               : encode_rows(&P.b[k], r.at<__nv_bfloat16>(r.p.wp) + ((size_t)k * h.V + v0) * r.p.dp, rows, r.p.dp, r.p.dp);
    if (!ok) return DP_ERR_CUDA;
  }
  static const unsigned char pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
  P.n_pairs = f32 ? 6 : 1;
  for (int k = 0; k < P.n_pairs; ++k) {
    P.pa[k] = f32 ? pa[k] : 0;
    P.pb[k] = f32 ? pb[k] : 0;
  }
  P.kb = ceil_div(h.d, 128);
  P.seg = f32 ? 4 : 16;
  P.nt = V_TILE;
  P.v0 = v0;
  P.V = h.V;
  P.status = r.status;
  return DP_OK;
}

// Pairs that share a line of K blocks: all, or fewer where a share would be shorter than four (one pair for fewer).  Small heads only, and
// no length is best for all: with shares of 1 / 2 / 4 / 8 blocks at least, replayed, the gradient of 16 x 20 bf16 tokens of width 512, 5003
// words takes 35 / 35 / 31 / 33 us, of 30 x 20 of width 1024, 300 words 35 / 38 / 48 / 50, the sum of 4 x 20 of width 256, 2000 words
// 29 / 25 / 29 / 38, of 2 x 60 of width 64, 20011 words 38 / 34 / 34 / 43.
static int share_units(long long line) {
  const long long most = sm_count() / 2;
  return (int)std::max<long long>(1, std::min<long long>(most, line / 4));
}

template <int MODE>
static int launch_product(const VRun& r, VParams& P) {
  const long long tiles = (long long)P.tiles_m * P.tiles_n, line = tiles * P.n_pairs * P.kb;
  if (tiles > 0x7fffffffll) return DP_ERR_UNSUPPORTED;
  if (MODE == V_LSE || MODE == V_GRAD) P.units = (int)std::min<long long>(tiles, sm_count() / 2);
  else P.units = share_units(line);
  const int shared = (int)tiles - whole_tiles(MODE, (int)tiles, P.units);
  P.sharers = std::min(P.units, share_units((long long)shared * P.n_pairs * P.kb));
  VOCAB_CUDA(launch_chained(k_vocab_gemm<MODE>, Pairs{(unsigned)P.units}, V_THREADS, v_smem<MODE>(), r.s, P));
  if constexpr (MODE == V_DX || MODE == V_DW) {
    if (P.sharers > 1 && shared)
      VOCAB_CUDA(P.sharers <= 8 * shared ? launch_chained(k_vocab_join<MODE, 1>, dim3((unsigned)shared, V_TILE / 4), 256, 0, r.s, P)
                                       : launch_chained(k_vocab_join<MODE, 4>, dim3((unsigned)shared, V_TILE), 256, 0, r.s, P));
  }
  return DP_OK;
}

// Tokens, planes of W, then G piece by piece; each piece is handed to `use`.
template <typename Use>
static int over_pieces(const VRun& r, const float* lse, const float* clip, float* bias_part, Use use) {
  const dp_vocab_head& h = r.h;
  const VPlan& p = r.p;
  const int N = h.B * h.T;
  const bool f32 = h.dtype == DP_F32;
  int rc;
  if (!p.direct && (rc = pack_rows(r, 0, 0)) != DP_OK) return rc;
  __nv_bfloat16 *xe = r.at<__nv_bfloat16>(p.xe), *x2 = r.at<__nv_bfloat16>(p.x2), *G = r.at<__nv_bfloat16>(p.G);
  const int columns = p.n_sub * p.sub;
  VOCAB_CUDA(launch_chained(k_vocab_tokens, (unsigned)ceil_div(std::max(N, columns / 64), 8), 256, 0, r.s, head_of(h), lse, clip, p.R, p.dp, p.dp > h.d && f32 && h.bias && !clip ? h.d : -1, xe, x2,
                            r.at<float4>(p.meta), r.at<float>(p.padded), columns, r.status));
  for (int s0 = 0; s0 < p.n_sub; s0 += p.piece_subs) {
    const int subs = std::min(p.piece_subs, p.n_sub - s0);
    VParams P = {};
    const int v0 = s0 * p.sub;
    if ((rc = logits_operands(r, P, v0, std::min(subs * p.sub, h.V - v0))) != DP_OK) return rc;
    if (!encode_rows(&P.a[0], xe, N, p.dp, (long long)p.R * p.dp)) return DP_ERR_CUDA;
    if (f32 && (!encode_rows(&P.a[1], xe + 2 * p.dp, N, p.dp, (long long)p.R * p.dp) || !encode_rows(&P.a[2], x2, N, p.dp, p.dp)))
      return DP_ERR_CUDA;
    const long long block = (long long)N * p.R * p.sub;
    const cuuint64_t dims[4] = {(cuuint64_t)p.sub, (cuuint64_t)p.R, (cuuint64_t)N, (cuuint64_t)subs};
    const cuuint64_t strides[3] = {(cuuint64_t)p.sub * 2, (cuuint64_t)p.R * p.sub * 2, (cuuint64_t)block * 2};
    const cuuint32_t box[4] = {(cuuint32_t)V_STAGE_COLS, 2u, 32u, 1u};
    if (!encode(&P.st, G, 4, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_64B)) return DP_ERR_CUDA;
    P.tiles_m = p.mt;
    P.tiles_n = subs * p.sub / V_TILE;
    P.M = N;
    P.N = subs * p.sub;
    P.sub = p.sub;
    P.bias = r.at<float>(p.padded);
    P.planes2 = f32;
    P.meta = r.at<float4>(p.meta);
    P.bias_part = bias_part;
    if ((rc = launch_product<V_GRAD>(r, P)) != DP_OK) return rc;
    if ((rc = use(s0, subs, block)) != DP_OK) return rc;
  }
  return DP_OK;
}

static int check_call(const dp_vocab_head* h, int op, void* workspace, size_t bytes, VPlan* p) {
  *p = plan_vocab(*h, op);
  if (p->total > ((size_t)1 << 40)) return DP_ERR_UNSUPPORTED;
  if (!workspace || misaligned(workspace, 256) || bytes < p->total) return DP_ERR_WORKSPACE;
  return DP_OK;
}

}  // namespace dpk

using namespace dpk;

extern "C" {

size_t dp_vocab_workspace_bytes(const dp_vocab_head* head) {
  if (check_head(head) != DP_OK) return 0;
  size_t most = (size_t)head->B * kCrossChunks * sizeof(float);
  for (int op = 0; op < 3; ++op) most = std::max(most, plan_vocab(*head, op).total);
  return most;
}

int dp_vocab_loss(const dp_vocab_head* head, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                  void* cuda_stream) {
  int rc = check_head(head);
  if (rc != DP_OK) return rc;
  if (!loss || !lse) return DP_ERR_ARG;
  if (misaligned(loss, 4) || misaligned(lse, 4)) return DP_ERR_ALIGN;
  VPlan p;
  if ((rc = check_call(head, 0, workspace, workspace_bytes, &p)) != DP_OK) return rc;
  const dp_vocab_head& h = *head;
  int* status = status_ptr();
  if (!status || !vocab_kernels_ready()) return DP_ERR_CUDA;
  const VRun r = {h, p, static_cast<char*>(workspace), static_cast<cudaStream_t>(cuda_stream), status};
  const int N = h.B * h.T;
  if (!p.direct && (rc = pack_rows(r, N, p.xp)) != DP_OK) return rc;
  float2* part = r.at<float2>(p.part);          // [what went before][column blocks], a value a token each
  for (int v0 = 0; v0 < h.V; v0 += p.loss_columns) {
    VParams P = {};
    if ((rc = logits_operands(r, P, v0, h.V - v0)) != DP_OK) return rc;
    for (int k = 0; k < (h.dtype == DP_F32 ? 3 : 1); ++k) {
      const bool ok = p.direct ? encode_rows(&P.a[k], h.X, N, h.d, h.ldx)
                               : encode_rows(&P.a[k], r.at<__nv_bfloat16>(p.xp) + (size_t)k * N * p.dp, N, p.dp, p.dp);
      if (!ok) return DP_ERR_CUDA;
    }
    const int columns = std::min(p.loss_columns, h.V - v0);
    const bool last = v0 + columns >= h.V;
    P.bias = h.bias;
    P.tiles_m = p.mt;
    P.tiles_n = ceil_div(columns, V_TILE);
    P.M = N;
    P.N = columns;
    P.labels = h.labels;
    P.part = part + N;
    if ((rc = launch_product<V_LSE>(r, P)) != DP_OK) return rc;
    VOCAB_CUDA(launch_chained(k_vocab_loss, (unsigned)ceil_div(N, 8), 256, 0, r.s, head_of(h), part + (v0 ? 0 : N),
                              2 * P.tiles_n + (v0 ? 1 : 0), last ? nullptr : part, loss, lse, status));
  }
  return DP_OK;
}

int dp_vocab_loss_backward(const dp_vocab_head* head, const float* lse, void* dx, int64_t ld_dx, float* sqnorm,
                           int accumulate_into, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_head(head);
  if (rc != DP_OK) return rc;
  if (!lse || (!dx && !sqnorm)) return DP_ERR_ARG;
  const dp_vocab_head& h = *head;
  if (dx && (ld_dx < h.d || ld_dx > 0x7fffffffll)) return DP_ERR_ARG;
  if (misaligned(lse, 4) || misaligned(sqnorm, 4) || misaligned(dx, h.dtype == DP_F32 ? 4 : 2)) return DP_ERR_ALIGN;
  VPlan p;
  if ((rc = check_call(head, 1, workspace, workspace_bytes, &p)) != DP_OK) return rc;
  if (dx && rows_meet(h.X, h.ldx, dx, ld_dx, (long long)h.B * h.T, h.d, h.dtype == DP_F32 ? 4 : 2)) return DP_ERR_ARG;
  int* status = status_ptr();
  if (!status || !vocab_kernels_ready()) return DP_ERR_CUDA;
  const VRun r = {h, p, static_cast<char*>(workspace), static_cast<cudaStream_t>(cuda_stream), status};
  const int N = h.B * h.T;
  const bool f32 = h.dtype == DP_F32;
  __nv_bfloat16* G = r.at<__nv_bfloat16>(p.G);
  try {                          // the layers' norm kernels keep lists of a piece's blocks
    return over_pieces(r, lse, nullptr, nullptr, [&](int s0, int subs, long long block) -> int {
      int rc = DP_OK;
      if (dx) {
        VParams P = {};
        const int v0 = s0 * p.sub, cols = std::min(subs * p.sub, h.V - v0);
        for (int k = 0; k < (f32 ? 2 : 1); ++k) {
          if (!encode_blocks(&P.a[k], G + (size_t)k * p.sub, N, p.sub, (long long)p.R * p.sub, subs, block)) return DP_ERR_CUDA;
          const bool ok = p.direct ? encode_rows(&P.b[k], h.W, h.V, h.d, h.ldw)
                                   : encode_rows(&P.b[k], r.at<__nv_bfloat16>(p.wp) + (size_t)k * h.V * p.dp, h.V, h.d, p.dp);
          if (!ok) return DP_ERR_CUDA;
        }
        static const unsigned char pa[4] = {1, 1, 0, 0}, pb[4] = {1, 0, 1, 0};
        P.n_pairs = f32 ? 4 : 1;
        for (int k = 0; k < P.n_pairs; ++k) {
          P.pa[k] = f32 ? pa[k] : 0;
          P.pb[k] = f32 ? pb[k] : 0;
        }
        P.kb = ceil_div(cols, 128);
        P.seg = 16;
        P.nt = h.d <= 128 ? 128 : V_TILE;
        P.tiles_m = p.mt;
        P.tiles_n = ceil_div(h.d, P.nt);
        P.M = N;
        P.N = h.d;
        P.sub = p.sub;
        P.v0 = v0;
        P.V = h.V;
        P.stride_c = (int)ld_dx;
        P.slots = r.at<float4>(p.slots);
        P.sum = p.pieces > 1 ? r.at<float>(p.dx) : nullptr;
        P.out = dx;
        P.out_bf16 = !f32;
        P.first = s0 == 0;
        P.last = s0 + subs >= p.n_sub;
        P.vec = !misaligned(dx, 16) && ld_dx % (f32 ? 4 : 8) == 0 && h.d % 4 == 0;
        P.status = status;
        if ((rc = launch_product<V_DX>(r, P)) != DP_OK) return rc;
      }
      const int add = accumulate_into || s0 > 0;
      if (sqnorm && p.short_examples) {
        NParams Q = {};
        const long long rows = (long long)N * p.R;
        if (!encode_rows(&Q.x, r.at<__nv_bfloat16>(p.xe), rows, p.dp, p.dp) || !encode_blocks(&Q.g, G, rows, p.sub, p.sub, subs, block))
          return DP_ERR_CUDA;
        Q.rows = p.R * h.T;
        Q.examples = p.short_examples;
        Q.B = h.B;
        Q.groups = ceil_div(h.B, Q.examples);
        Q.subs = subs;
        Q.sub = p.sub;
        Q.dp = p.dp;
        Q.splits = norm_splits(Q.groups, subs, p.sub, p.dp);
        Q.bias = h.bias && p.R == 2;
        Q.partial = r.at<float>(p.gram);
        Q.status = status;
        const long long items = (long long)Q.groups * Q.splits;
        if (items > 0x7fffffffll) return DP_ERR_UNSUPPORTED;
        VOCAB_CUDA(launch_chained(k_vocab_norms, (unsigned)std::min<long long>(items, sm_count()), N_THREADS, N_SMEM, r.s, Q));
        VOCAB_CUDA(launch_chained(k_vocab_norm_sum, (unsigned)ceil_div(h.B, 8), 256, 0, r.s, Q.partial, h.B, Q.splits, sqnorm, add));
      } else if (sqnorm) {
        std::vector<dp_layer> layers(subs);
        std::vector<int> idx(subs), way(subs, p.gram_way ? 1 : 0);
        std::vector<ColTaskHost> cols;
        for (int k = 0; k < subs; ++k) {
          layers[k] = piece_layer(h, p, r.at<__nv_bfloat16>(p.xe), G + (size_t)k * block);
          idx[k] = k;
        }
        float* partial = r.at<float>(p.gram);
        const int count = (int)umma_sqnorm_partials_per_example(layers.data(), idx.data(), subs, way.data());
        if ((rc = launch_umma_sqnorms(layers.data(), idx.data(), subs, way.data(), partial, count, 0, status, r.s, true)) != DP_OK) return rc;
        VOCAB_CUDA(launch_chained(k_vocab_norm_sum, (unsigned)ceil_div(h.B, 8), 256, 0, r.s, partial, h.B, count, sqnorm, add));
        if (!p.gram_way && h.bias && p.R == 2) {
          for (int k = 0; k < subs; ++k) cols.push_back({&layers[k], false, r.at<float>(p.cols) + (size_t)k * h.B * p.sub});
          if (launch_colsums_batched(cols.data(), (int)cols.size(), r.s) != cudaSuccess ||
              launch_rows_sqsum_batched(cols.data(), (int)cols.size(), sqnorm, r.s) != cudaSuccess) return DP_ERR_CUDA;
        }
      }
      return rc;
    });
  } catch (const std::bad_alloc&) {
    return DP_ERR_UNSUPPORTED;
  }
}

int dp_vocab_loss_clipped_accumulate(const dp_vocab_head* head, const float* lse, const float* clip, float* acc_w, float* acc_b,
                                     void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_head(head);
  if (rc != DP_OK) return rc;
  const dp_vocab_head& h = *head;
  if (!lse || !clip || !acc_w || (h.bias && !acc_b)) return DP_ERR_ARG;
  if (misaligned(lse, 4) || misaligned(clip, 4) || misaligned(acc_w, 4) || misaligned(acc_b, 4)) return DP_ERR_ALIGN;
  VPlan p;
  if ((rc = check_call(head, 2, workspace, workspace_bytes, &p)) != DP_OK) return rc;
  int* status = status_ptr();
  if (!status || !vocab_kernels_ready()) return DP_ERR_CUDA;
  const VRun r = {h, p, static_cast<char*>(workspace), static_cast<cudaStream_t>(cuda_stream), status};
  const int N = h.B * h.T;
  __nv_bfloat16* G = r.at<__nv_bfloat16>(p.G);
  float* bias_part = h.bias ? r.at<float>(p.bias) : nullptr;
  return over_pieces(r, lse, clip, bias_part, [&](int s0, int subs, long long block) -> int {
    int rc = DP_OK;
    VParams P = {};
    const int v0 = s0 * p.sub, cols = std::min(subs * p.sub, h.V - v0);
    const long long rows = (long long)N * p.R;
    if (!encode_blocks(&P.a[0], G, rows, p.sub, p.sub, subs, block) ||
        !encode_rows(&P.b[0], r.at<__nv_bfloat16>(p.xe), rows, p.dp, p.dp)) return DP_ERR_CUDA;
    P.n_pairs = 1;
    P.kb = (int)((rows + 127) / 128);
    P.seg = 16;
    P.nt = h.d <= 128 ? 128 : V_TILE;
    P.tiles_m = ceil_div(cols, V_TILE);
    P.tiles_n = ceil_div(h.d, P.nt);
    P.M = subs * p.sub;
    P.N = h.d;
    P.sub = p.sub;
    P.v0 = v0;
    P.V = h.V;
    P.stride_c = h.d;
    P.slots = r.at<float4>(p.slots);
    P.sum = acc_w;
    P.vec = !misaligned(acc_w, 16) && h.d % 4 == 0;
    P.status = status;
    if ((rc = launch_product<V_DW>(r, P)) != DP_OK) return rc;
    if (bias_part)
      VOCAB_CUDA(launch_chained(k_vocab_bias, (unsigned)ceil_div(cols, 32), 256, 0, r.s, bias_part, p.mt * 8, subs * p.sub, cols, acc_b + v0));
    return rc;
  });
}

int dp_vocab_loss_cross_sqnorms(const dp_vocab_head* head, const float* lse, const int32_t* ids, const void* G_emb, int64_t ld_emb,
                                int Tu, float* sqnorm, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const int rc = check_head(head);
  if (rc != DP_OK) return rc;
  if (!lse || !ids || !G_emb || !sqnorm || Tu <= 0 || ld_emb < head->d) return DP_ERR_ARG;
  if (Tu > (1 << 26) || ld_emb > (1ll << 36)) return DP_ERR_UNSUPPORTED;
  if (misaligned(lse, 4) || misaligned(ids, 4) || misaligned(sqnorm, 4) || misaligned(G_emb, head->dtype == DP_F32 ? 4 : 2))
    return DP_ERR_ALIGN;
  if (!workspace || misaligned(workspace, 256) || workspace_bytes < (size_t)head->B * kCrossChunks * sizeof(float))
    return DP_ERR_WORKSPACE;
  int* status = status_ptr();
  if (!status) return DP_ERR_CUDA;
  return launch_vocab_cross(*head, lse, ids, G_emb, ld_emb, Tu, sqnorm, static_cast<float*>(workspace), status,
                            static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
