// A learned relative position bias by buckets: table[num_buckets][n_heads], score bias
//   bias[h][q][k] = table[bucket(k - q - offset)][h]
// and every example's gradient of the table from the gradient G[b][h][q][k] of the scores,
//   rows[b][n][h] = sum over (q, k) with bucket(k - q - offset) = n of G[b][h][q][k].
//
// The bucket depends on k - q alone, so both are Toeplitz: the bias is one line of Tq + Tk - 1 values per head that
// every query reads at another place, and the gradient is a sum along diagonals first, over buckets last.  Both kernels
// are bound by memory: the bias by writing [H][Tq][Tk] (16 x 4096 x 4096 in bf16: 75 us, 7.2 TB/s), the gradient by reading
// G once (256 x 16 x 128 x 128 in bf16: 29 us, 4.6 TB/s; 64 x 16 x 512 x 512 padded at random: 45 us, 4.8 TB/s of what
// counts; a block has no loads in flight while it adds its strands and sums its diagonals).
#include <cstring>
#include <type_traits>

#include "dp_chain.cuh"
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

// 16 bytes of neighbouring values of a row.
template <typename T>
struct Strip {
  static constexpr int V = 16 / sizeof(T);
  uint32_t w[4];
  __device__ __forceinline__ void load(const T* p) {
    const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p));
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
  }
  __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0u; }
  // All bits of the first n values: what the mask takes away may be NaN.
  __device__ __forceinline__ void first(int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = n > i ? ~0u : 0u;
      else w[i] = n >= 2 * i + 2 ? ~0u : n == 2 * i + 1 ? 0xffffu : 0u;
    }
  }
  __device__ __forceinline__ void keep(const Strip& mask) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] &= mask.w[i];
  }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
    else return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
  }
};

// The same where rows start anywhere: the two 16-byte words of memory that the values lie in.
template <typename T>
struct Wide {
  uint32_t w[8];
  static __device__ __forceinline__ const uint4* words(const T* p) {
    return reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
  }
  // Both words lie inside the scores, [lo, hi).  Only the first and last few values of the whole array ever fail this.
  static __device__ __forceinline__ bool inside(const T* p, const T* lo, const T* hi) {
    return reinterpret_cast<const T*>(words(p)) >= lo && reinterpret_cast<const T*>(words(p) + 2) <= hi;
  }
  __device__ __forceinline__ void load(const T* p) {
    const uint4 u = __ldcs(words(p)), v = __ldcs(words(p) + 1);
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    w[4] = v.x; w[5] = v.y; w[6] = v.z; w[7] = v.w;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 0u;
  }
  __device__ __noinline__ static void gather(const T* p, const T* lo, const T* hi, uint32_t* out) {
    const T* q = reinterpret_cast<const T*>(words(p));
    for (int i = 0; i < 8; ++i) {
      uint32_t u = 0u;
      if constexpr (sizeof(T) == 4) {
        if (q + i >= lo && q + i < hi) u = *reinterpret_cast<const uint32_t*>(q + i);
      } else {
        for (int k = 0; k < 2; ++k)
          if (q + 2 * i + k >= lo && q + 2 * i + k < hi)
            u |= (uint32_t)*reinterpret_cast<const unsigned short*>(q + 2 * i + k) << (16 * k);
      }
      out[i] = u;
    }
  }
  // The strip that starts `s` values behind the first word's first.
  __device__ __forceinline__ Strip<T> at(int s) const {
    Strip<T> x;
    if constexpr (sizeof(T) == 4) {
      uint32_t t[5];
#pragma unroll
      for (int i = 0; i < 5; ++i) t[i] = s & 2 ? w[i + 2] : w[i];
#pragma unroll
      for (int i = 0; i < 4; ++i) x.w[i] = s & 1 ? t[i + 1] : t[i];
    } else {
      uint32_t t[6], u[5];
#pragma unroll
      for (int i = 0; i < 6; ++i) t[i] = s & 4 ? w[i + 2] : w[i];
#pragma unroll
      for (int i = 0; i < 5; ++i) u[i] = s & 2 ? t[i + 1] : t[i];
      const uint32_t pick = s & 1 ? 0x5432u : 0x3210u;
#pragma unroll
      for (int i = 0; i < 4; ++i) x.w[i] = __byte_perm(u[i], u[i + 1], pick);
    }
    return x;
  }
};

// ---------------------------------------------------------------------------------------------
// Forward.  A block of 8 warps writes a tile of columns x rows of one head; the line of bias values that the tile
// needs is looked up once into shared memory (in the output's type).  VEC: a lane owns 16 bytes of neighbouring columns
// and walks down the rows: from one row to the next its window of the line moves by one value, so it shifts its
// registers and reads a single new value.  Otherwise rows start anywhere: of each, the aligned 16-byte words are written
// whole, out of copies of the line that begin at every place of a word, and the few values before and behind them one by
// one (16 x 2047 x 2047: bf16 34 us value by value, 27 so; 2048 x 2048 23; fp32 51, 47 and 43).
// ---------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ T to_type(float x);
template <> __device__ __forceinline__ float to_type<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 to_type<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

constexpr int kBiasCols = 256, kBiasRowsPerWarp = 16;

template <typename T, typename TT, bool VEC>
__global__ void __launch_bounds__(256)
k_relpos_bias(const TT* table, const __grid_constant__ Buckets bk, int n_heads, int Tq, int Tk, int offset,
              T* out, long long stride_h, long long stride_q, int warps_x) {
  constexpr int V = 16 / sizeof(T);
  extern __shared__ __align__(16) unsigned char bias_smem[];
  wait_for_predecessor();
  let_successor_in();
  T* line = reinterpret_cast<T*>(bias_smem);
  const int warps_y = 8 / warps_x;
  const int cols = kBiasCols * warps_x, rows = kBiasRowsPerWarp * warps_y;
  const int c0 = blockIdx.x * cols, q0 = blockIdx.y * rows, h = blockIdx.z;
  const int n_line = cols + rows - 1 + (VEC ? 0 : V);      // words may end behind the tile's columns
  const int pitch = (n_line + V - 1) / V * V;
  // line[i]: relative position (c0 - q0 - offset) + i - (rows - 1)
  const int rel0 = c0 - q0 - offset - (rows - 1);
  T* o = out + (long long)h * stride_h + (long long)q0 * stride_q + c0;
  // Otherwise V copies of the line, copy s without its first s values, so that a row's words are words of one of them; which
  // ones occur repeats every V rows.
  const int off0 = (int)((reinterpret_cast<uintptr_t>(o) & 15) / sizeof(T));
  auto offset_of = [&](int r) { return (off0 + r * (int)(stride_q & (V - 1))) & (V - 1); };  // of a row's first column in its word
  unsigned need = 1u;
  if (!VEC)
    for (int r = 0; r < min(V, Tq - q0); ++r) need |= 1u << ((rows - 1 - r - offset_of(r)) & (V - 1));
  for (int i = threadIdx.x; i < n_line; i += 256) {
    const T x = to_type<T>(to_float(table[(long long)bk.of(rel0 + i) * n_heads + h]));
    line[i] = x;
    if (!VEC) {
#pragma unroll
      for (int s = 1; s < V; ++s)
        if ((need >> s & 1u) && i >= s) line[s * pitch + i - s] = x;
    }
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int wx = warp % warps_x, wy = warp / warps_x;
  const int r0 = wy * kBiasRowsPerWarp;
  const int r1 = min(r0 + kBiasRowsPerWarp, Tq - q0);
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
    const int seg = c0 + wx * kBiasCols, left = Tk - seg;            // the warp's first column, columns from there on
    if (left <= 0) return;
#pragma unroll 4
    for (int r = r0; r < r1; ++r) {
      T* row = o + (long long)r * stride_q + wx * kBiasCols;
      const int off = offset_of(r), head = off ? V - off : 0;          // columns before the first aligned word
      const int from = wx * kBiasCols - r + rows - 1, place = from + head, s = place & (V - 1);
      // the words that begin in the warp's columns, the last of which may end behind them; what a row has before its first
      // word and behind its last is written value by value
      const int most = (kBiasCols - head + V - 1) / V, have = left > head ? (left - head) / V : 0, words = min(most, have);
      const uint4* q = reinterpret_cast<const uint4*>(line + s * pitch + place - s);
#pragma unroll
      for (int k = lane; k < kBiasCols / V; k += 32)
        if (k < words) *reinterpret_cast<uint4*>(row + head + k * V) = q[k];
      const int before = seg == 0 ? min(head, left) : 0, behind = have < most ? max(left - head - have * V, 0) : 0;
      if (lane < before) row[lane] = line[from + lane];
      if (lane < behind) row[head + have * V + lane] = line[place + have * V + lane];
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Per-example gradient.  A block takes a tile of one (example, head), LG * V neighbouring columns wide; its groups of LG lanes
// (a warp or a part of one) take strands of RG rows below one another, V columns a lane.  Walking down the rows, a diagonal
// moves one column to the right per row: inside a lane that is another register of its V sums (renamed by unrolling the
// rows), at the lane's right edge the sum is handed to the next lane, and the one that leaves the last lane is complete and
// goes to the strand's line in shared memory.  That costs one add per element and one shuffle per V of them, with no atomic.
// Then the warps add the strands' lines into one line of the tile's diagonals and sum that by buckets, each sum in a fixed
// order.  A tile behind an example's lengths (or above the diagonal) only writes its zeros.
// ---------------------------------------------------------------------------------------------
// (a, b) + (x, y), two fp32 additions in one instruction.
__device__ __forceinline__ void add2(float& a, float& b, float x, float y) {
  asm("{.reg .b64 s, t, u;\n\tmov.b64 s, {%0, %1};\n\tmov.b64 t, {%2, %3};\n\tadd.rn.f32x2 u, s, t;\n\tmov.b64 {%0, %1}, u;}"
      : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}

// Measured (256 x 16 scores of 128 x 128; 64 x 16 of 512 x 512 padded at random; bf16, whole chain of calls):
//   (before the last steps)  rows per strand at most  16: 41 / 69 us, 32: 37 / 57, 64: 37 / 58
//                            threads at most  64: 37 / 65 us, 128: 37 / 57, 256: 37 / 58
//   blocks per SM  7: 38 / 56 us, 8: 37 / 53, 9: 37 / 53, 10: 47 / 91 (48 registers: up to 570 bytes of spills; at
//   64 they are 12 to 40)
constexpr int kGradThreads = 128, kGradMaxRows = 5;   // threads per block at most; log2 of the rows per strand at most
constexpr int kGradBlocks = 8;
constexpr int kGradRowBlock = 8;                 // rows whose loads are issued together

struct GradArgs {
  long long stride_b, stride_h, stride_q, extent;          // extent: from the first score to behind the last, in elements
  int B, H, Tq, Tk, offset, causal;
  int rg_log, n_ct, tiles;                       // log2 of the rows per strand; tiles of a head, side by side and all
  int accumulate;
};

// SHIFT: the rows do not all start and end on 16-byte boundaries.
template <typename T, int LGL, bool SHIFT>
__global__ void __launch_bounds__(kGradThreads, kGradBlocks)
k_relpos_grad(const T* G, const __grid_constant__ Buckets bk, const __grid_constant__ GradArgs a,
              const int32_t* q_len, const int32_t* k_len, float* partial,
              float* rows) {
  extern __shared__ float grad_smem[];
  wait_for_predecessor();
  let_successor_in();
  constexpr int V = Strip<T>::V, LG = 1 << LGL, CW = LG * V;
  const int RG = 1 << a.rg_log, LINE = RG + CW;  // a strand's line: diagonals -RG .. CW - 1
  const int lane = threadIdx.x & 31, li = lane & (LG - 1);
  const int gyi = threadIdx.x >> LGL, gy = blockDim.x >> LGL;
  float* buf = grad_smem + gyi * LINE;
  float* line = grad_smem + gy * LINE;           // the tile's: diagonals -(nr - 1) .. nc - 1
  const unsigned unit = blockIdx.x, bh = unit / (unsigned)a.tiles, u_in = unit - bh * (unsigned)a.tiles;
  const int rt = (int)(u_in / (unsigned)a.n_ct), ct = (int)u_in - rt * a.n_ct;
  const int b = (int)(bh / (unsigned)a.H), h = (int)bh - b * a.H;
  const int q_end = q_len ? min(max(q_len[b], 0), a.Tq) : a.Tq;
  const int k_end = k_len ? min(max(k_len[b], 0), a.Tk) : a.Tk;
  const int nb = bk.both ? 2 * bk.half : bk.half;
  const int R0 = rt * RG * gy, C0 = ct * CW;     // the tile's first row and column
  const int nr = min(RG * gy, q_end - R0), nc = min(CW, k_end - C0);           // what counts of it
  if (nr <= 0 || nc <= 0 || (a.causal && C0 > R0 + nr - 1 + a.offset)) {
    for (int k = threadIdx.x; k < nb; k += blockDim.x) {
      if (partial) partial[(long long)unit * nb + k] = 0.0f;
      else if (!a.accumulate) rows[((long long)b * nb + k) * a.H + h] = 0.0f;
    }
    return;
  }
  // the buckets' first and last diagonals, as places in the tile's line
  const int rel = C0 - R0 - a.offset - (nr - 1);           // relative position of line[0]
  const int n_line = nr + nc - 1;
  const int n_seen = a.causal ? min(n_line, 1 - rel) : n_line;      // causal: up to relative position 0
  int2* ends = reinterpret_cast<int2*>(line + ((RG * gy + CW + 31) & ~31));
  for (int k = threadIdx.x; k < nb; k += blockDim.x) {
    int lo, hi;
    bk.range(k, lo, hi);
    ends[k] = make_int2(max(lo - rel, 0), min(hi - rel, n_seen - 1));
  }
  const int q0 = R0 + gyi * RG, c = C0 + li * V;
  const int n = min(max(q_end - q0, 0), RG);     // rows of this strand
  const int valid = min(max(k_end - c, 0), V);   // columns of this lane
  // rows that this lane reads: [from, n); a causal lane starts where its first column is seen.  A lane behind the last key
  // reads what the last lane before it reads, and masks it.
  const int from = a.causal ? max(c - a.offset - q0, 0) : 0;
  const T* p = G + (long long)b * a.stride_b + (long long)h * a.stride_h + (long long)q0 * a.stride_q + min(c, (k_end - 1) / V * V);

  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.0f;
  // the strands of a warp walk together: blocks of rows [skip, rounds)
  const int rounds = (int)__reduce_max_sync(0xffffffffu, (unsigned)((n + kGradRowBlock - 1) / kGradRowBlock));
  const int skip = min(rounds, (int)__reduce_min_sync(0xffffffffu, (unsigned)from / kGradRowBlock));
  p += (long long)(skip * kGradRowBlock) * a.stride_q;
  const unsigned span = (unsigned)max(n - from, 0);
  const bool whole = __all_sync(0xffffffffu, valid == V);  // no lane of the warp reaches beyond the last key
  Strip<T> mask;
  mask.first(valid);
  // kAhead rows are in flight: a later row is fetched into a row's registers as soon as that is added up.  Where all the
  // warp's rows to be fetched count (and, shifted, lie well inside the scores), that takes no conditions.
  constexpr int kAhead = SHIFT ? kGradRowBlock / 2 : kGradRowBlock;
  std::conditional_t<SHIFT, Wide<T>, Strip<T>> x[kAhead];
  const T *lo_end = G, *hi_end = G + a.extent;
  int shift = SHIFT ? (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T)) : 0;       // of the row that is added next
  const int shift_step = (int)(a.stride_q & (V - 1));
  auto fetch = [&](const int r, bool counts) {
    x[r % kAhead].clear();
    if constexpr (SHIFT) {
      if (counts && Wide<T>::inside(p, lo_end, hi_end)) {
        x[r % kAhead].load(p);
      } else if (counts) {
        uint32_t t[8];
        Wide<T>::gather(p, lo_end, hi_end, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[r % kAhead].w[i] = t[i];
      }
    } else {
      if (counts) x[r % kAhead].load(p);
    }
    p += a.stride_q;
  };
  int row = skip * kGradRowBlock - from;         // the next row to be fetched, from the first that this lane reads
#pragma unroll
  for (int r = 0; r < kAhead; ++r) fetch(r, (unsigned)(row + r) < span);
  row += kAhead;
  float* edge = buf + (CW - 1 - skip * kGradRowBlock + RG);
  auto add_row = [&](const int r, bool masked) {
    Strip<T> y;
    if constexpr (SHIFT) {
      y = x[r % kAhead].at(shift);
      shift = (shift + shift_step) & (V - 1);
    } else {
      y = x[r % kAhead];
    }
    if (masked) y.keep(mask);
    // register i has, in row r, the diagonal of column (i + r) mod V
#pragma unroll
    for (int i = 0; i < V; i += 2) add2(acc[i], acc[i + 1], y.get((i + r) % V), y.get((i + 1 + r) % V));
  };
  auto hand_on = [&](const int r) {
    const int s = (V - 1 + kGradRowBlock * V - r) % V;
    const float out = acc[s];
    const float in = __shfl_up_sync(0xffffffffu, out, 1, LG);
    if (li == LG - 1) edge[-r] = out;
    acc[s] = li == 0 ? 0.0f : in;
  };
  for (int t = skip; t < rounds; ++t) {
    bool mine = row >= 0 && row + kGradRowBlock <= (int)span;
    if (SHIFT) mine = mine && Wide<T>::inside(p, lo_end, hi_end) && Wide<T>::inside(p + (kGradRowBlock - 1) * a.stride_q, lo_end, hi_end);
    const bool full = __all_sync(0xffffffffu, mine);
    if (full && whole) {
#pragma unroll
      for (int r = 0; r < kGradRowBlock; ++r) {
        add_row(r, false);
        x[r % kAhead].load(p);
        p += a.stride_q;
        hand_on(r);
      }
    } else if (full) {
#pragma unroll
      for (int r = 0; r < kGradRowBlock; ++r) {
        add_row(r, true);
        x[r % kAhead].load(p);
        p += a.stride_q;
        hand_on(r);
      }
    } else {
#pragma unroll
      for (int r = 0; r < kGradRowBlock; ++r) {
        add_row(r, true);
        fetch(r, (unsigned)(row + r) < span);
        hand_on(r);
      }
    }
    row += kGradRowBlock;
    edge -= kGradRowBlock;
  }
  // buf[d + RG]: diagonal d = column - row, both from the strand's first; those in [-walked, CW - skipped) are there, the
  // others of the line are 0.  (kGradRowBlock is a multiple of V.)
  const int walked = rounds * kGradRowBlock, skipped = skip * kGradRowBlock;
#pragma unroll
  for (int j = 0; j < V; ++j) buf[li * V + j - walked + RG] = acc[j];
  for (int i = li; i < RG - walked; i += LG) buf[i] = 0.0f;
  for (int i = LINE - skipped + li; i < LINE; i += LG) buf[i] = 0.0f;
  __syncthreads();
  // The tile's line, 32 diagonals per warp at a time: the strands' lines added up, then inside the 32 every diagonal is
  // summed with those before it that share its bucket, so that the last one of a bucket there holds their sum.
  const int my_lo = lane < nb ? ends[lane].x : 0x7fffffff, my_hi = lane < nb ? ends[lane].y : -1;
  for (int i0 = threadIdx.x & ~31; i0 < n_seen; i0 += blockDim.x) {
    const int i = i0 + lane, d = i - (nr - 1);
    // strand y has it as diagonal d + y RG, if that lies in [-RG, CW)
    const int y0 = d < -RG ? (-d - 1) >> a.rg_log : 0, y1 = min(gy, d < CW ? ((CW - 1 - d) >> a.rg_log) + 1 : 0);
    float s = 0.0f;
    for (int y = y0; y < y1; ++y) s += grad_smem[y * (LINE + RG) + d + RG];
    // where buckets begin among the 32
    unsigned begins = __reduce_or_sync(0xffffffffu, my_lo <= my_hi && my_lo >= i0 && my_lo < i0 + 32 ? 1u << (my_lo - i0) : 0u);
    for (int k = 32; k < nb; k += 32) {
      const int2 e = k + lane < nb ? ends[k + lane] : make_int2(0, -1);
      begins |= __reduce_or_sync(0xffffffffu, e.x <= e.y && e.x >= i0 && e.x < i0 + 32 ? 1u << (e.x - i0) : 0u);
    }
    const int head = 31 - __clz((int)(begins << (31 - lane) >> (31 - lane) | 1u));       // lane of this bucket's first here
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float other = __shfl_up_sync(0xffffffffu, s, o);
      if (lane - o >= head) s += other;
    }
    line[i] = s;                                 // the line has room for whole warps
  }
  __syncthreads();
  for (int k = threadIdx.x; k < nb; k += blockDim.x) {
    const int lo = ends[k].x, hi = ends[k].y;
    float s = 0.0f;
    for (int i = lo; i <= hi; i = (i | 31) + 1) s += line[min(i | 31, hi)];
    if (partial) {
      partial[(long long)unit * nb + k] = s;
    } else {
      float* w = rows + ((long long)b * nb + k) * a.H + h;
      *w = a.accumulate ? *w + s : s;
    }
  }
}

// rows[b][n][h] (+)= sum over the tiles of (b, h).  A block owns one (b, h); its threads stand as strands x buckets, a strand
// takes every (number of strands)-th tile and the strands are added in order.
__global__ void __launch_bounds__(1024)
k_relpos_units(const float* partial, int H, int nb, int units, float* rows, int add) {
  __shared__ float part[1024];
  wait_for_predecessor();
  let_successor_in();
  const int strands = blockDim.x / nb, n = threadIdx.x % nb, strand = threadIdx.x / nb;
  const long long bh = blockIdx.x, b = bh / H, h = bh - b * H;
  const float* p = partial + bh * units * nb + n;
  float s = 0.0f;
  if (strand < strands) {
#pragma unroll 8
    for (int u = strand; u < units; u += strands) s += p[(long long)u * nb];
  }
  part[threadIdx.x] = s;
  __syncthreads();
  if (strand == 0) {
    for (int k = 1; k < strands; ++k) s += part[k * nb + n];
    float* w = rows + (b * nb + n) * H + h;
    *w = add ? *w + s : s;
  }
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
  const bool vec = !misaligned(out, 16) && p.Tk % V == 0 && sh % V == 0 && sq % V == 0;
  const size_t smem = (vec ? cols + rows : (size_t)V * (cols + rows + 2 * V)) * sizeof(T);
  note_launch(1);
  return launch_chained(vec ? k_relpos_bias<T, TT, true> : k_relpos_bias<T, TT, false>, grid, 256, smem, s,
                        static_cast<const TT*>(table), bk, p.n_heads, p.Tq, p.Tk, (int)p.offset, static_cast<T*>(out), sh, sq, wx);
}

// How G is cut: V columns a lane, 2^lg lanes a strand, RG rows a strand, strands below one another in `threads` threads.
struct GradPlan { int lg, rg_log, threads, n_ct, n_rt; long long units; size_t smem; };
static GradPlan plan_grad(int B, const dp_relpos& p, int V) {
  GradPlan g;
  const int lanes = ceil_div(p.Tk, V);
  g.lg = 3;
  while (g.lg < 5 && (1 << g.lg) < lanes) ++g.lg;
  const int CW = V << g.lg;
  g.n_ct = ceil_div(p.Tk, CW);
  // Long strands amortise a tile's sums over diagonals and buckets, few of them leave warps without work: halved while the
  // GPU's warp slots would not be filled, or while a warp's strands reach far beyond the rows.
  g.rg_log = kGradMaxRows;
  while ((1 << g.rg_log) > kGradRowBlock &&
         ((((long long)B * p.n_heads * g.n_ct * ceil_div(p.Tq, 1 << g.rg_log)) << g.lg) < 148ll * 32 * 32 ||
          (1 << g.rg_log) * (32 >> g.lg) >= 2 * p.Tq))
    --g.rg_log;
  const int RG = 1 << g.rg_log;
  // then as many strands as there are rows, in at most 4 warps
  g.threads = 32;
  while (g.threads < kGradThreads && (g.threads >> g.lg) * RG < p.Tq) g.threads <<= 1;
  const int gy = g.threads >> g.lg;
  g.n_rt = ceil_div(p.Tq, gy * RG);
  g.units = (long long)B * p.n_heads * g.n_ct * g.n_rt;
  g.smem = ((size_t)gy * (RG + CW) + align_up((size_t)gy * RG + CW, 32)) * sizeof(float) + (size_t)p.num_buckets * sizeof(int2);
  return g;
}

template <typename T, int LGL>
static cudaError_t launch_grad_form(bool shift, const T* G, const Buckets& bk, const GradArgs& a, const GradPlan& g,
                             const int32_t* q_len, const int32_t* k_len, float* partial, float* rows, cudaStream_t s) {
  const unsigned n = (unsigned)g.units;
  note_launch(1);
  return launch_chained(shift ? k_relpos_grad<T, LGL, true> : k_relpos_grad<T, LGL, false>, n, g.threads, g.smem, s, G, bk, a,
                        q_len, k_len, partial, rows);
}

template <typename T>
static cudaError_t launch_grad(const void* G, const Buckets& bk, const GradArgs& a, const GradPlan& g, const int32_t* q_len,
                               const int32_t* k_len, float* partial, float* rows, cudaStream_t s) {
  const T* p = static_cast<const T*>(G);
  constexpr int V = Strip<T>::V;
  const bool shift = misaligned(G, 16) || a.Tk % V || a.stride_b % V || a.stride_h % V || a.stride_q % V;
  if (g.lg == 3) return launch_grad_form<T, 3>(shift, p, bk, a, g, q_len, k_len, partial, rows, s);
  if (g.lg == 4) return launch_grad_form<T, 4>(shift, p, bk, a, g, q_len, k_len, partial, rows, s);
  return launch_grad_form<T, 5>(shift, p, bk, a, g, q_len, k_len, partial, rows, s);
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
  const long long extent[2] = {p->n_heads, p->Tq}, stride[2] = {stride_h, stride_q};
  if (!lies_apart(p->Tk, 2, extent, stride)) return DP_ERR_ARG;
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
  long long most = 0;                            // bf16 and fp32 are cut differently
  for (int V : {8, 4}) {
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
  if (B == 1) stride_b = 0;                      // the stride of an extent of one, which nothing depends on
  if (p->n_heads == 1) stride_h = 0;
  if (p->Tq == 1) stride_q = 0;
  const GradPlan g = plan_grad(B, *p, dtype == DP_F32 ? 4 : 8);
  const int nb = p->num_buckets, per_bh = g.n_ct * g.n_rt;
  if (g.units > 0x7fffffffll) return DP_ERR_UNSUPPORTED;
  float* partial = nullptr;
  if (per_bh > 1) {
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < (size_t)g.units * nb * sizeof(float))
      return DP_ERR_WORKSPACE;
    partial = static_cast<float*>(workspace);
  }
  const GradArgs a = {stride_b, stride_h, stride_q, (B - 1) * stride_b + (p->n_heads - 1) * stride_h + (p->Tq - 1) * stride_q + p->Tk,
                      B, p->n_heads, p->Tq, p->Tk, (int)p->offset, causal ? 1 : 0,
                      g.rg_log, g.n_ct, g.n_ct * g.n_rt, accumulate_into ? 1 : 0};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (dtype == DP_F32) e = launch_grad<float>(G, bk, a, g, q_len, k_len, partial, rows, s);
  else e = launch_grad<__nv_bfloat16>(G, bk, a, g, q_len, k_len, partial, rows, s);
  if (e != cudaSuccess) return DP_ERR_CUDA;
  if (partial) {
    // enough strands that each has a handful of tiles, whose loads are all in flight.  The call in bf16 with one strand, this many,
    // as many as fit: 64 x 16 x 512 x 512 (16 tiles a head) 83.9, 83.9, 86.2 us; 4 x 16 x 1024 x 1024 (64) 29.4, 27.6, 27.9;
    // 1 x 16 x 2048 x 2048 (256) 32.7, 26.6, 27.5; 1 x 1 x 4096 x 4096 (2048) 94, 17.4, 17.4
    const int strands = per_bh <= 8 ? 1 : 1024 / nb < (per_bh + 7) / 8 ? 1024 / nb : (per_bh + 7) / 8;
    const int threads = (strands * nb + 31) / 32 * 32;
    e = launch_chained(k_relpos_units, B * p->n_heads, threads, 0, s, partial, p->n_heads, nb, per_bh, rows, a.accumulate);
    note_launch(1);
    if (e != cudaSuccess) return DP_ERR_CUDA;
  }
  return DP_OK;
}

}  // extern "C"
