// What the attention kernels share: rows of heads, the keys that a query sees, tiles in LDS, and the
// matrix instructions' operands.
//
// All products run on 32 x 32 tiles (32x32x16 instructions for 16-bit elements, 32x32x2 for fp32, four
// of them taken together). A lane (l, h) = (lane % 32, lane / 32) holds
//   a row operand       row l of a tile, elements of piece 2 step + h (16 bytes),
//   an accumulator      column l, rows 8 g + 4 h + i in element 4 g + i (g, i = 0 .. 3),
// and as the sum over a product's inner index may run in any order, an accumulator rounded to the
// element type is a column operand of the next product as it is: its elements 0 .. E - 1 are inner
// indices 8 g + 4 h + i, and the row operand of that product is read from the tile at the same ones
// (col_frag). So scores become weights and weights a factor without leaving their lanes.
#pragma once
#include "rows.h"

namespace eogp {

// Element (n, t, h, c) of a tensor of heads lies at p[n ld_n + t ld_t + h ld_h + c].
template <typename T>
struct Heads {
  T* p;
  int64_t ld_n, ld_t, ld_h;
  __device__ __forceinline__ T* row(int64_t n, int64_t t, int64_t h) const { return p + n * ld_n + t * ld_t + h * ld_h; }
};

template <typename T>
inline Heads<T> heads_of(const eogp_heads& x) {
  return Heads<T>{static_cast<T*>(x.data), x.ld_example, x.ld_token, x.ld_head};
}

// Which keys a query sees.
struct Sight {
  int causal;
  int window;                     // 0: no window
  int sinks;
  int Tq, Tk;
  const int64_t* q_start;         // position of an example's first query, or NULL: Tk - Tq
  const uint8_t *q_mask, *k_mask;

  __device__ __forceinline__ int64_t start(int64_t n) const { return q_start ? q_start[n] : (int64_t)Tk - Tq; }
};

// Keys [lo, hi) and [0, sk) of a query at position p.
struct Span {
  int lo, hi, sk;
};

__device__ __forceinline__ int clamp_key(int64_t j, int most) { return (int)(j < 0 ? 0 : j > most ? most : j); }

__device__ __forceinline__ Span span_of(const Sight& s, int64_t p) {
  // far positions see what positions 2^40 see: no sum below leaves 64 bits
  constexpr int64_t kFar = (int64_t)1 << 40;
  p = p < -kFar ? -kFar : p > kFar ? kFar : p;
  Span v;
  v.hi = clamp_key(s.causal ? p + 1 : s.window ? p + s.window : s.Tk, s.Tk);
  v.lo = s.window ? clamp_key(p - s.window + 1, v.hi) : 0;
  v.sk = clamp_key(s.causal ? p + 1 : s.Tk, s.sinks < s.Tk ? s.sinks : s.Tk);
  return v;
}

// (Without branches: what is tested is selected among values in matrix registers.)
__device__ __forceinline__ bool sees(const Span& v, int j) { return ((j >= v.lo) & (j < v.hi)) | (j < v.sk); }

// Division of numbers below 2^31 by one divisor.
struct Divide {
  uint32_t by = 1, mul = 0;
  int shift = 0;
  Divide() = default;
  explicit Divide(int64_t d) : by((uint32_t)d) {
    int s = 0;
    while (((int64_t)1 << s) < d) ++s;
    shift = 31 + s;
    mul = (uint32_t)((((uint64_t)1 << shift) / (uint64_t)d) + 1);   // at most 2^31 + 1, as 2^s < 2 d
  }
  __device__ __forceinline__ int quotient(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
  __device__ __forceinline__ int rest(int n, int q) const { return n - q * (int)by; }
};

// The three numbers of every row of a set of rows, as bounds: where any row sees keys, and where all do.
struct Bounds {
  int lo_min, hi_max, sk_max;     // outside [lo_min, hi_max) and [0, sk_max) no row sees a key
  int lo_max, hi_min;             // in [lo_max, hi_min) every row sees every key
};

__device__ __forceinline__ int wave_min_i(int v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) {
    const int o = __shfl_xor(v, m);
    v = o < v ? o : v;
  }
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max_i(int v) { return -wave_min_i(-v); }

// ---- tiles in LDS -------------------------------------------------------------------------------
// Rows of ROWB bytes (a multiple of 128), 16-byte pieces exchanged within a row by its number, so that
// both readings use all banks: the same piece of 16 consecutive rows (row_frag) and four pieces of 4
// consecutive rows (col_frag).
template <int ROWB>
__device__ __forceinline__ int piece_swap(int row) {
  if constexpr (ROWB == 128) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
  return (row & 3) << 2 | ((row >> 2) & 3);
}

template <int ROWB>
__device__ __forceinline__ int tile_at(int row, int piece) {
  return row * ROWB + ((piece ^ piece_swap<ROWB>(row)) << 4);
}

// ---- operands -----------------------------------------------------------------------------------
template <typename T>
using Frag = AlignedVec<T, kPiece<T>>;

template <typename T>
struct MmaStep;                   // inner indices of one operand pair

__device__ __forceinline__ void mma(f32x16& c, const Frag<__bf16>& a, const Frag<__bf16>& b) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16& c, const Frag<_Float16>& a, const Frag<_Float16>& b) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16& c, const Frag<float>& a, const Frag<float>& b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
}

// Row `row` of a tile (its lane's), piece 2 step + h.
template <typename T, int ROWB>
__device__ __forceinline__ Frag<T> row_frag(const char* tile, int row, int step) {
  return *reinterpret_cast<const Frag<T>*>(tile + tile_at<ROWB>(row, 2 * step + ((threadIdx.x >> 5) & 1)));
}

// Column 32 dt + l of a tile, rows base + 8 g + 4 h + i: g = 2 ks, 2 ks + 1 for 16-bit elements (a pair of
// transposing reads, each of which gives a lane of 16 its column of four rows), g = ks for fp32.
template <typename T, int ROWB>
__device__ __forceinline__ Frag<T> col_frag(const char* tile, int base, int ks, int dt) {
  const int lane = threadIdx.x & 63;
  if constexpr (sizeof(T) == 2) {
    typedef short s16x4 __attribute__((__vector_size__(8)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int col = 32 * dt + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const int row = base + 16 * ks + 4 * (lane >> 5) + ((lane >> 2) & 3);
    struct Pair {
      s16x4 a, b;
    } p;
    p.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + tile_at<ROWB>(row, col >> 3) + (col & 4) * 2));
    p.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + tile_at<ROWB>(row + 8, col >> 3) + (col & 4) * 2));
    return __builtin_bit_cast(Frag<T>, p);
  } else {
    const int col = 32 * dt + (lane & 31), row = base + 8 * ks + 4 * (lane >> 5);
    Frag<T> f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      f[i] = *reinterpret_cast<const float*>(tile + tile_at<ROWB>(row + i, col >> 2) + (col & 3) * 4);
    return f;
  }
}

// Elements of an accumulator as the column operand of inner step ks.
template <typename T>
__device__ __forceinline__ Frag<T> acc_frag(const f32x16& c, int ks) {
  Frag<T> f;
#pragma unroll
  for (int e = 0; e < kPiece<T>; ++e) f[e] = (T)c[kPiece<T> * ks + e];
  return f;
}

__device__ __forceinline__ f32x16 zeros16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// v and the other half wave's v of the same column.
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A row of D elements as the pieces of a row operand, zero past the end and where the row does not count.
template <typename T, int DP>
struct RowPieces {
  static constexpr int kSteps = DP * (int)sizeof(T) / 32;
  Frag<T> f[kSteps];
  __device__ __forceinline__ void load(const T* row, bool live, int D) {
    const int h = (threadIdx.x >> 5) & 1;
    AnyVec<T, kPiece<T>> x[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) x[s] = request_piece<T, kPiece<T>, false>(row, (2 * s + h) * kPiece<T>, D);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      settle_piece<T, kPiece<T>, false>(x[s], (2 * s + h) * kPiece<T>, D);
      const uint4 w = __builtin_bit_cast(uint4, x[s]);
      f[s] = __builtin_bit_cast(Frag<T>, live ? w : uint4{0, 0, 0, 0});
    }
  }
};

// ROWS x DP elements on their way from memory to a tile, NT threads. `row_at(r)` gives row r's address
// (always one that can be read), bit r of `live` whether it counts.
template <typename T, int DP, int ROWS, int NT>
struct Stage {
  static constexpr int E = kPiece<T>, kPieces = DP / E, kROWB = DP * (int)sizeof(T);
  static constexpr int kEach = ROWS * kPieces / NT;
  static_assert(ROWS * kPieces % NT == 0, "whole rounds");
  AnyVec<T, E> x[kEach];

  template <typename F>
  __device__ __forceinline__ void request(int tid, int D, F&& row_at) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int id = u * NT + tid;
      x[u] = request_piece<T, E, false>(row_at(id / kPieces), (id % kPieces) * E, D);
    }
  }
  __device__ __forceinline__ void store(int tid, int D, char* tile, uint64_t live) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int id = u * NT + tid, row = id / kPieces, piece = id % kPieces;
      settle_piece<T, E, false>(x[u], piece * E, D);
      const uint4 w = __builtin_bit_cast(uint4, x[u]);
      *reinterpret_cast<uint4*>(tile + tile_at<kROWB>(row, piece)) = (live >> row) & 1 ? w : uint4{0, 0, 0, 0};
    }
  }
};

// First and one past the last set byte of mask[lo .. hi), by a whole block of NT threads; {hi, hi} if none.
// `slot` is LDS for two numbers per wave.
template <int NT>
__device__ __forceinline__ int2 set_range(const uint8_t* __restrict__ mask, int lo, int hi, int* slot) {
  int last = lo, first = hi;
  for (int64_t top = hi; top > lo; top -= NT * 16) {      // from the end: padding is skipped 16 bytes a thread
    const int64_t from = top - 16 * ((int64_t)threadIdx.x + 1);
    int mine = lo;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int64_t j = from + i;
      if (j >= lo && mask[j]) mine = (int)j + 1;
    }
    mine = wave_max_i(mine);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = mine;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) last = slot[w] > last ? slot[w] : last;
    if (last > lo) break;
  }
  for (int64_t at = lo; at < last; at += NT * 16) {
    int mine = hi;
#pragma unroll
    for (int i = 15; i >= 0; --i) {
      const int64_t j = at + 16 * (int64_t)threadIdx.x + i;
      if (j < last && mask[j]) mine = (int)j;
    }
    mine = wave_min_i(mine);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = mine;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) first = slot[w] < first ? slot[w] : first;
    if (first < hi) break;
  }
  __syncthreads();
  return last > lo ? int2{first, last} : int2{hi, hi};
}

// Tiles of KB keys that rows with bounds b have to look at: [0, head) and [from, from + count - head).
struct Tiles {
  int head, from, count;
  __device__ __forceinline__ int at(int i) const { return i < head ? i : from + i - head; }
};

__device__ __forceinline__ Tiles tiles_of(const Bounds& b, int kb) {
  Tiles t;
  const int sk = (b.sk_max + kb - 1) / kb;
  const int end = (b.hi_max + kb - 1) / kb;
  t.from = b.lo_min < b.hi_max ? b.lo_min / kb : end;
  const int tail = b.lo_min < b.hi_max ? end - t.from : 0;
  if (tail == 0) t.from = sk;
  t.head = sk < t.from ? sk : t.from;
  int more = 0;
  if (tail && sk > end) more = sk - end;                  // sinks beyond the window's end (not causal)
  t.count = t.head + tail + more;
  return t;
}

}  // namespace eogp
