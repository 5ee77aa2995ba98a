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

// (Without branches: what is tested is selected among values that matrix instructions made.)
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
  int first = 0;                  // no row sees a key before this one
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

// ROWS rows of a tensor's heads, `ld` elements apart, as a source of tiles.
template <typename T>
struct RowSource {
  const T* base;                  // row 0
  int64_t ld;
  int rows;
};

// A buffer of `bytes` bytes for loads that take 0 past its end.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

// ROWS x DP elements on their way from memory to a tile, NT threads. FAST: rows of DP elements on 16-byte boundaries
// that lie less than 2^31 bytes apart over a tile: addresses are one scalar per tile and one constant per thread.
template <typename T, int DP, int ROWS, int NT, bool FAST>
struct Stage {
  static constexpr int E = kPiece<T>, kPieces = DP / E, kROWB = DP * (int)sizeof(T);
  static constexpr int kEach = ROWS * kPieces / NT;
  static_assert(ROWS * kPieces % NT == 0, "whole rounds");
  AnyVec<T, E> x[kEach];

  // Rows row0 .. of the source; those past its end are read as its last row or as zeros.
  __device__ __forceinline__ void request(const RowSource<T>& s, int row0, int tid, int D) {
    if constexpr (FAST) {
      const int left = s.rows - row0, some = left < ROWS ? left : ROWS;
      const auto r = buffer_of(s.base + (int64_t)row0 * s.ld, some > 0 ? (uint32_t)((some - 1) * s.ld + DP) * (uint32_t)sizeof(T) : 0u);
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const int id = u * NT + tid;
        const int at = (id / kPieces * (int)s.ld + id % kPieces * E) * (int)sizeof(T);
        x[u] = __builtin_bit_cast(AnyVec<T, E>, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
      }
    } else {
      request_each(tid, D, [&](int r) { return s.base + (int64_t)(row0 + r < s.rows ? row0 + r : s.rows - 1) * s.ld; });
    }
  }
  // `row_at(r)` gives row r's address (always one that can be read).
  template <typename F>
  __device__ __forceinline__ void request_each(int tid, int D, F&& row_at) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int id = u * NT + tid;
      x[u] = request_piece<T, E, false>(row_at(id / kPieces), (id % kPieces) * E, D);
    }
  }
  // To a tile; zeros for rows whose bit of `live` is not set.
  __device__ __forceinline__ void store(int tid, int D, char* tile, uint64_t live) {
    constexpr uint64_t kAll = ROWS == 64 ? ~0ull : (1ull << (ROWS & 63)) - 1;
    if constexpr (!FAST) {
#pragma unroll
      for (int u = 0; u < kEach; ++u) settle_piece<T, E, false>(x[u], (u * NT + tid) % kPieces * E, D);
    }
    if (live != kAll) {
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const uint4 w = __builtin_bit_cast(uint4, x[u]);
        x[u] = __builtin_bit_cast(AnyVec<T, E>, (live >> ((u * NT + tid) / kPieces)) & 1 ? w : uint4{0, 0, 0, 0});
      }
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int id = u * NT + tid;
      *reinterpret_cast<uint4*>(tile + tile_at<kROWB>(id / kPieces, id % kPieces)) = __builtin_bit_cast(uint4, x[u]);
    }
  }
};

// What a mask leaves of [lo, hi): first and one past the last set byte ({hi, hi} if none), and whether all between are.
struct MaskRange {
  int first, last;
  bool solid;
};

// By a whole block of NT threads, 64 bytes a thread at a time; `slot` is LDS for three numbers per wave.
template <int NT>
__device__ __forceinline__ MaskRange mask_range(const uint8_t* __restrict__ mask, int lo, int hi, int (*slot)[3]) {
  int first = hi, last = lo, count = 0;
  for (int64_t at = lo; at < hi; at += NT * 64) {
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(1)));
    words w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t from = at + (u * NT + (int)threadIdx.x) * 16;
      w[u] = words{0, 0, 0, 0};
      if (from + 16 <= hi) {
        w[u] = *reinterpret_cast<const words*>(mask + from);
      } else {
        for (int i = 0; i < 16; ++i)
          if (from + i < hi) w[u][i / 4] |= (uint32_t)mask[from + i] << (i % 4 * 8);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int from = (int)(at + (u * NT + (int)threadIdx.x) * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // a bit per byte that is not 0
        uint32_t z = w[u][i];
        z = (((z & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | z) & 0x80808080u;
        count += __builtin_popcount(z);
        if (z) {
          const int f = from + 4 * i + __builtin_ctz(z) / 8, l = from + 4 * i + 4 - __builtin_clz(z) / 8;
          first = f < first ? f : first;
          last = l > last ? l : last;
        }
      }
    }
  }
  first = wave_min_i(first);
  last = wave_max_i(last);
  for (int m = 32; m; m >>= 1) count += __shfl_xor(count, m);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    slot[threadIdx.x >> 6][0] = first;
    slot[threadIdx.x >> 6][1] = last;
    slot[threadIdx.x >> 6][2] = count;
  }
  __syncthreads();
  count = 0;
  for (int w = 0; w < NT / 64; ++w) {
    first = slot[w][0] < first ? slot[w][0] : first;
    last = slot[w][1] > last ? slot[w][1] : last;
    count += slot[w][2];
  }
  first = __builtin_amdgcn_readfirstlane(first);
  last = __builtin_amdgcn_readfirstlane(last);
  count = __builtin_amdgcn_readfirstlane(count);
  __syncthreads();
  return count > 0 ? MaskRange{first, last, count == last - first} : MaskRange{hi, hi, true};
}

// Bits a .. b - 1 of 32.
__device__ __forceinline__ uint32_t bits_between(int a, int b) {
  a = a < 0 ? 0 : a;
  b = b > 32 ? 32 : b;
  return b > a ? (uint32_t)((1ull << b) - (1ull << a)) : 0u;
}

// Keys j0 .. j0 + 31 that a row sees, as bits.
__device__ __forceinline__ uint32_t sight_bits(const Span& v, int j0) {
  return bits_between(v.lo - j0, v.hi - j0) | bits_between(0, v.sk - j0);
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
