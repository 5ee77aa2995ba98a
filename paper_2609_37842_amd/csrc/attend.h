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

  // (Positions further than 2^40 see what those see: no sum of a position leaves 64 bits.)
  __device__ __forceinline__ int64_t start(int64_t n) const {
    constexpr int64_t kFar = (int64_t)1 << 40;
    const int64_t p = q_start ? q_start[n] : (int64_t)Tk - Tq;
    return p < -kFar ? -kFar : p > kFar ? kFar : p;
  }
};

// Keys [lo, hi) and [0, sk) of a query at position p.
struct Span {
  int lo, hi, sk;
};

__device__ __forceinline__ int clamp_key(int64_t j, int most) { return (int)(j < 0 ? 0 : j > most ? most : j); }

__device__ __forceinline__ Span span_of(const Sight& s, int64_t p) {
  Span v;
  v.hi = clamp_key(s.causal ? p + 1 : s.window ? p + s.window : s.Tk, s.Tk);
  v.lo = s.window ? clamp_key(p - s.window + 1, v.hi) : 0;
  v.sk = clamp_key(s.causal ? p + 1 : s.Tk, s.sinks < s.Tk ? s.sinks : s.Tk);
  return v;
}

// Division of numbers below 2^31 by one divisor.
struct Divide {
  uint32_t by = 1, mul = 0;
  int shift = 0;
  Divide() = default;
  explicit Divide(int64_t d) : by((uint32_t)d) {
    int s = 0;
    while (((int64_t)1 << s) < d) ++s;
    shift = 31 + s;
    mul = (uint32_t)((((uint64_t)1 << shift) / (uint64_t)d) + 1);   // below 2^32, as 2^s < 2 d: a product with n fits 63 bits
  }
  __device__ __forceinline__ int quotient(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
  __device__ __forceinline__ int rest(int n, int q) const { return n - q * (int)by; }
};

// Where any of a set of rows sees keys: none outside [lo, hi) and [0, sk), none before `first`.
struct Bounds {
  int lo, hi, sk, first;
};

// Rows of a set that count, as bits of rows 0 .. 63 and 64 .. 127: none, or its first and last.
struct LiveRows {
  uint64_t low, high;
  __device__ __forceinline__ bool none() const { return !(low | high); }
  __device__ __forceinline__ int first() const { return low ? __builtin_ctzll(low) : 64 + __builtin_ctzll(high); }
  __device__ __forceinline__ int last() const { return high ? 127 - __builtin_clzll(high) : 63 - __builtin_clzll(low); }
};

// Minimum and maximum over a wave, in every lane.
__device__ __forceinline__ int wave_max_i(int v) {
  v = (int)scan_steps((uint32_t)v, [](uint32_t x, auto step) {
    const int y = (int)lane_before<decltype(step)::value>(x, x);
    return (uint32_t)(y > (int)x ? y : (int)x);
  });
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_min_i(int v) { return -wave_max_i(-v); }

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

// A piece that request_piece took at c of a row of d elements: zero past the row's end, by selects alone (once: what is
// there already would be moved again).
template <typename T>
__device__ __forceinline__ uint4 settled(uint4 x, int c, int d) {
  constexpr int E = kPiece<T>;
  const uint32_t down = (uint32_t)(c + E > d ? c + E - d : 0) * (uint32_t)sizeof(T);
  x = down & 8 ? uint4{x.z, x.w, 0, 0} : x;
  x = down & 4 ? uint4{x.y, x.z, x.w, 0} : x;
  if constexpr (sizeof(T) == 2) {
    const uint4 y{__builtin_amdgcn_alignbit(x.y, x.x, 16), __builtin_amdgcn_alignbit(x.z, x.y, 16),
                  __builtin_amdgcn_alignbit(x.w, x.z, 16), x.w >> 16};
    x = down & 2 ? y : x;
  }
  return down >= 16 ? uint4{0, 0, 0, 0} : x;
}

// A row of D elements as the pieces of a row operand, zero past the end and where the row does not count.
template <typename T, int DP, bool EXACT = false>
struct RowPieces {              // EXACT: D is DP
  static constexpr int kSteps = DP * (int)sizeof(T) / 32;
  Frag<T> f[kSteps];
  __device__ __forceinline__ static int at(int s) { return (2 * s + (int)((threadIdx.x >> 5) & 1)) * kPiece<T>; }
  __device__ __forceinline__ void request(const T* row, int D) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      f[s] = __builtin_bit_cast(Frag<T>, __builtin_bit_cast(uint4, request_piece<T, kPiece<T>, false>(row, at(s), EXACT ? DP : D)));
  }
  __device__ __forceinline__ void settle(bool live, int D) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      uint4 w = __builtin_bit_cast(uint4, f[s]);
      if constexpr (!EXACT) w = settled<T>(w, at(s), D);
      f[s] = __builtin_bit_cast(Frag<T>, live ? w : uint4{0, 0, 0, 0});
    }
  }
  __device__ __forceinline__ void load(const T* row, bool live, int D) {
    request(row, D);
    settle(live, D);
  }
};

// A buffer of `bytes` bytes for loads that take 0 past its end.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

// The tokens of one head as rows `ld` elements apart, a source of tiles.
template <typename T>
struct RowSource {
  const T* base;                  // row 0
  int64_t ld;
  int rows;
  __amdgpu_buffer_rsrc_t all;     // fast loads: the rows, less than 2^31 bytes

  __device__ __forceinline__ RowSource(const T* b, int64_t stride, int n, int width, bool fast)
      : base(b), ld(stride), rows(n),
        all(buffer_of(b, fast && n > 0 ? (uint32_t)((n - 1) * stride + width) * (uint32_t)sizeof(T) : 0u)) {}
};

// ROWS x DP elements on their way from memory to a tile, NT threads. FAST: all rows of DP elements lie on 16-byte
// boundaries within 2^31 bytes, so that an address is a number per tile plus one per thread.
template <typename T, int DP, int ROWS, int NT, bool FAST>
struct Stage {
  static constexpr int E = kPiece<T>, kPieces = DP / E, kROWB = DP * (int)sizeof(T);
  static constexpr int kEach = ROWS * kPieces / NT;
  static_assert(ROWS * kPieces % NT == 0, "whole rounds");
  AnyVec<T, E> x[kEach];

  // Rows row0 .. of the source; those past its end are read as its last row or as zeros.
  __device__ __forceinline__ void request(const RowSource<T>& s, int row0, int tid, int D) {
    if constexpr (FAST) {
      const int tile = row0 * (int)s.ld * (int)sizeof(T);
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const int id = u * NT + tid, at = (id / kPieces * (int)s.ld + id % kPieces * E) * (int)sizeof(T);
        x[u] = __builtin_bit_cast(AnyVec<T, E>, __builtin_amdgcn_raw_buffer_load_b128(s.all, at + tile, 0, 0));
      }
    } else {
      request_each(tid, D, [&](int r) { return s.base + (int64_t)(row0 + r < s.rows ? row0 + r : s.rows - 1) * s.ld; });
    }
  }
  // The thread's piece u at a byte of a buffer (FAST).
  __device__ __forceinline__ void request_one(int u, __amdgpu_buffer_rsrc_t all, int at) {
    x[u] = __builtin_bit_cast(AnyVec<T, E>, __builtin_amdgcn_raw_buffer_load_b128(all, at, 0, 0));
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
      for (int u = 0; u < kEach; ++u)
        x[u] = __builtin_bit_cast(AnyVec<T, E>, settled<T>(__builtin_bit_cast(uint4, x[u]), (u * NT + tid) % kPieces * E, D));
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

// By each wave for itself, 64 bytes a lane at a time; mask [rows].
__device__ __forceinline__ MaskRange mask_range(const uint8_t* __restrict__ mask, int rows, int lo, int hi) {
  int first = hi, last = lo, count = 0;
  for (int64_t at = lo; at < hi; at += 64 * 64) {
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(1)));
    words w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t from = at + (u * 64 + (int)(threadIdx.x & 63)) * 16;
      if (rows >= 16) {
        w[u] = *reinterpret_cast<const words*>(mask + (from + 16 <= rows ? from : rows - 16));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[u][i] = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (from + i < rows) w[u][i / 4] |= (uint32_t)mask[from + i] << (i % 4 * 8);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t from = at + (u * 64 + (int)(threadIdx.x & 63)) * 16;
      const int64_t begin = rows >= 16 && from + 16 > rows ? rows - 16 : from;     // of what was read
      uint32_t set = 0;                                    // a bit per byte that is not 0
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t z = w[u][i];
        z = (((z & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | z) & 0x80808080u;
        set |= ((z * 0x00204081u) >> 28) << (4 * i);
      }
      // bytes of [from, hi) alone
      const int skip = from - begin > 16 ? 16 : (int)(from - begin), keep = hi - begin > 16 ? 16 : hi < begin ? 0 : (int)(hi - begin);
      set = set >> skip << skip & ((1u << keep) - 1u);
      count += __builtin_popcount(set);
      const int f = (int)begin + __builtin_ctz(set | 0x10000u), l = (int)begin + 32 - __builtin_clz(set | 1u);
      first = set && f < first ? f : first;
      last = set && l > last ? l : last;
    }
  }
  first = wave_min_i(first);
  last = wave_max_i(last);
  uint32_t total = wave_scan((uint32_t)count);
  total = (uint32_t)__builtin_amdgcn_readlane((int)total, 63);
  return total > 0 ? MaskRange{first, last, (int)total == last - first} : MaskRange{hi, hi, true};
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

// Bounds of the keys that rows at positions `first` to `last` see (their numbers grow with the position), no further
// than the first and last key that the mask leaves; no mask any more where it leaves all between.
__device__ __forceinline__ Bounds bounds_of(const Sight& s, int64_t first, int64_t last, const MaskRange& m, const uint8_t*& kmask) {
  const Span f = span_of(s, first), l = span_of(s, last);
  Bounds b{f.lo, l.hi, l.sk, 0};
  if (!kmask) return b;
  b.lo = max(b.lo, m.first);
  b.hi = min(b.hi, m.last);
  b.sk = b.sk > m.first ? min(b.sk, m.last) : 0;
  b.first = m.first;
  if (m.solid) kmask = nullptr;
  return b;
}

// The mask's range for rows at those positions: of all keys where a wave reads them at once (which need not wait for the
// rows' own masks), else of the keys that the rows see.
constexpr int kMaskAtOnce = 4096;
__device__ __forceinline__ MaskRange range_of(const Sight& s, const uint8_t* kmask, int64_t first, int64_t last) {
  const Span f = span_of(s, first), l = span_of(s, last);
  const int to = max(l.hi, l.sk);
  return mask_range(kmask, s.Tk, l.sk > 0 ? 0 : min(f.lo, to), to);
}

// Keys of a tile that any row of the block sees, as bits, with the mask's byte of the lane's key (1 without a mask).
struct KeyMask {
  const uint8_t* bytes;           // without a mask, any that can be read: byte 0 is, and does not matter
  int index;                      // all bits set, or none without a mask
  int last;
  __device__ __forceinline__ KeyMask(const uint8_t* mask, const void* other, int Tk)
      : bytes(mask ? mask : static_cast<const uint8_t*>(other)), index(mask ? -1 : 0), last(Tk - 1) {}
  __device__ __forceinline__ uint8_t request(int j) const { return bytes[min(j, last) & index]; }
  __device__ __forceinline__ uint32_t bits(const Bounds& b, int j0, uint8_t byte) const {
    const uint32_t seen = (bits_between(b.lo - j0, b.hi - j0) | bits_between(0, b.sk - j0)) & ~bits_between(0, b.first - j0);
    return seen & ((uint32_t)__ballot(byte != 0) | ~(uint32_t)index);
  }
};

// Scores and references in powers of two from which on their own roundings count (half a step of 2^20 is 2^-5).
constexpr float kFar = 1048576.f;
constexpr float kLowest = -3.4028234e38f;   // reference of a row that has seen no key (finite: its difference to itself is 0)

// A product as it is rounded, whatever takes it. (The compiler makes one rounding of a product and a difference.)
__device__ __forceinline__ float rounded(float x) {
  asm("" : "+v"(x));
  return x;
}

// Scores that their row does not see become -inf.
__device__ __forceinline__ void hide(f32x16& s, const Span& span, uint32_t bits, int j0) {
  const uint32_t seen = (bits & sight_bits(span, j0)) >> (4 * ((threadIdx.x >> 5) & 1));
#pragma unroll
  for (int e = 0; e < 16; ++e) s[e] = (seen >> (8 * (e / 4) + e % 4)) & 1 ? s[e] : -INFINITY;
}

// Elements c .. c + 3 of a row of D (EXACT: D is a multiple of 4), by plain stores: the lines are filled by the two
// halves of the wave, one after the other.
template <typename T, bool EXACT>
__device__ __forceinline__ void put4(T* row, int c, int D, const float (&v)[4]) {
  if (EXACT || c + 4 <= D) {
    AnyVec<T, 4> x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (T)v[e];
    *reinterpret_cast<AnyVec<T, 4>*>(row + c) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < D) row[c + e] = (T)v[e];
  }
}

// Tiles of KB keys that rows with bounds b have to look at: [0, head) and [from, from + count - head).
struct Tiles {
  int head, from, count;
  __device__ __forceinline__ int at(int i) const { return i + (i < head ? 0 : from - head); }
};

__device__ __forceinline__ Tiles tiles_of(const Bounds& b, int kb) {
  Tiles t;
  const int sk = (b.sk + kb - 1) / kb;
  const int end = (b.hi + kb - 1) / kb;
  t.from = b.lo < b.hi ? b.lo / kb : end;
  const int tail = b.lo < b.hi ? end - t.from : 0;
  if (tail == 0) t.from = sk;
  t.head = sk < t.from ? sk : t.from;
  int more = 0;
  if (tail && sk > end) more = sk - end;                  // sinks beyond the window's end (not causal)
  t.count = t.head + tail + more;
  return t;
}

// Head widths that the kernels are built for.
inline constexpr int padded(int64_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
// Rows of exactly the built width on 16-byte boundaries, all heads of an example within 2^31 bytes.
inline bool fast_rows(const eogp_heads& x, int64_t rows, int64_t D, int size) {
  return D == padded(D) && (uintptr_t)x.data % 16 == 0 && x.ld_example * size % 16 == 0 && x.ld_token * size % 16 == 0 &&
         x.ld_head * size % 16 == 0 && (rows + 64) * x.ld_token < ((int64_t)1 << 30) / size && x.heads * x.ld_head < ((int64_t)1 << 30) / size;
}

}  // namespace eogp
