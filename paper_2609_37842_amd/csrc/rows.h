// Rows of fp32, bf16 or fp16 elements taken 16 bytes ("a piece") per lane, for the kernels that
// pass over rows once: embedding, layer norm, cross-entropy, sampling. Rows may start at any
// element; a row's last piece may be short.
#pragma once
#include <algorithm>
#include <type_traits>
#include <utility>

#include "common.h"

namespace eogp {

template <eogp_dtype D> struct ElemOf;
template <> struct ElemOf<EOGP_F32> { using type = float; };
template <> struct ElemOf<EOGP_BF16> { using type = __bf16; };
template <> struct ElemOf<EOGP_F16> { using type = _Float16; };

template <typename T> constexpr int kPiece = 16 / (int)sizeof(T);   // elements of a piece

// E elements at any element's address. (Plain typedefs: an alignment that depends on a template's
// parameters is dropped, and the compiler would take 16-byte boundaries for granted.)
template <typename T, int E> struct AnyVecOf;
#define EOGP_ANY_VEC(T, E)                                                  \
  template <> struct AnyVecOf<T, E> {                                       \
    typedef T type __attribute__((ext_vector_type(E), aligned(sizeof(T)))); \
  };
EOGP_ANY_VEC(float, 2)
EOGP_ANY_VEC(float, 4)
EOGP_ANY_VEC(float, 8)
EOGP_ANY_VEC(__bf16, 2)
EOGP_ANY_VEC(__bf16, 4)
EOGP_ANY_VEC(__bf16, 8)
EOGP_ANY_VEC(_Float16, 2)
EOGP_ANY_VEC(_Float16, 4)
EOGP_ANY_VEC(_Float16, 8)
#undef EOGP_ANY_VEC
template <typename T, int E>
using AnyVec = typename AnyVecOf<T, E>::type;

// E elements at a 16-byte boundary (LDS)
template <typename T, int E>
using AlignedVec = T __attribute__((ext_vector_type(E), aligned(16)));

// A piece as four words, moved down by a number of bytes with `fill` coming in above. (Only a row's last
// piece is ever short, by the same bytes in every row, so the tests are uniform.)
__device__ __forceinline__ uint4 words_down(uint4 x, uint32_t bytes, uint32_t fill) {
  if (bytes & 8) x = uint4{x.z, x.w, fill, fill};
  if (bytes & 4) x = uint4{x.y, x.z, x.w, fill};
  if (bytes & 2)
    x = uint4{__builtin_amdgcn_alignbit(x.y, x.x, 16), __builtin_amdgcn_alignbit(x.z, x.y, 16),
              __builtin_amdgcn_alignbit(x.w, x.z, 16), __builtin_amdgcn_alignbit(fill, x.w, 16)};
  return x;
}

// Elements c .. c + E - 1 of a row of d; `pad` in the place of those past the end, which are not read.
// The short last piece is one load of the row's last E elements, moved down. STREAM: rows that are read
// this once, past the L2s' other lines.
template <typename T, int E, bool STREAM = false>
__device__ __forceinline__ AnyVec<T, E> fetch_piece(const T* __restrict__ row, int64_t c, int64_t d, T pad) {
  AnyVec<T, E> x;
  if (c + E <= d) {
    const auto* p = reinterpret_cast<const AnyVec<T, E>*>(row + c);
    if constexpr (STREAM)
      x = __builtin_nontemporal_load(p);
    else
      x = *p;
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = pad;
    if (c < d) {
      if constexpr (E * sizeof(T) == 16) {
        if (d >= E) {
          uint32_t fill;
          if constexpr (sizeof(T) == 4)
            fill = __builtin_bit_cast(uint32_t, pad);
          else
            fill = __builtin_bit_cast(uint16_t, pad) * 0x10001u;
          const uint4 last = __builtin_bit_cast(uint4, *reinterpret_cast<const AnyVec<T, E>*>(row + d - E));
          return __builtin_bit_cast(AnyVec<T, E>, words_down(last, (uint32_t)(c + E - d) * (uint32_t)sizeof(T), fill));
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (c + e < d) x[e] = row[c + e];
    }
  }
  return x;
}

// The same in two steps, for several pieces at once: whole unconditional loads (a piece that would pass
// the end is taken E elements before it), then what such lanes hold put right. With the two in one step
// a wave that has such lanes waits for each load before it requests the next: the lanes' other value
// goes to the registers that the load is about to fill. NARROW: rows shorter than a piece, element by
// element (an instance of its own: a branch beside the loads would make them wait as well).
template <typename T, int E, bool NARROW, bool STREAM = false>
__device__ __forceinline__ AnyVec<T, E> request_piece(const T* __restrict__ row, int64_t c, int64_t d) {
  static_assert(E * sizeof(T) == 16, "one piece");
  if constexpr (NARROW) return fetch_piece<T, E>(row, c, d, (T)0.f);
  const auto* p = reinterpret_cast<const AnyVec<T, E>*>(row + (c < d - E ? c : d - E));
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  return *p;
}

// Zero past the row's end.
template <typename T, int E, bool NARROW>
__device__ __forceinline__ void settle_piece(AnyVec<T, E>& x, int64_t c, int64_t d) {
  if constexpr (!NARROW) {
    if (c + E > d) {
      const uint4 w = __builtin_bit_cast(uint4, x);
      x = __builtin_bit_cast(AnyVec<T, E>, c < d ? words_down(w, (uint32_t)(c + E - d) * (uint32_t)sizeof(T), 0)
                                                 : uint4{0, 0, 0, 0});
    }
  }
}

template <typename T, int E>
__device__ __forceinline__ void widen(const AnyVec<T, E>& x, float (&v)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = (float)x[e];
}

// The same elements as fp32.
template <typename T, int E>
__device__ __forceinline__ void load_piece(const T* __restrict__ row, int64_t c, int64_t d, float pad,
                                           float (&v)[E]) {
  widen<T, E>(fetch_piece<T, E>(row, c, d, (T)pad), v);
}

// The same elements rounded to T and stored, none past the end (a short piece in up to three stores).
// The stores are streaming: what these kernels write is not read again by them, and lines that go to HBM
// at once leave the L2s to what is (131,072 embedded rows of 768 fp32: 116 -> 75 us; layer norm of
// 65,536: 80 -> 71).
template <typename T, int E>
__device__ __forceinline__ void store_piece(T* __restrict__ row, int64_t c, int64_t d, const float (&v)[E]) {
  AnyVec<T, E> x;
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = (T)v[e];
  if (c + E <= d) {
    __builtin_nontemporal_store(x, reinterpret_cast<AnyVec<T, E>*>(row + c));
  } else if (c < d) {
    if constexpr (E * sizeof(T) == 16) {
      uint4 w = __builtin_bit_cast(uint4, x);
      T* to = row + c;
      const uint32_t bytes = (uint32_t)(d - c) * (uint32_t)sizeof(T);
      if (bytes & 8) {
        using Half = AnyVec<T, 8 / (int)sizeof(T)>;
        *reinterpret_cast<Half*>(to) = __builtin_bit_cast(Half, uint2{w.x, w.y});
        to += 8 / sizeof(T);
        w = words_down(w, 8, 0);
      }
      if constexpr (sizeof(T) == 4) {
        if (bytes & 4) *to = __builtin_bit_cast(T, w.x);
      } else {
        if (bytes & 4) {
          *reinterpret_cast<AnyVec<T, 2>*>(to) = __builtin_bit_cast(AnyVec<T, 2>, w.x);
          to += 2;
          w = words_down(w, 4, 0);
        }
        if (bytes & 2) *to = __builtin_bit_cast(T, (uint16_t)w.x);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (c + e < d) row[c + e] = x[e];
    }
  }
}

// Element c of an array whose type is known at run time (weights read once per wave).
__device__ __forceinline__ float load_any(const void* p, eogp_dtype t, int64_t c) {
  if (t == EOGP_F32) return static_cast<const float*>(p)[c];
  if (t == EOGP_BF16) return (float)static_cast<const __bf16*>(p)[c];
  return (float)static_cast<const _Float16*>(p)[c];
}

// Lane moves inside the vector unit (DPP): the value of the lane 1, 2, 4, 8 places before in a row of
// 16 lanes, then the last lane of the row before (rows 1 and 3), then lane 31 (rows 2 and 3); `other`
// where there is none. Six such steps make an inclusive scan of a wave, whose total is in lane 63.
template <int STEP>
__device__ __forceinline__ uint32_t lane_before(uint32_t x, uint32_t other) {
  constexpr int kCtrl[6] = {0x111, 0x112, 0x114, 0x118, 0x142, 0x143}, kRows[6] = {15, 15, 15, 15, 10, 12};
  return (uint32_t)__builtin_amdgcn_update_dpp((int)other, (int)x, kCtrl[STEP], kRows[STEP], 0xF, false);
}

template <typename F>
__device__ __forceinline__ uint32_t scan_steps(uint32_t v, F&& f) {
  v = f(v, std::integral_constant<int, 0>{});
  v = f(v, std::integral_constant<int, 1>{});
  v = f(v, std::integral_constant<int, 2>{});
  v = f(v, std::integral_constant<int, 3>{});
  v = f(v, std::integral_constant<int, 4>{});
  return f(v, std::integral_constant<int, 5>{});
}

__device__ __forceinline__ float last_lane(uint32_t v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)v, 63));
}

// Sum and maximum over a wave, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
  return last_lane(scan_steps(__float_as_uint(v), [](uint32_t x, auto step) {
    return __float_as_uint(__uint_as_float(x) + __uint_as_float(lane_before<decltype(step)::value>(x, 0)));
  }));
}

__device__ __forceinline__ float wave_max(float v) {
  return last_lane(scan_steps(__float_as_uint(v), [](uint32_t x, auto step) {
    return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(lane_before<decltype(step)::value>(x, x))));
  }));
}

// Inclusive sums over a wave.
template <int STEP>
__device__ __forceinline__ uint64_t add_before(uint64_t v) {
  return v + ((uint64_t)lane_before<STEP>((uint32_t)(v >> 32), 0) << 32 | lane_before<STEP>((uint32_t)v, 0));
}

__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
  v = add_before<1>(add_before<0>(v));
  v = add_before<3>(add_before<2>(v));
  return add_before<5>(add_before<4>(v));
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  return scan_steps(v, [](uint32_t x, auto step) { return x + lane_before<decltype(step)::value>(x, 0); });
}

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

__device__ __forceinline__ uint64_t wave_total(uint64_t v) { return lane_value(wave_scan(v), 63); }

// Calls f with the element type of a run-time dtype: f(T{}).
template <typename F>
inline eogp_status with_type(eogp_dtype t, F&& f) {
  if (t == EOGP_F32) return f(float{});
  if (t == EOGP_BF16) return f(__bf16{});
  return f(_Float16{});
}

}  // namespace eogp

namespace eogp {

// f(integral_constant<int, 0>), ..., f(integral_constant<int, N - 1>)
template <int... I, typename F>
__device__ __forceinline__ void unroll(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}

// A row that a block of NT threads keeps in registers as read: P pieces of 16 bytes per thread. In
// index order come groups of G pieces per thread, in a group the waves, in a wave its G pieces of 64
// lanes. A piece that would pass the end is taken E elements before the end instead, and its elements
// that other pieces hold read as -inf: so every load is whole and unconditional (a row has at least E
// elements). The passes over a row (each) take one piece at a time: groups past the end cost a scalar
// branch, and the compiler neither keeps one pass's conversions for the next nor interleaves pieces,
// both of which cost more registers than the row has left. The last pass over a row (each_then_load)
// requests each piece of the next row into the registers that it has just finished with, so that the
// next row arrives while this one's pass, sums and stores go on.
template <typename T, int NT, int P, int G = 1>
struct RegisterRow {
  static constexpr int E = kPiece<T>;
  static constexpr int kGroup = NT * G * E;                // elements of a group
  static_assert(P % G == 0, "whole groups");
  AnyVec<T, E> raw[P];

  // First element of piece p, from the thread's place (here). The place is hidden from the compiler
  // in each pass: it would keep the addresses of all pieces in registers from row to row.
  static __device__ __forceinline__ uint32_t here() {
    uint32_t b = ((threadIdx.x >> 6) * (G * 64) + (threadIdx.x & 63)) * E;
    asm volatile("" : "+v"(b));
    return b;
  }
  static __device__ __forceinline__ uint32_t at(uint32_t place, int p) {
    return place + (uint32_t)((p / G) * kGroup + (p % G) * 64 * E);
  }

  static __device__ __forceinline__ AnyVec<T, E> fetch(const T* row, uint32_t c, uint32_t width) {
    return *reinterpret_cast<const AnyVec<T, E>*>(row + (c < width - E ? c : width - E));
  }

  // f(p, c, first, v) with the elements v of indices c ..; those below `first` read as -inf.
  template <typename F>
  static __device__ __forceinline__ void take(int p, uint32_t c, uint32_t width, const AnyVec<T, E>& x, F&& f) {
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (float)x[e];
    const uint32_t from = c < width - E ? c : width - E;
    if (from != c) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (from + e < c) v[e] = -INFINITY;
    }
    f(p, from, c, v);
  }

  __device__ __forceinline__ void load(const T* row, uint32_t width) {
    const uint32_t place = here();
#pragma unroll
    for (int p = 0; p < P; ++p) raw[p] = fetch(row, at(place, p), width);
  }

  template <typename F>
  __device__ __forceinline__ void each(uint32_t width, F&& f) {
    const uint32_t place = here();
    unroll(std::make_integer_sequence<int, P>{}, [&](auto piece) {
      constexpr int p = decltype(piece)::value;
      if ((uint32_t)((p / G) * kGroup) < width) {          // uniform
        AnyVec<T, E> x = raw[p];
        asm volatile("" : "+v"(x));
        take(p, at(place, p), width, x, f);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  }

  template <typename F>
  __device__ __forceinline__ void each_then_load(uint32_t width, F&& f, const T* next) {
    const uint32_t place = here();
    unroll(std::make_integer_sequence<int, P>{}, [&](auto piece) {
      constexpr int p = decltype(piece)::value;
      if ((uint32_t)((p / G) * kGroup) < width) {          // uniform
        AnyVec<T, E> x = raw[p];
        asm volatile("" : "+v"(x));
        take(p, at(place, p), width, x, f);
      }
      raw[p] = fetch(next, at(place, p), width);
      __builtin_amdgcn_sched_barrier(0);
    });
  }
};

// The same passes over a row that is too long for the registers, or shorter than a piece: it is read
// in each.
template <typename T, int NT, int G>
struct RegisterRow<T, NT, 0, G> {
  using Shape = RegisterRow<T, NT, G, G>;
  static constexpr int E = kPiece<T>, kGroup = Shape::kGroup;
  const T* row;

  static __device__ __forceinline__ AnyVec<T, E> fetch(const T* row, uint32_t c, uint32_t width) {
    return fetch_piece<T, E>(row, c, width, (T)-INFINITY);
  }

  __device__ __forceinline__ void load(const T* r, uint32_t) { row = r; }

  template <typename F>
  __device__ __forceinline__ void each(uint32_t width, F&& f) {
    const uint32_t place = Shape::here();
    AnyVec<T, E> next[G];                                  // one group is on its way while another is taken
#pragma unroll
    for (int q = 0; q < G; ++q) next[q] = fetch(row, Shape::at(place, q), width);
    int p = 0;
    for (uint64_t base = 0; base < width; base += kGroup) {
      AnyVec<T, E> now[G];
#pragma unroll
      for (int q = 0; q < G; ++q) now[q] = next[q];
      if (base + kGroup < width) {
#pragma unroll
        for (int q = 0; q < G; ++q) next[q] = fetch(row, (uint32_t)(base + kGroup) + Shape::at(place, q), width);
      }
#pragma unroll
      for (int q = 0; q < G; ++q, ++p) {
        float v[E];
        widen<T, E>(now[q], v);
        const uint32_t c = (uint32_t)base + Shape::at(place, q);
        f(p, c, c, v);
      }
    }
  }

  template <typename F>
  __device__ __forceinline__ void each_then_load(uint32_t width, F&& f, const T* next) {
    each(width, f);
    row = next;
  }
};

// The rows of a block that stays for many: round i takes row i * blocks + (block + 97 i) mod blocks,
// so that rows that cost nothing (masked ends of examples of a power of two tokens) do not all fall to
// the same blocks. Against the same place in every round: cross-entropy of 4,096 bf16 places of 100,352, 75% valid,
// 311 and 324 us, sampling of 2,048 fp32 places of 50,257, 75% valid, 98 and 109; there the blocks with the most rows
// still have 7 or 8 where the mean is 6.3. (Numbering the valid rows by a scan over the mask and dealing those out
// evenly took that cross-entropy, in an earlier state, from 323 to 315 us and 24 rows of 50,257 fp32 from 11.8 to 14.8.)
struct RowWalk {
  uint32_t round = 0;
  // The next row for which work(row) holds, -1 at the end.
  template <typename Work>
  __device__ __forceinline__ int64_t next(int64_t n, Work&& work) {
    while ((int64_t)round * gridDim.x < n) {
      const int64_t row = (int64_t)round * gridDim.x + (blockIdx.x + 97u * round) % gridDim.x;
      ++round;
      if (row < n && work(row)) return row;
    }
    return -1;
  }
};

// Blocks of a launch that has one per row (a launch holds fewer than 2^32 threads).
constexpr int64_t kMostBlocks = 1 << 21;

// Blocks for n rows: those of 256 threads have one row each, the others stay, `per_cu` of them to a CU
// by their registers.
inline int64_t row_blocks(int64_t n, int nt, int per_cu) {
  return std::min<int64_t>(n, nt == 256 ? kMostBlocks : kCus * per_cu);
}

// Threads of the block that holds a row of `pieces` 16-byte pieces in registers, and pieces per
// thread; none (0) for rows longer than 1,024 threads x 16 pieces, which are read again instead, and
// for rows shorter than a piece.
template <typename T, typename F>
inline eogp_status with_row_shape(int64_t width, F&& f) {
  using std::integral_constant;
  using N256 = integral_constant<int, 256>;
  using N1024 = integral_constant<int, 1024>;
  const int64_t pieces = ceil_div(width, kPiece<T>);
  if (width < kPiece<T>) return f(N256{}, integral_constant<int, 0>{});
  if (pieces <= 512) return f(N256{}, integral_constant<int, 2>{});
  if (pieces <= 1024) return f(N256{}, integral_constant<int, 4>{});
  if (pieces <= 2048) return f(N256{}, integral_constant<int, 8>{});
  if (pieces <= 4096) return f(N1024{}, integral_constant<int, 4>{});
  if (pieces <= 8192) return f(N1024{}, integral_constant<int, 8>{});
  if (pieces <= 16384) return f(N1024{}, integral_constant<int, 16>{});
  return f(N1024{}, integral_constant<int, 0>{});
}
}  // namespace eogp
