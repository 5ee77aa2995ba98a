// Rows of fp32, bf16 or fp16 elements taken 16 bytes ("a piece") per lane, for the kernels that
// pass over rows once: embedding, layer norm, cross-entropy, sampling. Rows may start at any
// element; a row's last piece may be short.
#pragma once
#include <type_traits>

#include "common.h"

namespace eogp {

template <eogp_dtype D> struct ElemOf;
template <> struct ElemOf<EOGP_F32> { using type = float; };
template <> struct ElemOf<EOGP_BF16> { using type = __bf16; };
template <> struct ElemOf<EOGP_F16> { using type = _Float16; };

template <typename T> constexpr int kPiece = 16 / (int)sizeof(T);   // elements of a piece

// E elements at any element's address
template <typename T, int E>
using AnyVec = T __attribute__((ext_vector_type(E), aligned(sizeof(T))));

// Elements c .. c + E - 1 of a row of d as fp32; `pad` in the place of those past the end.
template <typename T, int E>
__device__ __forceinline__ void load_piece(const T* __restrict__ row, int64_t c, int64_t d, float pad,
                                           float (&v)[E]) {
  if (c + E <= d) {
    const AnyVec<T, E> x = *reinterpret_cast<const AnyVec<T, E>*>(row + c);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (float)x[e];
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = c + e < d ? (float)row[c + e] : pad;
  }
}

// The same elements rounded to T and stored; none past the end.
template <typename T, int E>
__device__ __forceinline__ void store_piece(T* __restrict__ row, int64_t c, int64_t d, const float (&v)[E]) {
  if (c + E <= d) {
    AnyVec<T, E> x;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = (T)v[e];
    *reinterpret_cast<AnyVec<T, E>*>(row + c) = x;
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (c + e < d) row[c + e] = (T)v[e];
  }
}

// Element c of an array whose type is known at run time (weights read once per wave).
__device__ __forceinline__ float load_any(const void* p, eogp_dtype t, int64_t c) {
  if (t == EOGP_F32) return static_cast<const float*>(p)[c];
  if (t == EOGP_BF16) return (float)static_cast<const __bf16*>(p)[c];
  return (float)static_cast<const _Float16*>(p)[c];
}

__device__ __forceinline__ float wave_sum(float v) {
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

__device__ __forceinline__ float wave_max(float v) {
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
  return v;
}

// Calls f with the element type of a run-time dtype: f(T{}).
template <typename F>
inline eogp_status with_type(eogp_dtype t, F&& f) {
  if (t == EOGP_F32) return f(float{});
  if (t == EOGP_BF16) return f(__bf16{});
  return f(_Float16{});
}

}  // namespace eogp

namespace eogp {

// A row that a block of NT threads keeps in registers as read: P pieces of 16 bytes per thread, piece
// p of thread t at element (p NT + t) E; past the row's end the elements are -inf. The passes over it
// (each) take one piece at a time: pieces past the end cost a scalar branch, and the compiler neither
// keeps one pass's conversions for the next nor interleaves pieces, both of which cost more registers
// than the row has left.
template <typename T, int NT, int P>
struct RegisterRow {
  static constexpr int E = kPiece<T>;
  AnyVec<T, E> raw[P];

  __device__ __forceinline__ void load(const T* row, int64_t width) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = (int64_t)(p * NT + threadIdx.x) * E;
      if (c + E <= width) {
        raw[p] = *reinterpret_cast<const AnyVec<T, E>*>(row + c);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) raw[p][e] = c + e < width ? row[c + e] : (T)-INFINITY;
      }
    }
  }

  // f(p, index of the piece's first element, its elements as fp32)
  template <typename F>
  __device__ __forceinline__ void each(int64_t width, F&& f) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if ((int64_t)p * NT * E >= width) break;             // uniform
      asm volatile("" : "+v"(raw[p]));
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = (float)raw[p][e];
      f(p, (int64_t)(p * NT + threadIdx.x) * E, v);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// The same passes over a row that is too long for the registers: it is read in each.
template <typename T, int NT>
struct RegisterRow<T, NT, 0> {
  static constexpr int E = kPiece<T>;
  const T* row;

  __device__ __forceinline__ void load(const T* r, int64_t) { row = r; }

  template <typename F>
  __device__ __forceinline__ void each(int64_t width, F&& f) {
    auto piece = [&](int64_t c) {
      AnyVec<T, E> x;
      if (c + E <= width) {
        x = *reinterpret_cast<const AnyVec<T, E>*>(row + c);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = c + e < width ? row[c + e] : (T)-INFINITY;
      }
      return x;
    };
    int64_t c = (int64_t)threadIdx.x * E;
    AnyVec<T, E> next = piece(c);                          // the next piece is on its way while one is taken
    for (int p = 0; (int64_t)p * NT * E < width; ++p, c += NT * E) {
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = (float)next[e];
      if ((int64_t)(p + 1) * NT * E < width) next = piece(c + NT * E);
      f(p, c, v);
    }
  }
};

// Threads of the block that holds a row of `pieces` 16-byte pieces in registers, and pieces per
// thread; none (0) for rows longer than 1,024 threads x 16 pieces, which are read again instead.
template <typename F>
inline eogp_status with_row_shape(int64_t pieces, F&& f) {
  using std::integral_constant;
  using N256 = integral_constant<int, 256>;
  using N1024 = integral_constant<int, 1024>;
  if (pieces <= 512) return f(N256{}, integral_constant<int, 2>{});
  if (pieces <= 1024) return f(N256{}, integral_constant<int, 4>{});
  if (pieces <= 4096) return f(N1024{}, integral_constant<int, 4>{});
  if (pieces <= 8192) return f(N1024{}, integral_constant<int, 8>{});
  if (pieces <= 16384) return f(N1024{}, integral_constant<int, 16>{});
  return f(N1024{}, integral_constant<int, 0>{});
}
}  // namespace eogp
