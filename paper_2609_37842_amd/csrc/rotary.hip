// Rotary positions: the table of cosines and sines, and the pass that norms heads and turns their pairs.
#include <algorithm>
#include <cmath>

#include "attend.h"
#include "timing.h"

namespace eogp {
namespace {

// table[p][i] = magnitude (cos, sin)(p f_i), f_i = base^(-2i/width) (g_i + (1 - g_i) / factor), where g_i
// runs from 0 to 1 as the pair's turns over the original length run from low to high (0 without one).
// A far position times a frequency is many turns: frequencies, angles, cosines and sines are fp64, rounded
// once. Each thread has one frequency and every 8th position of its block's.
__global__ __launch_bounds__(256) void k_rotary_table(int64_t positions, int pairs, double log2_step, double inv_factor,
                                                      double turns, double low, double inv_range, double magnitude,
                                                      float* __restrict__ table) {
  const int i = blockIdx.y * 32 + (threadIdx.x & 31);
  if (i >= pairs) return;
  double f = exp2((double)i * log2_step);
  double stay = 0.0;
  if (turns > 0.0) stay = fmin(fmax((f * turns - low) * inv_range, 0.0), 1.0);
  f *= stay + (1.0 - stay) * inv_factor;
  for (int64_t p = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); p < positions; p += (int64_t)gridDim.x * 8) {
    double s, c;
    sincos((double)p * f, &s, &c);
    typedef float f32x2 __attribute__((ext_vector_type(2), aligned(4)));
    *reinterpret_cast<f32x2*>(table + (p * pairs + i) * 2) = f32x2{(float)(c * magnitude), (float)(s * magnitude)};
  }
}

enum Norm { kNormNone = 0, kNormHead = 1, kNormRow = 2 };

template <typename T>
struct RotateArgs {
  Heads<const T> in[2];           // queries, keys: inputs of the norm (forward, and backward where there is one)
  Heads<const T> grad[2];         // backward: gradients of the outputs
  Heads<T> out[2];
  const void* weight[2];
  eogp_dtype wt;
  int heads[2];
  int D, width;                   // elements of a head, of its turned part
  int interleaved;
  float eps, sin_sign;
  const float* table;
  int64_t positions;              // rows of the table
  const int64_t* at;              // position of each token, or NULL: its index in the example
  const uint8_t* mask;
  int64_t T_, tokens;             // tokens of an example, of a group (one example, or all)
  int shift;                      // 2^shift lanes hold a head
  int chunks[2];                  // waves (row norm: blocks) that share a token's heads, of queries and keys
  int splits;                     // workers that share a group's tokens
  int64_t groups;
  float* part;                    // backward: [groups][splits][chunks][part_ld] sums, or NULL
  int64_t part_ld;
};

// What a lane has of a head: E pairs of the turned part (both members), or 2 E elements of the rest.
template <typename T>
struct Slot {
  static constexpr int E = kPiece<T>;
  int ca, cb, end_a, end_b;       // first elements of its two pieces, and where these have to end
  bool turned, together;          // a pair's members alternate in memory
  bool any;

  __device__ __forceinline__ void place(int slot, int D, int width, int interleaved) {
    const int half = width >> 1, turning = (half + E - 1) / E;
    turned = slot < turning;
    together = turned && interleaved;
    if (turned && !interleaved) {
      ca = slot * E;
      cb = half + ca;
      end_a = half;
      end_b = width;
    } else {
      ca = turned ? 2 * E * slot : width + 2 * E * (slot - turning);
      cb = ca + E;
      end_a = end_b = turned ? width : D;
    }
    any = ca < end_a;
  }
};

template <typename T>
struct Raw {
  AnyVec<T, kPiece<T>> a, b;
  __device__ __forceinline__ void request(const Slot<T>& s, const T* row, int D) {
    constexpr int E = kPiece<T>;
    if (D >= E) {
      a = request_piece<T, E, false>(row, s.ca, D);
      b = request_piece<T, E, false>(row, s.cb, D);
    } else {
      a = fetch_piece<T, E>(row, s.ca, D, (T)0.f);
      b = fetch_piece<T, E>(row, s.cb, D, (T)0.f);
    }
  }
};

// A slot's elements as fp32, zero past its end: pair members in a and b, or its first and second piece.
template <typename T>
struct Values {
  static constexpr int E = kPiece<T>;
  float a[E], b[E];

  __device__ __forceinline__ void take(const Slot<T>& s, Raw<T> r, int D) {
    if (D >= E) {
      settle_piece<T, E, false>(r.a, s.ca, D);
      settle_piece<T, E, false>(r.b, s.cb, D);
    }
    float u[E], v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u[e] = s.ca + e < s.end_a ? (float)r.a[e] : 0.f;
      v[e] = s.cb + e < s.end_b ? (float)r.b[e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float even = e < E / 2 ? u[2 * e % E] : v[2 * e % E], odd = e < E / 2 ? u[(2 * e + 1) % E] : v[(2 * e + 1) % E];
      a[e] = s.together ? even : u[e];
      b[e] = s.together ? odd : v[e];
    }
  }
  __device__ __forceinline__ void put(const Slot<T>& s, T* row) const {
    float u[E], v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float fu = e % 2 ? b[e / 2] : a[e / 2], fv = e % 2 ? b[E / 2 + e / 2] : a[E / 2 + e / 2];
      u[e] = s.together ? fu : a[e];
      v[e] = s.together ? fv : b[e];
    }
    store_piece<T, E>(row, s.ca, s.end_a, u);
    store_piece<T, E>(row, s.cb, s.end_b, v);
  }
  __device__ __forceinline__ float square() const {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += a[e] * a[e] + b[e] * b[e];
    return s;
  }
};

// Cosines and sines of a slot's pairs: 1 and 0 for the part that is not turned, NaN for a position that
// the table does not have.
template <typename T>
struct Turn {
  static constexpr int E = kPiece<T>;
  float c[E], s[E];
  __device__ __forceinline__ void load(const Slot<T>& slot, const float* table, int64_t positions, int64_t p, int width,
                                       float sign) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      c[e] = 1.f;
      s[e] = 0.f;
    }
    if (!slot.turned) return;
    const bool known = p >= 0 && p < positions;
    const float* row = table + (known ? p : 0) * width;
    const int first = slot.together ? slot.ca : 2 * slot.ca;
#pragma unroll
    for (int u = 0; u < E / 2; ++u) {
      const AnyVec<float, 4> x = fetch_piece<float, 4>(row, first + 4 * u, width, 0.f);
      c[2 * u] = known ? x[0] : NAN;
      s[2 * u] = known ? x[1] * sign : NAN;
      c[2 * u + 1] = known ? x[2] : NAN;
      s[2 * u + 1] = known ? x[3] * sign : NAN;
    }
  }
  __device__ __forceinline__ void apply(Values<T>& v) const {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float a = v.a[e], b = v.b[e];
      v.a[e] = a * c[e] - b * s[e];
      v.b[e] = a * s[e] + b * c[e];
    }
  }
};

// Tokens first, first + step, ... below n of a group, masks and positions of 64 at once.
struct TokenQueue {
  int64_t first, step, n, base, length;
  const uint8_t* mask;
  const int64_t* at;
  uint64_t left = 0;
  int lane_mask = 0;
  int64_t lane_at = 0;
  int64_t position;               // of the token that next returned
  bool live;

  __device__ __forceinline__ TokenQueue(const uint8_t* m, const int64_t* a, int64_t f, int64_t st, int64_t rows, int64_t b,
                                        int64_t len)
      : first(f - 64 * st), step(st), n(rows), base(b), length(len), mask(m), at(a) {}

  __device__ __forceinline__ int64_t next() {
    if (!left) {
      first += 64 * step;
      if (first >= n) return -1;
      const int64_t mine = first + (threadIdx.x & 63) * step;
      const bool in = mine < n;
      left = __ballot(in);
      lane_mask = in && (!mask || mask[base + mine] != 0);
      lane_at = !in ? 0 : at ? at[base + mine] : (base + mine) % length;
    }
    const int k = __builtin_ctzll(left);
    left &= left - 1;
    live = __builtin_amdgcn_readlane(lane_mask, k);
    position = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(lane_at >> 32), k) << 32 |
                         (uint32_t)__builtin_amdgcn_readlane((int)lane_at, k));
    return base + first + k * step;
  }
};

__device__ __forceinline__ float lanes_sum(float v, int shift) {
  for (int m = 1; m < 1 << shift; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

// Sums of two values over the threads of a block; `slot` is LDS for two floats a wave, another one for the next sums.
template <int NT>
__device__ __forceinline__ float2 block_sums(float u, float v, float2* slot) {
  u = wave_sum(u);
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = float2{u, v};
  __syncthreads();
  float2 s = slot[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) {
    s.x += slot[w].x;
    s.y += slot[w].y;
  }
  return s;
}

template <typename T>
__device__ __forceinline__ void load_weights(const RotateArgs<T>& a, const Slot<T>& s, int tensor, int64_t from, Values<T>& w) {
  constexpr int E = kPiece<T>;
  const void* p = a.weight[tensor];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int ia = s.together ? s.ca + 2 * e : s.ca + e, ib = s.together ? s.ca + 2 * e + 1 : s.cb + e;
    w.a[e] = p && ia < s.end_a ? load_any(p, a.wt, from + ia) : 1.f;
    w.b[e] = p && ib < s.end_b ? load_any(p, a.wt, from + ib) : 1.f;
  }
}

// y = R_p (x rstd w): each head is read once and written once. A wave holds 64 >> shift heads of a token at a
// time (row norm: a block of four waves the whole row), R of them after one another, and requests the next
// token's while it works; a token's cosines and sines are read once per wave.
template <typename T, int NORM, int NT, int R>
__global__ __launch_bounds__(NT) void k_rotate(const RotateArgs<T> a) {
  constexpr bool kRow = NORM == kNormRow;
  __shared__ float2 sums[2][kRow ? NT / 64 : 1];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int place = kRow ? (int)threadIdx.x : lane, width_of = kRow ? NT : 64;    // among the threads that share a token
  const int chunks = a.chunks[0] + a.chunks[1];
  const int64_t worker = kRow ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wid;
  if (worker >= (int64_t)chunks * a.splits) return;
  const int chunk = (int)(worker % chunks);
  const int64_t split = worker / chunks;
  const int tensor = chunk >= a.chunks[0], H = a.heads[tensor];
  const int head0 = (chunk - (tensor ? a.chunks[0] : 0)) * R * (width_of >> a.shift) + (place >> a.shift);
  Slot<T> slot;
  slot.place(place & ((1 << a.shift) - 1), a.D, a.width, a.interleaved);
  TokenQueue queue(a.mask, a.at, split, a.splits, a.tokens, 0, a.T_);
  const int step = width_of >> a.shift;
  Raw<T> raw[R];
  auto request = [&](int64_t token) {
    const T* base = a.in[tensor].row(token / a.T_, token % a.T_, 0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int head = head0 + r * step;
      raw[r].request(slot, base + (int64_t)(head < H ? head : 0) * a.in[tensor].ld_h, a.D);
    }
  };
  int turn_no = 0;
  int64_t token = queue.next();
  if (token >= 0 && queue.live) request(token);
  while (token >= 0) {
    const bool live = queue.live;
    T* out = a.out[tensor].row(token / a.T_, token % a.T_, 0);
    Values<T> v[R];
    if (live) {
      Turn<T> turn;
      turn.load(slot, a.table, a.positions, queue.position, a.width, a.sin_sign);
#pragma unroll
      for (int r = 0; r < R; ++r) v[r].take(slot, raw[r], a.D);
      token = queue.next();
      if (token >= 0 && queue.live) request(token);
      if constexpr (NORM != kNormNone) {
        float row = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int head = head0 + r * step;
          float s = slot.any && head < H ? v[r].square() : 0.f;
          if constexpr (kRow) {
            row += s;
          } else {
            s = lanes_sum(s, a.shift);
            const float rstd = 1.f / sqrtf(s / (float)a.D + a.eps);
            Values<T> w;
            load_weights<T>(a, slot, tensor, 0, w);
#pragma unroll
            for (int e = 0; e < kPiece<T>; ++e) {
              v[r].a[e] *= rstd * w.a[e];
              v[r].b[e] *= rstd * w.b[e];
            }
          }
        }
        if constexpr (kRow) {
          row = block_sums<NT>(row, 0.f, sums[turn_no]).x;
          turn_no ^= 1;
          const float rstd = 1.f / sqrtf(row / (float)((int64_t)H * a.D) + a.eps);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const int head = head0 + r * step;
            if (head >= H) continue;
            Values<T> w;
            load_weights<T>(a, slot, tensor, (int64_t)head * a.D, w);
#pragma unroll
            for (int e = 0; e < kPiece<T>; ++e) {
              v[r].a[e] *= rstd * w.a[e];
              v[r].b[e] *= rstd * w.b[e];
            }
          }
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) turn.apply(v[r]);
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < kPiece<T>; ++e) v[r].a[e] = v[r].b[e] = 0.f;
      token = queue.next();
      if (token >= 0 && queue.live) request(token);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int head = head0 + r * step;
      if (slot.any && head < H) v[r].put(slot, out + (int64_t)head * a.out[tensor].ld_h);
    }
  }
}

// With t = R_p^T dy, xh = x rstd: dx = rstd (t w - xh mean(t w xh)), and sums of t xh over the worker's tokens (and
// heads, where each has its own norm), which k_rotate_fold adds up in order.
template <typename T, int NORM, int NT, int R>
__global__ __launch_bounds__(NT) void k_rotate_back(const RotateArgs<T> a) {
  constexpr bool kRow = NORM == kNormRow;
  constexpr int E = kPiece<T>;
  __shared__ float2 sums[2][kRow ? NT / 64 : 1];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int place = kRow ? (int)threadIdx.x : lane, width_of = kRow ? NT : 64;
  const int chunks = a.chunks[0] + a.chunks[1];
  const int64_t worker = kRow ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wid;
  if (worker >= (int64_t)chunks * a.splits * a.groups) return;
  const int chunk = (int)(worker % chunks);
  const int64_t split = worker / chunks % a.splits, group = worker / chunks / a.splits;
  const int tensor = chunk >= a.chunks[0], H = a.heads[tensor];
  const int step = width_of >> a.shift;
  const int head0 = (chunk - (tensor ? a.chunks[0] : 0)) * R * step + (place >> a.shift);
  Slot<T> slot;
  slot.place(place & ((1 << a.shift) - 1), a.D, a.width, a.interleaved);
  TokenQueue queue(a.mask, a.at, split, a.splits, a.tokens, group * a.tokens, a.T_);
  Raw<T> rx[R], rg[R];
  auto request = [&](int64_t token) {
    const T* base = a.in[tensor].row(token / a.T_, token % a.T_, 0);
    const T* grad = a.grad[tensor].row(token / a.T_, token % a.T_, 0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int head = head0 + r * step, from = head < H ? head : 0;
      rx[r].request(slot, base + (int64_t)from * a.in[tensor].ld_h, a.D);
      rg[r].request(slot, grad + (int64_t)from * a.grad[tensor].ld_h, a.D);
    }
  };
  Values<T> dw[kRow ? R : 1];
#pragma unroll
  for (int r = 0; r < (kRow ? R : 1); ++r)
#pragma unroll
    for (int e = 0; e < E; ++e) dw[r].a[e] = dw[r].b[e] = 0.f;
  int turn_no = 0;
  int64_t token = queue.next();
  if (token >= 0 && queue.live) request(token);
  while (token >= 0) {
    const bool live = queue.live;
    T* out = a.out[tensor].row(token / a.T_, token % a.T_, 0);
    Values<T> x[R], t[R];
    if (live) {
      Turn<T> turn;
      turn.load(slot, a.table, a.positions, queue.position, a.width, -a.sin_sign);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        x[r].take(slot, rx[r], a.D);
        t[r].take(slot, rg[r], a.D);
        turn.apply(t[r]);
      }
      token = queue.next();
      if (token >= 0 && queue.live) request(token);
      float row = 0.f, dot = 0.f;
      Values<T> w[kRow ? R : 1];
      if constexpr (!kRow) load_weights<T>(a, slot, tensor, 0, w[0]);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int head = head0 + r * step;
        const bool in = slot.any && head < H;
        Values<T>& wr = w[kRow ? r : 0];
        if constexpr (kRow) load_weights<T>(a, slot, tensor, (int64_t)(head < H ? head : 0) * a.D, wr);
        float s = in ? x[r].square() : 0.f, d = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) d += t[r].a[e] * wr.a[e] * x[r].a[e] + t[r].b[e] * wr.b[e] * x[r].b[e];
        d = in ? d : 0.f;
        if constexpr (kRow) {
          row += s;
          dot += d;
        } else {
          s = lanes_sum(s, a.shift);
          d = lanes_sum(d, a.shift);
          const float rstd = 1.f / sqrtf(s / (float)a.D + a.eps), m = d * rstd / (float)a.D;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float ha = x[r].a[e] * rstd, hb = x[r].b[e] * rstd;
            if (in) {
              dw[0].a[e] += t[r].a[e] * ha;
              dw[0].b[e] += t[r].b[e] * hb;
            }
            x[r].a[e] = rstd * (t[r].a[e] * wr.a[e] - ha * m);
            x[r].b[e] = rstd * (t[r].b[e] * wr.b[e] - hb * m);
          }
        }
      }
      if constexpr (kRow) {
        const float n = (float)((int64_t)H * a.D);
        const float2 both = block_sums<NT>(row, dot, sums[turn_no]);
        turn_no ^= 1;
        const float rstd = 1.f / sqrtf(both.x / n + a.eps), m = both.y * rstd / n;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float ha = x[r].a[e] * rstd, hb = x[r].b[e] * rstd;
            dw[r].a[e] += t[r].a[e] * ha;
            dw[r].b[e] += t[r].b[e] * hb;
            x[r].a[e] = rstd * (t[r].a[e] * w[r].a[e] - ha * m);
            x[r].b[e] = rstd * (t[r].b[e] * w[r].b[e] - hb * m);
          }
      }
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < E; ++e) x[r].a[e] = x[r].b[e] = 0.f;
      token = queue.next();
      if (token >= 0 && queue.live) request(token);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int head = head0 + r * step;
      if (slot.any && head < H) x[r].put(slot, out + (int64_t)head * a.out[tensor].ld_h);
    }
  }
  if (!a.part) return;
  float* part = a.part + worker * a.part_ld;
#pragma unroll
  for (int r = 0; r < (kRow ? R : 1); ++r) {
    const int head = head0 + r * step;
    if constexpr (!kRow) {                     // the wave's heads
      for (int m = 1 << a.shift; m < 64; m <<= 1)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          dw[0].a[e] += __shfl_xor(dw[0].a[e], m);
          dw[0].b[e] += __shfl_xor(dw[0].b[e], m);
        }
    }
    if (!slot.any || (kRow ? head >= H : (place >> a.shift) != 0)) continue;
    float* to = part + (kRow ? (int64_t)head * a.D : 0);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int ia = slot.together ? slot.ca + 2 * e : slot.ca + e, ib = slot.together ? slot.ca + 2 * e + 1 : slot.cb + e;
      if (ia < slot.end_a) to[ia] = dw[r].a[e];
      if (ib < slot.end_b) to[ib] = dw[r].b[e];
    }
  }
}

// Sums of the workers' parts, in a fixed order: 32 columns x 8 slices of the workers per block.
__global__ __launch_bounds__(256) void k_rotate_fold(const float* __restrict__ part, int64_t part_ld, int64_t groups,
                                                     int splits, int chunks, int first, int count, int64_t n,
                                                     float* __restrict__ out) {
  __shared__ float sum[8][33];
  const int col = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int64_t col_blocks = (n + 31) / 32;
  for (int64_t unit = blockIdx.x; unit < groups * col_blocks; unit += gridDim.x) {
    const int64_t group = unit / col_blocks, c = unit % col_blocks * 32 + col;
    float s = 0.f;
    if (c < n)
      for (int64_t j = slice; j < (int64_t)splits * count; j += 8)
        s += part[((group * splits + j / count) * chunks + first + j % count) * part_ld + c];
    sum[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < n) {
#pragma unroll
      for (int k = 1; k < 8; ++k) s += sum[k][col];
      out[group * n + c] = s;
    }
    __syncthreads();
  }
}

// How a token's heads and a group's tokens are shared out.
struct RotatePlan {
  int shift, threads, reps, chunks[2];
  int64_t splits, part_ld;
};

constexpr int64_t kRotateWorkers = 8192;       // waves that are there at once, about

RotatePlan rotate_plan(eogp_dtype t, int norm, int Hq, int Hk, int64_t D, int64_t width, int64_t groups, int64_t tokens,
                       bool back) {
  RotatePlan p;
  const int E = t == EOGP_F32 ? 4 : 8;
  const int64_t slots = ceil_div(width / 2, E) + ceil_div(D - width, 2 * E);
  p.shift = 0;
  while ((1 << p.shift) < slots) ++p.shift;
  const int at_once = 64 >> p.shift;           // heads of a wave
  const int heads[2] = {Hq, Hk};
  p.threads = 256;
  if (norm == kNormRow) {
    const int64_t lanes = (int64_t)std::max(Hq, Hk) << p.shift;
    if (lanes > 512) p.threads = 1024;
    p.reps = 1;
    while (p.reps * p.threads < lanes) p.reps *= 2;
    for (int i = 0; i < 2; ++i) p.chunks[i] = heads[i] > 0;
    p.part_ld = std::max(Hq, Hk) * D;
  } else {
    // more heads a wave only where there are waves enough without
    p.reps = groups * tokens * ceil_div(Hq + Hk, at_once) >= 4 * kRotateWorkers ? 2 : 1;
    for (int i = 0; i < 2; ++i) p.chunks[i] = (int)ceil_div(heads[i], at_once * p.reps);
    p.part_ld = D;
  }
  const int64_t want = norm == kNormRow ? kRotateWorkers * 64 / p.threads : back ? kRotateWorkers / 2 : kRotateWorkers;
  p.splits = std::min(std::max<int64_t>(1, tokens), std::max<int64_t>(1, want / std::max<int64_t>(1, groups * (p.chunks[0] + p.chunks[1]))));
  return p;
}

template <typename T>
RotateArgs<T> rotate_args(const eogp_heads* in, const eogp_heads* grad, const eogp_heads* out, int64_t D, const void* qw,
                          const void* kw, eogp_dtype wt, float eps, const float* table, int64_t positions, int64_t width,
                          int interleaved, const int64_t* at, const uint8_t* mask, int64_t T_, const RotatePlan& p) {
  RotateArgs<T> a{};
  for (int i = 0; i < 2; ++i) {
    if (in) a.in[i] = Heads<const T>{static_cast<const T*>(in[i].data), in[i].ld_example, in[i].ld_token, in[i].ld_head};
    if (grad) a.grad[i] = Heads<const T>{static_cast<const T*>(grad[i].data), grad[i].ld_example, grad[i].ld_token, grad[i].ld_head};
    a.out[i] = heads_of<T>(out[i]);
    a.heads[i] = (int)out[i].heads;
    a.chunks[i] = p.chunks[i];
  }
  a.weight[0] = qw;
  a.weight[1] = kw;
  a.wt = wt;
  a.D = (int)D;
  a.width = (int)width;
  a.interleaved = interleaved;
  a.eps = eps;
  a.sin_sign = 1.f;
  a.table = table;
  a.positions = positions;
  a.at = at;
  a.mask = mask;
  a.T_ = T_;
  a.shift = p.shift;
  a.splits = (int)p.splits;
  a.part_ld = p.part_ld;
  a.groups = 1;
  return a;
}

// Threads of a block and heads that a lane holds. (fp32 rows of up to 8,192 elements in heads of 8 or more take up to
// 4,096 lanes, 16-bit ones 2,048.)
template <typename T, int NORM, typename F>
eogp_status with_shape(const RotatePlan& p, F&& f) {
  using std::integral_constant;
  using N256 = integral_constant<int, 256>;
  using N1024 = integral_constant<int, 1024>;
  using One = integral_constant<int, 1>;
  using Two = integral_constant<int, 2>;
  if (p.threads == 256) return p.reps == 1 ? f(N256{}, One{}) : f(N256{}, Two{});
  if constexpr (NORM == kNormRow) {
    if (p.reps == 1) return f(N1024{}, One{});
    if constexpr (sizeof(T) == 4)
      if (p.reps > 2) return f(N1024{}, integral_constant<int, 4>{});
    return f(N1024{}, Two{});
  }
  return EOGP_ERR_UNSUPPORTED;
}

template <typename F>
eogp_status with_norm(int norm, F&& f) {
  using std::integral_constant;
  if (norm == kNormHead) return f(integral_constant<int, kNormHead>{});
  if (norm == kNormRow) return f(integral_constant<int, kNormRow>{});
  return f(integral_constant<int, kNormNone>{});
}

unsigned rotate_blocks(int norm, int64_t workers) { return (unsigned)(norm == kNormRow ? workers : ceil_div(workers, 4)); }

}  // namespace

eogp_status rotary_table(int64_t positions, int64_t width, double base, double factor, double original, double low,
                         double high, double magnitude, float* table, hipStream_t s) {
  if (positions == 0) return EOGP_OK;
  timing::Scope ts(EOGP_KT_ROTARY, s);
  const int pairs = (int)(width / 2);
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(positions, 8), 2048), (unsigned)ceil_div(pairs, 32));
  hipLaunchKernelGGL(k_rotary_table, grid, dim3(256), 0, s, positions, pairs, -2.0 / (double)width * std::log2(base),
                     1.0 / factor, original / (2.0 * M_PI), low, 1.0 / (high - low), magnitude, table);
  EOGP_LAUNCH_CHECK("rotary_table");
  return EOGP_OK;
}

eogp_status rotate_heads(const eogp_heads* in, const eogp_heads* out, eogp_dtype t, int norm, const void* qw,
                         const void* kw, eogp_dtype wt, float eps, const float* table, int64_t positions, int64_t width,
                         int interleaved, bool back, const int64_t* at, const uint8_t* mask, int64_t N, int64_t T_,
                         int64_t D, hipStream_t s) {
  if (N * T_ == 0) return EOGP_OK;
  const RotatePlan p = rotate_plan(t, norm, (int)out[0].heads, (int)out[1].heads, D, width, 1, N * T_, false);
  timing::Scope ts(EOGP_KT_ROTARY, s);
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    RotateArgs<T> a = rotate_args<T>(in, nullptr, out, D, qw, kw, wt, eps, table, positions, width, interleaved, at, mask, T_, p);
    a.tokens = N * T_;
    a.sin_sign = back ? -1.f : 1.f;
    return with_norm(norm, [&](auto nm) {
      constexpr int NORM = decltype(nm)::value;
      return with_shape<T, NORM>(p, [&](auto nt, auto reps) {
        hipLaunchKernelGGL((k_rotate<T, NORM, decltype(nt)::value, decltype(reps)::value>),
                           dim3(rotate_blocks(norm, p.splits * (p.chunks[0] + p.chunks[1]))), dim3(p.threads), 0, s, a);
        EOGP_LAUNCH_CHECK("rotate_heads");
        return EOGP_OK;
      });
    });
  });
}

// Elements of a row that one norm takes.
int64_t rotate_max_row(int64_t D) { return D < 8 ? 2048 : 8192; }

size_t rotate_back_ws(eogp_dtype t, int norm, int64_t Hq, int64_t Hk, int64_t D, int64_t width, int64_t groups, int64_t tokens) {
  // the workers of any call of up to `groups` groups of up to `tokens` tokens, with one head a lane
  const RotatePlan p = rotate_plan(t, norm, (int)Hq, (int)Hk, D, width, 1, 1, true);
  const int64_t chunks = p.chunks[0] + p.chunks[1];
  const int64_t workers = std::min(groups * tokens * chunks, std::max(kRotateWorkers / 2, groups * chunks));
  return align256((size_t)std::max<int64_t>(workers, groups * chunks) * p.part_ld * sizeof(float));
}

eogp_status rotate_heads_back(const eogp_heads* in, const eogp_heads* grad, const eogp_heads* out, eogp_dtype t, int norm,
                              const void* qw, const void* kw, eogp_dtype wt, float eps, const float* table,
                              int64_t positions, int64_t width, int interleaved, const int64_t* at, const uint8_t* mask,
                              int64_t N, int64_t T_, int64_t D, bool per_example, float* dqw, float* dkw, void* ws,
                              hipStream_t s) {
  const int64_t groups = per_example ? N : 1, tokens = per_example ? T_ : N * T_;
  if (groups == 0) return EOGP_OK;
  const RotatePlan p = rotate_plan(t, norm, (int)out[0].heads, (int)out[1].heads, D, width, groups, tokens, true);
  const int chunks = p.chunks[0] + p.chunks[1];
  const int64_t workers = groups * p.splits * chunks;
  float* part = dqw || dkw ? static_cast<float*>(ws) : nullptr;
  timing::Scope ts(EOGP_KT_ROTARY, s);
  const eogp_status st = with_type(t, [&](auto el) {
    using T = decltype(el);
    RotateArgs<T> a = rotate_args<T>(in, grad, out, D, qw, kw, wt, eps, table, positions, width, interleaved, at, mask, T_, p);
    a.tokens = tokens;
    a.groups = groups;
    a.part = part;
    auto go = [&](auto nm) {
      constexpr int NORM = decltype(nm)::value;
      return with_shape<T, NORM>(p, [&](auto nt, auto reps) {
        hipLaunchKernelGGL((k_rotate_back<T, NORM, decltype(nt)::value, decltype(reps)::value>),
                           dim3(rotate_blocks(norm, workers)), dim3(p.threads), 0, s, a);
        EOGP_LAUNCH_CHECK("rotate_heads_backward");
        return EOGP_OK;
      });
    };
    using std::integral_constant;
    return norm == kNormRow ? go(integral_constant<int, kNormRow>{}) : go(integral_constant<int, kNormHead>{});
  });
  if (st != EOGP_OK) return st;
  float* outs[2] = {dqw, dkw};
  for (int i = 0; i < 2; ++i) {
    if (!outs[i] || !p.chunks[i]) continue;
    const int64_t n = norm == kNormRow ? out[i].heads * D : D;
    hipLaunchKernelGGL(k_rotate_fold, dim3((unsigned)std::min<int64_t>(groups * ceil_div(n, 32), 1 << 20)), dim3(256), 0, s,
                       part, p.part_ld, groups, (int)p.splits, chunks, i ? p.chunks[0] : 0, p.chunks[i], n, outs[i]);
    EOGP_LAUNCH_CHECK("rotate_heads_backward (fold)");
  }
  return EOGP_OK;
}

}  // namespace eogp
