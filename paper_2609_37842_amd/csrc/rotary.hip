// Rotary positions: the table of cosines and sines, and the pass that norms heads and turns their pairs.
#include <algorithm>
#include <cmath>

#include "attend.h"
#include "timing.h"
#include "token_walk.h"

namespace eogp {
namespace {

// table[p][i] = magnitude (cos, sin)(p f_i), f_i = base^(-2i/width) (g_i + (1 - g_i) / factor), where g_i
// runs from 0 to 1 as the pair's turns over the original length run from low to high (0 without one).
// A far position times a frequency is many turns: frequencies, angles, cosines and sines are fp64, rounded
// once. A thread has one frequency and K positions 8 apart: the sine and cosine of the first are computed,
// those of the others follow by K - 1 turns of 8 f (a product of complex numbers, 2^-52 of error each). 131,072 positions of
// 128: 13 us, the rate of a copy of its 67 MB; 24 us with a sine and a cosine each (bound by fp64 arithmetic).
__global__ __launch_bounds__(256) void k_rotary_table(int64_t positions, int pairs, int K, double log2_step, double inv_factor,
                                                      double turns, double low, double inv_range, double magnitude,
                                                      float* __restrict__ table) {
  const int i = blockIdx.y * 32 + (threadIdx.x & 31);
  int64_t p = (int64_t)blockIdx.x * 8 * K + (threadIdx.x >> 5);
  if (i >= pairs || p >= positions) return;
  double f = exp2((double)i * log2_step);
  double stay = 0.0;
  if (turns > 0.0) stay = fmin(fmax((f * turns - low) * inv_range, 0.0), 1.0);
  f *= stay + (1.0 - stay) * inv_factor;
  double s, c, ds = 0.0, dc = 1.0;
  sincos((double)p * f, &s, &c);
  s *= magnitude;
  c *= magnitude;
  if (K > 1) sincos(8.0 * f, &ds, &dc);
  for (int k = 0; k < K && p < positions; ++k, p += 8) {
    typedef float f32x2 __attribute__((ext_vector_type(2), aligned(4)));
    const f32x2 v{(float)c, (float)s};
    __builtin_nontemporal_store(v, reinterpret_cast<f32x2*>(table + (p * pairs + i) * 2));
    const double t = c * dc - s * ds;
    s = s * dc + c * ds;
    c = t;
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
  int tokens;                     // of a group (one example, or all)
  Divide by_length;               // tokens of an example
  int shift;                      // 2^shift lanes hold a head
  int chunks[2];                  // workers that share a token's heads, of queries and keys
  int splits;                     // blocks that share a group's tokens, for each chunk
  uint32_t block0;                // of the first block of the launch, among all of the call (fewer than 2^32)
  float* part;                    // backward: [groups][splits][chunks][part_ld] sums, or NULL
  int64_t part_ld;
};

// How a head lies in the lanes: any widths; or all pieces whole, with a pair's members in halves, or side by side.
enum Layout { kAny = 0, kHalves = 1, kPairs = 2 };

// What a lane has of a head: E pairs of the turned part (both members), or 2 E elements of the rest.
template <typename T, int LAYOUT>
struct Slot {
  static constexpr int E = kPiece<T>;
  int ca, cb, end_a, end_b;       // first elements of its two pieces, and where these have to end
  bool turned;
  bool pairs;                     // a pair's members alternate in memory
  bool any;

  __device__ __forceinline__ void place(int slot, int D, int width, int interleaved) {
    const int half = width >> 1, turning = (half + E - 1) / E;
    turned = slot < turning;
    pairs = turned && (LAYOUT == kAny ? interleaved != 0 : LAYOUT == kPairs);
    if (turned && !pairs) {
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
    if (!any) ca = cb = 0;
  }
  // The place in a head of element e of a and of b.
  __device__ __forceinline__ int at_a(int e) const { return pairs ? ca + 2 * e : ca + e; }
  __device__ __forceinline__ int at_b(int e) const { return pairs ? ca + 2 * e + 1 : cb + e; }
};

template <typename T, int LAYOUT>
struct Raw {
  static constexpr int E = kPiece<T>;
  AnyVec<T, E> a, b;
  __device__ __forceinline__ void request(const Slot<T, LAYOUT>& s, const T* row, int D) {
    if constexpr (LAYOUT != kAny) {
      a = *reinterpret_cast<const AnyVec<T, E>*>(row + s.ca);
      b = *reinterpret_cast<const AnyVec<T, E>*>(row + s.cb);
    } else if (D >= E) {
      a = request_piece<T, E, false>(row, s.ca, D);
      b = request_piece<T, E, false>(row, s.cb, D);
    } else {
      a = fetch_piece<T, E>(row, s.ca, D, (T)0.f);
      b = fetch_piece<T, E>(row, s.cb, D, (T)0.f);
    }
  }
};

// A slot's elements as fp32, zero past its end: pair members in a and b, or its first and second piece.
template <typename T, int LAYOUT>
struct Values {
  static constexpr int E = kPiece<T>;
  float a[E], b[E];

  __device__ __forceinline__ void take(const Slot<T, LAYOUT>& s, Raw<T, LAYOUT> r, int D) {
    if constexpr (LAYOUT == kAny) {
      if (D >= E) {
        settle_piece<T, E, false>(r.a, s.ca, D);
        settle_piece<T, E, false>(r.b, s.cb, D);
      }
    }
    float u[E], v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u[e] = (float)r.a[e];
      v[e] = (float)r.b[e];
      if constexpr (LAYOUT == kAny) {
        u[e] = s.ca + e < s.end_a ? u[e] : 0.f;
        v[e] = s.cb + e < s.end_b ? v[e] : 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float even = e < E / 2 ? u[2 * e % E] : v[2 * e % E], odd = e < E / 2 ? u[(2 * e + 1) % E] : v[(2 * e + 1) % E];
      a[e] = LAYOUT == kHalves ? u[e] : s.pairs ? even : u[e];
      b[e] = LAYOUT == kHalves ? v[e] : s.pairs ? odd : v[e];
    }
  }
  __device__ __forceinline__ void put(const Slot<T, LAYOUT>& s, T* row) const {
    AnyVec<T, E> x, y;
    float u[E], v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float fu = e % 2 ? b[e / 2] : a[e / 2], fv = e % 2 ? b[E / 2 + e / 2] : a[E / 2 + e / 2];
      u[e] = LAYOUT == kHalves ? a[e] : s.pairs ? fu : a[e];
      v[e] = LAYOUT == kHalves ? b[e] : s.pairs ? fv : b[e];
      x[e] = (T)u[e];
      y[e] = (T)v[e];
    }
    if constexpr (LAYOUT != kAny) {
      *reinterpret_cast<AnyVec<T, E>*>(row + s.ca) = x;
      *reinterpret_cast<AnyVec<T, E>*>(row + s.cb) = y;
    } else {
      store_piece<T, E>(row, s.ca, s.end_a, u);
      store_piece<T, E>(row, s.cb, s.end_b, v);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < E; ++e) a[e] = b[e] = 0.f;
  }
  __device__ __forceinline__ float square() const {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += a[e] * a[e] + b[e] * b[e];
    return s;
  }
};

// Cosines and sines of a slot's pairs, NaN for a position that the table does not have.
template <typename T, int LAYOUT>
struct Turn {
  static constexpr int E = kPiece<T>;
  AnyVec<float, 4> x[E / 2];
  bool known;
  __device__ __forceinline__ void request(const Slot<T, LAYOUT>& slot, const float* table, int64_t positions, int64_t p, int width) {
    known = p >= 0 && p < positions;
    if (!slot.turned) return;
    const float* row = table + (known ? p : 0) * width;
    const int first = slot.pairs ? slot.ca : 2 * slot.ca;
    if (positions == 0) return;
#pragma unroll
    for (int u = 0; u < E / 2; ++u) {
      if constexpr (LAYOUT != kAny)
        x[u] = *reinterpret_cast<const AnyVec<float, 4>*>(row + first + 4 * u);
      else
        x[u] = fetch_piece<float, 4>(row, first + 4 * u, width, 0.f);
    }
  }
  // (Selects, no product with 1 and 0: elements behind the turned part pass whatever their neighbours hold.)
  __device__ __forceinline__ void apply(const Slot<T, LAYOUT>& slot, float sign, Values<T, LAYOUT>& v) const {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float c = known ? x[e / 2][2 * (e % 2)] : NAN, s = known ? x[e / 2][2 * (e % 2) + 1] * sign : NAN;
      const float a = v.a[e], b = v.b[e];
      v.a[e] = slot.turned ? a * c - b * s : a;
      v.b[e] = slot.turned ? a * s + b * c : b;
    }
  }
};

// Tokens first, first + step, ... below n of a group, masks and positions of 64 at once.
struct TokenQueue {
  TokenWalk walk;
  int base;
  const uint8_t* mask;
  const int64_t* at;
  const Divide& by_length;
  uint64_t left = 0;
  int lane_mask = 0;
  int64_t lane_at = 0;
  int64_t position;               // of the token that next returned
  int example, index;
  bool live;

  __device__ __forceinline__ TokenQueue(const uint8_t* m, const int64_t* a, int f, int st, int rows, int b, const Divide& len)
      : walk(f, st, rows), base(b), mask(m), at(a), by_length(len) {}

  // False at the end.
  __device__ __forceinline__ bool next() {
    if (!left) {
      if (!walk.next()) return false;
      const int lane = threadIdx.x & 63;
      const bool in = walk.has(lane);
      const int64_t mine = base + walk.at(lane);
      left = __ballot(in);
      lane_mask = in && (!mask || mask[mine] != 0);
      lane_at = in && at ? at[mine] : 0;
    }
    const int k = __builtin_ctzll(left), token = base + (int)walk.at(k);
    left &= left - 1;
    live = __builtin_amdgcn_readlane(lane_mask, k);
    example = by_length.quotient(token);
    index = by_length.rest(token, example);
    position = at ? (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(lane_at >> 32), k) << 32 |
                              (uint32_t)__builtin_amdgcn_readlane((int)lane_at, k))
                  : index;
    return true;
  }
};

// Sum over the 2^shift lanes that hold a head.
__device__ __forceinline__ float lanes_sum(float v, int shift) {
  for (int m = 1; m < 1 << shift; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

// Sums of two values over the threads of a block (of one wave: over it); `slot` is LDS for two floats a wave, another
// one for the next sums.
template <int NT>
__device__ __forceinline__ float2 row_sums(float u, float v, float2* slot) {
  u = wave_sum(u);
  v = wave_sum(v);
  if constexpr (NT == 64) return float2{u, v};
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

// Who works on what: a worker of NW threads (a wave, or a block for long rows) has the heads of one chunk of a token at a
// time, R to a lane; the workers of a block take different tokens of the same group and chunk.
template <typename T, int NORM, int NW, int R, int LAYOUT>
struct Share {
  static constexpr int E = kPiece<T>, NT = NW == 64 ? 256 : NW, kWorkers = NT / NW;
  int place, tensor, H, head0, step, group, first_token, token_step, worker;
  uint32_t block;
  Slot<T, LAYOUT> slot;

  __device__ __forceinline__ Share(const RotateArgs<T>& a) {
    const uint32_t chunks = (uint32_t)a.chunks[0] + (uint32_t)a.chunks[1], unit = (block = a.block0 + blockIdx.x) / chunks;
    const int chunk = (int)(block - unit * chunks), split = (int)(unit % (uint32_t)a.splits);
    group = (int)(unit / (uint32_t)a.splits);
    worker = NW == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    place = NW == 64 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    tensor = chunk >= a.chunks[0];
    H = a.heads[tensor];
    step = NW >> a.shift;
    head0 = (chunk - (tensor ? a.chunks[0] : 0)) * R * step + (place >> a.shift);
    slot.place(place & ((1 << a.shift) - 1), a.D, a.width, a.interleaved);
    first_token = split * kWorkers + worker;
    token_step = a.splits * kWorkers;
  }
  __device__ __forceinline__ int head(int r) const { return head0 + r * step; }
  __device__ __forceinline__ bool has(int r) const { return slot.any && head(r) < H; }
};

// The weights in LDS as the lanes of a worker use them: 2 E a lane and head that it holds (for the norm of each head, 2 E),
// in 16-byte pieces, lanes side by side.
template <typename T, int NORM, int NW, int R, int LAYOUT>
struct Weights {
  static constexpr int E = kPiece<T>, kSets = NORM == kNormRow ? R : 1, kQuads = E / 2;
  float* lds;

  __device__ __forceinline__ void stage(const RotateArgs<T>& a, const Share<T, NORM, NW, R, LAYOUT>& s) {
    if (s.worker == 0) {
      const void* w = a.weight[s.tensor];
#pragma unroll
      for (int r = 0; r < kSets; ++r)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int64_t from = NORM == kNormRow ? (int64_t)s.head(r) * a.D : 0;
          const bool in = NORM == kNormRow ? s.has(r) : s.slot.any;
          const int ia = s.slot.at_a(e), ib = s.slot.at_b(e);
          put(s, r, e, w && in && ia < s.slot.end_a ? load_any(w, a.wt, from + ia) : in ? 1.f : 0.f);
          put(s, r, E + e, w && in && ib < s.slot.end_b ? load_any(w, a.wt, from + ib) : in ? 1.f : 0.f);
        }
    }
    __syncthreads();
  }
  __device__ __forceinline__ void put(const Share<T, NORM, NW, R, LAYOUT>& s, int r, int e, float v) {
    lds[((r * kQuads + e / 4) * NW + s.place) * 4 + e % 4] = v;
  }
  __device__ __forceinline__ void load(const Share<T, NORM, NW, R, LAYOUT>& s, int r, Values<T, LAYOUT>& w) const {
    const int set = NORM == kNormRow ? r : 0;
#pragma unroll
    for (int q = 0; q < kQuads; ++q) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(lds + ((set * kQuads + q) * NW + s.place) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) (4 * q + i < E ? w.a[(4 * q + i) % E] : w.b[(4 * q + i) % E]) = x[i];
    }
  }
};

constexpr int weight_floats(int norm, int nw, int r, int e) { return norm == kNormNone ? 4 : (norm == kNormRow ? r : 1) * 2 * e * nw; }

// y = R_p (x rstd w): each head is read once and written once, its next token's requested before this one is worked on; a
// token's cosines and sines are read once per worker. Bound by the bytes: bf16, 8 x 1,024 to 2,048 tokens of 16 + 16 heads of
// 128, a norm over each row: 52 us, 4.6 TB/s (63 a call; 163 with a block and a barrier to a row, weights in registers and tests as in the backward pass); 16
// tokens, 6 us, the launch and one trip to memory.
template <typename T, int NORM, int NW, int R, int LAYOUT>
__global__ __launch_bounds__(NW == 64 ? 256 : NW) void k_rotate(const RotateArgs<T> a) {
  constexpr bool kRow = NORM == kNormRow;
  constexpr int E = kPiece<T>;
  __shared__ float2 sums[2][kRow && NW > 64 ? NW / 64 : 1];
  __shared__ __align__(16) float staged[weight_floats(NORM, NW, R, E)];
  const Share<T, NORM, NW, R, LAYOUT> share(a);
  TokenQueue queue(a.mask, a.at, share.first_token, share.token_step, a.tokens, 0, a.by_length);
  Raw<T, LAYOUT> raw[R];
  Turn<T, LAYOUT> turn, turn_next;
  int n = 0, t = 0;
  bool live = false;
  auto request = [&]() {
    n = queue.example;
    t = queue.index;
    live = queue.live;
    if (!live) return;
    turn_next.request(share.slot, a.table, a.positions, queue.position, a.width);
    const T* base = a.in[share.tensor].row(n, t, 0);
#pragma unroll
    for (int r = 0; r < R; ++r) raw[r].request(share.slot, base + (share.has(r) ? share.head(r) : 0) * a.in[share.tensor].ld_h, a.D);
  };
  bool more = queue.next();
  if (more) request();
  Weights<T, NORM, NW, R, LAYOUT> weights{staged};
  if constexpr (NORM != kNormNone) weights.stage(a, share);
  int turn_no = 0;
  while (more) {
    T* out = a.out[share.tensor].row(n, t, 0);
    Values<T, LAYOUT> v[R];
    const bool now = live;
    if (now) {
#pragma unroll
      for (int r = 0; r < R; ++r) v[r].take(share.slot, raw[r], a.D);
      turn = turn_next;
    }
    more = queue.next();
    if (more) request();
    if (now) {
      if constexpr (NORM != kNormNone) {
        float part[R], row = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          part[r] = share.has(r) ? v[r].square() : 0.f;
          row += part[r];
        }
        if constexpr (kRow) {
          row = row_sums<NW>(row, 0.f, sums[turn_no]).x;
          turn_no ^= 1;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float s = kRow ? row / (float)(share.H * a.D) : lanes_sum(part[r], a.shift) / (float)a.D;
          const float rstd = 1.f / sqrtf(s + a.eps);
          Values<T, LAYOUT> w;
          weights.load(share, r, w);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            v[r].a[e] *= rstd * w.a[e];
            v[r].b[e] *= rstd * w.b[e];
          }
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) turn.apply(share.slot, a.sin_sign, v[r]);
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r) v[r].clear();
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (share.has(r)) v[r].put(share.slot, out + share.head(r) * a.out[share.tensor].ld_h);
  }
}

// With t = R_p^T dy, xh = x rstd: dx = rstd (t w - xh mean(t w xh)), and sums of t xh over the block's tokens (and
// heads, where each has its own norm), which k_rotate_fold adds up in order. Bound by the latency of one token's sums at 2.4
// waves a SIMD (registers; vector units busy 0.49): bf16, 4 x 1,024 to 2,048 tokens of 40 + 8 heads of 128, 252 MB: 64 us (3.9
// TB/s) and the fold 5. With two heads a lane 79 us (1.8 waves); 187 in all with weights in registers and each piece tested
// against its head's end.
template <typename T, int NORM, int NW, int R, int LAYOUT>
__global__ __launch_bounds__(NW == 64 ? 256 : NW) void k_rotate_back(const RotateArgs<T> a) {
  constexpr bool kRow = NORM == kNormRow;
  constexpr int E = kPiece<T>, kSets = kRow ? R : 1, NT = NW == 64 ? 256 : NW;
  __shared__ float2 sums[2][kRow && NW > 64 ? NW / 64 : 1];
  constexpr int kWeights = weight_floats(NORM, NW, R, E), kFold = NW == 64 ? 4 * kSets * 2 * E * 64 : 4;
  __shared__ __align__(16) float staged[kWeights > kFold ? kWeights : kFold];
  const Share<T, NORM, NW, R, LAYOUT> share(a);
  TokenQueue queue(a.mask, a.at, share.first_token, share.token_step, a.tokens, share.group * a.tokens, a.by_length);
  Raw<T, LAYOUT> rx[R], rg[R];
  Turn<T, LAYOUT> turn, turn_next;
  int n = 0, t = 0;
  bool live = false;
  auto request = [&]() {
    n = queue.example;
    t = queue.index;
    live = queue.live;
    if (!live) return;
    turn_next.request(share.slot, a.table, a.positions, queue.position, a.width);
    const T *base = a.in[share.tensor].row(n, t, 0), *grad = a.grad[share.tensor].row(n, t, 0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int from = share.has(r) ? share.head(r) : 0;
      rx[r].request(share.slot, base + from * a.in[share.tensor].ld_h, a.D);
      rg[r].request(share.slot, grad + from * a.grad[share.tensor].ld_h, a.D);
    }
  };
  bool more = queue.next();
  if (more) request();
  Weights<T, NORM, NW, R, LAYOUT> weights{staged};
  weights.stage(a, share);
  Values<T, LAYOUT> dw[kSets];
#pragma unroll
  for (int r = 0; r < kSets; ++r) dw[r].clear();
  int turn_no = 0;
  while (more) {
    T* out = a.out[share.tensor].row(n, t, 0);
    Values<T, LAYOUT> x[R], g[R];
    const bool now = live;
    if (now) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        x[r].take(share.slot, rx[r], a.D);
        g[r].take(share.slot, rg[r], a.D);
      }
      turn = turn_next;
    }
    more = queue.next();
    if (more) request();
    if (now) {
      float square[R], dot[R], row = 0.f, row_dot = 0.f;
      Values<T, LAYOUT> w;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        turn.apply(share.slot, -a.sin_sign, g[r]);
        weights.load(share, r, w);
        square[r] = x[r].square();
        dot[r] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) dot[r] += g[r].a[e] * w.a[e] * x[r].a[e] + g[r].b[e] * w.b[e] * x[r].b[e];
        square[r] = share.has(r) ? square[r] : 0.f;
        dot[r] = share.has(r) ? dot[r] : 0.f;
        row += square[r];
        row_dot += dot[r];
      }
      if constexpr (kRow) {
        const float2 both = row_sums<NW>(row, row_dot, sums[turn_no]);
        turn_no ^= 1;
        row = both.x;
        row_dot = both.y;
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float count = (float)(kRow ? share.H * a.D : a.D);
        const float s = kRow ? row : lanes_sum(square[r], a.shift), d = kRow ? row_dot : lanes_sum(dot[r], a.shift);
        const float rstd = 1.f / sqrtf(s / count + a.eps), m = d * rstd / count;
        const bool in = share.has(r);
        if constexpr (R > 1 || kRow) weights.load(share, r, w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float ha = x[r].a[e] * rstd, hb = x[r].b[e] * rstd;
          dw[kRow ? r : 0].a[e] += in ? g[r].a[e] * ha : 0.f;
          dw[kRow ? r : 0].b[e] += in ? g[r].b[e] * hb : 0.f;
          x[r].a[e] = rstd * (g[r].a[e] * w.a[e] - ha * m);
          x[r].b[e] = rstd * (g[r].b[e] * w.b[e] - hb * m);
        }
      }
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r) x[r].clear();
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (share.has(r)) x[r].put(share.slot, out + share.head(r) * a.out[share.tensor].ld_h);
  }
  if (!a.part) return;
  if constexpr (NW == 64) {                    // the block's four waves, in their order
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSets; ++r)
#pragma unroll
      for (int e = 0; e < 2 * E; ++e)
        staged[((share.worker * kSets + r) * 2 * E + e) * 64 + share.place] = e < E ? dw[r].a[e % E] : dw[r].b[e % E];
    __syncthreads();
    if (share.worker > 0) return;
#pragma unroll
    for (int r = 0; r < kSets; ++r)
#pragma unroll
      for (int e = 0; e < 2 * E; ++e) {
        float& v = e < E ? dw[r].a[e % E] : dw[r].b[e % E];
#pragma unroll
        for (int wv = 1; wv < 4; ++wv) v += staged[((wv * kSets + r) * 2 * E + e) * 64 + share.place];
      }
  }
  float* part = a.part + (int64_t)share.block * a.part_ld;
#pragma unroll
  for (int r = 0; r < kSets; ++r) {
    if constexpr (!kRow) {                     // the wave's heads
      for (int m = 1 << a.shift; m < 64; m <<= 1)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          dw[0].a[e] += __shfl_xor(dw[0].a[e], m);
          dw[0].b[e] += __shfl_xor(dw[0].b[e], m);
        }
    }
    if (kRow ? !share.has(r) : !share.slot.any || (share.place >> a.shift) != 0) continue;
    float* to = part + (kRow ? (int64_t)share.head(r) * a.D : 0);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int ia = share.slot.at_a(e), ib = share.slot.at_b(e);
      if (ia < share.slot.end_a) to[ia] = dw[r].a[e];
      if (ib < share.slot.end_b) to[ib] = dw[r].b[e];
    }
  }
}

// Rows that the registers of a block do not hold: it goes over the row twice, for its sums and for its results, a head of a lane
// at a time (of any width). bf16, 2,048 tokens of 128 + 16 heads of 256: 121 us (2.5 TB/s, the second reading from the L2s);
// the gradient 783 us, bound by the weights' sums, which it adds to in memory.
template <typename T>
struct LongRow {
  using Layout = Share<T, kNormRow, 1024, 1, kAny>;
  static constexpr int E = kPiece<T>;
  const RotateArgs<T>& a;
  const Layout& share;
  const int rounds;

  __device__ __forceinline__ LongRow(const RotateArgs<T>& args, const Layout& s)
      : a(args), share(s), rounds((s.H + s.step - 1) / s.step) {}
  __device__ __forceinline__ Values<T, kAny> load(const T* row, int64_t ld, int r) const {
    Raw<T, kAny> raw;
    raw.request(share.slot, row + (share.has(r) ? share.head(r) : 0) * ld, a.D);
    Values<T, kAny> v;
    v.take(share.slot, raw, a.D);
    return v;
  }
  __device__ __forceinline__ Values<T, kAny> weights(int r) const {
    const void* w = a.weight[share.tensor];
    if (w && (sizeof(T) == 4 || a.wt != EOGP_F32)) return load(static_cast<const T*>(w), a.D, r);
    const int64_t from = (int64_t)(share.has(r) ? share.head(r) : 0) * a.D;
    Values<T, kAny> v;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int ia = share.slot.at_a(e), ib = share.slot.at_b(e);
      v.a[e] = w && ia < share.slot.end_a ? load_any(w, a.wt, from + ia) : 1.f;
      v.b[e] = w && ib < share.slot.end_b ? load_any(w, a.wt, from + ib) : 1.f;
    }
    return v;
  }
  __device__ __forceinline__ void clear(T* out) const {
    Values<T, kAny> zero;
    zero.clear();
    for (int r = 0; r < rounds; ++r)
      if (share.has(r)) zero.put(share.slot, out + share.head(r) * a.out[share.tensor].ld_h);
  }
};

template <typename T>
__global__ __launch_bounds__(1024) void k_rotate_long(const RotateArgs<T> a) {
  constexpr int E = kPiece<T>;
  __shared__ float2 sums[2][16];
  const typename LongRow<T>::Layout share(a);
  const LongRow<T> row(a, share);
  TokenQueue queue(a.mask, a.at, share.first_token, share.token_step, a.tokens, 0, a.by_length);
  for (int turn_no = 0; queue.next();) {
    T* out = a.out[share.tensor].row(queue.example, queue.index, 0);
    if (!queue.live) {
      row.clear(out);
      continue;
    }
    const T* in = a.in[share.tensor].row(queue.example, queue.index, 0);
    const int64_t ld = a.in[share.tensor].ld_h;
    Turn<T, kAny> turn;
    turn.request(share.slot, a.table, a.positions, queue.position, a.width);
    float square = 0.f;
    for (int r = 0; r < row.rounds; ++r) {
      const float of = row.load(in, ld, r).square();
      square += share.has(r) ? of : 0.f;
    }
    square = row_sums<1024>(square, 0.f, sums[turn_no]).x;
    turn_no ^= 1;
    const float rstd = 1.f / sqrtf(square / (float)(share.H * a.D) + a.eps);
    for (int r = 0; r < row.rounds; ++r) {
      Values<T, kAny> v = row.load(in, ld, r), w = row.weights(r);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v.a[e] *= rstd * w.a[e];
        v.b[e] *= rstd * w.b[e];
      }
      turn.apply(share.slot, a.sin_sign, v);
      if (share.has(r)) v.put(share.slot, out + share.head(r) * a.out[share.tensor].ld_h);
    }
  }
}

// (The weights' sums lie in the block's part, each element with the thread that adds to it.)
template <typename T>
__global__ __launch_bounds__(1024) void k_rotate_back_long(const RotateArgs<T> a) {
  constexpr int E = kPiece<T>;
  __shared__ float2 sums[2][16];
  const typename LongRow<T>::Layout share(a);
  const LongRow<T> row(a, share);
  TokenQueue queue(a.mask, a.at, share.first_token, share.token_step, a.tokens, share.group * a.tokens, a.by_length);
  float* part = a.part ? a.part + (int64_t)share.block * a.part_ld : nullptr;
  auto each = [&](int r, auto&& f) {            // f(place in the part, element, of b)
    if (!part || !share.has(r)) return;
    float* to = part + (int64_t)share.head(r) * a.D;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int ia = share.slot.at_a(e), ib = share.slot.at_b(e);
      if (ia < share.slot.end_a) f(to[ia], e, false);
      if (ib < share.slot.end_b) f(to[ib], e, true);
    }
  };
  for (int r = 0; r < row.rounds; ++r) each(r, [](float& to, int, bool) { to = 0.f; });
  for (int turn_no = 0; queue.next();) {
    T* out = a.out[share.tensor].row(queue.example, queue.index, 0);
    if (!queue.live) {
      row.clear(out);
      continue;
    }
    const T *in = a.in[share.tensor].row(queue.example, queue.index, 0), *grad = a.grad[share.tensor].row(queue.example, queue.index, 0);
    const int64_t ld = a.in[share.tensor].ld_h, ld_g = a.grad[share.tensor].ld_h;
    Turn<T, kAny> turn;
    turn.request(share.slot, a.table, a.positions, queue.position, a.width);
    float square = 0.f, dot = 0.f;
    for (int r = 0; r < row.rounds; ++r) {
      const Values<T, kAny> x = row.load(in, ld, r), w = row.weights(r);
      Values<T, kAny> g = row.load(grad, ld_g, r);
      turn.apply(share.slot, -a.sin_sign, g);
      float of = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) of += g.a[e] * w.a[e] * x.a[e] + g.b[e] * w.b[e] * x.b[e];
      square += share.has(r) ? x.square() : 0.f;
      dot += share.has(r) ? of : 0.f;
    }
    const float2 both = row_sums<1024>(square, dot, sums[turn_no]);
    turn_no ^= 1;
    const float count = (float)(share.H * a.D), rstd = 1.f / sqrtf(both.x / count + a.eps), m = both.y * rstd / count;
    for (int r = 0; r < row.rounds; ++r) {
      Values<T, kAny> x = row.load(in, ld, r), g = row.load(grad, ld_g, r);
      const Values<T, kAny> w = row.weights(r);
      turn.apply(share.slot, -a.sin_sign, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x.a[e] *= rstd;
        x.b[e] *= rstd;
      }
      each(r, [&](float& to, int e, bool b) { to += b ? g.b[e] * x.b[e] : g.a[e] * x.a[e]; });
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x.a[e] = rstd * (g.a[e] * w.a[e] - x.a[e] * m);
        x.b[e] = rstd * (g.b[e] * w.b[e] - x.b[e] * m);
      }
      if (share.has(r)) x.put(share.slot, out + share.head(r) * a.out[share.tensor].ld_h);
    }
  }
}

// Sums of the blocks' parts, in a fixed order: 32 columns x 32 slices of the parts per block, eight requests of a thread
// at a time. Columns run over both tensors' weights.
__global__ __launch_bounds__(1024) void k_rotate_fold(const float* __restrict__ part, int64_t part_ld, int64_t groups, int splits,
                                                      int chunks_q, int chunks_k, int nq, int nk, float* __restrict__ dq,
                                                      float* __restrict__ dk) {
  __shared__ float sum[32][33];
  const int col = threadIdx.x & 31, slice = threadIdx.x >> 5, chunks = chunks_q + chunks_k;
  const int64_t blocks_q = (nq + 31) / 32, blocks = blocks_q + (nk + 31) / 32;
  for (int64_t unit = blockIdx.x; unit < groups * blocks; unit += gridDim.x) {
    const int64_t group = unit / blocks, b = unit % blocks;
    const bool of_k = b >= blocks_q;
    const int c = (int)(of_k ? b - blocks_q : b) * 32 + col, n = of_k ? nk : nq, count = of_k ? chunks_k : chunks_q;
    const float* from = part + (group * splits * chunks + (of_k ? chunks_q : 0)) * part_ld + c;
    float* out = of_k ? dk : dq;
    float s = 0.f;
    if (c < n && out) {
      const int all = splits * count;
      for (int j = slice; j < all; j += 8 * 32) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int at = j + k * 32;
          v[k] = at < all ? from[((int64_t)(at / count) * chunks + at % count) * part_ld] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[k];
      }
    }
    sum[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < n && out) {
#pragma unroll
      for (int k = 1; k < 32; ++k) s += sum[k][col];
      out[group * n + c] = s;
    }
    __syncthreads();
  }
}

// How a token's heads and a group's tokens are shared out.
struct RotatePlan {
  int shift, worker, reps, chunks[2], layout;  // lanes of a head, threads of a worker, heads of a lane (0: a long row's)
  int64_t splits, part_ld;
};

constexpr int64_t kRotateBlocks = 8 * kCus;    // that are there at once, about (of 256 threads)
constexpr int64_t kMostLaunched = 1 << 21;     // blocks of a launch (of up to 1,024 threads)

inline int64_t want_blocks(const RotatePlan& p) { return p.worker == 1024 ? kRotateBlocks / 4 : kRotateBlocks; }

RotatePlan rotate_plan(eogp_dtype t, int norm, int Hq, int Hk, int64_t D, int64_t width, int interleaved, int64_t groups,
                       int64_t tokens) {
  RotatePlan p;
  const int E = t == EOGP_F32 ? 4 : 8;
  const int64_t slots = ceil_div(width / 2, E) + ceil_div(D - width, 2 * E);
  p.shift = 0;
  while ((1 << p.shift) < slots) ++p.shift;
  const bool whole = width / 2 % E == 0 && (D - width) % (2 * E) == 0;
  p.layout = !whole ? kAny : interleaved ? kPairs : kHalves;
  const int heads[2] = {Hq, Hk};
  if (norm == kNormRow) {
    // a wave has the row while four heads a lane hold it: no barrier per token
    const int64_t lanes = (int64_t)std::max(Hq, Hk) << p.shift;
    p.worker = lanes <= 256 ? 64 : lanes <= 512 ? 256 : 1024;
    p.reps = 1;
    while (p.reps * p.worker < lanes) p.reps *= 2;
    if (lanes > (t == EOGP_F32 ? 2048 : 1024) * (whole ? 1 : 2)) p.reps = 0;
    for (int i = 0; i < 2; ++i) p.chunks[i] = heads[i] > 0;
    p.part_ld = std::max(Hq, Hk) * D;
  } else {
    // Two heads a lane where there are tokens enough for all waves, so that cosines and weights are read once for both; not
    // for 16-bit heads with a norm, whose registers then leave too few waves. Two and one, bf16: 32,768 tokens of 64 x 128
    // without a norm 217 and 231 us, 8,192 of 48 38 and 35, with a norm of each 42 and 36, its gradient 96 and 79; fp32, the
    // same: 420 and 452, 77 and 78, 80 and 83, 133 and 130.
    const int at_once = 64 >> p.shift;
    const int64_t waves = groups * tokens * ceil_div(Hq + Hk, at_once);
    p.worker = 64;
    p.reps = (E == 4 ? waves >= 16 * kRotateBlocks : norm == kNormNone && waves >= 64 * kRotateBlocks) ? 2 : 1;
    for (int i = 0; i < 2; ++i) p.chunks[i] = (int)ceil_div(heads[i], at_once * p.reps);
    p.part_ld = D;
  }
  const int64_t per_block = p.worker == 64 ? 4 : 1, want = want_blocks(p);
  p.splits = std::min(std::max<int64_t>(1, ceil_div(tokens, per_block)),
                      std::max<int64_t>(1, want / std::max<int64_t>(1, groups * ((int64_t)p.chunks[0] + p.chunks[1]))));
  return p;
}

template <typename T>
RotateArgs<T> rotate_args(const eogp_heads* in, const eogp_heads* grad, const eogp_heads* out, int64_t D, const void* qw,
                          const void* kw, eogp_dtype wt, float eps, const float* table, int64_t positions, int64_t width,
                          int interleaved, const int64_t* at, const uint8_t* mask, int64_t T_, int64_t tokens,
                          const RotatePlan& p) {
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
  a.tokens = (int)tokens;
  a.by_length = Divide(std::max<int64_t>(1, T_));
  a.shift = p.shift;
  a.splits = (int)p.splits;
  a.part_ld = p.part_ld;
  return a;
}

// The blocks of a call, in as many launches as they take (one but for millions of examples or heads).
template <typename K, typename T>
eogp_status launch_all(const char* what, K* kfn, RotateArgs<T>& a, const RotatePlan& p, int64_t groups, hipStream_t s) {
  const int64_t blocks = groups * p.splits * ((int64_t)p.chunks[0] + p.chunks[1]);
  for (int64_t from = 0; from < blocks; from += kMostLaunched) {
    a.block0 = (uint32_t)from;
    hipLaunchKernelGGL(kfn, dim3((unsigned)std::min(blocks - from, kMostLaunched)), dim3(std::max(256, p.worker)), 0, s, a);
    EOGP_LAUNCH_CHECK(what);
  }
  return EOGP_OK;
}

// f(threads of a worker, heads of a lane, layout), for rows that are not long. (Whole pieces take D / 2 E lanes a head, less than
// twice as many as a power of two. So rows of 8,192 elements have fewer than 2,048 lanes in fp32, 1,024 in 16 bits; other widths
// fewer than 4,096 and up to 2,048. Longer ones are held up to the same number of lanes.)
template <typename T, int NORM, typename F>
eogp_status with_shape(const RotatePlan& p, F&& f) {
  using std::integral_constant;
  auto go = [&](auto layout) {
    using One = integral_constant<int, 1>;
    using Two = integral_constant<int, 2>;
    using Four = integral_constant<int, 4>;
    using W64 = integral_constant<int, 64>;
    using W256 = integral_constant<int, 256>;
    using W1024 = integral_constant<int, 1024>;
    if (p.worker == 64) {
      if constexpr (NORM != kNormHead || sizeof(T) == 4)
        if (p.reps == 1) return f(W64{}, One{}, layout);
      if constexpr (NORM == kNormRow)
        if (p.reps == 4) return f(W64{}, Four{}, layout);
      if constexpr (NORM != kNormHead || sizeof(T) == 4) return f(W64{}, Two{}, layout);
      return f(W64{}, One{}, layout);
    }
    if constexpr (NORM == kNormRow) {
      if (p.worker == 256) return f(W256{}, Two{}, layout);
      constexpr bool kAnyWidth = decltype(layout)::value == kAny;
      if (p.reps == 1) return f(W1024{}, One{}, layout);
      if constexpr (sizeof(T) == 4 && kAnyWidth)
        if (p.reps > 2) return f(W1024{}, Four{}, layout);
      if constexpr (sizeof(T) == 4 || kAnyWidth) return f(W1024{}, Two{}, layout);
    }
    return EOGP_ERR_UNSUPPORTED;
  };
  if (p.layout == kHalves) return go(integral_constant<int, kHalves>{});
  if (p.layout == kPairs) return go(integral_constant<int, kPairs>{});
  return go(integral_constant<int, kAny>{});
}

template <typename F>
eogp_status with_norm(int norm, F&& f) {
  using std::integral_constant;
  if (norm == kNormHead) return f(integral_constant<int, kNormHead>{});
  if (norm == kNormRow) return f(integral_constant<int, kNormRow>{});
  return f(integral_constant<int, kNormNone>{});
}

}  // namespace

// Whether one norm takes a row of that many heads.
bool rotate_row_fits(int64_t heads, int64_t D) { return heads <= 128 || heads * D <= (D < 8 ? 2048 : 8192); }

eogp_status rotary_table(int64_t positions, int64_t width, double base, double factor, double original, double low,
                         double high, double magnitude, float* table, hipStream_t s) {
  if (positions == 0) return EOGP_OK;
  timing::Scope ts(EOGP_KT_ROTARY, s);
  const int64_t pairs = width / 2, columns = ceil_div(pairs, 32);
  // as many positions a thread as leave the chip full of threads
  int64_t K = 1;
  while (K < 32 && ceil_div(positions, 16 * K) * columns >= 8 * kCus) K *= 2;
  while (ceil_div(positions, 8 * K) > (1 << 23)) K *= 2;
  const dim3 grid((unsigned)ceil_div(positions, 8 * K), (unsigned)columns);
  hipLaunchKernelGGL(k_rotary_table, grid, dim3(256), 0, s, positions, (int)pairs, (int)K, -2.0 / (double)width * std::log2(base),
                     1.0 / factor, original / (2.0 * M_PI), low, 1.0 / (high - low), magnitude, table);
  EOGP_LAUNCH_CHECK("rotary_table");
  return EOGP_OK;
}

eogp_status rotate_heads(const eogp_heads* in, const eogp_heads* out, eogp_dtype t, int norm, const void* qw,
                         const void* kw, eogp_dtype wt, float eps, const float* table, int64_t positions, int64_t width,
                         int interleaved, bool back, const int64_t* at, const uint8_t* mask, int64_t N, int64_t T_,
                         int64_t D, hipStream_t s) {
  if (N * T_ == 0) return EOGP_OK;
  const RotatePlan p = rotate_plan(t, norm, (int)out[0].heads, (int)out[1].heads, D, width, interleaved, 1, N * T_);
  timing::Scope ts(EOGP_KT_ROTARY, s);
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    RotateArgs<T> a = rotate_args<T>(in, nullptr, out, D, qw, kw, wt, eps, table, positions, width, interleaved, at, mask, T_,
                                     N * T_, p);
    a.sin_sign = back ? -1.f : 1.f;
    if (p.reps == 0) return launch_all("rotate_heads", k_rotate_long<T>, a, p, 1, s);
    return with_norm(norm, [&](auto nm) {
      constexpr int NORM = decltype(nm)::value;
      return with_shape<T, NORM>(p, [&](auto nw, auto reps, auto layout) {
        return launch_all("rotate_heads", k_rotate<T, NORM, decltype(nw)::value, decltype(reps)::value, decltype(layout)::value>, a,
                          p, 1, s);
      });
    });
  });
}

size_t rotate_back_ws(eogp_dtype t, int norm, int64_t Hq, int64_t Hk, int64_t D, int64_t width, int64_t groups, int64_t tokens) {
  // the blocks of any call of up to `groups` groups of up to `tokens` tokens, with one head a lane
  const RotatePlan p = rotate_plan(t, norm, (int)Hq, (int)Hk, D, width, 0, 1, 1);
  const int64_t chunks = (int64_t)p.chunks[0] + p.chunks[1];
  const int64_t blocks = std::min(groups * std::max<int64_t>(1, tokens) * chunks, std::max(want_blocks(p), groups * chunks));
  return align256((size_t)blocks * p.part_ld * sizeof(float));
}

eogp_status rotate_heads_back(const eogp_heads* in, const eogp_heads* grad, const eogp_heads* out, eogp_dtype t, int norm,
                              const void* qw, const void* kw, eogp_dtype wt, float eps, const float* table,
                              int64_t positions, int64_t width, int interleaved, const int64_t* at, const uint8_t* mask,
                              int64_t N, int64_t T_, int64_t D, bool per_example, float* dqw, float* dkw, void* ws,
                              hipStream_t s) {
  const int64_t groups = per_example ? N : 1, tokens = per_example ? T_ : N * T_;
  if (groups == 0) return EOGP_OK;
  const RotatePlan p = rotate_plan(t, norm, (int)out[0].heads, (int)out[1].heads, D, width, interleaved, groups, tokens);
  float* part = dqw || dkw ? static_cast<float*>(ws) : nullptr;
  timing::Scope ts(EOGP_KT_ROTARY, s);
  const eogp_status st = with_type(t, [&](auto el) {
    using T = decltype(el);
    RotateArgs<T> a = rotate_args<T>(in, grad, out, D, qw, kw, wt, eps, table, positions, width, interleaved, at, mask, T_,
                                     tokens, p);
    a.part = part;
    if (p.reps == 0) return launch_all("rotate_heads_backward", k_rotate_back_long<T>, a, p, groups, s);
    auto go = [&](auto nm) {
      constexpr int NORM = decltype(nm)::value;
      return with_shape<T, NORM>(p, [&](auto nw, auto reps, auto layout) {
        return launch_all("rotate_heads_backward",
                          k_rotate_back<T, NORM, decltype(nw)::value, decltype(reps)::value, decltype(layout)::value>, a, p, groups, s);
      });
    };
    using std::integral_constant;
    return norm == kNormRow ? go(integral_constant<int, kNormRow>{}) : go(integral_constant<int, kNormHead>{});
  });
  if (st != EOGP_OK || !part) return st;
  const int64_t nq = norm == kNormRow ? out[0].heads * D : D, nk = p.chunks[1] ? (norm == kNormRow ? out[1].heads * D : D) : 0;
  hipLaunchKernelGGL(k_rotate_fold, dim3((unsigned)std::min<int64_t>(groups * (ceil_div(nq, 32) + ceil_div(nk, 32)), 1 << 20)),
                     dim3(1024), 0, s, part, p.part_ld, groups, (int)p.splits, p.chunks[0], p.chunks[1], (int)nq, (int)nk, dqw,
                     dkw);
  EOGP_LAUNCH_CHECK("rotate_heads_backward (fold)");
  return EOGP_OK;
}

}  // namespace eogp
