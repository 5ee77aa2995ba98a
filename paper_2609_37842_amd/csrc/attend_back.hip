// The gradients of attention at queries, keys and values.
#include <algorithm>

#include "attend.h"
#include "timing.h"

namespace eogp {
namespace {

template <typename T>
struct BackArgs {
  Heads<const T> q, k, v, dout;
  const void* out;                // the forward pass's output, rows of T or fp32
  int64_t out_n, out_t, out_h;
  int out_f32;
  Heads<T> dq, dk, dv;
  Sight sight;
  int N, Hq, Hkv, D;
  Divide by_group;                // query heads of a key head
  Divide by_splits, by_units, by_heads;   // splits; key heads of all examples, of one
  float scale, scale_log2;
  const float* lse;               // [N, Tq, Hq]
  // [N, Tq, Hq]: a weight is 2^(score - lse2 - low) (lse2 +inf: the row counts for nothing); dout . out
  float *lse2, *low, *delta;
  uint32_t* norms;                // fp16: [N Hkv][2] largest squared norms of a row of dout and of v, as bits
  int row_tiles, key_tiles, splits;
  float* part;                    // splits > 1: [splits][N Hkv][Tk][2][D]
};

// Weights times 2^kLiftBack: fp16 holds small ones as precisely as large ones. (Weights are at most 1.)
template <typename T> constexpr float kLiftBack = 0.f;
template <> constexpr float kLiftBack<_Float16> = 15.f;

// A log-sum-exp in fp32 holds a row's weights to 2^-22 of its size: below 2^10 (in powers of two) to 2^-12. Rows beyond have
// their scores' largest and the sum of the weights beside it made anew, lse2 and low, so that their weights add up to 1
// whatever the size. (lse2 is at most 29 below the log-sum-exp that made a row one of them.)
constexpr float kFarLse = 1024.f, kFarTile = 512.f;
__device__ __forceinline__ bool is_far(float lse2, float from) { return fabsf(lse2) >= from && fabsf(lse2) < INFINITY; }
__device__ __forceinline__ float far_score(float s, float scale_log2, float lse2) {
  return fabsf(lse2) < kFar ? __builtin_fmaf(s, scale_log2, -lse2) : rounded(s * scale_log2) - lse2;
}

// 16-bit weights P and score gradients dS are rounded to the type before the products that take them, which run at the 16-bit
// rate that way, and delta comes from the forward pass's output as it was rounded (in fp32 where the caller kept that):
// gradients are off by 0.0026 of their size (root mean square, bf16; fp16 0.00042) where one rounding at the end would leave
// 0.0017 (0.00021).
//
// fp16 score gradients P (dP - delta) are small where many keys share a row, and lie below fp16's normal range where
// the output gradients are small as well. They are held times 2^e, e from |dP - delta| <= 2 max |dout row| max |v row|
// of the key head's rows, so that none passes 2^14.
// (The gradients of queries take each row's own norm.)
template <typename T>
__device__ __forceinline__ int lift_of(const BackArgs<T>& a, int unit, float dout_square) {
  if constexpr (kLiftBack<T> == 0.f) return 0;
  const float bound = 2.f * sqrtf(dout_square) * sqrtf(__uint_as_float(a.norms[2 * unit + 1]));
  if (!(bound > 0.f) || isinf(bound)) return 0;
  const int e = 14 - (ilogbf(bound) + 1);
  return e < -100 ? -100 : e > 100 ? 100 : e;
}

// Waves that share tiles. fp32 products are bound by the matrix units alone: there two waves share theirs, so that short and
// ragged sequences leave fewer idle at another's pace (rows of more than 512 bytes aside); 16-bit ones would be bound by the
// tiles' way to LDS.
constexpr int back_share(int size, int dp) { return size == 4 && dp <= 128 ? 2 : 4; }

// Whether one kernel makes the gradients of keys and values. Together they take seven products where two kernels take eight
// (scores are made again), apart they leave two waves a SIMD: 16-bit heads of 128 are faster apart (2 x 2,048 tokens of
// 40 / 8 x 128 bf16, whole backward pass: 386 us, together 418), heads of 64 together (fp32, bound by the products, 32 x 512
// tokens of 12 x 64: 359 us, apart 399; bf16, 32 x 1,024: 320, apart 377; fp16, 32 x 512: 141, apart 165); wider ones do not
// fit the registers together.
constexpr bool kv_together(int dp) { return dp <= 64; }

// Waves of a SIMD, by the bytes of a row: so that registers are taken from one file without copies.
constexpr int back_waves(int row_bytes, int most) { return row_bytes <= most ? 2 : 1; }

__device__ __forceinline__ float sum_of(float v, int lanes) {
  for (int m = 1; m < lanes; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

__global__ __launch_bounds__(256) void k_attend_zero(uint32_t* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

// fp16: the largest norms of rows of v, of keys between the first and the last that queries of the example see (what others
// hold is nobody's). A row takes `lanes` lanes, 16 bytes each; a block has kNormSteps steps of an example's rows.
constexpr int kNormSteps = 16;
template <typename T>
__global__ __launch_bounds__(256) void k_attend_norms(const BackArgs<T> a, int lanes, int chunks) {
  constexpr int E = kPiece<T>;
  const int lane = threadIdx.x & 63, per = 64 / lanes, c = (lane % lanes) * E, rows = a.sight.Tk * a.Hkv;
  for (int64_t part = blockIdx.x; part < (int64_t)a.N * chunks; part += gridDim.x) {
    const int n = (int)(part / chunks), from = (int)(part - (int64_t)n * chunks) * kNormSteps * 4 * per;
    int i0 = 0, i1 = a.sight.Tq;
    if (a.sight.q_mask && i1 > 0) {
      const MaskRange r = mask_range(a.sight.q_mask + (int64_t)n * i1, i1, 0, i1);
      i0 = r.first;
      i1 = r.last;
    }
    if (i0 >= i1) continue;
    const int64_t start = a.sight.start(n);
    const Span first = span_of(a.sight, start + i0), last = span_of(a.sight, start + i1 - 1);
    for (int step = threadIdx.x >> 6; step < 4 * kNormSteps; step += 4) {
      const int id = from + step * per + lane / lanes, rc = id < rows ? id : rows - 1;
      const int j = rc / a.Hkv, h = rc - j * a.Hkv;
      const bool live = id < rows && ((j >= first.lo && j < last.hi) || j < last.sk) &&
                        (!a.sight.k_mask || a.sight.k_mask[(int64_t)n * a.sight.Tk + j]);
      float square = 0.f;
      if (live) {
        float x[E];
        load_piece<T, E>(a.v.row(n, j, h), c, a.D, 0.f, x);
#pragma unroll
        for (int e = 0; e < E; ++e) square += x[e] * x[e];
      }
      square = sum_of(square, lanes);
      // (the largest of a set does not depend on the order)
      if (live && lane % lanes == 0) atomicMax(a.norms + 2 * (n * a.Hkv + h) + 1, __float_as_uint(square == square ? square : 0.f));
    }
  }
}

// Gradients of keys and values: a wave has 32 keys, their rows of K and V and both gradients in registers; the
// block's waves share tiles of 32 rows of queries and output gradients, over all query heads of the key head.
// PARTS: 1 gradients of V, 2 of K, 3 both. Bound by the products at one or two waves a SIMD (registers) and the latency of a
// tile's scores, which the next product waits for: under a profiler, fp32, 32 x 64 to 512 tokens of 12 x 64, both 246 us (matrix
// units busy 0.34 of the SIMDs' time); bf16, 2 x 1,024 to 2,048 of 40 / 8 x 128, V 102 us (0.23, vector units 0.32), K 133
// (0.27, 0.33).
template <typename T, int DP, int PARTS, bool FAST>
__global__ __launch_bounds__(64 * back_share((int)sizeof(T), DP), back_waves(DP * (int)sizeof(T), PARTS == 3 ? 128 : 256)) void k_attend_back_kv(
    const BackArgs<T> a) {
  constexpr int NW = back_share((int)sizeof(T), DP), NT = 64 * NW;
  constexpr int kROWB = DP * (int)sizeof(T), RB = 32, kTile = RB * kROWB, kDt = DP / 32, kSteps = kROWB / 32;
  constexpr int kKs = 32 / (2 * kPiece<T>);
  constexpr bool kV = PARTS & 1, kK = PARTS & 2;
  extern __shared__ __align__(16) char lds[];            // [2][Q, dO]
  __shared__ __align__(16) float row_f[2][3][RB];        // rows of a tile: log-sum-exps and deltas; far ones' `low`
  __shared__ __align__(16) uint32_t seen[NW][RB];        // a wave's keys that each row sees
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 31, h = lane >> 5;
  const int units = a.N * a.Hkv, G = a.by_group.by;
  const int b = a.by_splits.quotient(blockIdx.x), split = a.by_splits.rest(blockIdx.x, b);
  // tiles of the first keys, which most queries see, first
  const int tile_key = a.by_units.quotient(b), unit = a.by_units.rest(b, tile_key);
  const int n = a.by_heads.quotient(unit), kvh = a.by_heads.rest(unit, n);
  const int64_t start = a.sight.start(n);
  // (the last keys of a causal tile have fewer queries: blocks of a CU, 256 apart, have them in opposite waves)
  const int k0 = tile_key * 32 * NW, j0 = k0 + ((blockIdx.x >> 8) & 1 ? NW - 1 - wid : wid) * 32, j = j0 + l;
  const int k1 = min(k0 + 32 * NW, a.sight.Tk);
  const bool key_live = j < a.sight.Tk && (!a.sight.k_mask || a.sight.k_mask[(int64_t)n * a.sight.Tk + j]);
  RowPieces<T, DP, FAST> kf, vf;
  const int jc = min(j, a.sight.Tk - 1);
  kf.request(a.k.row(n, jc, kvh), a.D);
  if constexpr (kK) vf.request(a.v.row(n, jc, kvh), a.D);

  // queries that can see one of the block's keys
  const bool sink = k0 < a.sight.sinks;
  const int64_t i_lo = a.sight.causal ? k0 - start : a.sight.window && !sink ? k0 - a.sight.window + 1 - start : 0;
  const int64_t i_hi = a.sight.window && !sink ? (int64_t)k1 - 1 + a.sight.window - start : a.sight.Tq;
  int i0 = clamp_key(i_lo, a.sight.Tq), i1 = clamp_key(i_hi, a.sight.Tq);
  if (a.sight.q_mask && i0 < i1) {
    const MaskRange r = mask_range(a.sight.q_mask + (int64_t)n * a.sight.Tq, a.sight.Tq, i0, i1);
    i0 = r.first;
    i1 = r.last;
  }
  const int some_keys = __syncthreads_or(key_live);
  const int rows_lo = i0 * G, rows_hi = i1 * G, row_tiles = some_keys && i1 > i0 ? (rows_hi - rows_lo + RB - 1) / RB : 0;
  int t = 0, t_end = row_tiles;
  if (a.splits > 1) {
    t = (int)((int64_t)row_tiles * split / a.splits);
    t_end = (int)((int64_t)row_tiles * (split + 1) / a.splits);
  }
  kf.settle(key_live, a.D);
  if constexpr (kK) vf.settle(key_live, a.D);
  f32x16 dv[kV ? kDt : 1], dk[kK ? kDt : 1];
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt) {
    if constexpr (kV) dv[dt] = zeros16();
    if constexpr (kK) dk[dt] = zeros16();
  }
  const int lift = kLiftBack<T> == 0.f ? 0 : lift_of(a, unit, __uint_as_float(a.norms[2 * unit]));
  const float ds_by = exp2f((float)lift - kLiftBack<T>);

  // Rows of the block from which on, and up to which, each sees all of the wave's keys (the sinks' share aside), and
  // those outside which none sees any.
  auto row_of = [&](int64_t p) { return (int)min(max(p - start, (int64_t)0), (int64_t)a.sight.Tq) * G; };
  const int64_t w = a.sight.window;
  const int full_lo = a.sight.causal ? row_of((int64_t)j0 + 31) : w ? row_of((int64_t)j0 + 32 - w) : 0;
  const int full_hi = w ? row_of((int64_t)j0 + w) : rows_hi;
  const bool wave_sink = j0 < a.sight.sinks;
  const int some_lo = a.sight.causal ? row_of(j0) : w && !wave_sink ? row_of((int64_t)j0 - w + 1) : 0;
  const int some_hi = w && !wave_sink ? row_of((int64_t)j0 + 31 + w) : rows_hi;

  // the first query head of the key head as rows: row r is query r / G of head r mod G
  const T *qbase = a.q.row(n, 0, kvh * G), *obase = a.dout.row(n, 0, kvh * G);
  auto span_bytes = [&](const Heads<const T>& x) {
    return (uint32_t)((a.sight.Tq - 1) * (int)x.ld_t + (G - 1) * (int)x.ld_h + DP) * (uint32_t)sizeof(T);
  };
  const auto qall = buffer_of(qbase, FAST ? span_bytes(a.q) : 0u), oall = buffer_of(obase, FAST ? span_bytes(a.dout) : 0u);
  const int64_t id0 = (int64_t)n * a.sight.Tq * a.Hq + kvh * G;
  Stage<T, DP, RB, NT, FAST> qs, os;
  constexpr int kEach = Stage<T, DP, RB, NT, FAST>::kEach, kPieces = DP / kPiece<T>;
  // What the thread asks for next: its rows' heads and first bytes (FAST), and the lane's row.
  int walk_g[kEach], walk_q[kEach], walk_o[kEach];
  const int step_i = a.by_group.quotient(RB), step_g = a.by_group.rest(RB, step_i);
  const int q_t = (int)a.q.ld_t * (int)sizeof(T), q_h = (int)a.q.ld_h * (int)sizeof(T);
  const int o_t = (int)a.dout.ld_t * (int)sizeof(T), o_h = (int)a.dout.ld_h * (int)sizeof(T);
  if constexpr (FAST) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int at = u * NT + (int)threadIdx.x, row = rows_lo + t * RB + at / kPieces, i = a.by_group.quotient(row);
      walk_g[u] = a.by_group.rest(row, i);
      walk_q[u] = i * q_t + walk_g[u] * q_h + at % kPieces * 16;
      walk_o[u] = i * o_t + walk_g[u] * o_h + at % kPieces * 16;
    }
  }
  auto id_of = [&](int row) {
    const int rc = min(row, rows_hi - 1), i = a.by_group.quotient(rc);
    return id0 + (int64_t)i * a.Hq + a.by_group.rest(rc, i);
  };
  float r_lse2 = 0.f, r_delta = 0.f;
  bool r_live = false;
  auto request = [&](int tile) {
    const int r0 = rows_lo + tile * RB;
    if constexpr (FAST) {
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        qs.request_one(u, qall, walk_q[u]);
        os.request_one(u, oall, walk_o[u]);
        walk_g[u] += step_g;
        const bool over = walk_g[u] >= G;
        walk_g[u] -= over ? G : 0;
        walk_q[u] += step_i * q_t + step_g * q_h + (over ? q_t - G * q_h : 0);
        walk_o[u] += step_i * o_t + step_g * o_h + (over ? o_t - G * o_h : 0);
      }
    } else {
      auto at = [&](const T* base, const Heads<const T>& x) {
        return [&, base](int r) {
          const int row = min(r0 + r, rows_hi - 1), i = a.by_group.quotient(row);
          return base + i * x.ld_t + a.by_group.rest(row, i) * x.ld_h;
        };
      };
      qs.request_each(threadIdx.x, a.D, at(qbase, a.q));
      os.request_each(threadIdx.x, a.D, at(obase, a.dout));
    }
    const int row = r0 + l;
    const int64_t id = id_of(row);
    r_lse2 = a.lse2[id];
    if constexpr (kK) r_delta = a.delta[id];
    r_live = row < rows_hi;
  };
  if (t < t_end) request(t);
  for (int turn = 0; t < t_end; ++t, turn ^= 1) {
    char *qt = lds + turn * 2 * kTile, *ot = qt + kTile;
    const int r0 = rows_lo + t * RB;
    r_lse2 = r_live ? r_lse2 : INFINITY;
    const uint64_t live = __ballot(r_lse2 != INFINITY) & 0xFFFFFFFFull;
    qs.store(threadIdx.x, a.D, qt, live);
    os.store(threadIdx.x, a.D, ot, live);
    const bool far = __ballot(is_far(r_lse2, kFarTile)) != 0;
    if (threadIdx.x < RB) {
      row_f[turn][0][l] = far ? r_lse2 : r_lse2 - kLiftBack<T>;
      if (__builtin_expect(far, 0)) row_f[turn][2][l] = a.low[id_of(r0 + l)] - kLiftBack<T>;
      if constexpr (kK) row_f[turn][1][l] = r_delta;
    }
    __syncthreads();
    if (t + 1 < t_end) request(t + 1);
    const bool full = r0 >= full_lo && r0 + RB <= full_hi;
    const bool some = live != 0 && r0 + RB > some_lo && r0 < some_hi;
    if (some && !full) {
      wave_lds_order();
      seen[wid][l] = sight_bits(span_of(a.sight, start + a.by_group.quotient(min(r0 + l, rows_hi - 1))), j0);
      wave_lds_order();
    }
    if (some) {
    f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      mma(s, row_frag<T, kROWB>(qt, l, k), kf.f[k]);
      if constexpr (kK) mma(dp, row_frag<T, kROWB>(ot, l, k), vf.f[k]);
    }
    if (__builtin_expect(far, 0)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int at = 8 * (e / 4) + 4 * h + e % 4;
        s[e] = __builtin_amdgcn_exp2f(far_score(s[e], a.scale_log2, row_f[turn][0][at]) - row_f[turn][2][at]);
      }
    } else {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 lse2 = *reinterpret_cast<const f32x4*>(&row_f[turn][0][8 * g + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * g + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * g + i], a.scale_log2, -lse2[i]));
      }
    }
    if (!full) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const i32x4 w = *reinterpret_cast<const i32x4*>(&seen[wid][8 * g + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (dP as well: a key that the row does not see may hold anything)
          const bool sees_it = ((uint32_t)w[i] >> l) & 1;
          s[4 * g + i] = sees_it ? s[4 * g + i] : 0.f;
          dp[4 * g + i] = sees_it ? dp[4 * g + i] : 0.f;
        }
      }
    }
    if constexpr (kV) {
      Frag<T> p[kKs];
#pragma unroll
      for (int k = 0; k < kKs; ++k) p[k] = acc_frag<T>(s, k);
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int k = 0; k < kKs; ++k) mma(dv[dt], col_frag<T, kROWB>(ot, 0, k, dt), p[k]);
    }
    if constexpr (kK) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 delta = *reinterpret_cast<const f32x4*>(&row_f[turn][1][8 * g + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float d = s[4 * g + i] * (dp[4 * g + i] - delta[i]);
          if constexpr (kLiftBack<T> != 0.f) d *= ds_by;
          dp[4 * g + i] = d;
        }
      }
      Frag<T> p[kKs];
#pragma unroll
      for (int k = 0; k < kKs; ++k) p[k] = acc_frag<T>(dp, k);
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int k = 0; k < kKs; ++k) mma(dk[dt], col_frag<T, kROWB>(qt, 0, k, dt), p[k]);
    }
    }
  }

  if (j >= a.sight.Tk) return;
  const float by_v = exp2f(-kLiftBack<T>), by_k = a.scale * exp2f(-(float)lift);
  const int D = FAST ? DP : a.D;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (!(which ? kK : kV)) continue;
    const Heads<T>& to = which ? a.dk : a.dv;
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = dt * 32 + 8 * g + 4 * h;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (PARTS == 1) v[i] = dv[dt][4 * g + i] * by_v;
          else if constexpr (PARTS == 2) v[i] = dk[dt][4 * g + i] * by_k;
          else v[i] = which ? dk[dt][4 * g + i] * by_k : dv[dt][4 * g + i] * by_v;
          v[i] = key_live ? v[i] : 0.f;
        }
        if (a.part)
          put4<float, FAST>(a.part + ((((int64_t)split * units + unit) * a.sight.Tk + j) * 2 + which) * D, c, D, v);
        else
          put4<T, FAST>(to.row(n, j, kvh), c, D, v);
      }
  }
}

// Sums of the splits' parts in their order, V elements of a gradient per thread (4 where D allows), four splits' asked for at
// once. Bound by reading the parts: bf16, 2 x 2,048 keys of 8 x 128, 4 splits, 134 MB: 24 us (6.4 TB/s; an element a thread,
// with 64-bit divisions, 42).
template <typename T, int V>
__global__ __launch_bounds__(256) void k_attend_back_join(const BackArgs<T> a) {
  using Piece = std::conditional_t<V == 4, AnyVec<float, 4>, float>;
  // (the parts of a launch are at most kSplitBlocks blocks of 128 keys: numbers of 32 bits)
  const uint32_t units = a.N * a.Hkv, wide = a.D / V, all = units * a.sight.Tk * 2 * wide;
  for (uint32_t id = blockIdx.x * 256 + threadIdx.x; id < all; id += gridDim.x * 256) {
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
    for (int s0 = 0; s0 < a.splits; s0 += 4) {
      Piece x[4];
#pragma unroll
      for (int s = 0; s < 4; ++s)
        x[s] = *reinterpret_cast<const Piece*>(a.part + ((int64_t)min(s0 + s, a.splits - 1) * all + id) * V);
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += s0 + s < a.splits ? reinterpret_cast<const float*>(&x[s])[e] : 0.f;
    }
    const uint32_t row = id / wide, c = (id - row * wide) * V, which = row & 1, key = row >> 1;
    const uint32_t unit = key / (uint32_t)a.sight.Tk, j = key - unit * a.sight.Tk, n = unit / (uint32_t)a.Hkv;
    T* to = (which ? a.dk : a.dv).row(n, j, unit - n * a.Hkv) + c;
    if constexpr (V == 4) {
      put4<T, true>(to, 0, 4, v);
    } else {
      to[0] = (T)v[0];
    }
  }
}

// Gradients of queries: a wave has 32 rows of queries, output gradients and the result in registers; the block's
// waves share tiles of keys and values. Before that each row's delta = dout . out is formed, and its log-sum-exp in powers
// of two, which the other kernels read (+inf: the row counts for nothing). Bound as k_attend_back_kv is: the fp32 batch
// there 165 us (matrix units busy 0.38), the bf16 one 156 (0.28, vector units 0.31).
template <typename T, int DP, bool FAST>
__global__ __launch_bounds__(64 * back_share((int)sizeof(T), DP), back_waves(DP * (int)sizeof(T), 256)) void k_attend_back_q(const BackArgs<T> a) {
  constexpr int NW = back_share((int)sizeof(T), DP), NT = 64 * NW, KB = 32;
  constexpr int kROWB = DP * (int)sizeof(T), kTile = KB * kROWB, kDt = DP / 32, kSteps = kROWB / 32;
  constexpr int kRows = 32 * NW, kKs = 32 / (2 * kPiece<T>);
  extern __shared__ __align__(16) char lds[];            // [2][K, V]
  __shared__ uint32_t all[NW];
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 31, h = lane >> 5;
  const int G = a.by_group.by, rows = G * a.sight.Tq;
  const int from_end = a.by_units.quotient(blockIdx.x), unit = a.by_units.rest(blockIdx.x, from_end);
  const int tile_row = a.row_tiles - 1 - from_end, n = a.by_heads.quotient(unit), kvh = a.by_heads.rest(unit, n);
  const int64_t start = a.sight.start(n);
  // (The first rows of a causal tile have fewer keys: blocks of a CU, 256 apart, have them in opposite waves.)
  const int group = (blockIdx.x >> 8) & 1 ? NW - 1 - wid : wid;
  const int r = tile_row * kRows + group * 32 + l, rc = min(r, rows - 1), i = a.by_group.quotient(rc),
            hq = kvh * G + a.by_group.rest(rc, i);
  RowPieces<T, DP, FAST> q, o;
  q.request(a.q.row(n, i, hq), a.D);
  o.request(a.dout.row(n, i, hq), a.D);
  const int64_t id = ((int64_t)n * a.sight.Tq + i) * a.Hq + hq;
  const float lse = r < rows && (!a.sight.q_mask || a.sight.q_mask[(int64_t)n * a.sight.Tq + i]) ? a.lse[id] : -INFINITY;
  const bool live = lse != -INFINITY;
  float lse2 = live ? lse * 1.4426950408889634f : INFINITY, low = 0.f;
  const uint32_t mine = (uint32_t)__ballot(live);
  if (lane == 0) all[group] = mine;
  q.settle(live, a.D);
  o.settle(live, a.D);
  float delta = 0.f, square = 0.f;
  {
    const int64_t at = n * a.out_n + i * a.out_t + hq * a.out_h;
    const int D = FAST ? DP : a.D;
    if (a.out_f32) {
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        float y[kPiece<T>];
        load_piece<float, kPiece<T>>(static_cast<const float*>(a.out) + at, RowPieces<T, DP, FAST>::at(st), D, 0.f, y);
#pragma unroll
        for (int e = 0; e < kPiece<T>; ++e) delta += (float)o.f[st][e] * y[e];
      }
    } else {
      RowPieces<T, DP, FAST> y;
      y.load(static_cast<const T*>(a.out) + at, live, a.D);
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
#pragma unroll
        for (int e = 0; e < kPiece<T>; ++e) delta += (float)o.f[st][e] * (float)y.f[st][e];
    }
    delta = half_sum(delta);
    delta = live ? delta : 0.f;                          // (whatever the output holds there)
    if constexpr (kLiftBack<T> != 0.f) {
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
#pragma unroll
        for (int e = 0; e < kPiece<T>; ++e) square += (float)o.f[st][e] * (float)o.f[st][e];
      square = half_sum(square);
      // (the largest of a set does not depend on the order)
      if (live && h == 0) atomicMax(a.norms + 2 * unit, __float_as_uint(square == square ? square : 0.f));
    }
  }
  // keys that any row of the block sees, those that any of the wave does, and those that every row of it does
  const bool far_row = is_far(lse2, kFarLse);
  const int far_block = __syncthreads_or(far_row);
  LiveRows block{all[0] | (uint64_t)all[1] << 32, 0};
  if constexpr (NW > 2) block.high = all[2] | (uint64_t)all[3] << 32;
  auto position = [&](int at) { return start + a.by_group.quotient(tile_row * kRows + at); };
  const uint8_t* kmask = a.sight.k_mask ? a.sight.k_mask + (int64_t)n * a.sight.Tk : nullptr;
  Bounds bd{0, 0, 0, 0};
  Span some{0, 0, 0};
  int lo_max = 0, hi_min = a.sight.Tk;
  if (!block.none()) {
    const int64_t p0 = position(block.first()), p1 = position(block.last());
    MaskRange range{0, 0, true};
    if (kmask) range = range_of(a.sight, kmask, p0, p1);
    bd = bounds_of(a.sight, p0, p1, range, kmask);
  }
  if (mine) {
    const Span f = span_of(a.sight, position(group * 32 + __builtin_ctz(mine)));
    const Span e = span_of(a.sight, position(group * 32 + 31 - __builtin_clz(mine)));
    some = Span{f.lo, e.hi, e.sk};
    lo_max = e.lo;
    hi_min = f.hi;
  }
  const Span span = live ? span_of(a.sight, start + i) : Span{0, 0, 0};
  const Tiles tiles = tiles_of(bd, KB);

  const RowSource<T> ksrc(a.k.row(n, 0, kvh), a.k.ld_t, a.sight.Tk, DP, FAST), vsrc(a.v.row(n, 0, kvh), a.v.ld_t, a.sight.Tk, DP, FAST);
  Stage<T, DP, KB, NT, FAST> ks, vs;
  const KeyMask km(kmask, ksrc.base, a.sight.Tk);
  if (far_block) {                                       // the far rows' largest scores, and their weights' sums
    float most = kLowest, total = 0.f;
    for (int t = 0; t < tiles.count; ++t) {
      const int j0 = tiles.at(t) * KB;
      ks.request(ksrc, j0, threadIdx.x, a.D);
      const uint32_t bits = km.bits(bd, j0, km.request(j0 + l));
      __syncthreads();
      ks.store(threadIdx.x, a.D, lds, bits);
      __syncthreads();
      f32x16 s = zeros16();
#pragma unroll
      for (int k = 0; k < kSteps; ++k) mma(s, row_frag<T, kROWB>(lds, l, k), q.f[k]);
      hide(s, span, bits, j0);
      float top = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
      const float next = fmaxf(most, rounded(half_max(top) * a.scale_log2));
      total *= __builtin_amdgcn_exp2f(most - next);
#pragma unroll
      for (int e = 0; e < 16; ++e) total += __builtin_amdgcn_exp2f(far_score(s[e], a.scale_log2, next));
      most = next;
    }
    total = half_sum(total);
    if (far_row) {
      lse2 = most;
      low = __builtin_amdgcn_logf(total);
    }
    __syncthreads();
  }
  if (r < rows && h == 0) {
    a.lse2[id] = lse2;
    a.low[id] = low;
    a.delta[id] = delta;
  }

  f32x16 dq[kDt];
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt) dq[dt] = zeros16();
  const int lift = kLiftBack<T> == 0.f ? 0 : lift_of(a, unit, square);
  const bool far = __ballot(far_row) != 0;
  const float ref = (far ? low : lse2) - kLiftBack<T>;
  const float ds_by = exp2f((float)lift - kLiftBack<T>);
  uint8_t byte = 0;
  auto request = [&](int tile) {
    const int j0 = tile * KB;
    ks.request(ksrc, j0, threadIdx.x, a.D);
    vs.request(vsrc, j0, threadIdx.x, a.D);
    byte = km.request(j0 + l);
  };
  if (tiles.count > 0) request(tiles.at(0));
  for (int t = 0, turn = 0; t < tiles.count; ++t, turn ^= 1) {
    char *kt = lds + turn * 2 * kTile, *vt = kt + kTile;
    const int j0 = tiles.at(t) * KB;
    const uint64_t bits = km.bits(bd, j0, byte);
    ks.store(threadIdx.x, a.D, kt, bits);
    vs.store(threadIdx.x, a.D, vt, bits);
    __syncthreads();
    if (t + 1 < tiles.count) request(tiles.at(t + 1));
    if (bits != 0 && ((j0 < some.hi && j0 + KB > some.lo) || j0 < some.sk)) {
      f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        mma(s, row_frag<T, kROWB>(kt, l, k), q.f[k]);
        mma(dp, row_frag<T, kROWB>(vt, l, k), o.f[k]);
      }
      const bool full = bits == 0xFFFFFFFFull && j0 >= lo_max && j0 + KB <= hi_min;
      if (!full) hide(s, span, (uint32_t)bits, j0);      // (weights 0)
      if (__builtin_expect(far, 0)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = far_score(s[e], a.scale_log2, lse2) - ref;
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], a.scale_log2, -ref);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float d = __builtin_amdgcn_exp2f(s[e]) * (dp[e] - delta);
        if constexpr (kLiftBack<T> != 0.f) d *= ds_by;
        s[e] = d;
      }
      Frag<T> ds[kKs];
#pragma unroll
      for (int k = 0; k < kKs; ++k) ds[k] = acc_frag<T>(s, k);
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int k = 0; k < kKs; ++k) mma(dq[dt], col_frag<T, kROWB>(kt, 0, k, dt), ds[k]);
    }
  }
  if (r >= rows) return;
  const float by = a.scale * exp2f(-(float)lift);
  T* to = a.dq.row(n, i, hq);
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = live ? dq[dt][4 * g + e] * by : 0.f;
      put4<T, FAST>(to, dt * 32 + 8 * g + 4 * h, FAST ? DP : a.D, v);
    }
}

constexpr int64_t kSplitBlocks = 4 * kCus;     // twice as many as are there at once: the first have more to do

// Workers that share a key tile's rows, none with fewer than 8 tiles.
int back_splits(int64_t N, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int share) {
  const int64_t blocks = N * Hkv * ceil_div(Tk, 32 * share), tiles = ceil_div(Hq / Hkv * Tq, 32);
  return (int)std::min<int64_t>(std::max<int64_t>(1, tiles / 8), std::max<int64_t>(1, kSplitBlocks * 4 / share / std::max<int64_t>(1, blocks)));
}

}  // namespace

// Bytes for any call of up to N examples, Tq queries and Tk keys: launches with several workers a key tile have at most
// kSplitBlocks blocks of 128 keys (or four times as many of 32), and a worker has no fewer than 8 tiles of 32 rows.
size_t attention_back_ws(eogp_dtype t, int64_t N, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D) {
  size_t bytes = 3 * align256((size_t)(N * Tq * Hq) * sizeof(float)) + 256;
  if (t == EOGP_F16) bytes += align256((size_t)(2 * N * Hkv) * sizeof(float));
  const int64_t most = ceil_div(Hq / Hkv * Tq, 32) / 8;
  if (most > 1)
    bytes += align256((size_t)std::min(most * (N * Hkv * Tk), kSplitBlocks * 128) * (2 * D) * sizeof(float));
  return bytes;
}

eogp_status attention_back(const eogp_heads& dout, const eogp_heads& q, const eogp_heads& k, const eogp_heads& v,
                           const eogp_heads& out, const eogp_heads& dq, const eogp_heads& dk, const eogp_heads& dv,
                           eogp_dtype t, eogp_dtype out_t, int64_t N, int64_t Tq, int64_t Tk, int64_t D, float scale,
                           int causal, int64_t window, int64_t sinks, const int64_t* q_start, const uint8_t* q_mask,
                           const uint8_t* k_mask, const float* lse, void* ws, hipStream_t s) {
  if (N == 0) return EOGP_OK;
  const int64_t Hq = q.heads, Hkv = k.heads, units = N * Hkv;
  timing::Scope ts(EOGP_KT_ATTENTION, s);
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    BackArgs<T> a{};
    auto in = [](const eogp_heads& x) {
      return Heads<const T>{static_cast<const T*>(x.data), x.ld_example, x.ld_token, x.ld_head};
    };
    a.q = in(q);
    a.k = in(k);
    a.v = in(v);
    a.dout = in(dout);
    a.out = out.data;
    a.out_n = out.ld_example;
    a.out_t = out.ld_token;
    a.out_h = out.ld_head;
    a.out_f32 = out_t == EOGP_F32;
    a.dq = heads_of<T>(dq);
    a.dk = heads_of<T>(dk);
    a.dv = heads_of<T>(dv);
    a.sight = Sight{causal, (int)std::min<int64_t>(window, 1 << 30), (int)std::min<int64_t>(sinks, 1 << 30), (int)Tq, (int)Tk,
                    q_start, q_mask, k_mask};
    a.N = (int)N;
    a.Hq = (int)Hq;
    a.Hkv = (int)Hkv;
    a.D = (int)D;
    a.by_group = Divide(Hq / Hkv);
    a.by_units = Divide(units);
    a.by_heads = Divide(Hkv);
    a.scale = scale;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.lse = lse;
    const int share = back_share((int)sizeof(T), padded(D));
    a.splits = back_splits(N, Tq, Tk, Hq, Hkv, share);
    a.by_splits = Divide(a.splits);
    a.key_tiles = (int)ceil_div(Tk, 32 * share);
    a.row_tiles = (int)ceil_div(Hq / Hkv * Tq, 32 * share);
    Carve w(ws, ~(size_t)0);
    a.lse2 = w.take<float>(N * Tq * Hq);
    a.low = w.take<float>(N * Tq * Hq);
    a.delta = w.take<float>(N * Tq * Hq);
    if (t == EOGP_F16) a.norms = w.take<uint32_t>(2 * units);
    a.part = a.splits > 1 ? w.take<float>((size_t)a.splits * (units * Tk * 2 * D)) : nullptr;

    const int64_t rows = N * Tq * Hq, keys = N * Tk * Hkv;
    if (t == EOGP_F16) {
      int lanes = 1;
      while (lanes * kPiece<T> < D) lanes *= 2;
      hipLaunchKernelGGL(k_attend_zero, dim3((unsigned)std::min<int64_t>(ceil_div(2 * units, 256), 4 * kCus)), dim3(256), 0, s,
                         a.norms, 2 * units);
      EOGP_LAUNCH_CHECK("attention_backward (zero)");
      if (keys > 0) {
        const int64_t chunks = ceil_div(Tk * Hkv, kNormSteps * 4 * (64 / lanes));
        hipLaunchKernelGGL(k_attend_norms<T>, dim3((unsigned)std::min<int64_t>(N * chunks, 16 * kCus)), dim3(256), 0, s, a, lanes,
                           (int)chunks);
        EOGP_LAUNCH_CHECK("attention_backward (norms)");
      }
    }
    const int size = (int)sizeof(T);
    const bool fast = fast_rows(q, Tq, D, size) && fast_rows(dout, Tq, D, size) && fast_rows(k, Tk, D, size) && fast_rows(v, Tk, D, size);
    auto go = [&](auto width, auto exact) {
      constexpr int DP = decltype(width)::value;
      constexpr bool FAST = decltype(exact)::value;
      constexpr int lds = 4 * 32 * DP * (int)sizeof(T);
      auto launch = [&](auto* kfn, int64_t blocks) {
        if (lds > (48 << 10)) {
          const eogp_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(kfn), lds);
          if (st != EOGP_OK) return st;
        }
        hipLaunchKernelGGL(kfn, dim3((unsigned)blocks), dim3(64 * back_share((int)sizeof(T), DP)), lds, s, a);
        EOGP_LAUNCH_CHECK("attention_backward");
        return EOGP_OK;
      };
      eogp_status st = EOGP_OK;
      if (rows > 0) st = launch(k_attend_back_q<T, DP, FAST>, units * a.row_tiles);
      if (st == EOGP_OK && keys > 0) {
        const int64_t blocks = units * a.key_tiles * a.splits;
        if constexpr (!kv_together(DP)) {
          st = launch(k_attend_back_kv<T, DP, 1, FAST>, blocks);
          if (st == EOGP_OK) st = launch(k_attend_back_kv<T, DP, 2, FAST>, blocks);
        } else {
          st = launch(k_attend_back_kv<T, DP, 3, FAST>, blocks);
        }
        if (st != EOGP_OK) return st;
        if (a.part) {
          const dim3 grid((unsigned)std::min<int64_t>(ceil_div(keys * 2 * D / (D % 4 ? 1 : 4), 256), 32 * kCus));
          if (D % 4 == 0)
            hipLaunchKernelGGL((k_attend_back_join<T, 4>), grid, dim3(256), 0, s, a);
          else
            hipLaunchKernelGGL((k_attend_back_join<T, 1>), grid, dim3(256), 0, s, a);
          EOGP_LAUNCH_CHECK("attention_backward (join)");
        }
      }
      return st;
    };
    auto with = [&](auto exact) {
      using std::integral_constant;
      return D <= 64    ? go(integral_constant<int, 64>{}, exact)
             : D <= 128 ? go(integral_constant<int, 128>{}, exact)
                        : go(integral_constant<int, 256>{}, exact);
    };
    return fast ? with(std::true_type{}) : with(std::false_type{});
  });
}

}  // namespace eogp
