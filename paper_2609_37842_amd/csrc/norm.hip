// Layer norm over the width of each row, forward and backward.
#include <algorithm>

#include "rows.h"
#include "timing.h"

namespace eogp {
namespace {

// WPR waves share a row: sum of v over the row, in every lane of its waves. `slot` is LDS of the
// block for 2 x 16 floats, used alternately so that one barrier per sum is enough.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* slot) {
  v = wave_sum(v);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slot[0];
#pragma unroll
    for (int w = 1; w < WPR; ++w) v += slot[w];
  }
  return v;
}

// A block's weights in LDS, fp32 (gamma 1 and beta 0 where there is none): as registers they would
// cost the kernels half of their waves. The places up to a whole piece of E hold zeros: what LDS held
// before may be a NaN, and 0 times it would be one.
template <int NT, int E>
__device__ __forceinline__ void stage_weights(float* lds, const void* w, eogp_dtype wt, int64_t d, float none) {
  for (int c = threadIdx.x; c < (d + E - 1) / E * E; c += NT) lds[c] = c >= d ? 0.f : w ? load_any(w, wt, c) : none;
}

// The valid rows among first, first + step, ... of a wave, in order. The masks (and the means
// and reciprocal deviations) of 64 rows are read at once, a row per lane, so that a row costs no wait
// for them. VALUES: 1 for the mask alone, 3 with the statistics.
template <int VALUES>
struct RowQueue {
  const uint8_t* mask;
  const float *means, *rstds;
  int64_t first, step, n;
  uint64_t live = 0, masked = 0;               // bits of the 64 rows from `first` on that are left
  float lane_mean = 0.f, lane_rstd = 0.f;

  __device__ __forceinline__ RowQueue(const uint8_t* m, const float* me, const float* rs, int64_t f, int64_t st,
                                      int64_t rows)
      : mask(m), means(me), rstds(rs), first(f - 64 * st), step(st), n(rows) {}

  // The next valid row, -1 at the end; skip(row) for the masked ones of a batch when it is taken up.
  template <typename Skip>
  __device__ __forceinline__ int64_t next(Skip&& skip) {
    while (!live) {
      first += 64 * step;
      if (first >= n) return -1;
      const int64_t mine = first + (threadIdx.x & 63) * step;
      const bool in = mine < n, ok = in && (!mask || mask[mine] != 0);
      live = __ballot(ok);
      masked = __ballot(in && !ok);
      if constexpr (VALUES > 1) {
        lane_mean = ok ? means[mine] : 0.f;
        lane_rstd = ok ? rstds[mine] : 0.f;
      }
      for (; masked; masked &= masked - 1) skip(first + __builtin_ctzll(masked) * step);
    }
    const int at = __builtin_ctzll(live);
    live &= live - 1;
    mean = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(__float_as_uint(lane_mean), at));
    rstd = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(__float_as_uint(lane_rstd), at));
    return first + at * step;
  }
  float mean = 0.f, rstd = 0.f;                // of the row that next returned
};

constexpr int norm_threads(int wpr) { return wpr > 4 ? 64 * wpr : 256; }

// Blocks of the forward pass on a CU, by its registers (elements of a lane).
constexpr int norm_per_cu(int wpr, int elements) {
  if (wpr > 4) return elements <= 8 ? 2 : 1;
  return elements <= 8 ? 8 : elements <= 12 ? 7 : elements <= 16 ? 6 : 4;
}

// y = (x - mean) rstd gamma + beta, rstd = (mean (x - mean)^2 + eps)^-1/2, one row at a time: the row stays in
// registers (P pieces of 16 bytes per lane), so the mean and the centred second moment are two passes over
// registers (no difference of large sums) and HBM sees one read and one write. Statistics and weights are
// fp32; y is rounded once.
// Bound by HBM. 65,536 places of 768 fp32, 56% of them valid, with the column of ones: 67 us, 4.7 TB/s; 16 rows
// (a token of a batch each): 5 us, a row's round trips.
template <typename TI, typename TO, int WPR, int SHAPE>
__global__ __launch_bounds__(norm_threads(WPR), norm_per_cu(WPR, SHAPE * kPiece<TI>) * norm_threads(WPR) / 256)
void k_layer_norm(
    const TI* __restrict__ x, int64_t ldx, const void* __restrict__ gamma, const void* __restrict__ beta,
    eogp_dtype wt, float eps, const uint8_t* __restrict__ mask, int64_t n, int64_t d, TO* __restrict__ y,
    int64_t ldy, int ones, float* __restrict__ mean_out, float* __restrict__ rstd_out) {
  constexpr int E = kPiece<TI>, NT = norm_threads(WPR), P = SHAPE ? SHAPE : 1;
  constexpr bool kNarrow = SHAPE == 0;
  constexpr int kRows = NT / 64 / WPR;                 // of a block at once
  extern __shared__ __align__(16) float weights[];     // gamma, beta: round_up(d, E) each
  __shared__ float slot[2][16];
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (rows and their addresses are scalar)
  const int t = WPR == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;   // place among the row's lanes
  float *g = weights, *b = weights + (d + E - 1) / E * E;
  const float width = (float)d;               // sums are divided by it: a constant row's mean is exact
  RowQueue<1> queue(mask, nullptr, nullptr, (int64_t)blockIdx.x * kRows + (WPR == 1 ? wid : 0),
                    (int64_t)gridDim.x * kRows, n);
  auto none = [&](int64_t row) {              // not read; zeros
    TO* yr = y + row * ldy;
    float zero[E] = {};
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = (int64_t)(p * 64 * WPR + t) * E;
      if (c < d) store_piece<TO, E>(yr, c, d, zero);
    }
    if (t == 0) {
      if (ones) yr[d] = (TO)0.f;
      if (mean_out) mean_out[row] = 0.f;
      if (rstd_out) rstd_out[row] = 0.f;
    }
  };
  AnyVec<TI, E> raw[P];
  auto load = [&](int64_t row) {
#pragma unroll
    for (int p = 0; p < P; ++p)
      raw[p] = request_piece<TI, E, kNarrow>(x + row * ldx, (int64_t)(p * 64 * WPR + t) * E, d);
  };
  int64_t row = queue.next(none);
  if (row >= 0) load(row);
  stage_weights<NT, E>(g, gamma, wt, d, 1.f);    // while the first row is on its way
  stage_weights<NT, E>(b, beta, wt, d, 0.f);
  __syncthreads();
  while (row >= 0) {
    float v[P][E];
    float s = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      settle_piece<TI, E, kNarrow>(raw[p], (int64_t)(p * 64 * WPR + t) * E, d);
      widen<TI, E>(raw[p], v[p]);
#pragma unroll
      for (int e = 0; e < E; ++e) s += v[p][e];
    }
    const int64_t after = queue.next(none);
    if (after >= 0) load(after);              // the next row, while this one is summed and written
    const float mean = row_sum<WPR>(s, slot[0]) / width;
    s = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int64_t c = (int64_t)(p * 64 * WPR + t) * E + e;
        v[p][e] = c < d ? v[p][e] - mean : 0.f;
        s += v[p][e] * v[p][e];
      }
    const float rstd = 1.f / sqrtf(row_sum<WPR>(s, slot[1]) / width + eps);
    TO* yr = y + row * ldy;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = (int64_t)(p * 64 * WPR + t) * E;
      if (c >= d) break;
      const AnyVec<float, E> gp = *reinterpret_cast<const AlignedVec<float, E>*>(g + c);
      const AnyVec<float, E> bp = *reinterpret_cast<const AlignedVec<float, E>*>(b + c);
#pragma unroll
      for (int e = 0; e < E; ++e) v[p][e] = v[p][e] * rstd * gp[e] + bp[e];
      store_piece<TO, E>(yr, c, d, v[p]);
    }
    if (t == 0) {
      if (ones) yr[d] = (TO)1.f;
      if (mean_out) mean_out[row] = mean;
      if (rstd_out) rstd_out[row] = rstd;
    }
    row = after;
  }
}

// dx = rstd (t - mean(t) - xh mean(t xh)) [+ residual gradient], t = dy gamma, xh = (x - mean) rstd,
// and the column sums of dy xh and dy over the block's rows, kept in registers from row to row.
// Group k (of rows_per_group rows) has `splits` blocks; block j takes its rows j, j + splits, ...
// (times the rows a block holds at once) and writes its sums to part[k][j][2][d]. A row's three
// inputs are requested together and stay as read (16-bit rows in half the registers); xh and t are
// formed twice, once for the sums and once for dx. All arithmetic is fp32; dx is rounded once.
// Bound by HBM. 65,536 places of 768 fp32, 56% of them valid, with the residual gradient and the weights'
// gradients of 128 examples: 120 us and 8 for the fold of their partial sums, 4.3 TB/s; 32,768 rows of 5120
// bf16: 242 us, 5.5 TB/s. Rows of more than 8,192 elements spill registers: 8,192 fp32 rows of 12,288 436 us,
// 2.8 TB/s (of 8,192 elements 145 us, 5.5 TB/s), 16,384 bf16 rows of 16,384 460 us, 3.5 TB/s.
template <typename T, int WPR, int SHAPE>
__global__ __launch_bounds__(norm_threads(WPR)) void k_layer_norm_back(
    const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx,
    const void* __restrict__ gamma, eogp_dtype wt, const float* __restrict__ mean_in,
    const float* __restrict__ rstd_in, const uint8_t* __restrict__ mask, const T* res,
    int64_t ldres, int64_t rows_per_group, int64_t d, int splits, T* dx, int64_t lddx,
    float* __restrict__ part, float* __restrict__ dgamma, float* __restrict__ dbeta) {
  constexpr int E = kPiece<T>, NT = norm_threads(WPR), P = SHAPE ? SHAPE : 1;
  constexpr bool kNarrow = SHAPE == 0;
  constexpr int kRows = NT / 64 / WPR;
  extern __shared__ __align__(16) float weights[];     // gamma: round_up(d, E)
  __shared__ float slot[2][2][16];
  __shared__ float fold[WPR == 1 ? 3 * 64 * E : 1];
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (rows and their addresses are scalar)
  const int t = WPR == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
  float ag[P][E], ab[P][E];
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int e = 0; e < E; ++e) ag[p][e] = ab[p][e] = 0.f;
  stage_weights<NT, E>(weights, gamma, wt, d, 1.f);
  __syncthreads();
  const float inv_width = 1.f / (float)d;
  const int64_t group = blockIdx.x / splits, split = blockIdx.x % splits;
  const int64_t row0 = group * rows_per_group;
  RowQueue<3> queue(mask ? mask + row0 : nullptr, mean_in + row0, rstd_in + row0,
                    split * kRows + (WPR == 1 ? wid : 0), (int64_t)splits * kRows, rows_per_group);
  auto none = [&](int64_t i) {               // not read; zeros
    float zero[E] = {};
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = (int64_t)(p * 64 * WPR + t) * E;
      if (c < d) store_piece<T, E>(dx + (row0 + i) * lddx, c, d, zero);
    }
  };
  // Rows ahead of their turn where two fit the registers (else the block's other waves and the CU's
  // other blocks have theirs on the way).
  constexpr bool kAhead = P * E <= (WPR <= 4 ? 16 : 8);
  struct Inputs {
    AnyVec<T, E> x[P], dy[P], res[P];
  };
  auto load = [&](int64_t i, Inputs& in) {
    const int64_t row = row0 + i;
    // (streaming loads: 32,768 rows of 5120 bf16 in 243 us, 248 without; 65,536 places of 768 fp32 127.6 and 130.8)
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = (int64_t)(p * 64 * WPR + t) * E;
      in.x[p] = request_piece<T, E, kNarrow, true>(x + row * ldx, c, d);
      in.dy[p] = request_piece<T, E, kNarrow, true>(dy + row * lddy, c, d);
    }
    if (res) {
#pragma unroll
      for (int p = 0; p < P; ++p)
        in.res[p] = request_piece<T, E, kNarrow, true>(res + row * ldres, (int64_t)(p * 64 * WPR + t) * E, d);
    }
  };
  int turn = 0;
  Inputs now, ahead;
  int64_t i = queue.next(none);
  if (kAhead && i >= 0) load(i, ahead);
  while (i >= 0) {
    const float mean = queue.mean, rstd = queue.rstd;
    T* out = dx + (row0 + i) * lddx;
    int64_t after;
    if constexpr (kAhead) {
      now = ahead;
      after = queue.next(none);
      if (after >= 0) load(after, ahead);
    } else {
      load(i, now);
      after = queue.next(none);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * 64 * WPR + t) * E;
      settle_piece<T, E, kNarrow>(now.x[p], c, d);
      settle_piece<T, E, kNarrow>(now.dy[p], c, d);             // (0 past the end: no sum sees x there)
      if (res) settle_piece<T, E, kNarrow>(now.res[p], c, d);
      AnyVec<float, E> gp;
      if (c < d) gp = *reinterpret_cast<const AlignedVec<float, E>*>(weights + c);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float xh = ((float)now.x[p][e] - mean) * rstd, g = (float)now.dy[p][e];
        ag[p][e] += g * xh;
        ab[p][e] += g;
        const float tv = c < d ? g * gp[e] : 0.f;
        s1 += tv;
        s2 += tv * xh;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if constexpr (WPR > 1) {
      float* q = &slot[turn][0][0];
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
        q[wid] = s1;
        q[16 + wid] = s2;
      }
      __syncthreads();
      s1 = q[0];
      s2 = q[16];
#pragma unroll
      for (int w = 1; w < WPR; ++w) {
        s1 += q[w];
        s2 += q[16 + w];
      }
    }
    s1 *= inv_width;
    s2 *= inv_width;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = (int64_t)(p * 64 * WPR + t) * E;
      if (c >= d) break;
      const AnyVec<float, E> gp = *reinterpret_cast<const AlignedVec<float, E>*>(weights + c);
      AnyVec<T, E> xc = now.x[p], dc = now.dy[p];
      asm volatile("" : "+v"(xc), "+v"(dc));           // formed again, not kept from the sums' pass
      float r[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float xh = ((float)xc[e] - mean) * rstd;
        r[e] = rstd * ((float)dc[e] * gp[e] - s1 - xh * s2) + (res ? (float)now.res[p][e] : 0.f);
      }
      store_piece<T, E>(out, c, d, r);
      __builtin_amdgcn_sched_barrier(0);
    }
    i = after;
  }
  // a group's only block writes its gradients, others their sums for k_norm_fold
  float *pg = part ? part + (int64_t)blockIdx.x * 2 * d : nullptr, *pb = part ? pg + d : nullptr;
  if (splits == 1) {
    pg = dgamma ? dgamma + group * d : nullptr;
    pb = dbeta ? dbeta + group * d : nullptr;
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int64_t c = (int64_t)(p * 64 * WPR + t) * E;
    if constexpr (WPR == 1) {                // the block's four rows at a time, in order of their waves
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        float(&a)[E] = which ? ab[p] : ag[p];
        __syncthreads();
        if (wid > 0)
#pragma unroll
          for (int e = 0; e < E; ++e) fold[((wid - 1) * 64 + t) * E + e] = a[e];
        __syncthreads();
        if (wid == 0)
#pragma unroll
          for (int e = 0; e < E; ++e)
            a[e] += fold[t * E + e] + fold[(64 + t) * E + e] + fold[(128 + t) * E + e];
      }
      if (wid > 0) continue;
    }
    if (c < d) {
      if (pg) store_piece<float, E>(pg, c, d, ag[p]);
      if (pb) store_piece<float, E>(pb, c, d, ab[p]);
    }
  }
}

// Column sums of the blocks' partial sums, in a fixed order: 32 columns x SLICES slices of the blocks
// per block, eight requests of a thread at a time.
template <int SLICES>
__global__ __launch_bounds__(32 * SLICES) void k_norm_fold(const float* __restrict__ part, int64_t groups, int splits,
                                                           int64_t d, float* __restrict__ dgamma,
                                                           float* __restrict__ dbeta) {
  __shared__ float sum[SLICES][33];
  const int col = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int64_t col_blocks = (2 * d + 31) / 32;
  for (int64_t unit = blockIdx.x; unit < groups * col_blocks; unit += gridDim.x) {
    const int64_t group = unit / col_blocks, c = unit % col_blocks * 32 + col;   // of the 2 d columns
    const float* from = part + group * splits * 2 * d + c;
    float s = 0.f;
    if (c < 2 * d) {
      for (int j = slice; j < splits; j += 8 * SLICES) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int at = j + k * SLICES;
          v[k] = at < splits ? from[(int64_t)at * 2 * d] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[k];
      }
    }
    sum[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < 2 * d) {
#pragma unroll
      for (int k = 1; k < SLICES; ++k) s += sum[k][col];
      float* out = c < d ? dgamma : dbeta;
      if (out) out[group * d + (c < d ? c : c - d)] = s;
    }
    __syncthreads();
  }
}

// Waves per row and 16-byte pieces per lane (0: a row is shorter than a piece) for rows of d: one wave while four pieces a
// lane hold the row (no barrier per row), then four waves, then sixteen. The backward pass goes over to
// sixteen waves at 512 pieces, the forward pass at 768: its three rows and two sums take a lane of three
// pieces too many registers, and blocks of many waves leave fewer partial sums (3,906 rows of 5120
// bf16 47 us, with four waves and three pieces 63; 18,310 of 8192 212 us, with four pieces 326).
template <typename T, bool BACK, typename F>
eogp_status with_shape(int64_t d, F&& f) {
  using std::integral_constant;
  using One = integral_constant<int, 1>;
  using Four = integral_constant<int, 4>;
  using Sixteen = integral_constant<int, 16>;
  const int64_t pieces = ceil_div(d, kPiece<T>);
  if (d < kPiece<T>) return f(One{}, integral_constant<int, 0>{});
  if (pieces <= 64) return f(One{}, integral_constant<int, 1>{});
  if (pieces <= 128) return f(One{}, integral_constant<int, 2>{});
  if (pieces <= 192) return f(One{}, integral_constant<int, 3>{});
  if (pieces <= 256) return f(One{}, integral_constant<int, 4>{});
  if (pieces <= 512) return f(Four{}, integral_constant<int, 2>{});
  if constexpr (!BACK)
    if (pieces <= 768) return f(Four{}, integral_constant<int, 3>{});
  if (pieces <= 1024) return f(Sixteen{}, integral_constant<int, 1>{});
  if constexpr (sizeof(T) == 4)              // (16-bit rows of up to 16,384 elements have 2,048 pieces)
    if (pieces > 2048) return f(Sixteen{}, integral_constant<int, 4>{});
  return f(Sixteen{}, integral_constant<int, 2>{});
}

int rows_per_block(int64_t pieces) { return pieces <= 256 ? 4 : 1; }

constexpr int kStaticLds = 48 << 10;         // dynamic LDS that needs no permission

int64_t weight_bytes(int64_t d, eogp_dtype t) { return round_up(d, t == EOGP_F32 ? 4 : 8) * (int64_t)sizeof(float); }

int64_t row_pieces(int64_t d, eogp_dtype t) { return ceil_div(d, t == EOGP_F32 ? 4 : 8); }

}  // namespace

int64_t norm_max_width() { return 16384; }   // 16 waves x 64 lanes x 4 pieces of 4 fp32

eogp_status layer_norm(const void* x, eogp_dtype xt, int64_t ldx, const void* gamma, const void* beta,
                       eogp_dtype wt, float eps, const uint8_t* mask, int64_t n, int64_t d, void* y,
                       eogp_dtype yt, int64_t ldy, int ones, float* mean, float* rstd, hipStream_t s) {
  if (n == 0) return EOGP_OK;
  const int64_t pieces = row_pieces(d, xt);
  timing::Scope ts(EOGP_KT_LAYER_NORM, s);
  return with_type(xt, [&](auto ti) {
    using TI = decltype(ti);
    auto go = [&](auto to) {
      using TO = decltype(to);
      return with_shape<TI, false>(d, [&](auto wpr, auto p) {
        constexpr int W = decltype(wpr)::value;
        auto* kfn = k_layer_norm<TI, TO, W, decltype(p)::value>;
        const int lds = 2 * (int)weight_bytes(d, xt);
        // no more blocks than are there at once: rows are dealt out to them, and each reads the weights
        const int64_t per_cu = std::min<int64_t>(norm_per_cu(W, decltype(p)::value * kPiece<TI>),
                                                 std::max<int64_t>(1, (160 << 10) / (lds + 256)));
        const int64_t blocks = std::min<int64_t>(ceil_div(n, rows_per_block(pieces)), per_cu * kCus);
        if (lds > kStaticLds) {
          const eogp_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(kfn), lds);
          if (st != EOGP_OK) return st;
        }
        hipLaunchKernelGGL(kfn, dim3((unsigned)blocks), dim3(norm_threads(W)), lds, s, static_cast<const TI*>(x), ldx,
                           gamma, beta, wt, eps, mask, n, d, static_cast<TO*>(y), ldy, ones, mean, rstd);
        EOGP_LAUNCH_CHECK("layer_norm");
        return EOGP_OK;
      });
    };
    return yt == xt ? go(TI{}) : go(float{});
  });
}

namespace {
// Blocks of a launch that sums columns, and the rows up to which a group has one block: so few that a second launch
// would cost more than their turns.
int64_t back_blocks(int64_t pieces) { return pieces <= 512 ? 4 * kCus : kCus; }
bool one_block(int64_t rows, int64_t pieces) { return rows <= 4 * rows_per_block(pieces); }

// Blocks of a group: as many as are there at once, no more than its rows need.
int back_splits(int64_t groups, int64_t rows, int64_t pieces) {
  if (one_block(rows, pieces)) return 1;
  return (int)std::min(ceil_div(rows, rows_per_block(pieces)), ceil_div(back_blocks(pieces), groups));
}
}  // namespace

size_t layer_norm_back_ws(int64_t groups, int64_t rows, int64_t d, eogp_dtype t) {
  // The partial sums of as many blocks as any launch of up to `groups` groups of up to `rows` rows writes, so that
  // the workspace for a batch serves every smaller one. A group's only block writes its gradients itself; those of
  // several, ceil(most / g) each, are at most g + most - 1 for g groups, and less than most groups have several.
  const int64_t pieces = row_pieces(d, t), most = back_blocks(pieces);
  const int64_t blocks = one_block(rows, pieces) ? 0
                                                 : std::min(groups * ceil_div(rows, rows_per_block(pieces)),
                                                            std::min(groups, most - 1) + most - 1);
  return align256(std::max<size_t>(1, (size_t)blocks * 2 * d * sizeof(float)));
}

eogp_status layer_norm_back(const void* dy, int64_t lddy, const void* x, int64_t ldx, eogp_dtype t,
                            const void* gamma, eogp_dtype wt, const float* mean, const float* rstd,
                            const uint8_t* mask, const void* res, int64_t ldres, int64_t groups,
                            int64_t rows, int64_t d, void* dx, int64_t lddx, float* dgamma,
                            float* dbeta, void* ws, hipStream_t s) {
  if (groups == 0) return EOGP_OK;
  const int64_t pieces = row_pieces(d, t);
  const int splits = back_splits(groups, rows, pieces);
  float* part = dgamma || dbeta ? static_cast<float*>(ws) : nullptr;   // (NULL: nobody wants the sums)
  timing::Scope ts(EOGP_KT_LAYER_NORM, s);
  const eogp_status st = with_type(t, [&](auto el) {
    using T = decltype(el);
    return with_shape<T, true>(d, [&](auto wpr, auto p) {
      constexpr int W = decltype(wpr)::value;
      auto* kfn = k_layer_norm_back<T, W, decltype(p)::value>;
      const int lds = (int)weight_bytes(d, t);
      if (lds > kStaticLds) {
        const eogp_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(kfn), lds);
        if (st != EOGP_OK) return st;
      }
      hipLaunchKernelGGL(kfn, dim3((unsigned)(groups * splits)), dim3(norm_threads(W)), lds, s,
                         static_cast<const T*>(dy), lddy, static_cast<const T*>(x), ldx, gamma, wt, mean, rstd, mask,
                         static_cast<const T*>(res), ldres, rows, d, splits, static_cast<T*>(dx), lddx, part, dgamma,
                         dbeta);
      EOGP_LAUNCH_CHECK("layer_norm_backward");
      return EOGP_OK;
    });
  });
  if (st != EOGP_OK) return st;
  if (splits == 1 || (!dgamma && !dbeta)) return EOGP_OK;
  const int64_t fold_blocks = std::min<int64_t>(groups * ceil_div(2 * d, 32), 1 << 20);
  const bool many = splits > 64;
  hipLaunchKernelGGL(many ? k_norm_fold<32> : k_norm_fold<8>, dim3((unsigned)fold_blocks), dim3(many ? 1024 : 256), 0,
                     s, part, groups, splits, d, dgamma, dbeta);
  EOGP_LAUNCH_CHECK("layer_norm_backward (fold)");
  return EOGP_OK;
}

}  // namespace eogp
