// Softmax attention over the keys that each query sees, for batches and for single tokens over a cache.
#include <algorithm>

#include "attend.h"
#include "timing.h"

namespace eogp {
namespace {

template <typename T>
struct AttendArgs {
  Heads<const T> q, k, v;
  void* out;                      // rows of T or fp32
  int64_t out_n, out_t, out_h;
  int out_f32;
  Sight sight;
  int N, Hq, Hkv, D;
  Divide by_group;                // query heads of a key head
  float scale_log2;               // scale log2(e): weights are powers of two of scores times it
  float* lse;                     // [N, Tq, Hq] or NULL
  int row_tiles, splits;
  float* part;                    // splits > 1 or several waves of keys: [workers][rows of all][D + 2]
};

// Weights are 2^(score - reference); the reference follows a row's maximum only when that has grown by 2^kLag,
// so sums and outputs are seldom rescaled. 16-bit weights keep their relative precision wherever the
// reference lies (fp16: 2^kLift keeps small ones out of its subnormals, and 2^(kLift + kLag) below its largest).
constexpr float kLag = 8.f;
template <typename T> constexpr float kLift = 0.f;
template <> constexpr float kLift<_Float16> = 7.f;
constexpr float kLowest = -1e30f;   // reference of a row that has seen no key (finite: differences stay numbers)

// What a lane knows of its rows. Rows of a head group: query i of head kvh G + g is row i G + g of key head kvh.
template <typename T, int QG>
struct Rows {
  int i[QG], h[QG];               // query and head of the lane's row in each group of 32
  bool live[QG];
  Span span[QG];
  Bounds b;                       // of the wave's rows

  __device__ __forceinline__ void place(const AttendArgs<T>& a, int n, int kvh, int first, int rows, int64_t start) {
    const int G = a.by_group.by;
    b = Bounds{a.sight.Tk, 0, 0, 0, a.sight.Tk};
#pragma unroll
    for (int qg = 0; qg < QG; ++qg) {
      const int r = first + qg * 32 + (int)(threadIdx.x & 31), rc = r < rows ? r : rows - 1;
      i[qg] = a.by_group.quotient(rc);
      h[qg] = kvh * G + a.by_group.rest(rc, i[qg]);
      live[qg] = r < rows && (!a.sight.q_mask || a.sight.q_mask[(int64_t)n * a.sight.Tq + i[qg]]);
      span[qg] = live[qg] ? span_of(a.sight, start + i[qg]) : Span{0, 0, 0};
      if (live[qg]) {
        const bool some = span[qg].hi > span[qg].lo;
        b.lo_min = min(b.lo_min, some ? span[qg].lo : a.sight.Tk);
        b.hi_max = max(b.hi_max, some ? span[qg].hi : 0);
        b.sk_max = max(b.sk_max, span[qg].sk);
        b.lo_max = max(b.lo_max, span[qg].lo);
        b.hi_min = min(b.hi_min, span[qg].hi);
      }
    }
    b.lo_max = wave_max_i(b.lo_max);
    b.hi_min = wave_min_i(b.hi_min);
    b.lo_min = wave_min_i(b.lo_min);
    b.hi_max = wave_max_i(b.hi_max);
    b.sk_max = wave_max_i(b.sk_max);
  }
};

// Bounds no further than the first and last key that the mask leaves, by the whole block; no mask any more where it
// leaves all between.
template <int NT>
__device__ __forceinline__ void clip_bounds(Bounds& b, const uint8_t*& kmask, int (*slot)[3]) {
  if (!kmask) return;
  const int from = b.sk_max > 0 ? 0 : b.lo_min, to = max(b.hi_max, b.sk_max);
  const MaskRange r = mask_range<NT>(kmask, min(from, to), to, slot);
  b.lo_min = max(b.lo_min, r.first);
  b.hi_max = min(b.hi_max, r.last);
  b.sk_max = b.sk_max > r.first ? min(b.sk_max, r.last) : 0;
  b.first = r.first;
  if (r.solid) kmask = nullptr;
}

// A row group's results: to the output, or unnormalised with their reference and sum to a worker's part.
template <typename T, int DP>
__device__ __forceinline__ void put_rows(const AttendArgs<T>& a, const f32x16* acc, float ref, float sum, int n, int r, int i,
                                         int hq, bool live, int64_t part_row) {
  const int h = (threadIdx.x >> 5) & 1;
  const float total = half_sum(sum);
  if (r < 0) return;
  if (a.part) {                                          // joined by k_attend_join
    float* to = a.part + part_row * (a.D + 2);
    if (h == 0) {
      to[0] = ref;
      to[1] = total;
    }
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float v[4] = {acc[dt][4 * g], acc[dt][4 * g + 1], acc[dt][4 * g + 2], acc[dt][4 * g + 3]};
        store_piece<float, 4>(to + 2, dt * 32 + 8 * g + 4 * h, a.D, v);
      }
    return;
  }
  const bool some = live && total != 0.f;
  const float inv = some ? 1.f / total : 0.f;
  if (a.lse && h == 0)
    a.lse[((int64_t)n * a.sight.Tq + i) * a.Hq + hq] =
        some ? (ref + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
  const int64_t at = n * a.out_n + i * a.out_t + hq * a.out_h;
#pragma unroll
  for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = dt * 32 + 8 * g + 4 * h;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = some ? acc[dt][4 * g + e] * inv : 0.f;
      if (a.out_f32)
        store_piece<float, 4>(static_cast<float*>(a.out) + at, c, a.D, v);
      else
        store_piece<T, 4>(static_cast<T*>(a.out) + at, c, a.D, v);
    }
}

// Keys of a tile that any row of the block sees, as bits, with the mask's byte of the lane's key (1 without a mask).
__device__ __forceinline__ uint32_t tile_bits(const Bounds& b, int j0, uint8_t mask) {
  const uint32_t seen = (bits_between(b.lo_min - j0, b.hi_max - j0) | bits_between(0, b.sk_max - j0)) & ~bits_between(0, b.first - j0);
  return seen & (uint32_t)__ballot(mask != 0);
}
__device__ __forceinline__ uint8_t mask_of(const uint8_t* kmask, int j, int Tk) {
  return kmask ? kmask[j < Tk ? j : Tk - 1] : 1;
}

// Scores that their row does not see become -inf.
__device__ __forceinline__ void hide(f32x16& s, const Span& span, uint32_t bits, int j0) {
  const uint32_t seen = (bits & sight_bits(span, j0)) >> (4 * ((threadIdx.x >> 5) & 1));
#pragma unroll
  for (int e = 0; e < 16; ++e) s[e] = (seen >> (8 * (e / 4) + e % 4)) & 1 ? s[e] : -INFINITY;
}

// Four waves side by side over rows (QG groups of 32 each) share tiles of 32 keys. A step works on three tiles at
// once, which depend on nothing of each other: the products of the next tile's scores, the weights of this one and the
// product of the last one's weights with V, so that the vector units make exponentials while the matrix units multiply.
// (A step's weights may move a row's reference: the output takes its factor at the step's end, when the last tile's
// product, made with the old one, is in.)
template <typename T, int DP, int QG, bool FAST>
__global__ __launch_bounds__(256, DP * QG * (int)sizeof(T) <= 256 ? 2 : 1) void k_attend(const AttendArgs<T> a) {
  constexpr int NWR = 4, NT = 256, KB = 32, kROWB = DP * (int)sizeof(T), kTile = KB * kROWB;
  constexpr int kRows = 32 * QG * NWR, kDt = DP / 32, kSteps = kROWB / 32, kKs = 32 / (2 * kPiece<T>);
  extern __shared__ __align__(16) char lds[];            // [2] K, [2] V
  __shared__ int slot[NWR][3], all[3][NWR];
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 31;
  const int tid = threadIdx.x;
  const int rows = a.by_group.by * a.sight.Tq, units = a.N * a.Hkv;
  // heavier row tiles (later positions) first
  int b = blockIdx.x;
  const int split = b % a.splits;
  b /= a.splits;
  const int unit = b % units, tile_row = a.row_tiles - 1 - b / units, n = unit / a.Hkv, kvh = unit % a.Hkv;
  const int64_t start = a.sight.start(n);
  const int first = tile_row * kRows + wid * QG * 32;
  Rows<T, QG> row;
  row.place(a, n, kvh, first, rows, start);
  Bounds bd = row.b;
  if (lane == 0) {
    all[0][wid] = bd.lo_min;
    all[1][wid] = bd.hi_max;
    all[2][wid] = bd.sk_max;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NWR; ++w) {
    bd.lo_min = min(bd.lo_min, all[0][w]);
    bd.hi_max = max(bd.hi_max, all[1][w]);
    bd.sk_max = max(bd.sk_max, all[2][w]);
  }
  const uint8_t* kmask = a.sight.k_mask ? a.sight.k_mask + (int64_t)n * a.sight.Tk : nullptr;
  clip_bounds<NT>(bd, kmask, slot);
  const Tiles tiles = tiles_of(bd, KB);
  const int t0 = (int)((int64_t)tiles.count * split / a.splits), t1 = (int)((int64_t)tiles.count * (split + 1) / a.splits);

  f32x16 acc[QG][kDt];
  float ref[QG], sum[QG];
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    ref[qg] = kLowest;
    sum[qg] = 0.f;
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) acc[qg][dt] = zeros16();
  }
  if (t0 < t1) {
    RowPieces<T, DP> q[QG];
#pragma unroll
    for (int qg = 0; qg < QG; ++qg) q[qg].load(a.q.row(n, row.i[qg], row.h[qg]), row.live[qg], a.D);
    const RowSource<T> ksrc{a.k.row(n, 0, kvh), a.k.ld_t, a.sight.Tk}, vsrc{a.v.row(n, 0, kvh), a.v.ld_t, a.sight.Tk};
    char *kt = lds, *vt = lds + 2 * kTile;
    Stage<T, DP, KB, NT, FAST> ks, vs;
    auto mask_at = [&](int t) { return mask_of(kmask, tiles.at(t) * KB + l, a.sight.Tk); };
    auto bits_at = [&](int t, uint8_t mask) { return t < t1 ? tile_bits(bd, tiles.at(t) * KB, mask) : 0; };
    uint32_t bits = bits_at(t0, mask_at(t0)), bits_next = bits_at(t0 + 1, mask_at(t0 + 1));   // of the step's tile and the one after it
    ks.request(ksrc, tiles.at(t0) * KB, tid, a.D);
    ks.store(tid, a.D, kt, bits);
    if (t0 + 1 < t1) {
      ks.request(ksrc, tiles.at(t0 + 1) * KB, tid, a.D);
      ks.store(tid, a.D, kt + kTile, bits_next);
    }
    // the first step's product with the tile before: weights 0 of values 0
    for (int c = tid * 16; c < kTile; c += NT * 16) *reinterpret_cast<uint4*>(vt + kTile + c) = uint4{0, 0, 0, 0};
    f32x16 s[2][QG];
    Frag<T> p[2][QG][kKs];
#pragma unroll
    for (int qg = 0; qg < QG; ++qg)
#pragma unroll
      for (int k = 0; k < kKs; ++k)
#pragma unroll
        for (int e = 0; e < kPiece<T>; ++e) p[1][qg][k][e] = (T)0.f;
    __syncthreads();
#pragma unroll
    for (int qg = 0; qg < QG; ++qg) s[0][qg] = zeros16();
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const Frag<T> kf = row_frag<T, kROWB>(kt, l, st);
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) mma(s[0][qg], kf, q[qg].f[st]);
    }
    // Step t, PAR = t - t0 mod 2: K of tile t + 1 and V of tile t - 1 are in the buffers of the other parity; K of
    // t + 2 and V of t are on their way to those of this one.
    auto step = [&](auto parity, int t) {
      constexpr int PAR = decltype(parity)::value;
      __syncthreads();
      const char *kn = kt + (1 - PAR) * kTile, *vl = vt + (1 - PAR) * kTile;
      const bool more = t + 2 < t1;
      if (more) ks.request(ksrc, tiles.at(t + 2) * KB, tid, a.D);
      vs.request(vsrc, tiles.at(t) * KB, tid, a.D);
      const uint8_t mask_after = mask_at(t + 2);
      const int j0 = tiles.at(t) * KB;
      if (!(bits == 0xFFFFFFFFu && j0 >= row.b.lo_max && j0 + KB <= row.b.hi_min)) {
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) hide(s[PAR][qg], row.span[qg], bits, j0);
      }
      float next[QG], by_sum[QG];
      bool moved = false;
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) {
        s[1 - PAR][qg] = zeros16();
        float most = s[PAR][qg][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) most = fmaxf(most, s[PAR][qg][e]);
        most = half_max(most) * a.scale_log2;
        const bool up = most > ref[qg] + (kLag + kLift<T>);
        next[qg] = up ? most - kLift<T> : ref[qg];
        moved |= up;
      }
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const Frag<T> kf = row_frag<T, kROWB>(kn, l, st);
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) mma(s[1 - PAR][qg], kf, q[qg].f[st]);
      }
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) {
        by_sum[qg] = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[PAR][qg][e], a.scale_log2, -next[qg]));
          s[PAR][qg][e] = w;
          by_sum[qg] += w;
        }
#pragma unroll
        for (int k = 0; k < kKs; ++k) p[PAR][qg][k] = acc_frag<T>(s[PAR][qg], k);
      }
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int k = 0; k < kKs; ++k) {
          const Frag<T> vf = col_frag<T, kROWB>(vl, 0, k, dt);
#pragma unroll
          for (int qg = 0; qg < QG; ++qg) mma(acc[qg][dt], vf, p[1 - PAR][qg][k]);
        }
      if (__ballot(moved)) {
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) {
          const float by = __builtin_amdgcn_exp2f(ref[qg] - next[qg]);
          ref[qg] = next[qg];
          sum[qg] *= by;
#pragma unroll
          for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[qg][dt][e] *= by;
        }
      }
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) sum[qg] += by_sum[qg];
      const uint32_t bits_after = bits_at(t + 2, mask_after);
      if (more) ks.store(tid, a.D, kt + PAR * kTile, bits_after);
      vs.store(tid, a.D, vt + PAR * kTile, bits);
      bits = bits_next;
      bits_next = bits_after;
    };
    auto finish = [&](auto parity) {                       // the last tile's product
      constexpr int PAR = decltype(parity)::value;
      __syncthreads();
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int k = 0; k < kKs; ++k) {
          const Frag<T> vf = col_frag<T, kROWB>(vt + PAR * kTile, 0, k, dt);
#pragma unroll
          for (int qg = 0; qg < QG; ++qg) mma(acc[qg][dt], vf, p[PAR][qg][k]);
        }
    };
    using Even = std::integral_constant<int, 0>;
    using Odd = std::integral_constant<int, 1>;
    int t = t0;
    for (; t + 1 < t1; t += 2) {
      step(Even{}, t);
      step(Odd{}, t + 1);
    }
    if (t < t1) {
      step(Even{}, t);
      finish(Even{});
    } else {
      finish(Odd{});
    }
  }
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    const int r = first + qg * 32 + l;
    put_rows<T, DP>(a, acc[qg], ref[qg], sum[qg], n, r < rows ? r : -1, row.i[qg], row.h[qg], row.live[qg],
                    ((int64_t)split * units + unit) * rows + r);
  }
}

// At most 32 rows a key head: single tokens, short chunks. The waves of a block take different keys, as splits do, so
// that a cache is read by many at once; each has tiles of its own and waits for nobody.
template <typename T, int DP, int NWK>
__global__ __launch_bounds__(64 * NWK) void k_attend_few(const AttendArgs<T> a) {
  constexpr int NT = 64 * NWK, KB = 32, kROWB = DP * (int)sizeof(T), kTile = KB * kROWB;
  constexpr int kDt = DP / 32, kSteps = kROWB / 32, kKs = 32 / (2 * kPiece<T>);
  extern __shared__ __align__(16) char lds[];            // [NWK] K, V
  __shared__ int slot[NWK][3];
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 31;
  const int rows = a.by_group.by * a.sight.Tq, units = a.N * a.Hkv;
  const int split = blockIdx.x % a.splits, unit = blockIdx.x / a.splits, n = unit / a.Hkv, kvh = unit % a.Hkv;
  Rows<T, 1> row;
  row.place(a, n, kvh, 0, rows, a.sight.start(n));
  Bounds bd = row.b;
  const uint8_t* kmask = a.sight.k_mask ? a.sight.k_mask + (int64_t)n * a.sight.Tk : nullptr;
  clip_bounds<NT>(bd, kmask, slot);
  const Tiles tiles = tiles_of(bd, KB);
  const int workers = a.splits * NWK, me = split * NWK + wid;
  int t = (int)((int64_t)tiles.count * me / workers);
  const int t_end = (int)((int64_t)tiles.count * (me + 1) / workers);

  RowPieces<T, DP> q;
  q.load(a.q.row(n, row.i[0], row.h[0]), row.live[0], a.D);
  f32x16 acc[kDt];
  float ref = kLowest, sum = 0.f;
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt) acc[dt] = zeros16();
  const RowSource<T> ksrc{a.k.row(n, 0, kvh), a.k.ld_t, a.sight.Tk}, vsrc{a.v.row(n, 0, kvh), a.v.ld_t, a.sight.Tk};
  Stage<T, DP, KB, 64, false> ks, vs;
  uint8_t mask = 0;
  auto request = [&](int tile) {
    ks.request(ksrc, tile * KB, lane, a.D);
    vs.request(vsrc, tile * KB, lane, a.D);
    mask = mask_of(kmask, tile * KB + l, a.sight.Tk);
  };
  char *kt = lds + wid * 2 * kTile, *vt = kt + kTile;
  if (t < t_end) request(tiles.at(t));
  for (; t < t_end; ++t) {
    const int j0 = tiles.at(t) * KB;
    const uint32_t bits = tile_bits(bd, j0, mask);
    wave_lds_order();
    ks.store(lane, a.D, kt, bits);
    vs.store(lane, a.D, vt, bits);
    wave_lds_order();
    if (t + 1 < t_end) request(tiles.at(t + 1));
    if (bits == 0) continue;
    f32x16 s[1] = {zeros16()};
#pragma unroll
    for (int st = 0; st < kSteps; ++st) mma(s[0], row_frag<T, kROWB>(kt, l, st), q.f[st]);
    if (!(bits == 0xFFFFFFFFu && j0 >= row.b.lo_max && j0 + KB <= row.b.hi_min)) hide(s[0], row.span[0], bits, j0);
    float most = s[0][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) most = fmaxf(most, s[0][e]);
    most = half_max(most) * a.scale_log2;
    if (__ballot(most > ref + (kLag + kLift<T>))) {
      const float next = fmaxf(ref, most - kLift<T>), by = __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      sum *= by;
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[dt][e] *= by;
    }
    Frag<T> p[kKs];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][e], a.scale_log2, -ref));
      s[0][e] = w;
      sum += w;
    }
#pragma unroll
    for (int k = 0; k < kKs; ++k) p[k] = acc_frag<T>(s[0], k);
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
      for (int k = 0; k < kKs; ++k) mma(acc[dt], col_frag<T, kROWB>(vt, 0, k, dt), p[k]);
  }
  put_rows<T, DP>(a, acc, ref, sum, n, l < rows ? l : -1, row.i[0], row.h[0], row.live[0], ((int64_t)me * units + unit) * rows + l);
}

// A wave joins the workers' parts of one row: references, sums and unnormalised outputs, in their order.
template <typename T>
__global__ __launch_bounds__(256) void k_attend_join(const AttendArgs<T> a, int workers) {
  const int G = a.Hq / a.Hkv, rows = G * a.sight.Tq, units = a.N * a.Hkv, lane = threadIdx.x & 63;
  const int64_t all = (int64_t)units * rows;
  for (int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); id < all; id += (int64_t)gridDim.x * 4) {
    const int unit = (int)(id / rows), r = (int)(id % rows), n = unit / a.Hkv, i = r / G, hq = unit % a.Hkv * G + r % G;
    const bool live = !a.sight.q_mask || a.sight.q_mask[(int64_t)n * a.sight.Tq + i];
    const float* from = a.part + id * (a.D + 2);
    const int64_t step = all * (a.D + 2);
    float ref = kLowest;
    for (int w = lane; w < workers; w += 64) ref = fmaxf(ref, from[w * step]);
    ref = wave_max(ref);
    float total = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};      // elements lane, lane + 64, ...
    for (int w = 0; w < workers; ++w) {
      const float by = __builtin_amdgcn_exp2f(from[w * step] - ref);
      total += by * from[w * step + 1];
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (lane + 64 * c < a.D) v[c] += by * from[w * step + 2 + lane + 64 * c];
    }
    const bool some = live && total != 0.f;
    const int64_t at = n * a.out_n + i * a.out_t + hq * a.out_h;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (lane + 64 * c < a.D) {
        const float o = some ? v[c] / total : 0.f;
        if (a.out_f32)
          static_cast<float*>(a.out)[at + lane + 64 * c] = o;
        else
          static_cast<T*>(a.out)[at + lane + 64 * c] = (T)o;
      }
    if (a.lse && lane == 0)
      a.lse[((int64_t)n * a.sight.Tq + i) * a.Hq + hq] =
          some ? (ref + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
  }
}

// Head widths that the kernels are built for.
constexpr int padded(int64_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
// Groups of 32 rows of a wave: as many as the registers hold.
constexpr int row_groups(int dp, int size) { return dp * size <= 128 ? 2 : 1; }
// Waves of a block that takes different keys, by the LDS of their tiles.
constexpr int waves_of_keys(int dp, int size) { return dp * size > 512 ? 2 : 4; }

struct Plan {
  bool few, wide;                 // one tile of rows a key head; two groups of rows a wave
  int waves_of_keys, row_tiles, splits;
  int workers() const { return splits * waves_of_keys; }
};

constexpr int kFewRows = 32;
constexpr int kMaxWorkers = 256;
constexpr int64_t kWantBlocks = 4 * kCus;      // of a launch that splits keys

Plan plan_of(eogp_dtype t, int64_t N, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D, int64_t window,
             int64_t sinks) {
  Plan p;
  const int64_t rows = Hq / Hkv * Tq, units = N * Hkv;
  const int size = t == EOGP_F32 ? 4 : 2;
  p.few = rows <= kFewRows;
  // a wave of two row groups reads each tile once for both: taken where the blocks still fill the chip
  p.wide = row_groups(padded(D), size) == 2 && units * ceil_div(rows, 256) >= 2 * kCus;
  p.waves_of_keys = p.few ? waves_of_keys(padded(D), size) : 1;
  p.row_tiles = (int)(p.few ? 1 : ceil_div(rows, p.wide ? 256 : 128));
  const int64_t keys = window > 0 ? std::min(Tk, window + sinks + Tq) : Tk;
  const int64_t most = std::max<int64_t>(1, keys / (2 * 32 * p.waves_of_keys));
  const int64_t blocks = std::max<int64_t>(1, units * p.row_tiles);
  p.splits = (int)std::min(std::min<int64_t>(most, kMaxWorkers / p.waves_of_keys), std::max<int64_t>(1, kWantBlocks / blocks));
  return p;
}

template <typename K, typename A>
eogp_status launch(K* kfn, const A& a, int64_t blocks, int threads, int lds, hipStream_t s) {
  if (lds > (48 << 10)) {
    const eogp_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(kfn), lds);
    if (st != EOGP_OK) return st;
  }
  hipLaunchKernelGGL(kfn, dim3((unsigned)blocks), dim3(threads), lds, s, a);
  EOGP_LAUNCH_CHECK("attention");
  return EOGP_OK;
}

// Rows of exactly the built width on 16-byte boundaries, a tile of which spans less than 2^31 bytes.
bool fast_rows(const eogp_heads& x, int64_t D, int size) {
  return D == padded(D) && (uintptr_t)x.data % 16 == 0 && x.ld_example * size % 16 == 0 && x.ld_token * size % 16 == 0 &&
         x.ld_head * size % 16 == 0 && x.ld_token * size * 32 < ((int64_t)1 << 31);
}

}  // namespace

// Bytes for the parts of any call of up to N examples, Tq queries and Tk keys: no launch that splits keys has more than
// kWantBlocks blocks, unless one worker a row tile is more, and no more workers than the longest keys give. (Fewer
// queries may be the few of a block whose waves take different keys: then every wave writes a part.)
size_t attention_ws(eogp_dtype t, int64_t N, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D) {
  if (N == 0 || Tq == 0) return 0;
  const int waves = waves_of_keys(padded(D), t == EOGP_F32 ? 4 : 2);
  const int64_t rows = Hq / Hkv * Tq, units = N * Hkv;
  // rows of the parts: (blocks at most) x rows a block x waves
  const int64_t few = std::min<int64_t>(units * std::min<int64_t>(rows, kFewRows) * kMaxWorkers,
                                        std::max(kWantBlocks, units) * std::min<int64_t>(rows, kFewRows) * waves);
  const int64_t many = rows <= kFewRows || ceil_div(Tk, 64) < 2 ? 0 : kWantBlocks * 128;
  return align256((size_t)std::max(few, many) * (D + 2) * sizeof(float));
}

eogp_status attention(const eogp_heads& q, const eogp_heads& k, const eogp_heads& v, const eogp_heads& out,
                      eogp_dtype t, eogp_dtype out_t, int64_t N, int64_t Tq, int64_t Tk, int64_t D, float scale,
                      int causal, int64_t window, int64_t sinks, const int64_t* q_start, const uint8_t* q_mask,
                      const uint8_t* k_mask, float* lse, void* ws, hipStream_t s) {
  if (N == 0 || Tq == 0) return EOGP_OK;
  const Plan p = plan_of(t, N, Tq, Tk, q.heads, k.heads, D, window, sinks);
  timing::Scope ts(EOGP_KT_ATTENTION, s);
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    AttendArgs<T> a;
    a.q = Heads<const T>{static_cast<const T*>(q.data), q.ld_example, q.ld_token, q.ld_head};
    a.k = Heads<const T>{static_cast<const T*>(k.data), k.ld_example, k.ld_token, k.ld_head};
    a.v = Heads<const T>{static_cast<const T*>(v.data), v.ld_example, v.ld_token, v.ld_head};
    a.out = out.data;
    a.out_n = out.ld_example;
    a.out_t = out.ld_token;
    a.out_h = out.ld_head;
    a.out_f32 = out_t == EOGP_F32;
    a.sight = Sight{causal, (int)std::min<int64_t>(window, 1 << 30), (int)std::min<int64_t>(sinks, 1 << 30), (int)Tq, (int)Tk,
                    q_start, q_mask, k_mask};
    a.N = (int)N;
    a.Hq = (int)q.heads;
    a.Hkv = (int)k.heads;
    a.D = (int)D;
    a.by_group = Divide(q.heads / k.heads);
    a.scale_log2 = scale * 1.4426950408889634f;
    a.lse = lse;
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    a.part = p.workers() > 1 ? static_cast<float*>(ws) : nullptr;
    const int64_t blocks = N * k.heads * p.row_tiles * p.splits;
    auto go = [&](auto width) {
      constexpr int DP = decltype(width)::value, size = (int)sizeof(T);
      constexpr int NWK = waves_of_keys(DP, size);
      if (p.few) return launch(k_attend_few<T, DP, NWK>, a, blocks, 64 * NWK, NWK * 2 * 32 * DP * size, s);
      constexpr int lds = 4 * 32 * DP * size;
      const bool fast = fast_rows(k, D, size) && fast_rows(v, D, size);
      if constexpr (row_groups(DP, size) == 2) {
        if (p.wide)
          return fast ? launch(k_attend<T, DP, 2, true>, a, blocks, 256, lds, s)
                      : launch(k_attend<T, DP, 2, false>, a, blocks, 256, lds, s);
      }
      return fast ? launch(k_attend<T, DP, 1, true>, a, blocks, 256, lds, s)
                  : launch(k_attend<T, DP, 1, false>, a, blocks, 256, lds, s);
    };
    using std::integral_constant;
    const eogp_status st = D <= 64    ? go(integral_constant<int, 64>{})
                           : D <= 128 ? go(integral_constant<int, 128>{})
                                      : go(integral_constant<int, 256>{});
    if (st != EOGP_OK || !a.part) return st;
    const int64_t rows = N * Tq * q.heads;
    hipLaunchKernelGGL(k_attend_join<T>, dim3((unsigned)std::min<int64_t>(ceil_div(rows, 4), 1 << 20)), dim3(256), 0, s, a,
                       p.workers());
    EOGP_LAUNCH_CHECK("attention (join)");
    return EOGP_OK;
  });
}

}  // namespace eogp
