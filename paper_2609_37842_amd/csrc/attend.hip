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
  Divide by_splits, by_units, by_heads, by_rows;   // splits; key heads of all examples, of one; rows of a key head
  float scale_log2;               // scale log2(e): weights are powers of two of scores times it
  float* lse;                     // [N, Tq, Hq] or NULL
  int row_tiles, splits;
  float *part, *part_stats;       // splits > 1: [splits][rows of all][D] unnormalised outputs, [..][2] references and sums
};

// Weights are 2^(score - reference); the reference follows a row's maximum only when that has grown by 2^kLag,
// so sums and outputs are seldom rescaled. 16-bit weights keep their relative precision wherever the
// reference lies (fp16: 2^kLift keeps small ones out of its subnormals, and 2^(kLift + kLag) below its largest).
// They are rounded to the type before the product with V, so that it runs at the 16-bit rate (fp32's is an eighth): outputs are
// off by 0.0022 of their size (root mean square, bf16; fp16 0.00029) where one rounding at the end would leave 0.0016 (0.00021).
constexpr float kLag = 8.f;
template <typename T> constexpr float kLift = 0.f;
template <> constexpr float kLift<_Float16> = 7.f;
// Exponents are scale_log2 score - reference in one rounding. The reference is a rounded product itself, so the largest
// weight of a row is 2 to the power of that rounding: with a reference of 2^20 and more (half a step: 2^-5) in any row of the
// wave, scores are rounded as the reference is before it is taken off, and the largest weight is what it is meant to be at any
// size. (Scores that far below a smaller reference have weights of 0 either way. References change with `moved` alone.)
__device__ __forceinline__ bool is_far(float ref) { return fabsf(ref) >= kFar && ref != kLowest; }
__device__ __forceinline__ void round_scores(f32x16& s, float by) {
#pragma unroll
  for (int e = 0; e < 16; ++e) s[e] = rounded(s[e] * by);
}
constexpr int kMaxSplits = 256;     // workers that share a row tile's keys
// Workers whose parts a wave a row joins; of more, a block a row. (bf16, 128 queries of 32 / 8 x 128 over 16,384 keys, 16
// splits: 60 us, by blocks 73; 33 queries of 8 x 128 over 32,768 keys, 64 splits: by blocks 31 us, by waves 37.)
constexpr int kFewSplits = 16;

// A row group's results: to the output, or unnormalised with their reference and sum to a worker's part.
template <typename T, int DP, bool EXACT>
__device__ __forceinline__ void put_rows(const AttendArgs<T>& a, const f32x16* acc, float ref, float sum, int n, int r, int i,
                                         int hq, bool live, int64_t part_row) {
  const int h = (threadIdx.x >> 5) & 1, D = EXACT ? DP : a.D;
  const float total = half_sum(sum);
  if (r < 0) return;
  if (a.part) {                                          // joined by k_attend_join
    float* to = a.part + part_row * D;
    if (h == 0) {
      a.part_stats[2 * part_row] = ref;
      a.part_stats[2 * part_row + 1] = total;
    }
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float v[4] = {acc[dt][4 * g], acc[dt][4 * g + 1], acc[dt][4 * g + 2], acc[dt][4 * g + 3]};
        put4<float, EXACT>(to, dt * 32 + 8 * g + 4 * h, D, v);
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
        put4<float, EXACT>(static_cast<float*>(a.out) + at, c, D, v);
      else
        put4<T, EXACT>(static_cast<T*>(a.out) + at, c, D, v);
    }
}

// Four waves side by side over rows (QG groups of 32 each) share tiles of 32 keys. A step works on three tiles at
// once, which depend on nothing of each other: the products of the next tile's scores, the weights of this one and the
// product of the last one's weights with V, so that the vector units make exponentials while the matrix units multiply.
// (A step's weights may move a row's reference: the output takes its factor at the step's end, when the last tile's
// product, made with the old one, is in.)
// Bound by its vector instructions and by LDS (each wave reads whole tiles for its 32 or 64 rows) between barriers every 32
// keys, with neither unit full: bf16 heads of 128, causal, 8 x 1,024 to 2,048 tokens of 16 heads 150 us (81 GFLOP, 540 TFLOP/s;
// vector units busy 0.39 of the SIMDs' time, matrix 0.29, and few blocks: 1.66 waves a SIMD), 2 x 8,192 tokens and more 860 to
// 910 TFLOP/s; heads of 64 720, of 256 (one wave a SIMD) 660; fp32 109 to 123 of the 154 that a large matrix product reaches, 27
// in heads of 256, whose rows do not fit the registers. With the three steps of one tile after another the first took
// 381 us; with three tiles at once but masks and rows' bounds read one after another before the first tile, 226.
template <typename T, int DP, int QG, bool FAST>
__global__ __launch_bounds__(256, DP * QG * (int)sizeof(T) <= 256 ? 2 : 1) void k_attend(const AttendArgs<T> a) {
  constexpr int NWR = 4, NT = 256, KB = 32, kROWB = DP * (int)sizeof(T), kTile = KB * kROWB;
  constexpr int kRows = 32 * QG * NWR, kDt = DP / 32, kSteps = kROWB / 32, kKs = 32 / (2 * kPiece<T>);
  extern __shared__ __align__(16) char lds[];            // [2] K, [2] V
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 31;
  const int tid = threadIdx.x;
  const int rows = a.by_group.by * a.sight.Tq, units = a.N * a.Hkv;
  // heavier row tiles (later positions) first
  const int b = a.by_splits.quotient(blockIdx.x), split = a.by_splits.rest(blockIdx.x, b);
  const int turn = a.by_units.quotient(b), unit = a.by_units.rest(b, turn), tile_row = a.row_tiles - 1 - turn;
  const int n = a.by_heads.quotient(unit), kvh = a.by_heads.rest(unit, n);
  const int64_t start = a.sight.start(n);
  const uint8_t* kmask = a.sight.k_mask ? a.sight.k_mask + (int64_t)n * a.sight.Tk : nullptr;
  const uint8_t* qmask = a.sight.q_mask ? a.sight.q_mask + (int64_t)n * a.sight.Tq : nullptr;

  // Row r of a key head is query r / G of query head kvh G + r mod G. Rows of the block that count, in halves of at most
  // 128; this wave's; and the lane's own.
  const int r0 = tile_row * kRows, first = r0 + wid * QG * 32;
  auto counts = [&](int r) { return r < rows && (!qmask || qmask[a.by_group.quotient(r)]); };
  LiveRows block[QG];
#pragma unroll
  for (int u = 0; u < QG; ++u) {
    block[u].low = __ballot(counts(r0 + u * 128 + lane));
    block[u].high = __ballot(counts(r0 + u * 128 + 64 + lane));
  }
  int row_i[QG], row_h[QG];
  RowPieces<T, DP, FAST> q[QG];
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    const int r = first + qg * 32 + l, rc = r < rows ? r : rows - 1;
    row_i[qg] = a.by_group.quotient(rc);
    row_h[qg] = kvh * (int)a.by_group.by + a.by_group.rest(rc, row_i[qg]);
    q[qg].request(a.q.row(n, row_i[qg], row_h[qg]), a.D);
  }
  MaskRange range{0, 0, true};
  const bool at_once = a.sight.Tk <= kMaskAtOnce;
  if (kmask && at_once) range = mask_range(kmask, a.sight.Tk, 0, a.sight.Tk);
  bool any = false;
  int block_first = 0, block_last = 0;
#pragma unroll
  for (int u = 0; u < QG; ++u)
    if (!block[u].none()) {
      if (!any) block_first = u * 128 + block[u].first();
      block_last = u * 128 + block[u].last();
      any = true;
    }
  auto position = [&](int r) { return start + a.by_group.quotient(r0 + r); };
  Bounds bd{0, 0, 0, 0};
  if (any) {
    if (kmask && !at_once) range = range_of(a.sight, kmask, position(block_first), position(block_last));
    bd = bounds_of(a.sight, position(block_first), position(block_last), range, kmask);
  }
  // the lane's spans, and the keys that all rows of the wave see
  bool live[QG];
  Span span[QG];
  int lo_max = 0, hi_min = a.sight.Tk;
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    const int at = (wid * QG + qg) * 32;
    const LiveRows& of = block[QG == 1 ? 0 : at / 128];
    const uint32_t mine = (uint32_t)((at % 128 < 64 ? of.low : of.high) >> (at % 64));
    live[qg] = (mine >> l) & 1;
    span[qg] = live[qg] ? span_of(a.sight, start + row_i[qg]) : Span{0, 0, 0};
    if (mine) {
      lo_max = max(lo_max, span_of(a.sight, position(at + 31 - __builtin_clz(mine))).lo);
      hi_min = min(hi_min, span_of(a.sight, position(at + __builtin_ctz(mine))).hi);
    }
    q[qg].settle(live[qg], a.D);
  }
  const Tiles tiles = tiles_of(bd, KB);
  int t0 = 0, t1 = tiles.count;
  if (a.splits > 1) {
    t0 = (int)((int64_t)tiles.count * split / a.splits);
    t1 = (int)((int64_t)tiles.count * (split + 1) / a.splits);
  }

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
    const RowSource<T> ksrc(a.k.row(n, 0, kvh), a.k.ld_t, a.sight.Tk, DP, FAST), vsrc(a.v.row(n, 0, kvh), a.v.ld_t, a.sight.Tk, DP, FAST);
    char *kt = lds, *vt = lds + 2 * kTile;
    Stage<T, DP, KB, NT, FAST> ks, vs;
    const KeyMask km(kmask, ksrc.base, a.sight.Tk);
    auto bits_at = [&](int t, uint8_t byte) { return t < t1 ? km.bits(bd, tiles.at(t) * KB, byte) : 0; };
    // bits of the step's tile and the one after it
    const uint8_t byte0 = km.request(tiles.at(t0) * KB + l), byte1 = km.request(tiles.at(t0 + 1) * KB + l);
    ks.request(ksrc, tiles.at(t0) * KB, tid, a.D);
    vs.request(ksrc, tiles.at(t0 + 1) * KB, tid, a.D);
    uint32_t bits = bits_at(t0, byte0), bits_next = bits_at(t0 + 1, byte1);
    ks.store(tid, a.D, kt, bits);
    vs.store(tid, a.D, kt + kTile, bits_next);
    // the first step's product with the tile before: weights 0 of values 0
    for (int c = tid * 16; c < kTile; c += NT * 16) *reinterpret_cast<uint4*>(vt + kTile + c) = uint4{0, 0, 0, 0};
    f32x16 s[2][QG];
    Frag<T> p[2][QG][kKs];
    bool far = false;
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
      ks.request(ksrc, tiles.at(t + 2) * KB, tid, a.D);   // (behind the last tile: not used)
      vs.request(vsrc, tiles.at(t) * KB, tid, a.D);
      const uint8_t byte_after = km.request(tiles.at(t + 2) * KB + l);
      const int j0 = tiles.at(t) * KB;
      // (One row group: before the maxima, the other order is 1% slower; two: behind the branch, 3% faster, without spills.)
      auto products = [&]() {
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) s[1 - PAR][qg] = zeros16();
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
          const Frag<T> kf = row_frag<T, kROWB>(kn, l, st);
#pragma unroll
          for (int qg = 0; qg < QG; ++qg) mma(s[1 - PAR][qg], kf, q[qg].f[st]);
        }
      };
      if constexpr (QG == 1) products();
      if (!(bits == 0xFFFFFFFFu && j0 >= lo_max && j0 + KB <= hi_min)) {
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) hide(s[PAR][qg], span[qg], bits, j0);
      }
      float next[QG], by_sum[QG];
      bool moved = false;
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) {
        float most = s[PAR][qg][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) most = fmaxf(most, s[PAR][qg][e]);
        most = rounded(half_max(most) * a.scale_log2);
        const bool up = most - ref[qg] > kLag + kLift<T>;   // (a sum with a large reference would round)
        next[qg] = up ? most - kLift<T> : ref[qg];
        moved |= up;
      }
      const bool any_moved = __ballot(moved) != 0;
      float per_score = a.scale_log2;
      if (__builtin_expect(any_moved || far, 0)) {
        bool some = false;
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) some |= is_far(next[qg]);
        far = __ballot(some) != 0;
        if (far) {
          per_score = 1.f;
#pragma unroll
          for (int qg = 0; qg < QG; ++qg) round_scores(s[PAR][qg], a.scale_log2);
        }
      }
      if constexpr (QG == 2) products();
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) {
        by_sum[qg] = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[PAR][qg][e], per_score, -next[qg]));
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
      if (any_moved) {
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
      const uint32_t bits_after = bits_at(t + 2, byte_after);
      ks.store(tid, a.D, kt + PAR * kTile, bits_after);
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
    put_rows<T, DP, FAST>(a, acc[qg], ref[qg], sum[qg], n, r < rows ? r : -1, row_i[qg], row_h[qg], live[qg],
                          ((int64_t)split * units + unit) * rows + r);
  }
}

// At most 32 rows a key head: single tokens, short chunks. The waves of a block take different keys, as splits do, so
// that a cache is read by many at once; each has tiles of its own and waits for nobody: one tile is on its way while one is
// multiplied. Bound by the cache's bytes: fp16, one token over 131,072 keys of 16 x 128, 1.07 GB, 200 us and the join 5
// (5.3 TB/s; matrix units busy 0.08 of the SIMDs' time, one wave a SIMD); bf16, 16 tokens of 40 / 8 x 128 over 512 to 4,096
// keys, 152 MB, 34 us and the join 5, where the longest sequence's blocks are a third of the time. With every wave's
// part joined behind the kernel (four times as many) the first took 493 us in all.
template <typename T, int DP, int NWK, bool FAST>
__global__ __launch_bounds__(64 * NWK) void k_attend_few(const AttendArgs<T> a) {
  constexpr int KB = 32, kROWB = DP * (int)sizeof(T), kTile = KB * kROWB;
  constexpr int kDt = DP / 32, kSteps = kROWB / 32, kKs = 32 / (2 * kPiece<T>);
  extern __shared__ __align__(16) char lds[];            // [NWK] K, V
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 31;
  const int rows = a.by_group.by * a.sight.Tq, units = a.N * a.Hkv;
  const int unit = a.by_splits.quotient(blockIdx.x), split = a.by_splits.rest(blockIdx.x, unit);
  const int n = a.by_heads.quotient(unit), kvh = a.by_heads.rest(unit, n);
  const int64_t start = a.sight.start(n);
  const uint8_t* kmask = a.sight.k_mask ? a.sight.k_mask + (int64_t)n * a.sight.Tk : nullptr;
  const int rc = l < rows ? l : rows - 1, row_i = a.by_group.quotient(rc);
  const int row_h = kvh * (int)a.by_group.by + a.by_group.rest(rc, row_i);
  RowPieces<T, DP, FAST> q;
  q.request(a.q.row(n, row_i, row_h), a.D);
  const bool live = l < rows && (!a.sight.q_mask || a.sight.q_mask[(int64_t)n * a.sight.Tq + row_i]);
  const uint32_t mine = (uint32_t)__ballot(live);
  const Span span = live ? span_of(a.sight, start + row_i) : Span{0, 0, 0};
  Bounds bd{0, 0, 0, 0};
  int lo_max = 0, hi_min = a.sight.Tk;
  if (mine) {
    const int64_t p0 = start + a.by_group.quotient(__builtin_ctz(mine)), p1 = start + a.by_group.quotient(31 - __builtin_clz(mine));
    MaskRange range{0, 0, true};
    if (kmask) range = range_of(a.sight, kmask, p0, p1);
    bd = bounds_of(a.sight, p0, p1, range, kmask);
    lo_max = span_of(a.sight, p1).lo;
    hi_min = span_of(a.sight, p0).hi;
  }
  q.settle(live, a.D);
  const Tiles tiles = tiles_of(bd, KB);
  const int workers = a.splits * NWK, me = split * NWK + wid;
  int t = (int)((int64_t)tiles.count * me / workers);
  const int t_end = (int)((int64_t)tiles.count * (me + 1) / workers);

  f32x16 acc[kDt];
  float ref = kLowest, sum = 0.f;
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt) acc[dt] = zeros16();
  const RowSource<T> ksrc(a.k.row(n, 0, kvh), a.k.ld_t, a.sight.Tk, DP, FAST), vsrc(a.v.row(n, 0, kvh), a.v.ld_t, a.sight.Tk, DP, FAST);
  Stage<T, DP, KB, 64, FAST> ks, vs;
  const KeyMask km(kmask, ksrc.base, a.sight.Tk);
  uint8_t byte = 0;
  auto request = [&](int tile) {
    ks.request(ksrc, tile * KB, lane, a.D);
    vs.request(vsrc, tile * KB, lane, a.D);
    byte = km.request(tile * KB + l);
  };
  char *kt = lds + wid * 2 * kTile, *vt = kt + kTile;
  bool far = false;
  if (t < t_end) request(tiles.at(t));
  for (; t < t_end; ++t) {
    const int j0 = tiles.at(t) * KB;
    const uint32_t bits = km.bits(bd, j0, byte);
    wave_lds_order();
    ks.store(lane, a.D, kt, bits);
    vs.store(lane, a.D, vt, bits);
    wave_lds_order();
    if (t + 1 < t_end) request(tiles.at(t + 1));
    if (bits == 0) continue;
    f32x16 s[1] = {zeros16()};
#pragma unroll
    for (int st = 0; st < kSteps; ++st) mma(s[0], row_frag<T, kROWB>(kt, l, st), q.f[st]);
    if (!(bits == 0xFFFFFFFFu && j0 >= lo_max && j0 + KB <= hi_min)) hide(s[0], span, bits, j0);
    float most = s[0][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) most = fmaxf(most, s[0][e]);
    most = rounded(half_max(most) * a.scale_log2);
    if (__ballot(most - ref > kLag + kLift<T>)) {
      const float next = fmaxf(ref, most - kLift<T>), by = __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      far = __ballot(is_far(ref)) != 0;
      sum *= by;
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[dt][e] *= by;
    }
    float per_score = a.scale_log2;
    if (far) {
      per_score = 1.f;
      round_scores(s[0], a.scale_log2);
    }
    Frag<T> p[kKs];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][e], per_score, -ref));
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
  // the waves' outputs to LDS (each over its own tiles, 16-byte pieces exchanged by row), and joined there
  constexpr int kPieces4 = DP / 4;
  static_assert(32 * DP * 4 <= 2 * kTile || sizeof(T) == 4, "a wave's output fits its tiles");
  __shared__ float stats[2][NWK][32];
  const float total = half_sum(sum);
  auto at = [&](int w, int r, int piece) {
    return reinterpret_cast<f32x4*>(lds + w * 2 * kTile + (r * kPieces4 + (piece ^ (r & (kPieces4 - 1 < 31 ? kPieces4 - 1 : 31)))) * 16);
  };
  wave_lds_order();
  if (l < rows) {
    if (lane < 32) {
      stats[0][wid][l] = ref;
      stats[1][wid][l] = total;
    }
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *at(wid, l, dt * 8 + 2 * g + (lane >> 5)) = f32x4{acc[dt][4 * g], acc[dt][4 * g + 1], acc[dt][4 * g + 2], acc[dt][4 * g + 3]};
  }
  __syncthreads();
  const int D = FAST ? DP : a.D;
  for (int e = threadIdx.x; e < rows * kPieces4; e += 64 * NWK) {
    const int r = e / kPieces4, c = e % kPieces4 * 4;
    float most = kLowest, all = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NWK; ++w) most = fmaxf(most, stats[0][w][r]);
#pragma unroll
    for (int w = 0; w < NWK; ++w) {
      const float by = __builtin_amdgcn_exp2f(stats[0][w][r] - most);
      const f32x4 x = *at(w, r, e % kPieces4);
      all += by * stats[1][w][r];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += by * x[i];
    }
    if (c >= D) continue;
    if (a.part) {
      const int64_t row = ((int64_t)split * units + unit) * rows + r;
      if (c == 0) {
        a.part_stats[2 * row] = most;
        a.part_stats[2 * row + 1] = all;
      }
      put4<float, FAST>(a.part + row * D, c, D, v);
      continue;
    }
    const int i = a.by_group.quotient(r), hq = kvh * (int)a.by_group.by + a.by_group.rest(r, i);
    const bool some = ((mine >> r) & 1) && all != 0.f;
    const float inv = some ? 1.f / all : 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = some ? v[k] * inv : 0.f;
    if (a.lse && c == 0)
      a.lse[((int64_t)n * a.sight.Tq + i) * a.Hq + hq] = some ? (most + __builtin_amdgcn_logf(all)) * 0.6931471805599453f : -INFINITY;
    const int64_t to = n * a.out_n + i * a.out_t + hq * a.out_h;
    if (a.out_f32)
      put4<float, FAST>(static_cast<float*>(a.out) + to, c, D, v);
    else
      put4<T, FAST>(static_cast<T*>(a.out) + to, c, D, v);
  }
}

// Where row `id` of all key heads' rows lies.
struct JoinRow {
  int n, i, hq;
};
template <typename T>
__device__ __forceinline__ JoinRow join_row(const AttendArgs<T>& a, int id) {
  const int unit = a.by_rows.quotient(id), r = a.by_rows.rest(id, unit), n = a.by_heads.quotient(unit);
  const int i = a.by_group.quotient(r);
  return JoinRow{n, i, a.by_heads.rest(unit, n) * (int)a.by_group.by + a.by_group.rest(r, i)};
}
template <typename T>
__device__ __forceinline__ bool counts(const AttendArgs<T>& a, const JoinRow& to, float total) {
  return total != 0.f && (!a.sight.q_mask || a.sight.q_mask[(int64_t)to.n * a.sight.Tq + to.i]);
}
template <typename T>
__device__ __forceinline__ void put_joined(const AttendArgs<T>& a, const JoinRow& to, int c, float v) {
  const int64_t at = to.n * a.out_n + to.i * a.out_t + to.hq * a.out_h + c;
  if (a.out_f32)
    static_cast<float*>(a.out)[at] = v;
  else
    static_cast<T*>(a.out)[at] = (T)v;
}
template <typename T>
__device__ __forceinline__ void put_lse(const AttendArgs<T>& a, const JoinRow& to, bool some, float ref, float total) {
  if (a.lse)
    a.lse[((int64_t)to.n * a.sight.Tq + to.i) * a.Hq + to.hq] =
        some ? (ref + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
}

// The splits' parts of a row joined: references, sums and unnormalised outputs, in the order of the splits. Bound by the
// reading of the parts. Few splits: a wave takes a row, D / 64 columns a lane, and asks for four splits' at once.
template <typename T, int COLS>
__global__ __launch_bounds__(256) void k_attend_join_few(const AttendArgs<T> a) {
  const int all = a.N * a.Hkv * (int)a.by_rows.by, lane = threadIdx.x & 63;
  const int64_t step = (int64_t)all * a.D;
  for (int id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); id < all; id += gridDim.x * 4) {
    const float* from = a.part + (int64_t)id * a.D;
    const int64_t at = 2 * ((int64_t)min(lane, a.splits - 1) * all + id);   // a lane has a split's weight
    const float ref = a.part_stats[at], sum = a.part_stats[at + 1], most = wave_max(ref);
    const float by = lane < a.splits ? __builtin_amdgcn_exp2f(ref - most) : 0.f, total = wave_sum(by * sum);
    float v[COLS / 64];
#pragma unroll
    for (int k = 0; k < COLS / 64; ++k) v[k] = 0.f;
    for (int w0 = 0; w0 < a.splits; w0 += 4) {
      float x[4][COLS / 64];
#pragma unroll
      for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int k = 0; k < COLS / 64; ++k) x[w][k] = from[min(w0 + w, a.splits - 1) * step + min(lane + 64 * k, a.D - 1)];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float of = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(by), min(w0 + w, 63)));
#pragma unroll
        for (int k = 0; k < COLS / 64; ++k) v[k] += w0 + w < a.splits ? of * x[w][k] : 0.f;
      }
    }
    const JoinRow to = join_row(a, id);
    const bool some = counts(a, to, total);
#pragma unroll
    for (int k = 0; k < COLS / 64; ++k)
      if (lane + 64 * k < a.D) put_joined(a, to, lane + 64 * k, some ? v[k] / total : 0.f);
    if (lane == 0) put_lse(a, to, some, most, total);
  }
}

// Many splits: a block takes a row, COLS columns a slice of its threads, each slice every SLICES-th split in order, four
// requests of a thread at a time; the slices' sums in their order.
template <typename T, int COLS>
__global__ __launch_bounds__(1024) void k_attend_join(const AttendArgs<T> a) {
  constexpr int SLICES = 1024 / COLS;
  __shared__ float weight[kMaxSplits], parts[SLICES][COLS], both[2];
  const int all = a.N * a.Hkv * (int)a.by_rows.by;
  const int col = threadIdx.x % COLS, slice = threadIdx.x / COLS;
  for (int id = blockIdx.x; id < all; id += gridDim.x) {
    __syncthreads();
    if (threadIdx.x < 64) {                              // the first wave: weights of the splits, and the row's sum
      const int lane = threadIdx.x;
      float ref[kMaxSplits / 64], sum[kMaxSplits / 64], most = kLowest, total = 0.f;
#pragma unroll
      for (int k = 0; k < kMaxSplits / 64; ++k) {
        const int w = min(lane + 64 * k, a.splits - 1);
        ref[k] = a.part_stats[2 * ((int64_t)w * all + id)];
        sum[k] = lane + 64 * k < a.splits ? a.part_stats[2 * ((int64_t)w * all + id) + 1] : 0.f;
        most = fmaxf(most, ref[k]);
      }
      most = wave_max(most);
#pragma unroll
      for (int k = 0; k < kMaxSplits / 64; ++k) {
        const float by = __builtin_amdgcn_exp2f(ref[k] - most);
        weight[lane + 64 * k] = by;
        total += by * sum[k];
      }
      total = wave_sum(total);
      if (lane == 0) {
        both[0] = most;
        both[1] = total;
      }
    }
    __syncthreads();
    float v = 0.f;
    const float* from = a.part + (int64_t)id * a.D + min(col, a.D - 1);
    const int64_t step = (int64_t)all * a.D;
    for (int w = slice; w < a.splits; w += 4 * SLICES) {
      float x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = from[min(w + k * SLICES, a.splits - 1) * step];
#pragma unroll
      for (int k = 0; k < 4; ++k) v += w + k * SLICES < a.splits ? x[k] * weight[min(w + k * SLICES, a.splits - 1)] : 0.f;
    }
    parts[slice][col] = v;
    __syncthreads();
    const float total = both[1];
    const JoinRow to = join_row(a, id);
    const bool some = counts(a, to, total);
    if (slice == 0 && col < a.D) {
#pragma unroll
      for (int k = 1; k < SLICES; ++k) v += parts[k][col];
      put_joined(a, to, col, some ? v / total : 0.f);
    }
    if (threadIdx.x == 0) put_lse(a, to, some, both[0], total);
  }
}

// Groups of 32 rows of a wave: as many as the registers hold.
constexpr int row_groups(int dp, int size) { return dp * size <= 128 ? 2 : 1; }
// Waves of a block that takes different keys, by the LDS of their tiles.
constexpr int waves_of_keys(int dp, int size) { return dp * size > 512 ? 2 : 4; }

struct Plan {
  bool few, wide;                 // one tile of rows a key head; two groups of rows a wave
  int waves_of_keys, row_tiles, splits;
};

constexpr int kFewRows = 32;
// Blocks that a launch which splits keys goes up to: of rows, what is there at once (2 x 2,048 tokens of 16 x 128 bf16, not
// causal, 512 blocks: 97 us, in two splits 217 when the join took 100; 1,024 x 8,192 tokens, 128 blocks of rows: 102 us in
// four splits, 122 in two); of few rows, four times as many as CUs.
constexpr int64_t kWantBlocks = 2 * kCus, kWantFew = 4 * kCus;

Plan plan_of(eogp_dtype t, int64_t N, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D, int64_t window,
             int64_t sinks) {
  Plan p;
  const int64_t rows = Hq / Hkv * Tq, units = N * Hkv;
  const int size = t == EOGP_F32 ? 4 : 2;
  p.few = rows <= kFewRows;
  // A wave of two row groups reads each tile once for both: taken where the blocks still fill the chip (so that keys are not
  // split then: the workspace is that of 128 rows a block). Two groups and one, heads of 64: fp16, 8 x 4,096 tokens of 16
  // 416 and 427 us; bf16, 2 x 2,048 of 40 / 8 75 and 77, 32 x 1,024 of 12 133 and 131, 8 x 2,048 99 and 90; of 40, whose tiles
  // take more instructions on their way to LDS, 32 x 1,024 of 12 224 and 317.
  p.wide = row_groups(padded(D), size) == 2 && units * ceil_div(rows, 256) >= 2 * kCus;
  p.waves_of_keys = p.few ? waves_of_keys(padded(D), size) : 1;
  p.row_tiles = (int)(p.few ? 1 : ceil_div(rows, p.wide ? 256 : 128));
  const int64_t keys = window > 0 ? std::min(Tk, window + sinks + Tq) : Tk;
  const int64_t want = p.few ? kWantFew : kWantBlocks, least = p.few ? 64 * p.waves_of_keys : 256;   // keys of a split
  const int64_t most = std::max<int64_t>(1, keys / least);
  const int64_t blocks = std::max<int64_t>(1, units * p.row_tiles);
  p.splits = (int)std::min(std::min<int64_t>(most, kMaxSplits), std::max<int64_t>(1, want / blocks));
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

}  // namespace

// Bytes for the parts of any call of up to N examples, Tq queries and Tk keys: a launch that splits keys has at most
// kWantFew blocks of at most 32 rows or kWantBlocks of 128, and at most kMaxSplits splits.
size_t attention_ws(eogp_dtype t, int64_t N, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D) {
  if (N == 0 || Tq == 0 || Tk < 256) return 0;
  const int64_t rows = Hq / Hkv * Tq, all = N * Hkv * rows;
  const int64_t most = std::max(kWantFew * std::min<int64_t>(rows, kFewRows), rows <= kFewRows ? 0 : kWantBlocks * 128);
  return align256((size_t)std::min(all * kMaxSplits, most) * (D + 2) * sizeof(float));
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
    AttendArgs<T> a{};
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
    a.by_splits = Divide(p.splits);
    a.by_units = Divide(N * k.heads);
    a.by_heads = Divide(k.heads);
    a.by_rows = Divide(q.heads / k.heads * Tq);
    a.scale_log2 = scale * 1.4426950408889634f;
    a.lse = lse;
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    if (p.splits > 1) {
      a.part = static_cast<float*>(ws);
      a.part_stats = a.part + p.splits * (N * Tq * q.heads) * D;
    }
    const int64_t blocks = N * k.heads * p.row_tiles * p.splits;
    auto go = [&](auto width) {
      constexpr int DP = decltype(width)::value, size = (int)sizeof(T);
      constexpr int NWK = waves_of_keys(DP, size);
      const bool fast = fast_rows(k, Tk, D, size) && fast_rows(v, Tk, D, size);
      if (p.few)
        return fast ? launch(k_attend_few<T, DP, NWK, true>, a, blocks, 64 * NWK, NWK * 2 * 32 * DP * size, s)
                    : launch(k_attend_few<T, DP, NWK, false>, a, blocks, 64 * NWK, NWK * 2 * 32 * DP * size, s);
      constexpr int lds = 4 * 32 * DP * size;
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
    auto join = [&](auto width) {
      constexpr int DP = decltype(width)::value;
      if (p.splits <= kFewSplits)
        hipLaunchKernelGGL((k_attend_join_few<T, DP>), dim3((unsigned)ceil_div(rows, 4)), dim3(256), 0, s, a);
      else
        hipLaunchKernelGGL((k_attend_join<T, DP>), dim3((unsigned)rows), dim3(1024), 0, s, a);
    };
    if (D <= 64)
      join(integral_constant<int, 64>{});
    else if (D <= 128)
      join(integral_constant<int, 128>{});
    else
      join(integral_constant<int, 256>{});
    EOGP_LAUNCH_CHECK("attention (join)");
    return EOGP_OK;
  });
}

}  // namespace eogp
