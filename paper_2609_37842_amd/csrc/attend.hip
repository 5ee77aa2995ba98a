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

// Rows of a head group: query i of head kvh G + g is row i G + g of key head kvh.
// NWR waves side by side over rows (QG times 32 each) share tiles of KB keys; NWK waves (or groups of
// them) take different keys, as different splits do.
template <typename T, int DP, int QG, int NWR, int NWK, int KB>
__global__ __launch_bounds__(64 * NWR * NWK) void k_attend(const AttendArgs<T> a) {
  constexpr int NT = 64 * NWR * NWK, kROWB = DP * (int)sizeof(T), kTile = KB * kROWB;
  constexpr int kRows = 32 * QG * NWR, kSub = KB / 32, kDt = DP / 32, kSteps = kROWB / 32;
  constexpr int kKs = 32 / (2 * kPiece<T>);             // operands of 32 inner indices
  constexpr int kTurns = NWR > 1 ? 2 : 1;               // a wave of its own tiles is in order with itself
  extern __shared__ __align__(16) char lds[];           // [NWK][kTurns][K, V]
  __shared__ int slot[NT / 64];
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wid % NWR, wk = wid / NWR, lane = threadIdx.x & 63, l = lane & 31, h = lane >> 5;
  const int tid = threadIdx.x - wk * 64 * NWR;          // place among the waves that share tiles
  const int G = a.Hq / a.Hkv, rows = G * a.sight.Tq;
  // heavier row tiles (later positions) first; blocks of one key head keep to one XCD where their number divides
  const int units = a.N * a.Hkv;
  int b = blockIdx.x;
  const int split = b % a.splits;
  b /= a.splits;
  const int unit = b % units, tile_row = a.row_tiles - 1 - b / units;
  const int n = unit / a.Hkv, kvh = unit % a.Hkv;
  const int64_t start = a.sight.start(n);

  // this lane's rows
  Span span[QG];
  bool live[QG];
  int row_i[QG], row_h[QG];
  Bounds bd{a.sight.Tk, 0, 0, 0, a.sight.Tk};
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    const int r = tile_row * kRows + (wr * QG + qg) * 32 + l;
    const int rc = r < rows ? r : rows - 1;
    row_i[qg] = a.by_group.quotient(rc);
    row_h[qg] = kvh * G + a.by_group.rest(rc, row_i[qg]);
    live[qg] = r < rows && (!a.sight.q_mask || a.sight.q_mask[(int64_t)n * a.sight.Tq + row_i[qg]]);
    span[qg] = live[qg] ? span_of(a.sight, start + row_i[qg]) : Span{0, 0, 0};
    if (live[qg]) {
      bd.lo_min = min(bd.lo_min, span[qg].hi > span[qg].lo ? span[qg].lo : a.sight.Tk);
      bd.hi_max = max(bd.hi_max, span[qg].hi > span[qg].lo ? span[qg].hi : 0);
      bd.sk_max = max(bd.sk_max, span[qg].sk);
      bd.lo_max = max(bd.lo_max, span[qg].lo);
      bd.hi_min = min(bd.hi_min, span[qg].hi);
    }
  }
  const int lo_max = wave_max_i(bd.lo_max), hi_min = wave_min_i(bd.hi_min);     // of this wave's rows
  bd.lo_min = wave_min_i(bd.lo_min);
  bd.hi_max = wave_max_i(bd.hi_max);
  bd.sk_max = wave_max_i(bd.sk_max);
  if constexpr (NWR > 1) {                               // (waves of other keys have the same rows)
    __shared__ int all[3][NWR];
    if (lane == 0 && wk == 0) {
      all[0][wr] = bd.lo_min;
      all[1][wr] = bd.hi_max;
      all[2][wr] = bd.sk_max;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NWR; ++w) {
      bd.lo_min = min(bd.lo_min, all[0][w]);
      bd.hi_max = max(bd.hi_max, all[1][w]);
      bd.sk_max = max(bd.sk_max, all[2][w]);
    }
  }
  const uint8_t* kmask = a.sight.k_mask ? a.sight.k_mask + (int64_t)n * a.sight.Tk : nullptr;
  if (kmask) {                                           // no further than the first and last key that count
    const int from = bd.sk_max > 0 ? 0 : bd.lo_min, to = max(bd.hi_max, bd.sk_max);
    const int2 r = set_range<NT>(kmask, min(from, to), to, slot);
    bd.lo_min = max(bd.lo_min, r.x);
    bd.hi_max = min(bd.hi_max, r.y);
    bd.sk_max = bd.sk_max > r.x ? min(bd.sk_max, r.y) : 0;
  }
  const Tiles tiles = tiles_of(bd, KB);
  const int workers = a.splits * NWK, me = split * NWK + wk;
  int t = (int)((int64_t)tiles.count * me / workers);
  const int t_end = (int)((int64_t)tiles.count * (me + 1) / workers);

  RowPieces<T, DP> q[QG];
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) q[qg].load(a.q.row(n, row_i[qg], row_h[qg]), live[qg], a.D);

  f32x16 acc[QG][kDt];
  float ref[QG], sum[QG];
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    ref[qg] = kLowest;
    sum[qg] = 0.f;
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) acc[qg][dt] = zeros16();
  }

  const T *kbase = a.k.row(n, 0, kvh), *vbase = a.v.row(n, 0, kvh);
  Stage<T, DP, KB, 64 * NWR> ks, vs;
  bool key_live = false;
  auto request = [&](int tile) {
    const int j0 = tile * KB;
    auto at = [&](const T* base, int64_t ld) {
      return [=](int r) { return base + (int64_t)min(j0 + r, a.sight.Tk - 1) * ld; };
    };
    ks.request(tid, a.D, at(kbase, a.k.ld_t));
    vs.request(tid, a.D, at(vbase, a.v.ld_t));
    const int j = j0 + lane % KB;
    key_live = ((j >= bd.lo_min && j < bd.hi_max) || j < bd.sk_max) && (!kmask || kmask[j]);
  };
  char* mine = lds + wk * 2 * kTurns * kTile;
  if (t < t_end) request(tiles.at(t));
  for (int turn = 0; t < t_end; ++t, turn ^= kTurns - 1) {
    char *ktile = mine + turn * 2 * kTile, *vtile = ktile + kTile;
    uint64_t bits = __ballot(key_live);
    if constexpr (KB == 32) bits &= 0xFFFFFFFFull;
    const int j0 = tiles.at(t) * KB;
    if constexpr (NWR == 1) wave_lds_order();
    ks.store(tid, a.D, ktile, bits);
    vs.store(tid, a.D, vtile, bits);
    if constexpr (NWR > 1)
      __syncthreads();
    else
      wave_lds_order();
    if (t + 1 < t_end) request(tiles.at(t + 1));
    if (bits == 0) continue;

    f32x16 s[QG][kSub];
#pragma unroll
    for (int sub = 0; sub < kSub; ++sub) {
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) s[qg][sub] = zeros16();
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const Frag<T> kf = row_frag<T, kROWB>(ktile, sub * 32 + l, st);
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) mma(s[qg][sub], kf, q[qg].f[st]);
      }
    }
    constexpr uint64_t kAll = KB == 64 ? ~0ull : 0xFFFFFFFFull;
    if (!(bits == kAll && j0 >= lo_max && j0 + KB <= hi_min)) {
#pragma unroll
      for (int qg = 0; qg < QG; ++qg)
#pragma unroll
        for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int at = sub * 32 + 8 * (e / 4) + 4 * h + e % 4;
            const bool seen = (bool)((bits >> at) & 1) & sees(span[qg], j0 + at);
            s[qg][sub][e] = seen ? s[qg][sub][e] : -INFINITY;
          }
    }
    Frag<T> p[QG][kSub * kKs];
#pragma unroll
    for (int qg = 0; qg < QG; ++qg) {
      float most = s[qg][0][0];
#pragma unroll
      for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
        for (int e = 0; e < 16; ++e) most = fmaxf(most, s[qg][sub][e]);
      most = half_max(most) * a.scale_log2;
      if (__ballot(most > ref[qg] + (kLag + kLift<T>))) {
        const float next = fmaxf(ref[qg], most - kLift<T>);
        const float by = __builtin_amdgcn_exp2f(ref[qg] - next);
        ref[qg] = next;
        sum[qg] *= by;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[qg][dt][e] *= by;
      }
#pragma unroll
      for (int sub = 0; sub < kSub; ++sub) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qg][sub][e], a.scale_log2, -ref[qg]));
          s[qg][sub][e] = w;
          sum[qg] += w;
        }
#pragma unroll
        for (int k = 0; k < kKs; ++k) p[qg][sub * kKs + k] = acc_frag<T>(s[qg][sub], k);
      }
    }
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
      for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
        for (int k = 0; k < kKs; ++k) {
          const Frag<T> vf = col_frag<T, kROWB>(vtile, sub * 32, k, dt);
#pragma unroll
          for (int qg = 0; qg < QG; ++qg) mma(acc[qg][dt], vf, p[qg][sub * kKs + k]);
        }
  }

#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    const int r = tile_row * kRows + (wr * QG + qg) * 32 + l;
    const float total = half_sum(sum[qg]);
    if (r >= rows) continue;
    if (a.part) {                                        // joined by k_attend_join
      float* to = a.part + (((int64_t)me * units + unit) * rows + r) * (a.D + 2);
      if (h == 0) {
        to[0] = ref[qg];
        to[1] = total;
      }
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float v[4] = {acc[qg][dt][4 * g], acc[qg][dt][4 * g + 1], acc[qg][dt][4 * g + 2], acc[qg][dt][4 * g + 3]};
          const int c = dt * 32 + 8 * g + 4 * h;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (c + i < a.D) to[2 + c + i] = v[i];
        }
      continue;
    }
    const float inv = live[qg] && total != 0.f ? 1.f / total : 0.f;
    if (a.lse && h == 0)
      a.lse[((int64_t)n * a.sight.Tq + row_i[qg]) * a.Hq + row_h[qg]] =
          live[qg] && total != 0.f ? (ref[qg] + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
    const int64_t at = n * a.out_n + row_i[qg] * a.out_t + row_h[qg] * a.out_h;
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = dt * 32 + 8 * g + 4 * h;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = inv == 0.f ? 0.f : acc[qg][dt][4 * g + i] * inv;
        if (a.out_f32)
          store_piece<float, 4>(static_cast<float*>(a.out) + at, c, a.D, v);
        else
          store_piece<T, 4>(static_cast<T*>(a.out) + at, c, a.D, v);
      }
  }
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

struct Plan {
  bool few;                       // one tile of rows a key head: waves take different keys
  int rows_per_block, keys_per_tile, waves_of_keys, row_tiles, splits;
  int workers() const { return splits * waves_of_keys; }
};

constexpr int kFewRows = 32;
// Waves of a block that takes different keys, by the LDS of their tiles.
constexpr int waves_of_keys(int dp, int size) { return dp * size > 512 ? 2 : 4; }
// Head widths that the kernels are built for.
constexpr int padded(int64_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
constexpr int kMaxWorkers = 256;
constexpr int64_t kWantBlocks = 4 * kCus;      // of a launch that splits keys

Plan plan_of(eogp_dtype t, int64_t N, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D, int64_t window,
             int64_t sinks) {
  Plan p;
  const int64_t rows = Hq / Hkv * Tq, units = N * Hkv;
  p.few = rows <= kFewRows;
  p.rows_per_block = p.few ? 32 : 128;
  p.keys_per_tile = 32;
  p.waves_of_keys = p.few ? waves_of_keys(padded(D), t == EOGP_F32 ? 4 : 2) : 1;
  p.row_tiles = (int)ceil_div(rows, p.rows_per_block);
  const int64_t keys = window > 0 ? std::min(Tk, window + sinks + Tq) : Tk;
  const int64_t most = std::max<int64_t>(1, keys / (2 * p.keys_per_tile * p.waves_of_keys));
  const int64_t blocks = std::max<int64_t>(1, units * p.row_tiles);
  p.splits = (int)std::min(std::min<int64_t>(most, kMaxWorkers / p.waves_of_keys), std::max<int64_t>(1, kWantBlocks / blocks));
  return p;
}

template <typename T, int DP, int QG, int NWR, int NWK, int KB>
eogp_status launch(const AttendArgs<T>& a, int64_t blocks, hipStream_t s) {
  auto* kfn = k_attend<T, DP, QG, NWR, NWK, KB>;
  const int lds = NWK * (NWR > 1 ? 4 : 2) * KB * DP * (int)sizeof(T);
  if (lds > (48 << 10)) {
    const eogp_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(kfn), lds);
    if (st != EOGP_OK) return st;
  }
  hipLaunchKernelGGL(kfn, dim3((unsigned)blocks), dim3(64 * NWR * NWK), lds, s, a);
  EOGP_LAUNCH_CHECK("attention");
  return EOGP_OK;
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
      constexpr int DP = decltype(width)::value;
      constexpr int NWK = waves_of_keys(DP, sizeof(T));
      return p.few ? launch<T, DP, 1, 1, NWK, 32>(a, blocks, s) : launch<T, DP, 1, 4, 1, 32>(a, blocks, s);
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
