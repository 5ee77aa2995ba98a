// Token embedding: rows of a table by token, and the table's gradient by sorted tokens.
#include <algorithm>

#include "rows.h"
#include "timing.h"

namespace eogp {
namespace {

// One wave per row and 64 P pieces of it; a lane's P pieces are requested together. A token
// outside [0, V) gives NaN, a masked row zeros (neither reads the table).
template <typename TT, typename TO, int P>
__global__ __launch_bounds__(256) void k_embed(const TT* __restrict__ table, int64_t ldt, int64_t V, int64_t d,
                                               const int64_t* __restrict__ tokens,
                                               const uint8_t* __restrict__ mask, int64_t n, float scale,
                                               int accumulate, TO* __restrict__ out, int64_t ldo,
                                               int64_t col_units) {
  constexpr int E = kPiece<TT>;
  const int lane = threadIdx.x & 63;
  const int64_t units = n * col_units;
  for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t row = u / col_units, c0 = (u % col_units) * (64 * P * E);
    const bool live = !mask || mask[row] != 0;
    const int64_t tok = live ? tokens[row] : 0;
    const bool inside = tok >= 0 && tok < V;
    const TT* src = table + (live && inside ? tok : 0) * ldt;
    TO* dst = out + row * ldo;
    float v[P][E];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = c0 + (int64_t)(p * 64 + lane) * E;
      if (live && inside) {
        load_piece<TT, E>(src, c, d, 0.f, v[p]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[p][e] = live ? __builtin_nanf("") : 0.f;
      }
    }
    if (!live && accumulate) continue;         // nothing to add
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = c0 + (int64_t)(p * 64 + lane) * E;
      if (c >= d) break;
      float old[E] = {};
      if (accumulate) load_piece<TO, E>(dst, c, d, 0.f, old);
#pragma unroll
      for (int e = 0; e < E; ++e) v[p][e] = accumulate ? old[e] + v[p][e] * scale : v[p][e] * scale;
      store_piece<TO, E>(dst, c, d, v[p]);
    }
  }
}

// ---- sorting the tokens ----------------------------------------------------------
// Stable least-significant-digit radix sort of (token, row) pairs; rows that count for no token
// (masked, or a token outside [0, V)) get key V and end up last. A tile is what one block sorts:
// its waves take 64 rows at a time in order, so equal digits keep the order of their rows and the
// result does not depend on any race.
constexpr int kTile = 2048, kSortWaves = 4, kMaxDigit = 9;

__device__ __forceinline__ uint32_t token_key(const int64_t* tokens, const uint8_t* mask, int64_t i, int64_t V) {
  if (mask && mask[i] == 0) return (uint32_t)V;
  const int64_t t = tokens[i];
  return t >= 0 && t < V ? (uint32_t)t : (uint32_t)V;
}

// Digit counts of each tile: hist[digit][tile].
template <bool FIRST>
__global__ __launch_bounds__(256) void k_sort_count(const int64_t* __restrict__ tokens,
                                                    const uint8_t* __restrict__ mask, int64_t V,
                                                    const uint32_t* __restrict__ keys, int64_t n, int shift,
                                                    int bits, uint32_t* __restrict__ hist, int64_t tiles) {
  __shared__ uint32_t count[1 << kMaxDigit];
  const uint32_t dmask = (1u << bits) - 1;
  for (int b = threadIdx.x; b <= (int)dmask; b += 256) count[b] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kTile;
  for (int64_t i = base + threadIdx.x; i < std::min<int64_t>(base + kTile, n); i += 256) {
    const uint32_t k = FIRST ? token_key(tokens, mask, i, V) : keys[i];
    atomicAdd(&count[(k >> shift) & dmask], 1u);
  }
  __syncthreads();
  for (int b = threadIdx.x; b <= (int)dmask; b += 256) hist[b * tiles + blockIdx.x] = count[b];
}

// One wave per digit: its counts become the rows of earlier tiles with that digit; totals[digit].
__global__ __launch_bounds__(64) void k_sort_scan(uint32_t* __restrict__ hist, int64_t tiles,
                                                  uint32_t* __restrict__ totals) {
  uint32_t* h = hist + (int64_t)blockIdx.x * tiles;
  const int lane = threadIdx.x;
  uint32_t carry = 0;
  for (int64_t base = 0; base < tiles; base += 64) {
    const uint32_t v = base + lane < tiles ? h[base + lane] : 0;
    uint32_t incl = v;
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t o = __shfl_up(incl, off);
      if (lane >= off) incl += o;
    }
    if (base + lane < tiles) h[base + lane] = carry + incl - v;
    carry += __shfl(incl, 63);
  }
  if (lane == 0) totals[blockIdx.x] = carry;
}

template <bool FIRST>
__global__ __launch_bounds__(256) void k_sort_scatter(const int64_t* __restrict__ tokens,
                                                      const uint8_t* __restrict__ mask, int64_t V,
                                                      const uint32_t* __restrict__ keys,
                                                      const uint32_t* __restrict__ rows, int64_t n, int shift,
                                                      int bits, const uint32_t* __restrict__ hist, int64_t tiles,
                                                      const uint32_t* __restrict__ totals,
                                                      uint32_t* __restrict__ keys_out,
                                                      uint32_t* __restrict__ rows_out) {
  __shared__ uint32_t at[kSortWaves][1 << kMaxDigit];   // next place of a digit for a wave
  __shared__ uint32_t wave_total[kSortWaves];
  const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int nd = 1 << bits;
  const uint32_t dmask = (uint32_t)nd - 1;
  for (int b = threadIdx.x; b < kSortWaves << kMaxDigit; b += 256) at[b >> kMaxDigit][b & ((1 << kMaxDigit) - 1)] = 0;
  __syncthreads();
  constexpr int R = kTile / 256;                        // rounds of 64 rows per wave
  const int64_t base = (int64_t)blockIdx.x * kTile + (int64_t)wid * R * 64;
  uint32_t key[R], row[R], rank[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t i = base + r * 64 + lane;
    const bool in = i < n;
    key[r] = !in ? 0u : FIRST ? token_key(tokens, mask, i, V) : keys[i];
    row[r] = !in ? 0u : FIRST ? (uint32_t)i : rows[i];
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool in = base + r * 64 + lane < n;
    const uint32_t dig = (key[r] >> shift) & dmask;
    uint64_t peers = __ballot(in);                      // lanes with the same digit
    for (int b = 0; b < bits; ++b) {
      const uint64_t m = __ballot((dig >> b) & 1);
      peers &= (dig >> b) & 1 ? m : ~m;
    }
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(peers >> 32),
                                                 __builtin_amdgcn_mbcnt_lo((uint32_t)peers, 0));
    wave_lds_order();
    rank[r] = in ? at[wid][dig] + before : 0;
    wave_lds_order();
    if (in && before == 0) at[wid][dig] += (uint32_t)__popcll(peers);
  }
  __syncthreads();
  // at[w][dig]: the first place of wave w's rows with this digit. Exclusive sum over the digits'
  // totals (each thread holds nd / 256 or fewer neighbouring digits), plus earlier tiles and waves.
  const int per = nd > 256 ? nd / 256 : 1;
  uint32_t mine = 0, tot[2] = {0, 0};
  const int d0 = threadIdx.x * per;
  for (int k = 0; k < per; ++k)
    if (d0 + k < nd) mine += tot[k] = totals[d0 + k];
  uint32_t incl = mine;
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
  }
  if (lane == 63) wave_total[wid] = incl;
  __syncthreads();
  uint32_t first = incl - mine;
  for (int w = 0; w < wid; ++w) first += wave_total[w];
  for (int k = 0; k < per; ++k)
    if (d0 + k < nd) {
      uint32_t run = first + hist[(int64_t)(d0 + k) * tiles + blockIdx.x];
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = at[w][d0 + k];
        at[w][d0 + k] = run;
        run += c;
      }
      first += tot[k];
    }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (base + r * 64 + lane < n) {
      const uint32_t to = at[wid][(key[r] >> shift) & dmask] + rank[r];
      keys_out[to] = key[r];
      rows_out[to] = row[r];
    }
}

// ---- sums over the sorted rows -----------------------------------------------------
__global__ __launch_bounds__(256) void k_zero(float* __restrict__ p, int64_t ld, int64_t rows, int64_t d) {
  const int lane = threadIdx.x & 63;
  for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += (int64_t)gridDim.x * 4) {
    float z[4] = {};
    for (int64_t c = 4 * lane; c < d; c += 256) store_piece<float, 4>(p + r * ld, c, d, z);
  }
}

// A wave sums the rows of a chunk of sorted places, for 64 pieces of their columns, eight rows in
// flight, token by token. A token whose rows all lie in the chunk is finished here; the sum of one
// that goes on beyond an end of the chunk is written to part[chunk][0] (it began in an earlier
// chunk) or part[chunk][1] (it begins here and goes on), and k_embed_join adds those in order.
constexpr int kChunk = 64;

template <typename T>
__global__ __launch_bounds__(256) void k_embed_sum(const T* __restrict__ dout, int64_t ldd, int64_t d,
                                                   const uint32_t* __restrict__ keys,
                                                   const uint32_t* __restrict__ rows, int64_t n, uint32_t V,
                                                   float scale, int accumulate, float* __restrict__ dtable,
                                                   int64_t ldt, float* __restrict__ part, int64_t col_units) {
  constexpr int E = kPiece<T>, U = 8;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t chunk = unit / col_units, p0 = chunk * kChunk;
  if (p0 >= n) return;
  const int64_t c = (unit % col_units * 64 + lane) * E;
  const int count = (int)std::min<int64_t>(kChunk, n - p0);
  // lane l holds place p0 + l
  const uint32_t mykey = lane < count ? keys[p0 + lane] : V;
  const uint32_t myrow = lane < count ? rows[p0 + lane] : 0;
  const uint32_t before = p0 > 0 ? keys[p0 - 1] : V, after = p0 + count < n ? keys[p0 + count] : V;
  float acc[E] = {};
  uint32_t cur = __builtin_amdgcn_readlane(mykey, 0);
  bool from_before = cur == before;
  auto flush = [&](bool goes_on) {
    if (c >= d) return;
    if (from_before || goes_on) {
      store_piece<float, E>(part + (chunk * 2 + (from_before ? 0 : 1)) * d, c, d, acc);
    } else {
      float* t = dtable + (int64_t)cur * ldt;
      float old[E] = {};
      if (accumulate) load_piece<float, E>(t, c, d, 0.f, old);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = old[e] + acc[e] * scale;
      store_piece<float, E>(t, c, d, acc);
    }
  };
  for (int i = 0; i < count; i += U) {
    float v[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = std::min(i + u, count - 1);
      const uint32_t k = __builtin_amdgcn_readlane(mykey, j), r = __builtin_amdgcn_readlane(myrow, j);
      if (k < V) load_piece<T, E>(dout + (int64_t)r * ldd, c, d, 0.f, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= count) break;
      const uint32_t k = __builtin_amdgcn_readlane(mykey, i + u);
      if (k != cur) {
        flush(false);
        cur = k;
        from_before = false;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
      }
      if (k >= V) return;                      // the rows that count for no token are last
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += v[u][e];
    }
  }
  flush(cur == after);
}

// One block per chunk and 256 columns: if a token's rows begin in the chunk and go on beyond it, the
// sums of its chunks are added (its four waves take every fourth following chunk) and the row is
// finished.
__global__ __launch_bounds__(256) void k_embed_join(const uint32_t* __restrict__ keys, int64_t n, uint32_t V,
                                                    const float* __restrict__ part, int64_t d, float scale,
                                                    int accumulate, float* __restrict__ dtable, int64_t ldt,
                                                    int64_t col_blocks) {
  __shared__ float fold[4][256];
  const int64_t chunk = blockIdx.x / col_blocks, p1 = (chunk + 1) * kChunk;
  if (p1 >= n) return;
  const uint32_t k = keys[p1 - 1];
  if (k >= V || keys[p1] != k || (chunk > 0 && keys[chunk * kChunk] == k && keys[chunk * kChunk - 1] == k)) return;
  const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t c = (blockIdx.x % col_blocks) * 256 + lane * 4;
  float acc[4] = {};
  if (wid == 0 && c < d) load_piece<float, 4>(part + (chunk * 2 + 1) * d, c, d, 0.f, acc);
  for (int64_t j = chunk + 1 + wid; j * kChunk < n && keys[j * kChunk] == k; j += 4) {
    float v[4];
    load_piece<float, 4>(part + j * 2 * d, c, d, 0.f, v);
    for (int e = 0; e < 4; ++e) acc[e] += v[e];
  }
  for (int e = 0; e < 4; ++e) fold[wid][lane * 4 + e] = acc[e];
  __syncthreads();
  const int64_t col = (blockIdx.x % col_blocks) * 256 + threadIdx.x;
  if (col >= d) return;
  float s = fold[0][threadIdx.x];
  for (int w = 1; w < 4; ++w) s += fold[w][threadIdx.x];
  float* t = dtable + (int64_t)k * ldt + col;
  *t = (accumulate ? *t : 0.f) + s * scale;
}

struct SortShape {
  int passes, bits;
};

SortShape sort_shape(int64_t V) {
  int b = 1;
  while (((int64_t)1 << b) <= V) ++b;        // keys 0 .. V
  const int passes = (b + kMaxDigit - 1) / kMaxDigit;
  return {passes, (b + passes - 1) / passes};
}

struct BackWs {
  uint32_t *keys[2], *rows[2], *hist, *totals;
  float* part;
  size_t bytes;
};

BackWs carve_back(void* ws, int64_t n, int64_t d) {
  Carve cv(ws, ~(size_t)0);
  BackWs w;
  for (int k = 0; k < 2; ++k) {
    w.keys[k] = cv.take<uint32_t>(n);
    w.rows[k] = cv.take<uint32_t>(n);
  }
  w.hist = cv.take<uint32_t>((size_t)ceil_div(n, kTile) << kMaxDigit);
  w.totals = cv.take<uint32_t>(1 << kMaxDigit);
  w.part = cv.take<float>((size_t)ceil_div(n, kChunk) * 2 * d);
  w.bytes = cv.used;
  return w;
}

}  // namespace

eogp_status embed_tokens(const void* table, eogp_dtype tt, int64_t ldt, int64_t V, int64_t d,
                         const int64_t* tokens, const uint8_t* mask, int64_t n, float scale, int accumulate,
                         void* out, eogp_dtype ot, int64_t ldo, hipStream_t s) {
  if (n == 0) return EOGP_OK;
  timing::Scope ts(EOGP_KT_EMBED, s);
  return with_type(tt, [&](auto el) {
    using TT = decltype(el);
    auto go = [&](auto to, auto pp) {
      using TO = decltype(to);
      constexpr int P = decltype(pp)::value;
      const int64_t col_units = ceil_div(d, 64 * P * kPiece<TT>);
      const int64_t blocks = std::min<int64_t>(ceil_div(n * col_units, 4), 8 * kCus * 4);
      hipLaunchKernelGGL((k_embed<TT, TO, P>), dim3((unsigned)blocks), dim3(256), 0, s,
                         static_cast<const TT*>(table), ldt, V, d, tokens, mask, n, scale, accumulate,
                         static_cast<TO*>(out), ldo, col_units);
      EOGP_LAUNCH_CHECK("embed_tokens");
      return EOGP_OK;
    };
    auto pick = [&](auto to) {
      const int64_t pieces = ceil_div(d, kPiece<TT>);
      return pieces <= 64    ? go(to, std::integral_constant<int, 1>{})
             : pieces <= 128 ? go(to, std::integral_constant<int, 2>{})
             : pieces <= 192 ? go(to, std::integral_constant<int, 3>{})
                             : go(to, std::integral_constant<int, 4>{});
    };
    return ot == tt ? pick(TT{}) : pick(float{});
  });
}

size_t embed_back_ws(int64_t n, int64_t d) { return carve_back(nullptr, n, d).bytes; }

eogp_status embed_back(const void* dout, eogp_dtype t, int64_t ldd, const int64_t* tokens, const uint8_t* mask,
                       int64_t n, int64_t V, int64_t d, float scale, int accumulate, float* dtable, int64_t ldt,
                       void* ws, hipStream_t s) {
  timing::Scope ts(EOGP_KT_EMBED, s);
  if (!accumulate) {
    hipLaunchKernelGGL(k_zero, dim3((unsigned)std::min<int64_t>(ceil_div(V, 4), 8 * kCus)), dim3(256), 0, s, dtable,
                       ldt, V, d);
    EOGP_LAUNCH_CHECK("embed_backward (zeros)");
  }
  if (n == 0) return EOGP_OK;
  const BackWs w = carve_back(ws, n, d);
  const int64_t tiles = ceil_div(n, kTile);
  const SortShape sh = sort_shape(V);
  for (int p = 0; p < sh.passes; ++p) {
    const int shift = p * sh.bits;
    const uint32_t *ki = w.keys[(p + 1) & 1], *ri = w.rows[(p + 1) & 1];
    auto* count = p == 0 ? k_sort_count<true> : k_sort_count<false>;
    auto* scatter = p == 0 ? k_sort_scatter<true> : k_sort_scatter<false>;
    hipLaunchKernelGGL(count, dim3((unsigned)tiles), dim3(256), 0, s, tokens, mask, V, ki, n, shift, sh.bits, w.hist,
                       tiles);
    hipLaunchKernelGGL(k_sort_scan, dim3(1u << sh.bits), dim3(64), 0, s, w.hist, tiles, w.totals);
    hipLaunchKernelGGL(scatter, dim3((unsigned)tiles), dim3(256), 0, s, tokens, mask, V, ki, ri, n, shift, sh.bits,
                       w.hist, tiles, w.totals, w.keys[p & 1], w.rows[p & 1]);
    EOGP_LAUNCH_CHECK("embed_backward (sort)");
  }
  const uint32_t *keys = w.keys[(sh.passes - 1) & 1], *rows = w.rows[(sh.passes - 1) & 1];
  const int64_t chunks = ceil_div(n, kChunk);
  const eogp_status st = with_type(t, [&](auto el) {
    using T = decltype(el);
    const int64_t col_units = ceil_div(d, 64 * kPiece<T>);
    hipLaunchKernelGGL(k_embed_sum<T>, dim3((unsigned)ceil_div(chunks * col_units, 4)), dim3(256), 0, s,
                       static_cast<const T*>(dout), ldd, d, keys, rows, n, (uint32_t)V, scale, accumulate, dtable,
                       ldt, w.part, col_units);
    EOGP_LAUNCH_CHECK("embed_backward (sums)");
    return EOGP_OK;
  });
  if (st != EOGP_OK || chunks == 1) return st;
  const int64_t col_blocks = ceil_div(d, 256);
  hipLaunchKernelGGL(k_embed_join, dim3((unsigned)(chunks * col_blocks)), dim3(256), 0, s, keys, n, (uint32_t)V,
                     w.part, d, scale, accumulate, dtable, ldt, col_blocks);
  EOGP_LAUNCH_CHECK("embed_backward (join)");
  return EOGP_OK;
}

}  // namespace eogp
