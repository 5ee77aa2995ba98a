// Token embedding: rows of a table by token, and the table's gradient by sorted tokens.
#include <algorithm>

#include "rows.h"
#include "timing.h"

namespace eogp {
namespace {

// out[n] = scale table[token n] (+ out[n]), in fp32 and rounded once to out's type. A token outside [0, V) gives
// NaN, a masked row zeros (neither reads the table).
// Bound by the writes (the rows of common tokens stay in the caches). One wave per row and 64 P pieces of it; a
// lane's P pieces are requested together, so a row costs one round trip. 131,072 places of 768 fp32, 56% of
// them valid: 73 us, 6.2 TB/s of reads and writes (a fill runs at 6.8, a copy at 4.7).
template <typename TT, typename TO, int SHAPE>
__global__ __launch_bounds__(256) void k_embed(const TT* __restrict__ table, int64_t ldt, int64_t V, int64_t d,
                                               const int64_t* __restrict__ tokens,
                                               const uint8_t* __restrict__ mask, int64_t n, float scale,
                                               int accumulate, TO* __restrict__ out, int64_t ldo,
                                               int64_t col_units) {
  constexpr int E = kPiece<TT>, P = SHAPE ? SHAPE : 1;      // SHAPE 0: rows shorter than a piece
  constexpr bool kNarrow = SHAPE == 0;
  const int lane = threadIdx.x & 63;
  const int64_t units = n * col_units;
  for (int64_t u = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); u < units;
       u += (int64_t)gridDim.x * 4) {
    const int64_t row = u / col_units, c0 = (u % col_units) * (64 * P * E);
    const bool live = !mask || mask[row] != 0;
    const int64_t tok = live ? tokens[row] : 0;
    const bool inside = tok >= 0 && tok < V;
    const TT* src = table + (live && inside ? tok : 0) * ldt;
    TO* dst = out + row * ldo;
    AnyVec<TT, E> raw[P];
    if (live && inside) {
#pragma unroll
      for (int p = 0; p < P; ++p) raw[p] = request_piece<TT, E, kNarrow>(src, c0 + (int64_t)(p * 64 + lane) * E, d);
    }
    if (!live && accumulate) continue;         // nothing to add
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = c0 + (int64_t)(p * 64 + lane) * E;
      if (c >= d) break;
      float v[E], old[E] = {};
      if (live && inside) {
        settle_piece<TT, E, kNarrow>(raw[p], c, d);
        widen<TT, E>(raw[p], v);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = live ? __builtin_nanf("") : 0.f;
      }
      if (accumulate) load_piece<TO, E>(dst, c, d, 0.f, old);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = accumulate ? old[e] + v[e] * scale : v[e] * scale;
      store_piece<TO, E>(dst, c, d, v);
    }
  }
}

// ---- sorting the tokens ----------------------------------------------------------
// The gradient of row v of the table is the sum of the output's gradients over the rows with token v. They are
// added in the order of their rows by whoever owns the token, so no atomic decides the result: the rows are
// sorted by token first, which costs a few passes over 8 bytes a row where the sums read d elements of it.
// Stable least-significant-digit radix sort of (token, row) pairs; rows that count for no token
// (masked, or a token outside [0, V)) get key V and end up last. A tile is what one block sorts:
// its waves take 64 rows at a time in order, so equal digits keep the order of their rows and the
// result does not depend on any race.
constexpr int kTile = 2048, kSortWaves = 4, kMaxDigit = 9;

// Keys of rows i0, i0 + step, ..., all requested together (rows past the end read the last one): with a branch at
// the mask each row would wait for its mask and then for its token.
template <bool FIRST, int R>
__device__ __forceinline__ void load_keys(const int64_t* tokens, const uint8_t* mask, int64_t V, const uint32_t* keys,
                                          int64_t n, int64_t i0, int64_t step, uint32_t (&key)[R]) {
  if constexpr (FIRST) {
    const uint8_t* live = mask ? mask : reinterpret_cast<const uint8_t*>(tokens);   // (some byte that is there)
    int64_t t[R];
    uint8_t m[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t i = std::min<int64_t>(i0 + r * step, n - 1);
      t[r] = tokens[i];
      m[r] = live[i];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = (!mask || m[r]) && t[r] >= 0 && t[r] < V ? (uint32_t)t[r] : (uint32_t)V;
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = keys[std::min<int64_t>(i0 + r * step, n - 1)];
  }
}

// Zeros `words` words of flags.
__global__ __launch_bounds__(256) void k_clear(uint32_t* __restrict__ flags, int64_t words) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (int64_t)gridDim.x * 256) flags[i] = 0;
}

// Zeros rows row0 .. row1 - 1 of the table but for flagged ones (their sums are written later). Streaming
// stores: call after call, 154 MB of zeros and 512 rows take 36 us so, 42 with plain ones. Rows are
// written from a cache line on: 8,997 rows of 7,875 (283 MB) 61 us, from wherever they begin 73.
__device__ void fill_zero(float* __restrict__ dtable, int64_t ldt, int64_t d, const uint8_t* __restrict__ flags,
                          int64_t block, int64_t blocks, int64_t row0, int64_t row1) {
  const int lane = threadIdx.x & 63;
  const AnyVec<float, 4> z = {};
  for (int64_t r = row0 + block * 4 + (threadIdx.x >> 6); r < row1; r += blocks * 4) {
    if (flags && flags[r]) continue;
    float* row = dtable + r * ldt;
    const int64_t head = std::min<int64_t>(d, -(reinterpret_cast<uintptr_t>(row) >> 2) & 31);   // to a cache line
    if (lane < head) row[lane] = 0.f;
    const int64_t rest = d - head;
    row += head;
    for (int64_t c = 4 * lane; c + 4 <= rest; c += 256)
      __builtin_nontemporal_store(z, reinterpret_cast<AnyVec<float, 4>*>(row + c));
    if (lane < (rest & 3)) row[(rest & ~(int64_t)3) + lane] = 0.f;
  }
}

// Digit counts of each tile: hist[digit][tile]. The first pass flags the tokens that have rows.
template <bool FIRST>
__global__ __launch_bounds__(256) void k_sort_count(const int64_t* __restrict__ tokens,
                                                    const uint8_t* __restrict__ mask, int64_t V,
                                                    const uint32_t* __restrict__ keys, int64_t n, int shift,
                                                    int bits, uint32_t* __restrict__ hist, int64_t tiles,
                                                    uint8_t* __restrict__ flags) {
  __shared__ uint32_t count[1 << kMaxDigit];
  const uint32_t dmask = (1u << bits) - 1;
  for (int b = threadIdx.x; b <= (int)dmask; b += 256) count[b] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kTile;
  uint32_t key[kTile / 256];
  load_keys<FIRST>(tokens, mask, V, keys, n, base + threadIdx.x, 256, key);
#pragma unroll
  for (int r = 0; r < kTile / 256; ++r) {
    if (base + r * 256 + threadIdx.x >= n) break;
    const uint32_t k = key[r];
    if (FIRST && flags && k < V) flags[k] = 1;         // (whoever writes it, it is 1)
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
                                                      uint32_t* __restrict__ rows_out, float* __restrict__ dtable,
                                                      int64_t ldt, int64_t d, const uint8_t* __restrict__ flags,
                                                      int64_t row0, int64_t row1) {
  if (blockIdx.x >= tiles) {                            // blocks beside the sort's: its latency hides the zeros
    fill_zero(dtable, ldt, d, flags, blockIdx.x - tiles, gridDim.x - tiles, row0, row1);
    return;
  }
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
  load_keys<FIRST>(tokens, mask, V, keys, n, base + lane, 64, key);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t i = std::min<int64_t>(base + r * 64 + lane, n - 1);
    row[r] = FIRST ? (uint32_t)i : rows[i];
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
  // Without `totals` the counts are as k_sort_count left them, and the block sums the tiles itself.
  const int per = nd > 256 ? nd / 256 : 1;
  uint32_t mine = 0, tot[2] = {0, 0}, earlier[2] = {0, 0};
  const int d0 = threadIdx.x * per;
  for (int k = 0; k < per; ++k)
    if (d0 + k < nd) {
      const uint32_t* h = hist + (int64_t)(d0 + k) * tiles;
      if (totals) {
        tot[k] = totals[d0 + k];
        earlier[k] = h[blockIdx.x];
      } else {
        for (int64_t j0 = 0; j0 < tiles; j0 += 8) {
          uint32_t c[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) c[q] = h[std::min<int64_t>(j0 + q, tiles - 1)];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int64_t j = j0 + q;
            tot[k] += j < tiles ? c[q] : 0;
            earlier[k] += j < blockIdx.x ? c[q] : 0;   // (blockIdx.x < tiles)
          }
        }
      }
      mine += tot[k];
    }
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
      uint32_t run = first + earlier[k];
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

// Few rows: each one's place is the number of rows before it, found by comparing it with all of them
// (an eighth of them per thread); one launch instead of the radix sort's four or more. Blocks beside them write
// the table's zeros. Whole calls with comparisons / with the sort: 2,049 fp32 rows of 768 into 8,204 tokens 29 / 39 us,
// 4,000 into 50,257 46 / 54, 6,000 of 100 into 5,000 37 / 42, 8,192 of 1,543 into 8,204 59 / 56.
constexpr int kFew = 6144, kRankRows = 32;    // rows of a block that ranks them

__global__ __launch_bounds__(256) void k_rank(const int64_t* __restrict__ tokens, const uint8_t* __restrict__ mask,
                                              int64_t V, int n, uint32_t* __restrict__ keys_out,
                                              uint32_t* __restrict__ rows_out, int rank_blocks, float* __restrict__ dtable, int64_t ldt, int64_t d) {
  __shared__ __align__(16) uint32_t key[kFew];
  if ((int)blockIdx.x >= rank_blocks) {
    fill_zero(dtable, ldt, d, nullptr, blockIdx.x - rank_blocks, gridDim.x - rank_blocks, 0, V);
    return;
  }
  for (int base = 0; base < n; base += kTile) {        // (kFew is a multiple of kTile)
    const int i0 = base + threadIdx.x;
    uint32_t some[kTile / 256];
    load_keys<true>(tokens, mask, V, nullptr, n, i0, 256, some);
#pragma unroll
    for (int r = 0; r < kTile / 256; ++r) key[i0 + r * 256] = i0 + r * 256 < n ? some[r] : 0xFFFFFFFFu;
  }
  __syncthreads();
  const int i = blockIdx.x * kRankRows + (threadIdx.x >> 3), part = threadIdx.x & 7;
  const uint32_t mine = i < n ? key[i] : 0;
  uint32_t before = 0;
  for (int j0 = 4 * part; j0 < n; j0 += 256) {         // (eight reads in flight; places past n hold the last of all keys)
    uint4 k[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) k[q] = *reinterpret_cast<const uint4*>(key + j0 + q * 32);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int j = j0 + q * 32;                       // earlier rows come first among equal keys
      before += (k[q].x < mine + (j < i)) + (k[q].y < mine + (j + 1 < i)) + (k[q].z < mine + (j + 2 < i)) +
                (k[q].w < mine + (j + 3 < i));
    }
  }
  before += __shfl_xor(before, 1);
  before += __shfl_xor(before, 2);
  before += __shfl_xor(before, 4);
  if (i < n && part == 0) {
    keys_out[before] = mine;
    rows_out[before] = (uint32_t)i;
  }
}

// ---- sums over the sorted rows -----------------------------------------------------
// Bound by HBM: the rows are read once, in the order of their tokens, and each finished row of the table is
// written once (196,600 bf16 rows of 2048, 805 MB, into a table of 100,352: 230 us; with the sort, the zeros of
// the other tokens' rows and the join 392 us, 4.2 TB/s).
// A wave sums the rows of a chunk of CHUNK sorted places, for 64 pieces of their columns, eight rows in
// flight, token by token, in fp32. A token whose rows all lie in the chunk is finished here; the sum of one
// that goes on beyond an end of the chunk is written to part[chunk][0] (it began in an earlier
// chunk) or part[chunk][1] (it begins here and goes on: begins[chunk]), and k_embed_join adds those in
// order.
template <typename T, int CHUNK, bool NARROW>
__global__ __launch_bounds__(256) void k_embed_sum(const T* __restrict__ dout, int64_t ldd, int64_t d,
                                                   const uint32_t* __restrict__ keys,
                                                   const uint32_t* __restrict__ rows, int64_t n, uint32_t V,
                                                   float scale, int accumulate, float* __restrict__ dtable,
                                                   int64_t ldt, float* __restrict__ part, int64_t col_units,
                                                   uint8_t* __restrict__ begins) {
  constexpr int E = kPiece<T>, U = 8;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t chunk = unit / col_units, p0 = chunk * CHUNK;
  if (p0 >= n) return;
  const int64_t c = (unit % col_units * 64 + lane) * E;
  const int count = (int)std::min<int64_t>(CHUNK, n - p0);
  // lane l holds place p0 + l
  const uint32_t mykey = lane < count ? keys[p0 + lane] : V;
  const uint32_t myrow = lane < count ? rows[p0 + lane] : 0;
  const uint32_t before = p0 > 0 ? keys[p0 - 1] : V, after = p0 + count < n ? keys[p0 + count] : V;
  float acc[E] = {};
  uint32_t cur = __builtin_amdgcn_readlane(mykey, 0);
  const uint32_t row0 = __builtin_amdgcn_readlane(myrow, 0);
  if (cur >= V) {                              // the rows that count for no token are last
    if (unit % col_units == 0 && lane == 0) begins[chunk] = 0;
    return;
  }
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
    AnyVec<T, E> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = std::min(i + u, count - 1);
      const uint32_t k = __builtin_amdgcn_readlane(mykey, j), r = __builtin_amdgcn_readlane(myrow, j);
      v[u] = request_piece<T, E, NARROW, true>(dout + (int64_t)(k < V ? r : row0) * ldd, c, d);
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
      if (k >= V) {                            // (the requests of such rows were the first row's again)
        if (unit % col_units == 0 && lane == 0) begins[chunk] = 0;
        return;
      }
      settle_piece<T, E, NARROW>(v[u], c, d);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += (float)v[u][e];
    }
  }
  if (unit % col_units == 0 && lane == 0) begins[chunk] = cur == after && !from_before;
  flush(cur == after);
}

// A block takes chunks in which a token begins that goes on, 256 columns at a time (a unit; the flags of
// 64 units are read at once): the sums of that token's chunks are added, a quarter of them per wave, and
// its row is finished. Most such tokens span two or three chunks, so a unit is a chain of waits and as
// many units as fit are wanted: for 196,000 rows of 2048 with Zipf-distributed tokens 16 waves per block
// take 105 us, 4 waves with eight requests each 36, with four (fewer registers) 25. Eight waves with four
// requests help long chains and cost short ones: 74,562 rows of 158 into 7,642 tokens 81 us (the whole call) against
// 92, 196,000 of 2048 408 against 390; four it is. A chain of thousands of chunks is one block's: 262,144 fp32 rows of
// 256 that all have one token take 564 us, of a thousand tokens 89.
template <int CHUNK>
__global__ __launch_bounds__(256) void k_embed_join(const uint32_t* __restrict__ keys, int64_t n,
                                                    const float* __restrict__ part, int64_t d, float scale,
                                                    int accumulate, float* __restrict__ dtable, int64_t ldt,
                                                    int64_t col_blocks, const uint8_t* __restrict__ begins) {
  __shared__ float fold[4][256];
  const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t units = (n + CHUNK - 1) / CHUNK * col_blocks;
  uint64_t todo = 0;
  int64_t base = blockIdx.x - 64 * (int64_t)gridDim.x;
  for (;;) {
    while (!todo) {                                    // (uniform across the block)
      base += 64 * (int64_t)gridDim.x;
      if (base >= units) return;
      const int64_t u = base + lane * (int64_t)gridDim.x;
      todo = __ballot(u < units && begins[u < units ? u / col_blocks : 0]);
    }
    const int64_t unit = base + __builtin_ctzll(todo) * (int64_t)gridDim.x;
    todo &= todo - 1;
    const int64_t first = unit / col_blocks;
    const uint32_t k = keys[(first + 1) * CHUNK - 1];
    // Chunks after the first that begin with its rows: 64 ends of equal parts are looked at at a time.
    int64_t more = 0, end = (n + CHUNK - 1) / CHUNK - first - 1;
    while (more < end) {
      const int64_t part_len = (end - more + 63) / 64, at = more + (lane + 1) * part_len - 1;
      const bool same = at < end && keys[(first + 1 + at) * CHUNK] == k;
      more += __popcll(__ballot(same)) * part_len;
      if (part_len == 1) break;
      end = std::min(end, more + part_len - 1);
    }
    const int64_t c = unit % col_blocks * 256 + lane * 4;
    float acc[4] = {};
    for (int64_t j = wid; j <= more; j += 4 * 4) {    // chunk first + j: its own part 1, the others' part 0
      AnyVec<float, 4> v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t q = j + u * 4;
        v[u] = fetch_piece<float, 4>(part + ((first + q) * 2 + (q == 0)) * d, c, q <= more ? d : 0, 0.f);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += v[u][e];
    }
    __syncthreads();                                   // the unit before has been read
#pragma unroll
    for (int e = 0; e < 4; ++e) fold[wid][lane * 4 + e] = acc[e];
    __syncthreads();
    const int64_t col = unit % col_blocks * 256 + threadIdx.x;
    if (col < d) {
      float s = fold[0][threadIdx.x];
#pragma unroll
      for (int w = 1; w < 4; ++w) s += fold[w][threadIdx.x];
      float* t = dtable + (int64_t)k * ldt + col;
      *t = (accumulate ? *t : 0.f) + s * scale;
    }
  }
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

constexpr int64_t kFlagBytes = 256 << 20;
constexpr int64_t kTilesInline = 64;         // tiles whose counts a scatter block sums itself

// Sorted places per wave: 64, fewer where those would leave most of the chip's waves without rows. Shorter chunks
// give the sums more waves and the join longer chains. Whole calls with chunks of 16 / 32, one after the other: 74,562 rows of 158 into
// 7,642 tokens 121 / 92 us, 65,536 bf16 rows of 768 into 50,257 132 / 108, 8,000 rows of 1,543 into 8,204 60 / 58.
constexpr int kChunk = 64, kShortChunk = 32, kFewChunk = 8;
constexpr int64_t kFewChunkRows = 2048;

constexpr int64_t kFullWaves = 16 * kCus;    // waves from which 64 places each keep the chip busy

int chunk_of(int64_t n, int64_t d, eogp_dtype t) {
  if (n <= kFewChunkRows) return kFewChunk;
  const int64_t waves = ceil_div(n, kChunk) * ceil_div(d, t == EOGP_F32 ? 256 : 512);
  return waves >= kFullWaves ? kChunk : kShortChunk;
}

// The most chunks, and the most chunks times d, of any list of up to n rows of up to d elements: the
// workspace for a batch holds that of every smaller one, though longer lists may have fewer chunks. Short
// chunks are taken for fewer than kFullWaves chunks of 64 places and 512 (fp32: 256) columns, so no
// such list has more than 2 kFullWaves of them, or more than that times 512 elements.
struct ChunkRoom {
  int64_t chunks, elements;
};

ChunkRoom chunk_room(int64_t n, int64_t d) {
  const int64_t few = ceil_div(std::min(n, kFewChunkRows), kFewChunk), shorts = ceil_div(n, kShortChunk),
                longs = ceil_div(n, kChunk);
  return {std::max({few, std::min(shorts, 2 * kFullWaves), longs}),
          std::max({few * d, std::min(shorts * d, 2 * kFullWaves * 512), longs * d})};
}

struct BackWs {
  uint32_t *keys[2], *rows[2], *hist, *totals;
  uint8_t *flags, *begins;
  float* part;
  size_t bytes;
};

BackWs carve_back(void* ws, int64_t n, int64_t V, int64_t d) {
  Carve cv(ws, ~(size_t)0);
  const bool few = n <= kFew;
  const ChunkRoom room = chunk_room(n, d);
  BackWs w;
  for (int k = 0; k < (few ? 1 : 2); ++k) {
    w.keys[k] = cv.take<uint32_t>(n);
    w.rows[k] = cv.take<uint32_t>(n);
  }
  w.hist = cv.take<uint32_t>(few ? 0 : (size_t)ceil_div(n, kTile) << kMaxDigit);
  w.totals = cv.take<uint32_t>(few ? 0 : 1 << kMaxDigit);
  w.flags = cv.take<uint8_t>(few ? 0 : round_up(V, 4));
  w.begins = cv.take<uint8_t>(room.chunks);
  w.part = cv.take<float>((size_t)room.elements * 2);
  w.bytes = cv.used;
  return w;
}

// Sums of the sorted rows, then of the tokens that several chunks hold.
template <int CHUNK>
eogp_status sum_sorted(const BackWs& w, const uint32_t* keys, const uint32_t* rows, const void* dout, eogp_dtype t,
                       int64_t ldd, int64_t n, int64_t V, int64_t d, float scale, int accumulate, float* dtable,
                       int64_t ldt, hipStream_t s) {
  const int64_t chunks = ceil_div(n, CHUNK);
  const eogp_status st = with_type(t, [&](auto el) {
    using T = decltype(el);
    const int64_t col_units = ceil_div(d, 64 * kPiece<T>);
    auto* kfn = d < kPiece<T> ? k_embed_sum<T, CHUNK, true> : k_embed_sum<T, CHUNK, false>;
    hipLaunchKernelGGL(kfn, dim3((unsigned)ceil_div(chunks * col_units, 4)), dim3(256), 0, s,
                       static_cast<const T*>(dout), ldd, d, keys, rows, n, (uint32_t)V, scale, accumulate, dtable,
                       ldt, w.part, col_units, w.begins);
    EOGP_LAUNCH_CHECK("embed_backward (sums)");
    return EOGP_OK;
  });
  if (st != EOGP_OK || chunks == 1) return st;
  const int64_t col_blocks = ceil_div(d, 256);
  hipLaunchKernelGGL(k_embed_join<CHUNK>, dim3((unsigned)std::min<int64_t>((chunks - 1) * col_blocks, 8 * kCus)),
                     dim3(256), 0, s, keys, n, w.part, d, scale, accumulate, dtable, ldt, col_blocks, w.begins);
  EOGP_LAUNCH_CHECK("embed_backward (join)");
  return EOGP_OK;
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
      const int64_t col_units = ceil_div(d, 64 * std::max(P, 1) * kPiece<TT>);
      const int64_t blocks = std::min<int64_t>(ceil_div(n * col_units, 4), 8 * kCus * 4);
      hipLaunchKernelGGL((k_embed<TT, TO, P>), dim3((unsigned)blocks), dim3(256), 0, s,
                         static_cast<const TT*>(table), ldt, V, d, tokens, mask, n, scale, accumulate,
                         static_cast<TO*>(out), ldo, col_units);
      EOGP_LAUNCH_CHECK("embed_tokens");
      return EOGP_OK;
    };
    auto pick = [&](auto to) {
      const int64_t pieces = ceil_div(d, kPiece<TT>);
      return d < kPiece<TT> ? go(to, std::integral_constant<int, 0>{})
             : pieces <= 64  ? go(to, std::integral_constant<int, 1>{})
             : pieces <= 128 ? go(to, std::integral_constant<int, 2>{})
             : pieces <= 192 ? go(to, std::integral_constant<int, 3>{})
                             : go(to, std::integral_constant<int, 4>{});
    };
    return ot == tt ? pick(TT{}) : pick(float{});
  });
}

size_t embed_back_ws(int64_t n, int64_t V, int64_t d) { return carve_back(nullptr, n, V, d).bytes; }

eogp_status embed_back(const void* dout, eogp_dtype t, int64_t ldd, const int64_t* tokens, const uint8_t* mask,
                       int64_t n, int64_t V, int64_t d, float scale, int accumulate, float* dtable, int64_t ldt,
                       void* ws, hipStream_t s) {
  timing::Scope ts(EOGP_KT_EMBED, s);
  const unsigned fill_blocks = accumulate ? 0 : (unsigned)std::min<int64_t>(ceil_div(V, 4), 4 * kCus);
  const BackWs w = n > 0 ? carve_back(ws, n, V, d) : BackWs{};
  auto chunks = [&](const uint32_t* keys, const uint32_t* rows) {
    const int chunk = chunk_of(n, d, t);
    const auto sum = chunk == kChunk ? sum_sorted<kChunk> : chunk == kShortChunk ? sum_sorted<kShortChunk> : sum_sorted<kFewChunk>;
    return sum(w, keys, rows, dout, t, ldd, n, V, d, scale, accumulate, dtable, ldt, s);
  };
  if (n <= kFew) {
    const int rank_blocks = (int)ceil_div(n, kRankRows);
    if (rank_blocks + fill_blocks == 0) return EOGP_OK;
    hipLaunchKernelGGL(k_rank, dim3(rank_blocks + fill_blocks), dim3(256), 0, s, tokens, mask, V, (int)n, w.keys[0],
                       w.rows[0], rank_blocks, dtable, ldt, d);
    EOGP_LAUNCH_CHECK("embed_backward (ranks)");
    if (n == 0) return EOGP_OK;
    return chunks(w.keys[0], w.rows[0]);
  }
  const int64_t tiles = ceil_div(n, kTile);
  const SortShape sh = sort_shape(V);
  // Zeros of a table of up to 256 MB cost less beside the sort than knowing which rows need none.
  const bool flagged = !accumulate && V * d * (int64_t)sizeof(float) > kFlagBytes;
  if (flagged) {
    const int64_t words = round_up(V, 4) / 4;
    hipLaunchKernelGGL(k_clear, dim3((unsigned)std::min<int64_t>(ceil_div(words, 256), kCus)), dim3(256), 0, s,
                       reinterpret_cast<uint32_t*>(w.flags), words);
    EOGP_LAUNCH_CHECK("embed_backward (flags)");
  }
  const bool scan = tiles > kTilesInline;
  for (int p = 0; p < sh.passes; ++p) {
    const int shift = p * sh.bits;
    const uint32_t *ki = w.keys[(p + 1) & 1], *ri = w.rows[(p + 1) & 1];
    auto* count = p == 0 ? k_sort_count<true> : k_sort_count<false>;
    auto* scatter = p == 0 ? k_sort_scatter<true> : k_sort_scatter<false>;
    hipLaunchKernelGGL(count, dim3((unsigned)tiles), dim3(256), 0, s, tokens, mask, V, ki, n, shift, sh.bits, w.hist,
                       tiles, flagged ? w.flags : nullptr);
    if (scan) hipLaunchKernelGGL(k_sort_scan, dim3(1u << sh.bits), dim3(64), 0, s, w.hist, tiles, w.totals);
    // an equal share of the table's zeros beside each pass
    hipLaunchKernelGGL(scatter, dim3((unsigned)tiles + fill_blocks), dim3(256), 0, s, tokens, mask, V, ki, ri, n,
                       shift, sh.bits, w.hist, tiles, scan ? w.totals : nullptr, w.keys[p & 1], w.rows[p & 1], dtable,
                       ldt, d, flagged ? w.flags : nullptr, V * p / sh.passes, V * (p + 1) / sh.passes);
    EOGP_LAUNCH_CHECK("embed_backward (sort)");
  }
  const int last = (sh.passes - 1) & 1;
  return chunks(w.keys[last], w.rows[last]);
}

}  // namespace eogp
