// One token per row of logits, drawn with given uniform numbers.
//
// Everything after the logits' differences is integer arithmetic, so the answer does not depend on
// the order of a sum, on the block's shape or on the GPU:
//   t_i = (l_i - max l) * (log2 e / temperature)      fp32, each operation rounded once
//   w_i = floor(2^30 * 2^t_i)                         by a degree-5 polynomial, each operation rounded once
// Order: logit descending, index ascending. Kept are the first top_k; of these the shortest prefix
// whose mass reaches top_p of theirs; of these the ones with w_i >= min_p * 2^30 (the largest weight
// is 2^30). The answer is the lowest kept index whose running mass exceeds floor(u * mass).
#include <algorithm>
#include <cmath>

#include "rows.h"
#include "timing.h"

namespace eogp {
namespace {

constexpr int kBins = 2048;        // first digit of the selection: 64 per octave of weight, 32 octaves
constexpr float kBinsPerOctave = 64.f;
constexpr int64_t kMaxVocab = (int64_t)1 << 20;

// 2^30 2^f on [-1/2, 1/2]: a least-squares fit of (2^f - 1) / f reweighted until its relative error
// was level (1.1e-7, and 1.9e-7 with fp32's roundings); scaling by 2^30 changes no rounding.
constexpr float kTwo30 = 1073741824.f;
constexpr float kC1 = 0.6931470036506653f * kTwo30, kC2 = 0.24022242426872253f * kTwo30,
                kC3 = 0.05550733581185341f * kTwo30, kC4 = 0.009671512991189957f * kTwo30,
                kC5 = 0.001326472731307149f * kTwo30;

// A row's largest logit and the scale of the differences from it. With a largest of +inf only the
// logits of +inf count: inf - FLT_MAX is inf, every other difference times inf is -inf or NaN.
struct Scale {
  float most, c;
};

__device__ __forceinline__ Scale scale_of(float most, float c) {
  return most == INFINITY ? Scale{3.4028234663852886e38f, INFINITY} : Scale{most, c};
}

// t in [-31, 0]; below -31 the weight is 0 as it is at -31. The median of a NaN (a NaN logit) and two
// numbers is the lesser number, so it weighs nothing.
__device__ __forceinline__ float exponent_of(float l, Scale s) {
#pragma clang fp contract(off)
  const float diff = l - s.most;
  return __builtin_amdgcn_fmed3f(diff * s.c, -31.f, 0.f);
}

// Adding 1.5 * 2^23 rounds t to a whole number k (nearest, ties to even) and leaves it in the sum's low
// bits, which go to the exponent of 2^30 2^f as they are (k >= -31: it stays a normal number).
__device__ __forceinline__ uint32_t weight_of(float t) {
#pragma clang fp contract(off)
  const float shifted = t + 12582912.f;
  const float k = shifted - 12582912.f;
  const float f = t - k;
  float p = f * kC5;
  p = p + kC4;
  p = p * f;
  p = p + kC3;
  p = p * f;
  p = p + kC2;
  p = p * f;
  p = p + kC1;
  p = p * f;
  p = p + kTwo30;
  return (uint32_t)__uint_as_float(__float_as_uint(p) + (__float_as_uint(shifted) << 23));
}

// Sum of up to eight weights of at most 2^30 each: three fit 32 bits, four might not.
template <int E>
__device__ __forceinline__ uint64_t sum_weights(const uint32_t (&w)[E]) {
  if constexpr (E == 4) return (uint64_t)(w[0] + w[1] + w[2]) + w[3];
  return (uint64_t)(w[0] + w[1] + w[2]) + (w[3] + w[4] + w[5]) + (w[6] + w[7]);
}

__device__ __forceinline__ int bin_of(float t) { return std::min((int)(t * -kBinsPerOctave), kBins - 1); }

// Ascending order of these keys is descending order of the logits.
__device__ __forceinline__ uint32_t order_key(float l) {
  const uint32_t u = __float_as_uint(l + 0.f);         // -0 becomes +0
  return u & 0x80000000u ? u : ~(u | 0x80000000u);
}

// floor(total * part / 2^24) for total < 2^62, part <= 2^24
__device__ __forceinline__ uint64_t share_of(uint64_t total, uint32_t part) {
  return (total >> 24) * part + (((total & 0xFFFFFF) * part) >> 24);
}

// Sum over the block, in every thread; `slot` is free again after the next barrier.
template <int NT>
__device__ __forceinline__ uint64_t block_total(uint64_t v, uint64_t* slot) {
  v = wave_total(v);
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
  __syncthreads();
  v = slot[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v += slot[w];
  return v;
}

// floor(u * total), u in steps of 2^-24 and clamped to [0, 1)
__device__ __forceinline__ uint64_t target_of(uint64_t total, float u) {
  return share_of(total, (uint32_t)fminf(fmaxf(floorf(u * 16777216.f), 0.f), 16777215.f));
}

// The largest logit of the row, in every thread (-inf if there is none); `mine`: this thread's.
template <typename Row, int NT>
__device__ __forceinline__ float row_max(Row& r, int64_t V, float* slot, float& mine) {
  float m = -INFINITY;
  r.each((uint32_t)V, [&](int, uint32_t, uint32_t, const auto& v) {
#pragma unroll
    for (int e = 0; e < Row::E; ++e) m = fmaxf(m, v[e]);   // (passes over NaN)
  });
  mine = m;
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) m = fmaxf(m, slot[w]);
  return m;
}

// Pieces of a wave whose weights are summed at once, and how many such groups a row has at most.
constexpr int group_of(int p) { return p == 2 ? 2 : 4; }
template <typename T, int NT, int P>
constexpr int kGroups = P > 0 ? P / group_of(P) : (int)(kMaxVocab / (NT * group_of(P) * kPiece<T>));

// The token drawn from the weights kept(logit, index), of which group_mass holds each wave's sums,
// group by group (in index order come groups, then waves): the wave that holds it reads its group's
// pieces again.
template <typename T, int NT, int G, typename Kept>
__device__ void find_token(const T* l, int64_t V, float u, const uint64_t* group_mass, int64_t* out, Kept&& kept) {
  constexpr int E = kPiece<T>, kWaves = NT / 64, kGroup = NT * G * E;
  const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int sums = (int)((V + kGroup - 1) / kGroup) * kWaves;
  const uint64_t mine = lane < sums ? group_mass[lane] : 0, scan = wave_scan(mine);
  uint64_t total = lane_value(scan, 63);
  for (int b = 64; b < sums; b += 64) total += wave_total(b + lane < sums ? group_mass[b + lane] : 0);
  const uint64_t target = target_of(total, u);         // below the total
  uint64_t before = 0;
  int hit = -1;
  for (int b = 0; b < sums && hit < 0; b += 64) {
    const uint64_t v = b == 0 ? mine : b + lane < sums ? group_mass[b + lane] : 0;
    const uint64_t incl = before + (b == 0 ? scan : wave_scan(v));
    const uint64_t over = __ballot(incl > target);
    const int at = over ? __builtin_ctzll(over) : 63;
    if (over) hit = b + at;
    before = lane_value(over ? incl - v : incl, at);
  }
  if (hit < 0 || hit % kWaves != wid) return;
  const int64_t c0 = (int64_t)(hit / kWaves) * kGroup + ((int64_t)wid * G * 64 + lane) * E;
  AnyVec<T, E> raw[G];                                 // requested together
#pragma unroll
  for (int q = 0; q < G; ++q) raw[q] = fetch_piece<T, E>(l, c0 + q * 64 * E, V, (T)-INFINITY);
#pragma unroll
  for (int q = 0; q < G; ++q) {
    const int64_t c = c0 + q * 64 * E;
    uint32_t w[E];
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = kept((float)raw[q][e], (uint32_t)c + e);
    const uint64_t s = sum_weights<E>(w), incl = before + wave_scan(s);
    uint64_t run = incl - s;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (run <= target && target < run + w[e]) *out = c + e;
      run += w[e];
    }
    before = lane_value(incl, 63);
  }
}

// Adds a piece's weights to its group's sum; the group's last piece stores the wave's.
template <int NT, int G, int E, typename Kept>
__device__ __forceinline__ void add_piece(int p, uint32_t c, const float (&v)[E], uint64_t& sum, uint64_t* group_mass,
                                          Kept&& kept) {
  uint32_t w[E];
#pragma unroll
  for (int e = 0; e < E; ++e) w[e] = kept(v[e], c + e);
  sum += sum_weights<E>(w);
  if (p % G == G - 1) {
    const uint64_t total = wave_scan(sum);
    if ((threadIdx.x & 63) == 63) group_mass[(p / G) * (NT / 64) + (threadIdx.x >> 6)] = total;
    sum = 0;
  }
}

// From the whole distribution (or its w >= min_w). A block takes a row at a time. P > 0: the row stays
// in registers as read, and the next one is requested piece by piece as the weights' pass lets go of
// this one; P = 0: it is read in both passes.
// MIN: only weights of at least min_w count (a compare and a select per logit that the plain draw is spared).
// Bound by the vector ALU of the blocks with the most rows: 37 vector instructions a logit (18 of them the
// whole-number weight of 30 bits, since the hardware's exponential has no rounding that another machine repeats; the
// others the maximum, 64-bit sums and addresses) keep it busy for 0.72 of the launch on average over the CUs, where the
// mean block has 6.3 rows and those with the most 7 or 8. 2,048 fp32 places of 50,257, 75% of them valid: 93 to 101 us,
// 3.1 to 3.3 TB/s; 1,536 unmasked rows, six a block: 91; the first reading of the row is its only one.
// With P = 0 it is read twice (1,024 fp32 rows of 100,352: 145 us, 2.8 TB/s of one reading); 16-bit rows of 8,193 to
// 16,384 pieces spill 4 registers, with MIN 11 (2,048 bf16 rows of 100,352: 174 and 183 us, 2.4 and 2.2 TB/s).
template <typename T, int NT, int P, bool MIN>
__global__ __launch_bounds__(NT) void k_sample(
    const T* __restrict__ logits, int64_t ldl, int64_t n, int64_t V, const float* __restrict__ uniforms,
    const uint8_t* __restrict__ mask, float c, uint32_t min_w, int64_t* __restrict__ out) {
  constexpr int E = kPiece<T>, G = group_of(P);
  __shared__ uint64_t group_mass[2][kGroups<T, NT, P> * (NT / 64)];
  __shared__ float slot[2][NT / 64];
  using Row = RegisterRow<T, NT, P, G>;
  RowWalk walk;
  auto live = [&](int64_t row) {
    if (!mask || mask[row] != 0) return true;
    if (threadIdx.x == 0) out[row] = -1;
    return false;
  };
  Row r;
  int64_t row = walk.next(n, live);
  if (row < 0) return;
  r.load(logits + row * ldl, (uint32_t)V);
  for (int turn = 0;; turn ^= 1) {                     // rows alternate between the two sets of sums
    const T* l = logits + row * ldl;
    float mine;
    const float m = row_max<Row, NT>(r, V, slot[turn], mine);
    const int64_t after = walk.next(n, live);
    const Scale scale = scale_of(m, c);
    auto kept = [&](float v, uint32_t) -> uint32_t {
      const uint32_t w = weight_of(exponent_of(v, scale));
      return !MIN || w >= min_w ? w : 0;
    };
    uint64_t sum = 0;
    auto add = [&](int p, uint32_t i0, uint32_t, const float(&v)[E]) {
      add_piece<NT, G, E>(p, i0, v, sum, group_mass[turn], kept);
    };
    if (after < 0)
      r.each((uint32_t)V, add);
    else
      r.each_then_load((uint32_t)V, add, logits + after * ldl);
    __syncthreads();
    if (m == -INFINITY) {                              // nothing to draw from
      if (threadIdx.x == 0) out[row] = -1;
    } else {
      find_token<T, NT, G>(l, V, uniforms[row], group_mass[turn], out + row, kept);
    }
    if (after < 0) return;
    row = after;
  }
}

// ---- with top_k or top_p -------------------------------------------------------------
// Candidates that are settled against each other in LDS, each against all, which takes the square of their
// number (1,024: some 40 us): the most there is room for; with top_k, where the alternative is the histogram's
// passes; and where it is a list of one bin and a pass over the row (about 10 us for 50,257 logits).
constexpr int kList = 1024, kListTopK = 512, kListAll = 256;

// What is kept: every element up to this one in the order.
struct Bound {
  uint32_t key, index;
  __device__ __forceinline__ bool keeps(uint32_t k, uint32_t i) const {
    return k < key || (k == key && i <= index);
  }
};

struct Found {
  uint32_t digit;
  uint64_t before, amount;
};

template <int NT>
struct SelectLds {
  unsigned long long hist[kBins];
  alignas(16) uint32_t reach[2][256];
  alignas(16) uint32_t key[kList + 4], index[kList + 4], weight[kList + 4];
  uint64_t sum[NT / 64], sum2[NT / 64];
  uint32_t listed;
  float slot[NT / 64], cut;
  Bound bound;
  Found found;
};

// The digit at which the running sum of hist, from `before` on, reaches `want`. One exists.
template <int NT>
__device__ Found find_digit(SelectLds<NT>& sh, int digits, uint64_t before, uint64_t want) {
  constexpr int kMost = kBins / NT;
  const int per = std::max(1, digits / NT), wid = threadIdx.x >> 6;
  uint64_t h[kMost], s = 0;
  __syncthreads();                                     // the histogram is complete
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const int b = threadIdx.x * per + k;
    s += h[k] = k < per && b < digits ? sh.hist[b] : 0;
  }
  const uint64_t incl = wave_scan(s);
  if ((threadIdx.x & 63) == 63) sh.sum[wid] = incl;
  __syncthreads();
  uint64_t run = before + incl - s;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const uint64_t others = sh.sum[w];
    run += w < wid ? others : 0;
  }
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    if (run < want && want <= run + h[k]) sh.found = Found{(uint32_t)(threadIdx.x * per + k), run, h[k]};
    run += h[k];
  }
  __syncthreads();
  return sh.found;
}

template <int NT>
__device__ void clear_hist(SelectLds<NT>& sh, int digits) {
  __syncthreads();
  for (int b = threadIdx.x; b < digits; b += NT) sh.hist[b] = 0;
  __syncthreads();
}

template <int NT>
__device__ void clear_list(SelectLds<NT>& sh) {
  __syncthreads();
  if (threadIdx.x == 0) sh.listed = 0;
  __syncthreads();
}

template <int NT>
__device__ __forceinline__ void append(SelectLds<NT>& sh, uint32_t key, uint32_t index, uint32_t weight) {
  const uint32_t at = atomicAdd(&sh.listed, 1u);
  if (at < kList) {
    sh.key[at] = key;
    sh.index[at] = index;
    sh.weight[at] = weight;
  }
}

// Four places past the list's n elements that are read with them and stand for nothing.
template <int NT>
__device__ __forceinline__ void end_list(SelectLds<NT>& sh, int n) {
  if (threadIdx.x < 4) {
    sh.key[n + threadIdx.x] = sh.index[n + threadIdx.x] = 0xFFFFFFFFu;
    sh.weight[n + threadIdx.x] = 0;
  }
  __syncthreads();
}

// Place and mass before element i of the list among its n elements.
template <int NT>
__device__ __forceinline__ void settle(const SelectLds<NT>& sh, int n, int i, uint32_t& rank, uint64_t& mass) {
  const uint64_t mine = (uint64_t)sh.key[i] << 32 | sh.index[i];
  rank = 0;
  mass = 0;
  for (int j = 0; j < n; j += 4) {
    const uint4 k = *reinterpret_cast<const uint4*>(sh.key + j), x = *reinterpret_cast<const uint4*>(sh.index + j),
                w = *reinterpret_cast<const uint4*>(sh.weight + j);
    auto one = [&](uint32_t kj, uint32_t xj, uint32_t wj) {
      const bool first = ((uint64_t)kj << 32 | xj) < mine;
      rank += first;
      mass += first ? wj : 0;
    };
    one(k.x, x.x, w.x);
    one(k.y, x.y, w.y);
    one(k.z, x.z, w.z);
    one(k.w, x.w, w.w);
  }
}

// The draw when the list holds every element that can be kept: top_k by rank (0: all of them),
// top_p of `mass` (of the top_k's own mass if there is a top_k), min_w, then the running mass by
// index; each element against all others.
template <int NT>
__device__ void draw_from_list(SelectLds<NT>& sh, uint32_t top_k, uint32_t top_p24, uint32_t min_w, uint64_t mass,
                               float u, int64_t* out) {
  constexpr int kMine = kList / NT;
  const int n = (int)sh.listed;
  end_list(sh, n);
  uint32_t rank[kMine];
  uint64_t before[kMine], s = 0;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int i = k * NT + threadIdx.x;
    if (i >= n) break;
    settle(sh, n, i, rank[k], before[k]);
    if (!top_k || rank[k] < top_k) s += sh.weight[i];
  }
  s = block_total<NT>(s, sh.sum);
  if (top_k) mass = s;
  const uint64_t want = std::max<uint64_t>(1, share_of(mass, top_p24));
  uint64_t kept = 0;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int i = k * NT + threadIdx.x;
    if (i >= n) break;
    const uint32_t w = sh.weight[i];
    if ((top_k && rank[k] >= top_k) || before[k] >= want || w < min_w) sh.weight[i] = 0;   // all have read it
    kept += sh.weight[i];
  }
  const uint64_t target = target_of(block_total<NT>(kept, sh.sum2), u);
  for (int i = threadIdx.x; i < n; i += NT) {
    const uint32_t w = sh.weight[i], x = sh.index[i];
    uint64_t run = 0;
    for (int j = 0; j < n; j += 4) {
      const uint4 xs = *reinterpret_cast<const uint4*>(sh.index + j),
                  ws = *reinterpret_cast<const uint4*>(sh.weight + j);
      run += (uint64_t)((xs.x < x ? ws.x : 0) + (xs.y < x ? ws.y : 0) + (xs.z < x ? ws.z : 0)) +
             (xs.w < x ? ws.w : 0);
    }
    if (run <= target && target < run + w) *out = x;
  }
}

// A lower bound of the top_k-th largest logit (1 <= top_k <= NT): of the upper 16 bits of the threads'
// own largest logits (as order keys), the least that top_k of them reach; the logit with that key and
// its lower bits set. Found a byte at a time: every wave scans the counts of the byte's 256 values.
template <int NT>
__device__ float lower_bound_of(SelectLds<NT>& sh, uint32_t key, uint32_t top_k) {
  const int lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i < 512; i += NT) (&sh.reach[0][0])[i] = 0;
  if (threadIdx.x == 0) sh.listed = 0;
  __syncthreads();
  uint32_t found = 0, below = 0;                       // below: threads whose key is below the bytes found
#pragma unroll
  for (int byte = 0; byte < 2; ++byte) {
    if (byte == 0 || key >> 24 == found >> 8) atomicAdd(&sh.reach[byte][(key >> (24 - 8 * byte)) & 255], 1u);
    __syncthreads();
    const uint4 c = *reinterpret_cast<const uint4*>(&sh.reach[byte][4 * lane]);
    const uint32_t sum = c.x + c.y + c.z + c.w, incl = below + wave_scan(sum);
    const int at = __builtin_ctzll(__ballot(incl >= top_k));        // (all NT threads reach it at the latest)
    uint32_t run = (uint32_t)__builtin_amdgcn_readlane((int)(incl - sum), at), digit = 4 * at;
    const uint32_t part[3] = {(uint32_t)__builtin_amdgcn_readlane((int)c.x, at),
                              (uint32_t)__builtin_amdgcn_readlane((int)c.y, at),
                              (uint32_t)__builtin_amdgcn_readlane((int)c.z, at)};
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (digit == 4u * at + k && run + part[k] < top_k) {
        run += part[k];
        ++digit;
      }
    below = run;
    found |= digit << (8 - 8 * byte);
  }
  const uint32_t last = found << 16 | 0xFFFFu;
  const uint32_t bits = last & 0x80000000u ? last : ~last & 0x7FFFFFFFu;
  return last >= 0xFF800000u ? -INFINITY : __uint_as_float(bits);   // (-inf's own key, or beyond)
}

// The last kept element when more of a bin's elements tie than the list holds: the bin is split by the
// key's four digits, then the index's. `row` is read once per digit.
template <typename T, int NT>
__device__ Bound split_bin(SelectLds<NT>& sh, RegisterRow<T, NT, 0, 4>& row, int64_t V, Scale scale, Bound within,
                           bool by_mass, Found f, uint64_t want) {
  constexpr int E = kPiece<T>;
  const int bin = (int)f.digit;
  Bound b{0, 0};
  uint64_t before = f.before;
  for (int level = 0; level < 8; ++level) {
    const int shift = 24 - 8 * (level & 3);
    clear_hist(sh, 256);
    row.each((uint32_t)V, [&](int, uint32_t i0, uint32_t, const float(&v)[E]) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t i = i0 + e;
        const float x = fmaxf(v[e], -INFINITY), t = exponent_of(x, scale);
        if (i >= V || bin_of(t) != bin) continue;
        const uint32_t k = order_key(x);
        if (!within.keeps(k, i)) continue;
        uint32_t dig;
        if (level < 4) {
          if (level > 0 && ((k ^ b.key) >> (shift + 8)) != 0) continue;
          dig = (k >> shift) & 255;
        } else {
          if (k != b.key || (level > 4 && ((i ^ b.index) >> (shift + 8)) != 0)) continue;
          dig = (i >> shift) & 255;
        }
        atomicAdd(&sh.hist[dig], by_mass ? (unsigned long long)weight_of(t) : 1ull);
      }
    });
    f = find_digit<NT>(sh, 256, before, want);
    before = f.before;
    if (level < 4)
      b.key |= f.digit << shift;
    else
      b.index |= f.digit << shift;
    if (level == 3 && !by_mass && f.before + f.amount == want) {   // all of the last key's elements
      b.index = 0xFFFFFFFFu;
      break;
    }
  }
  return b;
}

// One block per row, since all its steps meet in one list. 256 bf16 rows of 100,352 (a row per CU) with
// top_k 50, top_p 0.9 and min_p: 20 us, 2.6 TB/s of one reading; one fp16 row of 50,257 with top_p 0.95: 19 us where
// few tokens reach it (59 where thousands do), dependent steps (maximum, histogram, its scan, list, order, draw) of one
// CU, where several CUs for the row would pay a launch of 4 us or a wait between blocks for each. The histogram
// and the list read the row again, from the caches, and the bound and scale lie in scratch (64 to 72 bytes a lane). Wide filters read
// it up to five times: 256 bf16 rows of 100,352 with a top_p that keeps thousands 124 us, top_k 2,000 101, both 167.
// 1. top_k up to the block's threads: the top_k-th largest of the threads' own maxima is a lower
//    bound of the top_k-th largest logit, so the elements at or above it (few more than top_k) hold
//    all that is kept; they are settled in LDS.
// 2. Otherwise the row is read again: a histogram over bins of t (monotone in the logit) shows the
//    bin in which the count or the mass is reached. The elements up to that bin, if the list holds
//    them, are settled as in 1; if not, only that bin's are, which gives the last kept element; if
//    even those are too many (ties), the bin is split digit by digit.
// t_cut: elements below it weigh so little together that top_p is reached before them.
template <typename T, int NT, int P>
__global__ __launch_bounds__(NT) void k_sample_select(const T* __restrict__ logits, int64_t ldl, int64_t V,
                                                      const float* __restrict__ uniforms,
                                                      const uint8_t* __restrict__ mask, float c, uint32_t top_k,
                                                      uint32_t top_p24, uint32_t min_w, float t_cut,
                                                      int64_t* __restrict__ out) {
  constexpr int E = kPiece<T>;
  __shared__ SelectLds<NT> sh;
  constexpr int kSums = (int)(((P > 0 ? P * NT * E : kMaxVocab) + NT * 4 * E - 1) / (NT * 4 * E)) * (NT / 64);
  __shared__ uint64_t group_mass[kSums];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  if (mask && mask[row] == 0) {
    if (tid == 0) out[row] = -1;
    return;
  }
  const T* l = logits + row * ldl;
  const float u = uniforms[row];
  Scale scale;
  {
    RegisterRow<T, NT, P> r;
    r.load(l, (uint32_t)V);
    float mine;
    const float m = row_max<RegisterRow<T, NT, P>, NT>(r, V, sh.slot, mine);
    if (m == -INFINITY) {                              // nothing to draw from
      if (tid == 0) out[row] = -1;
      return;
    }
    scale = scale_of(m, c);
    if (top_k && top_k <= NT) {
      const float cut = lower_bound_of<NT>(sh, order_key(mine), top_k);
      // Which of the thread's pieces reach the bound; those few are read again and taken apart.
      uint64_t hits = 0;
      if (mine >= cut)
        r.each((uint32_t)V, [&](int p, uint32_t, uint32_t, const float(&v)[E]) {
          float top = v[0];
#pragma unroll
          for (int e = 1; e < E; ++e) top = fmaxf(top, v[e]);
          if (top >= cut) hits |= 1ull << (P > 0 ? p : p & 63);
        });
      using Shape = RegisterRow<T, NT, 1>;
      const uint32_t place = Shape::here();
      for (; hits; hits &= hits - 1) {
        for (int64_t i0 = place + (int64_t)__builtin_ctzll(hits) * NT * E; i0 < V; i0 += 64 * NT * E) {
          float v[E];
          load_piece<T, E>(l, i0, V, -INFINITY, v);
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (v[e] >= cut && i0 + e < V)
              append(sh, order_key(v[e]), (uint32_t)i0 + e, weight_of(exponent_of(v[e], scale)));
          if (P > 0) break;
        }
      }
      __syncthreads();
      if (sh.listed <= kListTopK) {
        draw_from_list<NT>(sh, top_k, top_p24, min_w, 0, u, out + row);
        return;
      }
    }
  }
  RegisterRow<T, NT, 0, 4> r;
  r.load(l, (uint32_t)V);
  Bound bound{0xFFFFFFFFu, 0xFFFFFFFFu};               // everything
  for (int by_mass = 0; by_mass < 2; ++by_mass) {
    if (by_mass ? top_p24 == 1u << 24 : top_k == 0) continue;
    clear_hist(sh, kBins);
    const bool bounded = by_mass && top_k;
    uint64_t mass = 0;
    r.each((uint32_t)V, [&](int, uint32_t i0, uint32_t, const float(&v)[E]) {
      if ((uint32_t)__builtin_amdgcn_readfirstlane((int)i0) >= V) return;   // past the end for the whole wave
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t i = i0 + e;
        const float t = exponent_of(v[e], scale);
        if (by_mass) {
          uint32_t w = weight_of(t);                   // (0 past the row's end)
          if (bounded && !bound.keeps(order_key(fmaxf(v[e], -INFINITY)), i)) w = 0;
          mass += w;
          if (t >= t_cut && w) atomicAdd(&sh.hist[bin_of(t)], (unsigned long long)w);
        } else if (i < V) {
          atomicAdd(&sh.hist[bin_of(t)], 1ull);
        }
      }
    });
    mass = block_total<NT>(mass, sh.sum2);
    const uint64_t want = by_mass ? std::max<uint64_t>(1, share_of(mass, top_p24)) : top_k;
    const Found f = find_digit<NT>(sh, kBins, 0, want);
    // Elements up to the bin, then of the bin alone; the bin's t are above `low` and at most `high`.
    const float low = -((float)f.digit + 1.f) / kBinsPerOctave, high = -(float)f.digit / kBinsPerOctave;
    bool all = true;
    for (int only = 0; only < 2; ++only) {
      all = !only;
      clear_list(sh);
      r.each((uint32_t)V, [&](int, uint32_t i0, uint32_t, const float(&v)[E]) {
        float top = v[0];
#pragma unroll
        for (int e = 1; e < E; ++e) top = fmaxf(top, v[e]);
        if (exponent_of(top, scale) <= low) return;    // none of the piece
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint32_t i = i0 + e;
          const float x = fmaxf(v[e], -INFINITY), t = exponent_of(x, scale);
          if (t <= low || (only && t > high) || i >= V) continue;
          const uint32_t k = order_key(x);
          if (bound.keeps(k, i)) append(sh, k, i, weight_of(t));
        }
      });
      __syncthreads();
      if (sh.listed <= (only ? kList : kListAll)) break;
      if (!only) __syncthreads();                      // all have seen the count before it is cleared
    }
    const int n = (int)sh.listed;
    if (n > kList) {
      bound = split_bin<T, NT>(sh, r, V, scale, bound, by_mass, f, want);
      continue;
    }
    if (all) {
      draw_from_list<NT>(sh, by_mass ? 0 : top_k, top_p24, min_w, mass, u, out + row);
      return;
    }
    end_list(sh, n);
    for (int i = tid; i < n; i += NT) {
      uint32_t rank;
      uint64_t before;
      settle(sh, n, i, rank, before);
      const bool is_last = by_mass ? f.before + before < want && want <= f.before + before + sh.weight[i]
                                   : f.before + rank == want - 1;
      if (is_last) sh.bound = Bound{sh.key[i], sh.index[i]};
    }
    __syncthreads();
    bound = sh.bound;
  }
  auto kept = [&](float v, uint32_t i) -> uint32_t {
    const float x = fmaxf(v, -INFINITY);
    if (!bound.keeps(order_key(x), i)) return 0;
    const uint32_t w = weight_of(exponent_of(x, scale));
    return w >= min_w ? w : 0;
  };
  uint64_t sum = 0;
  r.each((uint32_t)V, [&](int p, uint32_t i0, uint32_t, const float(&v)[E]) {
    add_piece<NT, 4, E>(p, i0, v, sum, group_mass, kept);
  });
  __syncthreads();
  find_token<T, NT, 4>(l, V, u, group_mass, out + row, kept);
}

// Temperature 0: the lowest index of the largest logit, one block per row (bound by HBM for many rows, by the
// row's round trips for few). 2,048 fp32 rows of 50,257: 75 us, 5.5 TB/s; 256 bf16 rows of 100,352 13 us, one row 7.
template <typename T>
__global__ __launch_bounds__(1024) void k_argmax(const T* __restrict__ logits, int64_t ldl, int64_t V,
                                                 const uint8_t* __restrict__ mask, int64_t* __restrict__ out) {
  constexpr int E = kPiece<T>;
  __shared__ uint64_t best[16];
  const int64_t row = blockIdx.x;
  if (mask && mask[row] == 0) {
    if (threadIdx.x == 0) out[row] = -1;
    return;
  }
  uint64_t b = ~0ull;                                  // (order key, index), the least is the answer
  for (int64_t at = (int64_t)threadIdx.x * E; at < V; at += 1024 * E) {
    float v[E];
    load_piece<T, E>(logits + row * ldl, at, V, -INFINITY, v);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (v[e] > -INFINITY)                            // (false for NaN)
        b = std::min(b, (uint64_t)order_key(v[e]) << 32 | (uint64_t)(at + e));
  }
  for (int off = 32; off > 0; off >>= 1) b = std::min<uint64_t>(b, __shfl_xor((unsigned long long)b, off));
  if ((threadIdx.x & 63) == 0) best[threadIdx.x >> 6] = b;
  __syncthreads();
  if (threadIdx.x) return;
  for (int w = 1; w < 16; ++w) b = std::min(b, best[w]);
  out[row] = b == ~0ull ? -1 : (int64_t)(b & 0xFFFFFFFFu);
}

}  // namespace

int64_t sample_max_vocab() { return kMaxVocab; }

eogp_status sample_tokens(const void* logits, eogp_dtype t, int64_t ldl, int64_t n, int64_t V,
                          const float* uniforms, const uint8_t* mask, double temperature, int64_t top_k,
                          double top_p, double min_p, int64_t* out, hipStream_t s) {
  if (n == 0) return EOGP_OK;
  timing::Scope ts(EOGP_KT_SAMPLE, s);
  const float c = (float)std::min(1.4426950408889634 / temperature, 3.0e38);
  const uint32_t k = top_k >= V ? 0 : (uint32_t)top_k;           // all of them: no limit
  const uint32_t p24 = (uint32_t)std::floor(top_p * 16777216.0 + 0.5);
  const uint32_t min_w = (uint32_t)std::ceil(min_p * 1073741824.0);
  const bool select = k || p24 < 1u << 24;
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    const T* l = static_cast<const T*>(logits);
    // f(first row, rows) for launches with a block per row
    auto in_parts = [&](auto&& f) {
      for (int64_t r = 0; r < n; r += kMostBlocks) {
        f(r, (unsigned)std::min<int64_t>(n - r, kMostBlocks));
        EOGP_LAUNCH_CHECK("sample_tokens");
      }
      return EOGP_OK;
    };
    if (temperature == 0)
      return in_parts([&](int64_t r, unsigned rows) {
        hipLaunchKernelGGL(k_argmax<T>, dim3(rows), dim3(1024), 0, s, l + r * ldl, ldl, V, mask ? mask + r : nullptr,
                           out + r);
      });
    return with_row_shape<T>(V, [&](auto nt, auto p) -> eogp_status {
      constexpr int NT = decltype(nt)::value, P = decltype(p)::value;
      if (select) {
        // V weights of at most 2^(30 + t_cut) each come to less than the (1 - top_p) 2^30 beyond top_p
        const float t_cut = (float)(std::log2((16777216.0 - p24) / 16777216.0 / (double)V) - 0.01);
        return in_parts([&](int64_t r, unsigned rows) {
          hipLaunchKernelGGL((k_sample_select<T, NT, P>), dim3(rows), dim3(NT), 0, s, l + r * ldl, ldl, V,
                             uniforms + r, mask ? mask + r : nullptr, c, k, p24, min_w, t_cut, out + r);
        });
      }
      auto* kfn = min_w > 1 ? k_sample<T, NT, P, true> : k_sample<T, NT, P, false>;
      hipLaunchKernelGGL(kfn, dim3((unsigned)row_blocks(n, NT, 1)), dim3(NT), 0, s, l, ldl, n, V, uniforms, mask, c,
                         min_w, out);
      EOGP_LAUNCH_CHECK("sample_tokens");
      return EOGP_OK;
    });
  });
}

}  // namespace eogp
