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
// was level (9e-8); scaling by 2^30 changes no rounding.
constexpr float kTwo30 = 1073741824.f;
constexpr float kC1 = 0.6931470036506653f * kTwo30, kC2 = 0.24022242426872253f * kTwo30,
                kC3 = 0.05550733581185341f * kTwo30, kC4 = 0.009671512991189957f * kTwo30,
                kC5 = 0.001326472731307149f * kTwo30;

// t in [-31, 0]; below -31 the weight is 0 as it is at -31. fminf takes the NaN of inf - inf to 0.
__device__ __forceinline__ float exponent_of(float l, float m, float c) {
#pragma clang fp contract(off)
  const float diff = l - m;
  const float t = diff * c;
  return fmaxf(fminf(t, 0.f), -31.f);
}

__device__ __forceinline__ uint32_t weight_of(float t) {
#pragma clang fp contract(off)
  const float k = rintf(t);
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
  return (uint32_t)p >> (uint32_t)(int)-k;
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

// What is kept so far: every element before (bin, key, index) in the order, that one included.
struct Bound {
  int bin = kBins;
  uint32_t key = 0xFFFFFFFFu, index = 0xFFFFFFFFu;
  __device__ __forceinline__ bool keeps(int b, uint32_t k, uint32_t i) const {
    return b < bin || (b == bin && (k < key || (k == key && i <= index)));
  }
  __device__ __forceinline__ Bound least(const Bound& o) const { return keeps(o.bin, o.key, o.index) ? o : *this; }
};

struct Found {
  uint32_t digit, count_before, count;
  uint64_t mass_before, mass;
};

// Inclusive sum over a wave.
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
  const int lane = threadIdx.x & 63;
  for (int off = 1; off < 64; off <<= 1) {
    const uint64_t o = __shfl_up((unsigned long long)v, off);
    if (lane >= off) v += o;
  }
  return v;
}

template <int NT>
struct Shared {
  uint32_t count[kBins];
  unsigned long long mass[kBins];
  uint64_t wave_count[NT / 64], wave_mass[NT / 64];
  float slot[NT / 64];
  Found found;
};

// The digit at which the running count reaches `want` (BY_MASS: the running mass), starting from
// (count0, mass0) before the first digit. One exists by the caller's choice of `want`.
template <int NT, bool BY_MASS>
__device__ Found find_digit(Shared<NT>& sh, int digits, uint32_t count0, uint64_t mass0, uint64_t want) {
  constexpr int kMost = kBins / NT;
  const int per = std::max(1, digits / NT), wid = threadIdx.x >> 6;
  uint32_t cn[kMost];
  uint64_t ms[kMost], cs = 0, mm = 0;
  __syncthreads();                                     // the histogram is complete
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const int b = threadIdx.x * per + k;
    const bool in = k < per && b < digits;
    cn[k] = in ? sh.count[b] : 0;
    ms[k] = in ? sh.mass[b] : 0;
    cs += cn[k];
    mm += ms[k];
  }
  const uint64_t ci = wave_scan(cs), mi = wave_scan(mm);
  if ((threadIdx.x & 63) == 63) {
    sh.wave_count[wid] = ci;
    sh.wave_mass[wid] = mi;
  }
  __syncthreads();
  uint64_t c = count0 + ci - cs, m = mass0 + mi - mm;
  for (int w = 0; w < wid; ++w) {
    c += sh.wave_count[w];
    m += sh.wave_mass[w];
  }
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const uint64_t b0 = BY_MASS ? m : c, b1 = b0 + (BY_MASS ? ms[k] : (uint64_t)cn[k]);
    if (b0 < want && want <= b1) sh.found = Found{(uint32_t)(threadIdx.x * per + k), (uint32_t)c, cn[k], m, ms[k]};
    c += cn[k];
    m += ms[k];
  }
  __syncthreads();
  return sh.found;
}

// One block per row. P > 0: the row stays in registers as read; P = 0: it is read in every pass.
template <typename T, int NT, int P, bool SELECT>
__global__ __launch_bounds__(NT) void k_sample(const T* __restrict__ logits, int64_t ldl, int64_t V,
                                               const float* __restrict__ uniforms,
                                               const uint8_t* __restrict__ mask, float c, uint32_t top_k,
                                               uint32_t top_p24, uint32_t min_w, int64_t* __restrict__ out) {
  constexpr int E = kPiece<T>;
  constexpr bool kResident = P > 0;
  constexpr int kTurns = kResident ? P : (int)(kMaxVocab / (NT * E));
  __shared__ Shared<NT> sh;
  __shared__ uint64_t turn_mass[kTurns][NT / 64];      // kept mass of a wave's 64 pieces, in index order
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, wid = tid >> 6, lane = tid & 63;
  if (mask && mask[row] == 0) {
    if (tid == 0) out[row] = -1;
    return;
  }
  const T* l = logits + row * ldl;
  AnyVec<T, E> raw[kResident ? P : 1];
  auto load_raw = [&](int64_t at) {
    AnyVec<T, E> r;
    if (at + E <= V) {
      r = *reinterpret_cast<const AnyVec<T, E>*>(l + at);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) r[e] = at + e < V ? l[at + e] : (T)-INFINITY;
    }
    return r;
  };
  if constexpr (kResident) {
#pragma unroll
    for (int p = 0; p < P; ++p) raw[p] = load_raw((int64_t)(p * NT + tid) * E);
  }
  const int turns = kResident ? P : (int)((V + NT * E - 1) / (NT * E));
  // f(turn, index of the piece's first element, its logits with NaN as -inf)
  auto each = [&](auto&& f) {
    auto one = [&](int p, const AnyVec<T, E>& r) {
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = fmaxf((float)r[e], -INFINITY);
      f(p, (uint32_t)(p * NT + tid) * E, v);
    };
    if constexpr (kResident) {
#pragma unroll
      for (int p = 0; p < P; ++p) one(p, raw[p]);
    } else {
      for (int p = 0; p < turns; ++p) one(p, load_raw((int64_t)(p * NT + tid) * E));
    }
  };
  float m = -INFINITY;
  each([&](int, uint32_t, const float(&v)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) m = fmaxf(m, v[e]);
  });
  m = wave_max(m);
  if (lane == 0) sh.slot[wid] = m;
  __syncthreads();
  for (int w = 0; w < NT / 64; ++w) m = fmaxf(m, sh.slot[w]);
  if (m == -INFINITY) {                                // nothing to draw from
    if (tid == 0) out[row] = -1;
    return;
  }
  Bound bound;
  if constexpr (SELECT) {
    const uint32_t n_el = (uint32_t)V;
    auto clear = [&](int digits) {
      __syncthreads();
      for (int b = tid; b < digits; b += NT) {
        sh.count[b] = 0;
        sh.mass[b] = 0;
      }
      __syncthreads();
    };
    // The last kept element when `want` elements (or that mass) are to be reached, given the
    // histogram over the bins; `within` limits the candidates. Each pass splits the boundary digit
    // by the next one: the bits of the key, then of the index. A digit that is taken whole, or
    // holds one element, ends it. Returns the bound and adds up the mass kept.
    auto refine = [&](auto by_mass, Found f, const Bound& within, uint64_t want, uint64_t& kept_mass) {
      constexpr bool kByMass = decltype(by_mass)::value;
      Bound b;
      b.bin = (int)f.digit;
      uint32_t key = 0, index = 0;                     // digits found so far
      for (int level = 0; level < 8; ++level) {
        const bool whole = kByMass ? f.count == 1 : f.count_before + f.count == want;
        if (whole) break;
        clear(256);
        const int shift = 24 - 8 * (level & 3);
        each([&](int, uint32_t i0, const float(&v)[E]) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const uint32_t i = i0 + e;
            const float t = exponent_of(v[e], m, c);
            if (i >= n_el || bin_of(t) != b.bin) continue;
            const uint32_t k = order_key(v[e]);
            if (!within.keeps(b.bin, k, i)) continue;
            uint32_t dig;
            if (level < 4) {
              if (level > 0 && ((k ^ key) >> (shift + 8)) != 0) continue;
              dig = (k >> shift) & 255;
            } else {
              if (k != key || (level > 4 && ((i ^ index) >> (shift + 8)) != 0)) continue;
              dig = (i >> shift) & 255;
            }
            atomicAdd(&sh.count[dig], 1u);
            atomicAdd(&sh.mass[dig], (unsigned long long)weight_of(t));
          }
        });
        f = find_digit<NT, kByMass>(sh, 256, f.count_before, f.mass_before, want);
        if (level < 4) {
          key |= f.digit << shift;
          b.key = key | ((1u << shift) - 1);
        } else {
          index |= f.digit << shift;
          b.index = index | ((1u << shift) - 1);
        }
      }
      kept_mass = f.mass_before + f.mass;
      return b.least(within);
    };
    clear(kBins);
    each([&](int, uint32_t i0, const float(&v)[E]) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (i0 + e >= n_el) continue;
        const float t = exponent_of(v[e], m, c);
        const int b = bin_of(t);
        atomicAdd(&sh.count[b], 1u);
        atomicAdd(&sh.mass[b], (unsigned long long)weight_of(t));
      }
    });
    uint64_t mass = 0;
    Found fk{}, fp{};
    if (top_k) fk = find_digit<NT, false>(sh, kBins, 0, 0, top_k);
    if (top_k && top_p24 == 1u << 24) bound = refine(std::false_type{}, fk, bound, top_k, mass);
    if (top_p24 < 1u << 24) {
      if (top_k) {                                     // the bins' sums once more, of what top_k keeps
        bound = refine(std::false_type{}, fk, bound, top_k, mass);
        clear(kBins);
        each([&](int, uint32_t i0, const float(&v)[E]) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            if (i0 + e >= n_el) continue;
            const float t = exponent_of(v[e], m, c);
            const int b = bin_of(t);
            if (!bound.keeps(b, order_key(v[e]), i0 + e)) continue;
            atomicAdd(&sh.count[b], 1u);
            atomicAdd(&sh.mass[b], (unsigned long long)weight_of(t));
          }
        });
      } else {
        uint64_t part = 0;
        __syncthreads();
        for (int b = tid; b < kBins; b += NT) part += sh.mass[b];
        part = wave_scan(part);
        if (lane == 63) sh.wave_mass[wid] = part;
        __syncthreads();
        for (int w = 0; w < NT / 64; ++w) mass += sh.wave_mass[w];
        __syncthreads();
      }
      const uint64_t want = std::max<uint64_t>(1, share_of(mass, top_p24));
      fp = find_digit<NT, true>(sh, kBins, 0, 0, want);
      const Bound within = bound;
      bound = refine(std::true_type{}, fp, within, want, mass);
    }
  }
  // Kept mass of each wave's pieces, turn by turn; turns and waves are in index order.
  auto kept_weight = [&](float v, uint32_t i) -> uint32_t {
    const float t = exponent_of(v, m, c);
    if constexpr (SELECT) {
      if (!bound.keeps(bin_of(t), order_key(v), i)) return 0;
    }
    const uint32_t w = weight_of(t);
    return w >= min_w ? w : 0;
  };
  each([&](int p, uint32_t i0, const float(&v)[E]) {
    uint64_t s = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) s += kept_weight(v[e], i0 + e);
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor((unsigned long long)s, off);
    if (lane == 0) turn_mass[p][wid] = s;
  });
  __syncthreads();
  // Every wave finds the turn and the wave that hold the drawn element: 64 sums at a time.
  const uint64_t* flat = &turn_mass[0][0];
  const int sums = turns * (NT / 64);
  uint64_t total = 0;
  for (int b = lane; b < sums; b += 64) total += flat[b];
  for (int off = 32; off > 0; off >>= 1) total += __shfl_xor((unsigned long long)total, off);
  const float u24 = floorf(uniforms[row] * 16777216.f);
  const uint32_t r = (uint32_t)fminf(fmaxf(u24, 0.f), 16777215.f);
  const uint64_t target = share_of(total, r);          // below total
  uint64_t before = 0;
  int hit = -1;
  for (int b = 0; b < sums; b += 64) {
    const uint64_t v = b + lane < sums ? flat[b + lane] : 0;
    const uint64_t incl = before + wave_scan(v);
    const uint64_t over = __ballot(incl > target);
    if (over) {
      const int at = __builtin_ctzll(over);
      hit = b + at;
      before = __shfl((unsigned long long)(incl - v), at);
      break;
    }
    before = __shfl((unsigned long long)incl, 63);
  }
  if (hit < 0 || hit % (NT / 64) != wid) return;
  const int turn = hit / (NT / 64);
  each([&](int p, uint32_t i0, const float(&v)[E]) {
    if (p != turn) return;
    uint64_t w[E], s = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) s += w[e] = kept_weight(v[e], i0 + e);
    uint64_t run = before + wave_scan(s) - s;
    if (run <= target && target < run + s) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (run <= target && target < run + w[e]) out[row] = i0 + e;
        run += w[e];
      }
    }
  });
}

// Temperature 0: the lowest index of the largest logit.
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
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    if (temperature == 0) {
      hipLaunchKernelGGL(k_argmax<T>, dim3((unsigned)n), dim3(1024), 0, s, static_cast<const T*>(logits), ldl, V,
                         mask, out);
      EOGP_LAUNCH_CHECK("sample_tokens (argmax)");
      return EOGP_OK;
    }
    return with_row_shape(ceil_div(V, kPiece<T>), [&](auto nt, auto p) {
      constexpr int NT = decltype(nt)::value, P = decltype(p)::value;
      auto* kfn = k || p24 < 1u << 24 ? k_sample<T, NT, P, true> : k_sample<T, NT, P, false>;
      hipLaunchKernelGGL(kfn, dim3((unsigned)n), dim3(NT), 0, s, static_cast<const T*>(logits), ldl, V, uniforms,
                         mask, c, k, p24, min_w, out);
      EOGP_LAUNCH_CHECK("sample_tokens");
      return EOGP_OK;
    });
  });
}

}  // namespace eogp
