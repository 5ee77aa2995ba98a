// Softmax cross-entropy of one label per row, with its gradient at the logits.
#include <algorithm>

#include "rows.h"
#include "timing.h"

namespace eogp {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

template <int NT>
__device__ __forceinline__ float block_max(float v, float* slot) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
  __syncthreads();
  v = slot[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = fmaxf(v, slot[w]);
  return v;
}

template <int NT>
__device__ __forceinline__ float block_sum(float v, float* slot) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
  __syncthreads();
  v = slot[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v += slot[w];
  return v;
}

constexpr int xent_per_cu(int nt, int p) { return nt == 256 ? 6 : p >= 1 && p <= 4 ? 2 : 1; }

// loss = ln sum_i exp(l_i - m) - (l_label - m), m = max l;
// dl_i = g (exp(l_i - m) / sum - [i = label]) = g (2^((l_i - m) log2 e - log2 sum) - [i = label]).
// The maximum is exact; exponentials, their sum and its logarithm are fp32, and only the gradient is rounded
// to the logits' type.
// Bound by HBM. A block takes a row at a time. With P > 0 the row stays in registers as read, so HBM sees
// one read and one write, and the next row is requested piece by piece as the gradient's pass lets go of
// this one; P = 0 reads the row three times, for rows longer than the registers hold. 4,096 bf16 places of
// 100,352, 75% of them valid, with their gradients take 311 to 315 us, 4.6 TB/s; 24 fp32 rows of 50,257 take 12 us,
// three passes over a row's registers by one CU (a row over several CUs would need a second launch, 4 us, or a wait
// between blocks). With P = 0, 2,048 fp32 rows of 100,352: 510 us, 3.2 TB/s of one reading and the writing (6.4 of all
// three), the loss alone 250. The six blocks of 16-bit rows of 1,025 to 2,048 pieces on a CU spill two registers each
// (8,192 rows of 16,384: 101 us, 5.3 TB/s).
template <typename T, int NT, int P, bool GRAD>
__global__ __launch_bounds__(NT, xent_per_cu(NT, P) * NT / 256) void k_xent(
    const T* logits, int64_t ldl, const int64_t* __restrict__ labels, const uint8_t* __restrict__ mask, int64_t n,
    int64_t V, float gscale, float* __restrict__ loss, T* dlogits, int64_t ldd) {
  constexpr int E = kPiece<T>;
  __shared__ float slot[2][NT / 64];
  RowWalk walk;
  auto live = [&](int64_t row) {                       // rows without a loss are not read
    if ((!mask || mask[row] != 0) && labels[row] >= 0 && labels[row] < V) return true;
    if (threadIdx.x == 0 && loss) loss[row] = 0.f;
    float zero[E] = {};
    if (GRAD)
      for (int64_t c = (int64_t)threadIdx.x * E; c < V; c += NT * E)
        store_piece<T, E>(dlogits + row * ldd, c, V, zero);
    return false;
  };
  RegisterRow<T, NT, P> r;
  int64_t row = walk.next(n, live);
  if (row < 0) return;
  r.load(logits + row * ldl, V);
  for (;;) {
    const uint32_t label = (uint32_t)labels[row];
    const float at_label = threadIdx.x == 0 ? (float)logits[row * ldl + label] : 0.f;
    // A NaN among the logits shows in the sum (fmaxf passes over it).
    float m = -INFINITY;
    r.each(V, [&](int, uint32_t, uint32_t, const float(&v)[E]) {
#pragma unroll
      for (int e = 0; e < E; ++e) m = fmaxf(m, v[e]);
    });
    m = block_max<NT>(m, slot[0]);
    float s = 0.f;
    r.each(V, [&](int, uint32_t, uint32_t, const float(&v)[E]) {
#pragma unroll
      for (int e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f((v[e] - m) * kLog2e);
    });
    // Over the logits in place, other waves write this element after the barrier: it has to be here by then.
    asm volatile("" ::"v"(at_label));
    s = block_sum<NT>(s, slot[1]);
    if (threadIdx.x == 0 && loss) loss[row] = logf(s) - (at_label - m);
    const int64_t after = walk.next(n, live);
    T* dl = dlogits + row * ldd;
    const float log2s = log2f(s);
    auto gradient = [&](int, uint32_t c, uint32_t first, const float(&v)[E]) {
      if constexpr (GRAD) {
        AnyVec<T, E> g;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float p = __builtin_amdgcn_exp2f((v[e] - m) * kLog2e - log2s);
          g[e] = (T)((c + e == label ? p - 1.f : p) * gscale);
        }
        if (P > 0 ? c == first : c + E <= V) {
          __builtin_nontemporal_store(g, reinterpret_cast<AnyVec<T, E>*>(dl + c));
        } else {                                       // other pieces hold what lies before `first`
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (c + e >= first && c + e < V) dl[c + e] = g[e];
        }
      }
    };
    if (after < 0) {
      r.each(V, gradient);
      return;
    }
    r.each_then_load(V, gradient, logits + after * ldl);
    row = after;
  }
}

}  // namespace

eogp_status softmax_xent(const void* logits, eogp_dtype t, int64_t ldl, const int64_t* labels,
                         const uint8_t* mask, int64_t n, int64_t V, float gscale, float* loss, void* dlogits,
                         int64_t ldd, hipStream_t s) {
  if (n == 0) return EOGP_OK;
  timing::Scope ts(EOGP_KT_XENT, s);
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    auto go = [&](auto nt, auto p) {
      constexpr int NT = decltype(nt)::value;
      constexpr int P = decltype(p)::value;
      const int64_t blocks = row_blocks(n, NT, xent_per_cu(NT, P));
      auto* kfn = dlogits ? k_xent<T, NT, P, true> : k_xent<T, NT, P, false>;
      hipLaunchKernelGGL(kfn, dim3((unsigned)blocks), dim3(NT), 0, s, static_cast<const T*>(logits), ldl, labels, mask,
                         n, V, gscale, loss, static_cast<T*>(dlogits), ldd);
      EOGP_LAUNCH_CHECK("softmax_xent");
      return EOGP_OK;
    };
    return with_row_shape<T>(V, go);
  });
}

}  // namespace eogp
