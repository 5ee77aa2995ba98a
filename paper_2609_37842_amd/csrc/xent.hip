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

// One block per row. loss = ln sum_i exp(l_i - m) - (l_label - m), m = max l;
// dl_i = g (exp(l_i - m) / sum - [i = label]) = g (2^((l_i - m) log2 e - log2 sum) - [i = label]).
// With P > 0 the row stays in registers as read (P pieces of 16 bytes per lane), so HBM sees one
// read and one write; P = 0 reads it three times, for rows longer than the registers hold.
template <typename T, int NT, int P>
__global__ __launch_bounds__(NT) void k_xent(const T* logits, int64_t ldl, const int64_t* __restrict__ labels,
                                             const uint8_t* __restrict__ mask, int64_t V, float gscale,
                                             float* __restrict__ loss, T* dlogits, int64_t ldd) {
  constexpr int E = kPiece<T>;
  __shared__ float slot[2][NT / 64];
  const int64_t row = blockIdx.x;
  const T* l = logits + row * ldl;
  T* dl = dlogits ? dlogits + row * ldd : nullptr;
  const int64_t label = labels[row];
  if ((mask && mask[row] == 0) || label < 0 || label >= V) {   // no loss; not read
    if (threadIdx.x == 0 && loss) loss[row] = 0.f;
    float zero[E] = {};
    if (dl)
      for (int64_t c = (int64_t)threadIdx.x * E; c < V; c += NT * E) store_piece<T, E>(dl, c, V, zero);
    return;
  }
  const float at_label = threadIdx.x == 0 ? (float)l[label] : 0.f;
  RegisterRow<T, NT, P> r;
  r.load(l, V);
  // A NaN among the logits shows in the sum (fmaxf passes over it).
  float m = -INFINITY;
  r.each(V, [&](int, int64_t, const float(&v)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) m = fmaxf(m, v[e]);
  });
  m = block_max<NT>(m, slot[0]);
  float s = 0.f;
  r.each(V, [&](int, int64_t, const float(&v)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f((v[e] - m) * kLog2e);
  });
  s = block_sum<NT>(s, slot[1]);
  if (threadIdx.x == 0 && loss) loss[row] = logf(s) - (at_label - m);
  if (!dl) return;
  const float log2s = log2f(s);
  r.each(V, [&](int, int64_t c, const float(&v)[E]) {
    if (c >= V) return;
    float g[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      g[e] = __builtin_amdgcn_exp2f((v[e] - m) * kLog2e - log2s);
      if (c + e == label) g[e] -= 1.f;
      g[e] *= gscale;
    }
    store_piece<T, E>(dl, c, V, g);
  });
}

}  // namespace

eogp_status softmax_xent(const void* logits, eogp_dtype t, int64_t ldl, const int64_t* labels,
                         const uint8_t* mask, int64_t n, int64_t V, float gscale, float* loss, void* dlogits,
                         int64_t ldd, hipStream_t s) {
  if (n == 0) return EOGP_OK;
  timing::Scope ts(EOGP_KT_XENT, s);
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    const int64_t pieces = ceil_div(V, kPiece<T>);
    auto go = [&](auto nt, auto p) {
      constexpr int NT = decltype(nt)::value;
      hipLaunchKernelGGL((k_xent<T, NT, decltype(p)::value>), dim3((unsigned)n), dim3(NT), 0, s,
                         static_cast<const T*>(logits), ldl, labels, mask, V, gscale, loss,
                         static_cast<T*>(dlogits), ldd);
      EOGP_LAUNCH_CHECK("softmax_xent");
      return EOGP_OK;
    };
    return with_row_shape(pieces, go);
  });
}

}  // namespace eogp
