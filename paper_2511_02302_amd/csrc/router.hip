// The router in front of the experts: top-k experts and their routing weights from the logits of
// T tokens, and the gradient of the logits, for gfx950.
//
// Mathematics.  A token's score of expert i is softmax(l)_i or sigmoid(l_i).  The k experts are
// those of the largest key, the key being the logit itself (both scores grow with it) or, with a
// balancing bias, score + bias; ties go to the lower index.  A weight is c * score, or normalized
// over the chosen, c * score_j / sum(chosen scores).  The latter is computed as a softmax over the
// chosen of v_j = l_j (softmax scores: the sum over all experts cancels) or of v_j = log sigmoid(l_j),
// so that scores too small for float32 give weights and not 0 / 0.  Gradients, with dp of the weights:
//   softmax             dl_i = c s_i (dp_i [i chosen] - sum_j s_j dp_j)
//   sigmoid             dl_j = c s_j (1 - s_j) dp_j
//   normalized, r_j     dl_j = c g_j r_j (dp_j - sum_m r_m dp_m),  g = 1 or sigmoid(-l_j)
// and zero for experts that are not chosen in the last two.

#include <math.h>

#include "ff8_device.hpp"
#include "ff8_launch.hpp"

namespace ff8 {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load_logit(const float* p) { return *p; }
__device__ __forceinline__ float load_logit(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store_logit(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_logit(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16(v); }

__device__ __forceinline__ double max_key(double a, double b) { return a > b ? a : b; }
__device__ __forceinline__ float max_key(float a, float b) { return a > b ? a : b; }

// Over the aligned group of L lanes (every lane gets the result).
template <int L, typename V>
__device__ __forceinline__ V group_max(V v) {
#pragma unroll
  for (int d = 1; d < L; d <<= 1) v = max_key(v, __shfl_xor(v, d));
  return v;
}
template <int L>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int d = 1; d < L; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }
__device__ __forceinline__ float log_sigmoid(float x) { return fminf(x, 0.0f) - log1pf(expf(-fabsf(x))); }

// L lanes a token, V consecutive experts a lane (L * V >= E), so that among lanes of equal keys the
// lowest has the lowest expert.  K is the key's type: the logit as it is in float32; score + bias in
// float64, as a rounding of the sum would decide between experts.
template <int L, int V, bool kSigmoid, bool kNormalize, typename K, typename X>
__global__ __launch_bounds__(kThreads) void topk_kernel(const X* __restrict__ logits, const float* __restrict__ bias,
                                                        int64_t T, int E, int k, float scale,
                                                        int32_t* __restrict__ topk_idx, float* __restrict__ probs) {
  constexpr bool kBias = sizeof(K) == 8;
  constexpr int kSlots = L == 64 ? 1 : (64 + L - 1) / L;  // slots a lane holds: k <= 64
  const int lane = threadIdx.x & (L - 1);
  const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  if (t >= T) return;  // whole groups of L lanes
  float l[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = lane * V + v;
    l[v] = i < E ? load_logit(logits + t * E + i) : -INFINITY;
  }
  float m = -INFINITY, sum = 0.0f;
  const bool full = !kSigmoid && (kBias || !kNormalize);  // the softmax over all experts is needed
  if (full) {
#pragma unroll
    for (int v = 0; v < V; ++v) m = fmaxf(m, l[v]);
    m = group_max<L>(m);
    if (m == -INFINITY) m = 0.0f;  // no expert can be chosen
  }
  K key[V];
  if (kBias) {
    double z = 1.0;
    if (!kSigmoid) {
      z = 0.0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        key[v] = exp((double)l[v] - (double)m);
        z += key[v];
      }
#pragma unroll
      for (int d = 1; d < L; d <<= 1) z += __shfl_xor(z, d);
      sum = (float)z;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = lane * V + v;
      const double s = kSigmoid ? 1.0 / (1.0 + exp(-(double)l[v])) : key[v] / z;
      key[v] = (i < E && l[v] > -INFINITY) ? s + (double)bias[i] : -INFINITY;
    }
  } else {
    if (full) {
#pragma unroll
      for (int v = 0; v < V; ++v) sum += expf(l[v] - m);
      sum = group_sum<L>(sum);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = l[v];
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (!(key[v] > -INFINITY)) key[v] = -INFINITY;  // NaN is never chosen
  // k rounds: the largest key of the group, the lowest lane that has it, its lowest expert
  int my_idx[kSlots];
  float my_l[kSlots];
#pragma unroll
  for (int q = 0; q < kSlots; ++q) {
    my_idx[q] = -1;
    my_l[q] = -INFINITY;
  }
  for (int j = 0; j < k; ++j) {
    K best = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = max_key(best, key[v]);
    const K top = group_max<L>(best);
    const unsigned long long who = __ballot(best == top) >> (threadIdx.x & 63 & ~(L - 1));
    const int win = __ffsll(who) - 1;  // the group's own bits come first
    int vi = 0;
    float vl = 0.0f;
#pragma unroll
    for (int v = V - 1; v >= 0; --v)
      if (key[v] == top) {
        vi = v;
        vl = l[v];
      }
    const bool some = top > -INFINITY;
    if (some && lane == win) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (v == vi) key[v] = -INFINITY;
    }
    const int at = (threadIdx.x & 63 & ~(L - 1)) + win;
    const int ji = some ? win * V + __shfl(vi, at) : -1;
    const float jl = some ? __shfl(vl, at) : -INFINITY;
#pragma unroll
    for (int q = 0; q < kSlots; ++q)
      if (j == q * L + lane) {
        my_idx[q] = ji;
        my_l[q] = jl;
      }
  }
  float vmax = -INFINITY, total = 0.0f;
  float w[kSlots];
#pragma unroll
  for (int q = 0; q < kSlots; ++q) {
    const int j = q * L + lane;
    const bool have = j < k && my_idx[q] >= 0;
    if (kNormalize) {
      w[q] = have ? (kSigmoid ? log_sigmoid(my_l[q]) : my_l[q]) : -INFINITY;
      vmax = fmaxf(vmax, w[q]);
    } else {
      w[q] = have ? (kSigmoid ? sigmoid(my_l[q]) : expf(my_l[q] - m) / sum) : 0.0f;
    }
  }
  if (kNormalize) {
    vmax = group_max<L>(vmax);
#pragma unroll
    for (int q = 0; q < kSlots; ++q) {
      w[q] = w[q] > -INFINITY ? expf(w[q] - vmax) : 0.0f;
      total += w[q];
    }
    total = group_sum<L>(total);
  }
#pragma unroll
  for (int q = 0; q < kSlots; ++q) {
    const int j = q * L + lane;
    if (j < k) {
      topk_idx[t * k + j] = my_idx[q];
      probs[t * k + j] = my_idx[q] < 0 ? 0.0f : scale * (kNormalize ? w[q] / total : w[q]);
    }
  }
}

template <int L, int V, bool kSigmoid, bool kNormalize, typename X>
__global__ __launch_bounds__(kThreads) void topk_bwd_kernel(const X* __restrict__ logits,
                                                            const int32_t* __restrict__ topk_idx,
                                                            const float* __restrict__ dprobs, int64_t T, int E, int k,
                                                            float scale, X* __restrict__ dlogits) {
  constexpr int kSlots = L == 64 ? 1 : (64 + L - 1) / L;
  const int lane = threadIdx.x & (L - 1);
  const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  if (t >= T) return;
  const X* row = logits + t * E;
  // the chosen: index, logit and weight's gradient, slot q * L + lane
  int idx[kSlots];
  float cl[kSlots], g[kSlots];
#pragma unroll
  for (int q = 0; q < kSlots; ++q) {
    const int j = q * L + lane;
    idx[q] = j < k ? topk_idx[t * k + j] : -1;
    if (idx[q] >= E) idx[q] = -1;
    cl[q] = idx[q] >= 0 ? load_logit(row + idx[q]) : -INFINITY;
    g[q] = idx[q] >= 0 ? dprobs[t * k + j] : 0.0f;
  }
  const bool dense = !kSigmoid && !kNormalize;
  float l[V], m = -INFINITY, sum = 0.0f, dot = 0.0f;
  if (dense) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = lane * V + v;
      l[v] = i < E ? load_logit(row + i) : -INFINITY;
      m = fmaxf(m, l[v]);
    }
    m = group_max<L>(m);
    if (m == -INFINITY) m = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      l[v] = expf(l[v] - m);
      sum += l[v];
    }
    sum = group_sum<L>(sum);
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] *= inv;
#pragma unroll
    for (int q = 0; q < kSlots; ++q)
      if (idx[q] >= 0) dot += expf(cl[q] - m) * inv * g[q];
    dot = group_sum<L>(dot);
  } else if (kNormalize) {
    float vmax = -INFINITY, total = 0.0f, r[kSlots];
#pragma unroll
    for (int q = 0; q < kSlots; ++q) {
      r[q] = idx[q] >= 0 ? (kSigmoid ? log_sigmoid(cl[q]) : cl[q]) : -INFINITY;
      vmax = fmaxf(vmax, r[q]);
    }
    vmax = group_max<L>(vmax);
#pragma unroll
    for (int q = 0; q < kSlots; ++q) {
      r[q] = r[q] > -INFINITY ? expf(r[q] - vmax) : 0.0f;
      total += r[q];
    }
    total = group_sum<L>(total);
#pragma unroll
    for (int q = 0; q < kSlots; ++q) {
      r[q] = total > 0.0f || total != total ? r[q] / total : 0.0f;
      dot += r[q] * g[q];
    }
    dot = group_sum<L>(dot);
#pragma unroll
    for (int q = 0; q < kSlots; ++q) g[q] = scale * r[q] * (g[q] - dot) * (kSigmoid ? sigmoid(-cl[q]) : 1.0f);
  } else {
#pragma unroll
    for (int q = 0; q < kSlots; ++q) {
      g[q] = idx[q] >= 0 ? scale * g[q] * sigmoid(cl[q]) * sigmoid(-cl[q]) : 0.0f;
    }
  }
  float d[V];
#pragma unroll
  for (int v = 0; v < V; ++v) d[v] = 0.0f;
  const int base = threadIdx.x & 63 & ~(L - 1);
#pragma unroll
  for (int q = 0; q < kSlots; ++q) {
    const int n = k - q * L < L ? k - q * L : L;
    for (int j = 0; j < n; ++j) {
      const int at = __shfl(idx[q], base + j) - lane * V;  // of an index of -1 below zero for every lane
      const float gj = __shfl(g[q], base + j);
#pragma unroll
      for (int v = 0; v < V; ++v) d[v] += at == v ? gj : 0.0f;
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = lane * V + v;
    if (i < E) store_logit(dlogits + t * E + i, dense ? scale * l[v] * (d[v] - dot) : d[v]);
  }
}

template <int L, int V, typename X>
hipError_t topk_launch(const X* logits, const float* bias, int64_t T, int E, int k, bool sig, bool norm, float scale,
                       int32_t* idx, float* probs, hipStream_t st) {
  const unsigned grid = (unsigned)((T + kThreads / L - 1) / (kThreads / L));
#define FF8_GO(S, N)                                                                                             \
  if (bias)                                                                                                      \
    topk_kernel<L, V, S, N, double, X><<<grid, kThreads, 0, st>>>(logits, bias, T, E, k, scale, idx, probs);     \
  else                                                                                                           \
    topk_kernel<L, V, S, N, float, X><<<grid, kThreads, 0, st>>>(logits, bias, T, E, k, scale, idx, probs);
  if (sig && norm) {
    FF8_GO(true, true)
  } else if (sig) {
    FF8_GO(true, false)
  } else if (norm) {
    FF8_GO(false, true)
  } else {
    FF8_GO(false, false)
  }
#undef FF8_GO
  return hipGetLastError();
}

template <int L, int V, typename X>
hipError_t topk_bwd_launch(const X* logits, const int32_t* idx, const float* dprobs, int64_t T, int E, int k, bool sig,
                           bool norm, float scale, X* dlogits, hipStream_t st) {
  const unsigned grid = (unsigned)((T + kThreads / L - 1) / (kThreads / L));
#define FF8_GO(S, N) \
  topk_bwd_kernel<L, V, S, N, X><<<grid, kThreads, 0, st>>>(logits, idx, dprobs, T, E, k, scale, dlogits)
  if (sig && norm)
    FF8_GO(true, true);
  else if (sig)
    FF8_GO(true, false);
  else if (norm)
    FF8_GO(false, true);
  else
    FF8_GO(false, false);
#undef FF8_GO
  return hipGetLastError();
}

// Lanes and experts a lane by E: 16 lanes (four tokens a wave) up to 256 experts, the whole wave above.
#define FF8_BY_E(E, CALL)                  \
  if ((E) <= 16) return CALL(16, 1);       \
  if ((E) <= 32) return CALL(16, 2);       \
  if ((E) <= 64) return CALL(16, 4);       \
  if ((E) <= 128) return CALL(16, 8);      \
  if ((E) <= 256) return CALL(16, 16);     \
  if ((E) <= 512) return CALL(64, 8);      \
  return CALL(64, 16);

template <typename X>
hipError_t topk_impl(const X* logits, const float* bias, int64_t T, int E, int k, bool sig, bool norm, float scale,
                     int32_t* idx, float* probs, hipStream_t st) {
  if (T == 0) return hipSuccess;
#define FF8_CALL(L, V) topk_launch<L, V, X>(logits, bias, T, E, k, sig, norm, scale, idx, probs, st)
  FF8_BY_E(E, FF8_CALL)
#undef FF8_CALL
}

template <typename X>
hipError_t topk_bwd_impl(const X* logits, const int32_t* idx, const float* dprobs, int64_t T, int E, int k, bool sig,
                         bool norm, float scale, X* dlogits, hipStream_t st) {
  if (T == 0) return hipSuccess;
#define FF8_CALL(L, V) topk_bwd_launch<L, V, X>(logits, idx, dprobs, T, E, k, sig, norm, scale, dlogits, st)
  FF8_BY_E(E, FF8_CALL)
#undef FF8_CALL
}

}  // namespace

hipError_t launch_router_topk(const float* logits, const float* bias, int64_t T, int E, int k, bool sig, bool norm,
                              float scale, int32_t* idx, float* probs, hipStream_t st) {
  return topk_impl(logits, bias, T, E, k, sig, norm, scale, idx, probs, st);
}
hipError_t launch_router_topk(const uint16_t* logits, const float* bias, int64_t T, int E, int k, bool sig, bool norm,
                              float scale, int32_t* idx, float* probs, hipStream_t st) {
  return topk_impl(logits, bias, T, E, k, sig, norm, scale, idx, probs, st);
}
hipError_t launch_router_topk_bwd(const float* logits, const int32_t* idx, const float* dprobs, int64_t T, int E, int k,
                                  bool sig, bool norm, float scale, float* dlogits, hipStream_t st) {
  return topk_bwd_impl(logits, idx, dprobs, T, E, k, sig, norm, scale, dlogits, st);
}
hipError_t launch_router_topk_bwd(const uint16_t* logits, const int32_t* idx, const float* dprobs, int64_t T, int E,
                                  int k, bool sig, bool norm, float scale, uint16_t* dlogits, hipStream_t st) {
  return topk_bwd_impl(logits, idx, dprobs, T, E, k, sig, norm, scale, dlogits, st);
}

}  // namespace ff8
