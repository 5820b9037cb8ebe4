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
//
// What bounds it.  The floor is one read of the logits (8.4 MB at 16384 tokens x 256 experts: 1.4 us, of which
// the choice with a bias is measured at 7.5 and the gradient, 17.8 MB and 2.7 us, at 6.2: a launch alone is about 2
// and the rest is instructions: 709 and 435 vector instructions a wave, of which a SIMD has four waves, are 4.7 and 2.9 us
// at 4 cycles each).  So those are kept few: a token is held by 16 lanes (or by a wave, for few tokens or many
// experts), its experts in registers, reductions run on DPP and lane swaps instead of LDS, bf16 logits carry
// their expert's number in the low half of one word for the k rounds of the maximum, and where they cannot, the
// candidates for the k places are found and ranked by counting.

#include <math.h>

#include "ff8_device.hpp"
#include "ff8_launch.hpp"

namespace ff8 {

namespace {

constexpr int kThreads = 256;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---- reductions over the aligned group of L = 16 or 64 lanes (every lane gets the result) ----

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, 0xF, 0xF, false);
}
// f over xor 1, xor 2, half-row mirror and row mirror; then the rows' values by lane swaps.
template <int L, typename F>
__device__ __forceinline__ uint32_t group_reduce(uint32_t v, F f) {
  static_assert(L == 16 || L == 64, "a row of 16 lanes or the wave");
  v = f(v, dpp<0xB1>(v));
  v = f(v, dpp<0x4E>(v));
  v = f(v, dpp<0x141>(v));
  v = f(v, dpp<0x140>(v));
  if (L == 64) {
    auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = f(r[0], r[1]);
    r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = f(r[0], r[1]);
  }
  return v;
}
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  return group_reduce<L>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int L>
__device__ __forceinline__ float group_max(float v) {
  return __uint_as_float(group_reduce<L>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}
template <int L>
__device__ __forceinline__ float group_sum(float v) {
  return __uint_as_float(group_reduce<L>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}

// ---- a row's logits: V consecutive experts a lane ----

template <int kBytes>
struct Piece;
template <>
struct Piece<2> { typedef uint16_t type; };
template <>
struct Piece<4> { typedef uint32_t type; };
template <>
struct Piece<8> { typedef u32x2 type; };
template <>
struct Piece<16> { typedef u32x4 type; };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void from_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void from_f32(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16(v); }

// How a row's experts are moved: one by one, in a lane's pieces, or through LDS.
enum class Rows { kSingle, kPieces, kStaged };

// vec: E is a multiple of V and the tensor is aligned to a lane's piece (at most 16 bytes), so a lane's experts
// are all there or all missing.
template <int V, typename X>
__device__ __forceinline__ void load_row(const X* row, int lane, int E, bool vec, X missing, X (&x)[V]) {
  constexpr int kBytes = V * sizeof(X) < 16 ? V * sizeof(X) : 16, kPer = kBytes / sizeof(X);
  typedef typename Piece<kBytes>::type P;
#pragma unroll
  for (int v = 0; v < V; ++v) x[v] = missing;
  if (vec) {
    if (lane * V < E) {
#pragma unroll
      for (int v = 0; v < V; v += kPer) {
        const P p = *reinterpret_cast<const P*>(row + lane * V + v);
        __builtin_memcpy(&x[v], &p, kBytes);
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (lane * V + v < E) x[v] = row[lane * V + v];
  }
}
template <int V, typename X>
__device__ __forceinline__ void store_row(X* row, int lane, int E, bool vec, const float (&d)[V]) {
  constexpr int kBytes = V * sizeof(X) < 16 ? V * sizeof(X) : 16, kPer = kBytes / sizeof(X);
  typedef typename Piece<kBytes>::type P;
  X x[V];
#pragma unroll
  for (int v = 0; v < V; ++v) from_f32(&x[v], d[v]);
  if (vec) {
    if (lane * V < E) {
#pragma unroll
      for (int v = 0; v < V; v += kPer) {
        P p;
        __builtin_memcpy(&p, &x[v], kBytes);
        *reinterpret_cast<P*>(row + lane * V + v) = p;
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (lane * V + v < E) row[lane * V + v] = x[v];
  }
}

// Rows that are not aligned to a lane's piece (E no multiple of it) go through LDS: the 16 rows of a workgroup are
// one run of memory that begins at a multiple of 16 bytes, so they are moved in whole pieces, and a lane takes its
// experts from LDS.  One by one, an access meets 16 lines and more for 64 elements.
constexpr int kStagedRows = kThreads / 16;
template <int L, int V>
constexpr bool kCanStage = L == 16 && V >= 8;
extern __shared__ u32x4 stage[];  // where rows are staged: kThreads * V elements, and 16 * V of the bias

// The workgroup's elements, from global memory to LDS or back.
template <typename X>
__device__ __forceinline__ void move_staged(const X* from, X* to, int n) {
  constexpr int kPer = 16 / sizeof(X);
  for (int i = (int)threadIdx.x * kPer; i + kPer <= n; i += kThreads * kPer)
    *reinterpret_cast<u32x4*>(to + i) = *reinterpret_cast<const u32x4*>(from + i);
  const int i = n / kPer * kPer + (int)threadIdx.x;
  if (i < n) to[i] = from[i];
}
__device__ __forceinline__ int staged_elements(int64_t T, int E) {
  const int64_t left = T - (int64_t)blockIdx.x * kStagedRows;
  return (int)(left < kStagedRows ? left : kStagedRows) * E;
}

// Experts a lane holds, from per * lane on: V in pieces, otherwise as many as spread them over all 16 lanes.  Where the
// experts are chosen by ranks they are spread, and so staged, up to 10 V too: with few lanes the lanes' largest keys
// are a poor bound for the candidates.  By E alone, so that results do not depend on the address.
// 16384 tokens with a bias, k = 8, us, staged / in pieces: 144 experts 8.5 / 12.0, 160 8.7 / 10.5, 192 9.0 / 9.0, 256 7.9 /
// 7.5; over packed keys 160 8.6 / 8.0, the gradient 6.4 / 5.0.  And staged and spread / one by one: 129 8.5 / 21.8, 255 9.3 /
// 18.6, the gradient 7.6 / 20.2; 49 experts (V = 4) 7.0 / 7.3 and 4.5 / 4.5.
template <int L, int V>
__host__ __device__ __forceinline__ int experts_per_lane(int E, bool ranked) {
  return kCanStage<L, V> && (E % V != 0 || (ranked && E <= 10 * V)) ? (E + 15) / 16 : V;
}
template <int V, typename X>
__device__ __forceinline__ void load_experts(const X* row, int lane, int per, int E, X missing, X (&x)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) x[v] = v < per && lane * per + v < E ? row[lane * per + v] : missing;
}
template <int V, typename X>
__device__ __forceinline__ void store_experts(X* row, int lane, int per, int E, const float (&d)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (v < per && lane * per + v < E) from_f32(&row[lane * per + v], d[v]);
}

// ---- scores ----

// e^d for d <= 0 to about one unit in the last place: the hardware 2^x of the product's head, times
// 1 + ln 2 * (the product's rounding and log2(e)'s own).  Below e^-200, 0; NaN stays.
__device__ __forceinline__ float exp_neg(float d) {
  constexpr float kLog2e = 1.44269504f, kLog2eLow = 1.92596303e-8f, kLn2 = 0.693147181f;
  d = d < -200.0f ? -200.0f : d;
  const float hi = d * kLog2e;
  const float lo = fmaf(d, kLog2e, -hi) + d * kLog2eLow;
  const float e = __builtin_amdgcn_exp2f(hi);
  return fmaf(e, lo * kLn2, e);
}
__device__ __forceinline__ float sigmoid(float x) {
  const float e = exp_neg(-fabsf(x));
  return (x < 0.0f ? e : 1.0f) / (1.0f + e);
}
__device__ __forceinline__ float log_sigmoid(float x) { return fminf(x, 0.0f) - log1pf(exp_neg(-fabsf(x))); }

// Ordered key of a bf16 logit with its expert's number: larger for larger logits, and for lower experts among
// equal ones; 0 for a logit that is never chosen (-inf, NaN).
__device__ __forceinline__ uint32_t packed_key(uint16_t b, int i) {
  const uint32_t u = b == 0x8000 ? 0u : b;
  const uint32_t ord = u & 0x8000 ? ~u & 0xFFFFu : u | 0x8000u;
  const bool never = (u & 0x7FFFu) > 0x7F80u || u == 0xFF80u;
  return never ? 0u : ord << 16 | (0xFFFFu - (uint32_t)i);
}
__device__ __forceinline__ float packed_logit(uint32_t key) {
  const uint32_t ord = key >> 16;
  return __uint_as_float((ord & 0x8000u ? ord ^ 0x8000u : ~ord & 0xFFFFu) << 16);
}

// What a round has found, by slot of a group.
struct Choice {
  int idx;
  float logit, key, bias;
};
template <int kSlots>
struct Choices {
  int idx[kSlots];
  float logit[kSlots], key[kSlots], bias[kSlots];
  __device__ __forceinline__ void put(int i, const Choice& c) {
    idx[i] = c.idx;
    logit[i] = c.logit;
    key[i] = c.key;
    bias[i] = c.bias;
  }
  __device__ __forceinline__ Choice get(int i) const { return {idx[i], logit[i], key[i], bias[i]}; }
};
// Whether the float32 keys of two experts tell their order: they are further apart than both may be off, or come
// from equal logits and biases.
__device__ __forceinline__ bool certain(const Choice& a, const Choice& b, float err) {
  return (a.key - b.key > err + 0x1p-21f * fabsf(a.key)) | ((a.logit == b.logit) & (a.bias == b.bias));
}

// k rounds over keys of type K (-inf: never chosen): the largest of the group, the lowest lane that has it, its
// lowest expert.  Slot j of `out` is written by the lane that held it; chosen keys become -inf.
template <int L, int V, typename K, typename Out>
__device__ __forceinline__ void choose_rounds(K (&key)[V], const float (&l)[V], int per, int k, Out& out) {
  const int lane = threadIdx.x & (L - 1), base = threadIdx.x & 63 & ~(L - 1);
  for (int j = 0; j < k; ++j) {
    K best = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = key[v] > best ? key[v] : best;
    K top = best;
    if constexpr (sizeof(K) == 4) {
      top = group_max<L>(best);
    } else {
#pragma unroll
      for (int d = 1; d < L; d <<= 1) {
        const K o = __shfl_xor(top, d);
        top = o > top ? o : top;
      }
    }
    const int win = __ffsll(__ballot(best == top) >> base) - 1;  // the group's own bits come first
    bool mine = lane == win;
    int at = -1;
    float logit = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const bool hit = mine && key[v] == top;
      at = hit ? v : at;
      logit = hit ? l[v] : logit;
      key[v] = hit ? (K)-INFINITY : key[v];
      mine = mine && !hit;
    }
    if (lane == win) out.put(j, {top > -INFINITY ? lane * per + at : -1, logit, (float)top, 0.0f});
  }
}

// The same by ranks, for 16 lanes (k <= 16), where that takes a fraction of the rounds' instructions (16384 x 256 biased
// 7.5 us; over packed keys, whose rounds are short, ranks were no faster: 8.2 us against 7.9): the k-th of the
// lanes' largest keys bounds the k-th of all from below; the keys from there on (11 of 256 for k = 8, on average) go
// to the lanes in expert order, one each (two where a group of the wave has more than 16), and each lane counts the
// better ones.  With a bias the candidates begin as far below that as float32 may be off, and where the order
// of two of them is not certain they are ranked again in float64: a few tokens in a thousand, and only these
// experts (all 256 in float64 made such waves, and with them the launch, 8 us longer).
// False, with nothing chosen, where there are more than 32.  Leaves the keys as they are.
template <int N>
__device__ __forceinline__ float from_left(float v) {  // of the lane N to the left, around the row
  return __uint_as_float(dpp<0x120 + N>(__float_as_uint(v)));
}
template <int N>
__device__ __forceinline__ double from_left(double v) {
  const u32x2 u = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(double, u32x2{dpp<0x120 + N>(u[0]), dpp<0x120 + N>(u[1])});
}
template <int N>
__device__ __forceinline__ int count_larger(float v, int n) {
  if constexpr (N < 16) return count_larger<N + 1>(v, n + (from_left<N>(v) > v));
  return n;
}
// Of the row's values `o`, how many come before this lane's v: larger, or equal and in a lane below `lane`
// (kSelf: the lane's own `o` is another value, and counts as one in a lane below).
template <int N, bool kSelf, typename K>
__device__ __forceinline__ int count_before(K o, K v, int lane, int n) {
  if constexpr (N < 16) {
    const K f = N == 0 ? o : from_left<N == 0 ? 1 : N>(o);
    if (N > 0 || kSelf) n += (f > v) | ((f == v) & (lane >= N));
    return count_before<N + 1, kSelf>(o, v, lane, n);
  }
  return n;
}
// Ranks of the lanes' first keys c and, with `two`, second keys d, in the order of the list c0 .. c15 d0 .. d15.
template <typename K>
__device__ __forceinline__ void ranks(K c, K d, bool two, int lane, int& rank_c, int& rank_d) {
  rank_c = count_before<0, false>(c, c, lane, 0);
  if (two) {
    rank_c += count_before<0, true>(d, c, -1, 0);
    rank_d = count_before<0, false>(d, d, lane, 0) + count_before<0, true>(c, d, 16, 0);
  }
}
__device__ __forceinline__ int row_inclusive_sum(int v) {
  v += (int)dpp<0x111>((uint32_t)v);
  v += (int)dpp<0x112>((uint32_t)v);
  v += (int)dpp<0x114>((uint32_t)v);
  v += (int)dpp<0x118>((uint32_t)v);
  return v;
}
// Score + bias in float64: sigmoid, or for softmax exp(l - m) / z with z the row's sum.
template <bool kSigmoid>
__device__ __forceinline__ double key64(float l, float b, float m, double z) {
  const double s = kSigmoid ? 1.0 / (1.0 + exp(-(double)l)) : exp((double)l - (double)m) / z;
  const double k = s + (double)b;
  return ((l > -INFINITY) & (k > -INFINITY)) ? k : -INFINITY;
}
template <int L, int V, bool kSigmoid>
__device__ __forceinline__ double row_sum64(const float (&l)[V], float m) {
  double z = 0.0;
  if (!kSigmoid) {
#pragma unroll
    for (int v = 0; v < V; ++v) z += exp((double)l[v] - (double)m);
#pragma unroll
    for (int d = 1; d < L; d <<= 1) z += __shfl_xor(z, d);
  }
  return z;
}
template <int V, bool kSigmoid, bool kBias, typename Out>
__device__ __forceinline__ bool choose_ranked(const float (&key)[V], const float (&l)[V], const float* b, int per,
                                              int k, float err, float m, Out& out) {
  const int lane = threadIdx.x & 15;
  float best = key[0];
#pragma unroll
  for (int v = 1; v < V; ++v) best = fmaxf(best, key[v]);
  float bound = -group_max<16>(count_larger<1>(best, 0) < k ? -best : -INFINITY);
  if (kBias) bound -= err + 0x1p-21f * fabsf(bound);
  bound = fmaxf(bound, -3.402823466e38f);  // the lowest finite number: a key of -inf is no candidate
  int n = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) n += key[v] >= bound;
  const int end = row_inclusive_sum(n), total = (int)dpp<0x15F>((uint32_t)end);
  if (__any(total > 32)) return false;
  const bool two = __any(total > 16);
  int at = end - n;
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (key[v] >= bound) out.put(at++, {lane * per + v, l[v], key[v], kBias ? b[v] : 0.0f});
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  Choice c = {-1, -INFINITY, -INFINITY, 0.0f}, d = c;
  if (lane < total) c = out.get(lane);
  if (two && lane + 16 < total) d = out.get(lane + 16);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  int rank_c, rank_d = 32;
  ranks(c.key, d.key, two, lane, rank_c, rank_d);
  out.put(rank_c, c);  // (missing ones behind)
  if (two) out.put(rank_d, d);
  if (kBias) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // every two neighbours down to where the keys are clearly below the k-th
    const float last = total >= k ? out.key[k - 1] : -INFINITY, near = last - (err + 0x1p-21f * fabsf(last));
    bool unsure = false;
    for (int r = lane; r + 1 < total; r += 16) {
      const Choice x = out.get(r);
      unsure |= !(x.key < near) & !certain(x, out.get(r + 1), err);
    }
    if (__any(unsure)) {
      const double z = row_sum64<16, V, kSigmoid>(l, m);
      ranks(key64<kSigmoid>(c.logit, c.bias, m, z), key64<kSigmoid>(d.logit, d.bias, m, z), two, lane, rank_c, rank_d);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      out.put(rank_c, c);
      if (two) out.put(rank_d, d);
    }
  }
  return true;
}

template <int L, int V, bool kSigmoid, bool kNormalize, bool kBias, typename X>
__global__ __launch_bounds__(kThreads) void topk_kernel(const X* __restrict__ logits, const float* __restrict__ bias,
                                                        int64_t T, int E, int k, float scale, Rows rows,
                                                        bool vec_bias, int32_t* __restrict__ topk_idx, float* __restrict__ probs) {
  constexpr bool kPacked = sizeof(X) == 2 && !kBias;
  constexpr bool kFull = !kSigmoid && (kBias || !kNormalize);  // the softmax over all experts is needed
  constexpr int kFound = L == 16 ? 32 : 64;  // slots a group: k, or the candidates for them
  __shared__ Choices<kFound> found[kPacked ? 1 : kThreads / L];
  const int lane = threadIdx.x & (L - 1);
  Choices<kFound>& mine = found[kPacked ? 0 : threadIdx.x / L];
  const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  X raw[V], missing;
  from_f32(&missing, -INFINITY);
  const bool staged = kCanStage<L, V> && rows == Rows::kStaged;
  const int per = experts_per_lane<L, V>(E, !kPacked);
  float* const bias_stage = reinterpret_cast<float*>(reinterpret_cast<X*>(stage) + kThreads * V);
  if (staged) {
    X* const in = reinterpret_cast<X*>(stage);
    move_staged(logits + (int64_t)blockIdx.x * kStagedRows * E, in, staged_elements(T, E));
    if (kBias && (int)threadIdx.x < E) bias_stage[threadIdx.x] = bias[threadIdx.x];
    __syncthreads();
    load_experts<V>(in + threadIdx.x / L * E, lane, per, E, missing, raw);
  }
  if (t >= T) return;  // whole groups of L lanes
  if (!staged) {
    if (kCanStage<L, V> && rows == Rows::kSingle)
      load_experts<V>(logits + t * E, lane, per, E, missing, raw);
    else
      load_row<V>(logits + t * E, lane, E, rows == Rows::kPieces, missing, raw);
  }
  float l[V], m = 0.0f, sum = 1.0f, e[kFull ? V : 1];
#pragma unroll
  for (int v = 0; v < V; ++v) l[v] = to_f32(raw[v]);
  if (kFull) {
    m = l[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, l[v]);
    m = group_max<L>(m);
    if (m == -INFINITY) m = 0.0f;  // no expert can be chosen
    sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      e[v] = exp_neg(l[v] - m);
      sum += e[v];
    }
    sum = group_sum<L>(sum);
  }
  Choice c = {-1, -INFINITY, -INFINITY};
  if constexpr (kPacked) {
    uint32_t key[V], word = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = packed_key(raw[v], lane * per + v);
    for (int j = 0; j < k; ++j) {
      uint32_t top = key[0];
#pragma unroll
      for (int v = 1; v < V; ++v) top = key[v] > top ? key[v] : top;
      top = group_max<L>(top);
      word = lane == j ? top : word;
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = key[v] == top ? 0u : key[v];
    }
    if (word) c = {(int)(0xFFFFu - (word & 0xFFFFu)), packed_logit(word), 0.0f};
  } else {
    float key[V];
    if (!kBias) {
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = l[v] > -INFINITY ? l[v] : -INFINITY;  // NaN is never chosen
      if (L != 16 || !choose_ranked<V, kSigmoid, false>(key, l, nullptr, per, k, 0.0f, 0.0f, mine))
        choose_rounds<L, V>(key, l, per, k, mine);
    } else {
      // In float32 first.  Both scores are off by less than 2^-21 (sigmoid: the exponential's and the
      // reciprocal's unit, damped) or 2^-18 of the row's largest (softmax: a sum of up to 1024), the sum by
      // half a unit; `err` is over twice that.  What float32 does not tell is decided in float64.
      const float inv = 1.0f / sum;
      float b[V];
      if (staged || (kCanStage<L, V> && rows == Rows::kSingle))
        load_experts<V>(staged ? bias_stage : bias, lane, per, E, 0.0f, b);
      else
        load_row<V>(bias, lane, E, vec_bias, 0.0f, b);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float s = kSigmoid ? __builtin_amdgcn_rcpf(1.0f + __expf(-l[v])) : e[kFull ? v : 0] * inv;
        const float sum_b = s + b[v];
        key[v] = ((l[v] > -INFINITY) & (sum_b > -INFINITY)) ? sum_b : -INFINITY;
      }
      const float err = kSigmoid ? 0x1p-19f : 0x1p-16f * inv;
      if (L != 16 || !choose_ranked<V, kSigmoid, true>(key, l, b, per, k, err, m, mine)) {
        choose_rounds<L, V>(key, l, per, k, mine);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        bool unsure = false;
        auto of = [&](int j) {
          Choice x = mine.get(j);
          x.bias = x.idx >= 0 ? bias[x.idx] : 0.0f;
          return x;
        };
        if (lane + 1 < k && mine.idx[lane + 1] >= 0) unsure = !certain(of(lane), of(lane + 1), err);
        if (mine.idx[k - 1] >= 0) {  // the others (the rounds leave -inf in the place of a chosen key) below the last
          const Choice last = of(k - 1);
#pragma unroll
          for (int v = 0; v < V; ++v)
            unsure |= (key[v] > -INFINITY) & !certain(last, {lane * per + v, l[v], key[v], b[v]}, err);
        }
        if (__any(unsure)) {
          const double z = row_sum64<L, V, kSigmoid>(l, m);
          double wide[V];
#pragma unroll
          for (int v = 0; v < V; ++v) wide[v] = key64<kSigmoid>(l[v], b[v], m, z);  // a missing expert's l is -inf
          choose_rounds<L, V>(wide, l, per, k, mine);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (lane < k) c = mine.get(lane);
  }
  float w = 0.0f;
  if (kNormalize) {
    w = c.idx >= 0 ? (kSigmoid ? log_sigmoid(c.logit) : c.logit) : -INFINITY;
    const float top = group_max<L>(w);
    w = w > -INFINITY ? exp_neg(w - top) : 0.0f;
    w = w / group_sum<L>(w);
  } else {
    w = kSigmoid ? sigmoid(c.logit) : exp_neg(c.logit - m) / sum;
  }
  if (lane < k) {
    topk_idx[t * k + lane] = c.idx;
    probs[t * k + lane] = c.idx < 0 ? 0.0f : scale * w;
  }
}

// d[v] += g of every slot whose expert is the lane's v-th; slots in order, so that the sum of an expert that is
// there twice has one order.
template <int L, int V, int J>
__device__ __forceinline__ void spread_slot(int idx, float g, int k, int lane, float (&d)[V]) {
  if constexpr (J < 16) {
    if (J >= k) return;  // uniform
    // lane J of the row to all its lanes
    const int at = (int)dpp<0x150 + J>((uint32_t)idx) - lane * V;
    const float gj = __uint_as_float(dpp<0x150 + J>(__float_as_uint(g)));
#pragma unroll
    for (int v = 0; v < V; ++v) d[v] += at == v ? gj : 0.0f;
    spread_slot<L, V, J + 1>(idx, g, k, lane, d);
  }
}
// From eight experts a lane on the sums are made in LDS (`row`: the group's L * V floats, a lane's four in a piece
// and the lanes side by side): the slots' lanes add theirs one behind the other.  16384 tokens x 256 experts 6.2 us, in
// registers 7.3; x 96 experts 4.2 both ways.
template <int L, int V>
constexpr bool kSpreadInLds = L == 16 && V >= 8;
template <int L, int V>
__device__ __forceinline__ void spread(int idx, float g, int k, int lane, int per, float* row, float (&d)[V]) {
  if constexpr (kSpreadInLds<L, V>) {
    f32x4* const pieces = reinterpret_cast<f32x4*>(row) + lane;
#pragma unroll
    for (int q = 0; q < V / 4; ++q) pieces[q * 16] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int i = idx < 0 ? 0 : idx, owner = (int)((unsigned)i / (unsigned)per), v = i - owner * per;
    float* const at = row + ((v / 4) * 16 + owner) * 4 + v % 4;
    for (int j = 0; j < k; ++j)
      if (lane == j && idx >= 0) __hip_atomic_fetch_add(at, g, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      const f32x4 p = pieces[q * 16];
#pragma unroll
      for (int u = 0; u < 4; ++u) d[4 * q + u] = p[u];
    }
    return;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) d[v] = 0.0f;
  if constexpr (L == 16) {
    spread_slot<L, V, 0>(idx, g, k, lane, d);
  } else {
    for (int j = 0; j < k; ++j) {
      const int at = __builtin_amdgcn_readlane(idx, j) - lane * V;
      const float gj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), j));
#pragma unroll
      for (int v = 0; v < V; ++v) d[v] += at == v ? gj : 0.0f;
    }
  }
}

template <int L, int V, bool kSigmoid, bool kNormalize, typename X>
__global__ __launch_bounds__(kThreads) void topk_bwd_kernel(const X* __restrict__ logits,
                                                            const int32_t* __restrict__ topk_idx,
                                                            const float* __restrict__ dprobs, int64_t T, int E, int k,
                                                            float scale, Rows rows, X* __restrict__ dlogits) {
  constexpr bool kDense = !kSigmoid && !kNormalize;
  const int lane = threadIdx.x & (L - 1);
  int64_t t = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const bool staged = kCanStage<L, V> && rows == Rows::kStaged;
  const int per = experts_per_lane<L, V>(E, false);
  X* const in_stage = reinterpret_cast<X*>(stage);
  const int64_t first = (int64_t)blockIdx.x * kStagedRows * E;  // (staged)
  if (staged) {  // the last workgroup's missing rows go along as the last row
    if (kDense) {
      move_staged(logits + first, in_stage, staged_elements(T, E));
      __syncthreads();
    }
  } else if (t >= T) {
    return;
  }
  const int local = (int)(t < T ? threadIdx.x / L : T - 1 - (t - threadIdx.x / L));  // row of the workgroup
  t = t < T ? t : T - 1;
  const X* row = logits + t * E;
  __shared__ __align__(16) float in_lds[kSpreadInLds<L, V> ? kThreads * V : 4];
  float* const sums = in_lds + (kSpreadInLds<L, V> ? threadIdx.x / L * (L * V) : 0);
  float d[V];
  // slot `lane`: its expert (-1: none) and its weight's gradient
  int idx = lane < k ? topk_idx[t * k + lane] : -1;
  if (idx >= E) idx = -1;
  float g = lane < k ? dprobs[t * k + lane] : 0.0f;
  if (idx < 0) g = 0.0f;
  if (kDense) {
    X raw[V], missing;
    from_f32(&missing, -INFINITY);
    if (staged || (kCanStage<L, V> && rows == Rows::kSingle))
      load_experts<V>(staged ? in_stage + local * E : row, lane, per, E, missing, raw);
    else
      load_row<V>(row, lane, E, rows == Rows::kPieces, missing, raw);
    float p[V], m = -INFINITY, sum = 0.0f, dot = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      p[v] = to_f32(raw[v]);
      m = fmaxf(m, p[v]);
    }
    m = group_max<L>(m);
    if (m == -INFINITY) m = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      p[v] = exp_neg(p[v] - m);
      sum += p[v];
    }
    sum = group_sum<L>(sum);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    spread<L, V>(idx, g, k, lane, per, sums, d);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      p[v] *= inv;
      dot = fmaf(p[v], d[v], dot);
    }
    dot = group_sum<L>(dot);
#pragma unroll
    for (int v = 0; v < V; ++v) d[v] = scale * p[v] * (d[v] - dot);
  } else {
    const float l = idx >= 0 ? to_f32(row[idx]) : -INFINITY;
    if (kNormalize) {
      float r = idx >= 0 ? (kSigmoid ? log_sigmoid(l) : l) : -INFINITY;
      const float top = group_max<L>(r);
      r = r > -INFINITY ? exp_neg(r - top) : 0.0f;
      const float total = group_sum<L>(r);
      r = total == 0.0f ? 0.0f : r / total;
      const float dot = group_sum<L>(r * g);
      g = scale * r * (g - dot) * (kSigmoid ? sigmoid(-l) : 1.0f);
    } else if (idx >= 0) {
      g = scale * g * sigmoid(l) * sigmoid(-l);
    }
    spread<L, V>(idx, g, k, lane, per, sums, d);
  }
  if (staged) {
    __syncthreads();
    store_experts<V>(in_stage + local * E, lane, per, E, d);
    __syncthreads();
    move_staged<X>(in_stage, dlogits + first, staged_elements(T, E));
  } else if (kCanStage<L, V> && rows == Rows::kSingle) {
    store_experts<V>(dlogits + t * E, lane, per, E, d);
  } else {
    store_row<V>(dlogits + t * E, lane, E, rows == Rows::kPieces, d);
  }
}

// Lanes a token.  Sixteen (four tokens a wave) take a quarter of the reductions of a whole wave but hold four
// times the experts a lane.  The wave is for k above 16 (a lane holds a slot), for more than 256 experts, and for
// few tokens where the experts are chosen by rounds over packed keys (`rounds`: bf16 logits without a bias), as a
// round's latency counts there: 256 experts, k = 8, 16 against 64 lanes, us: 1 token 3.4 2.1, 64 4.1 3.2, 2048 4.4 3.6,
// 4096 4.7 4.8, 16384 7.8 11.0.  Up to 64 experts sixteen are as fast or faster from 64 tokens on (64: 2.5 2.9,
// 16384: 4.2 8.0), and so they are at any number where 16 lanes choose by ranks (1 token 2.9 3.1 in float32, 3.6
// 3.9 with a bias; 2048 tokens 4.7 5.0 and 5.5 8.7) and in the gradient (1 token 2.2 2.4, of all logits 2.6 2.1,
// 64 3.0 3.9, 3.1 2.9, 2048 3.4 3.5, 3.5 3.5, 16384 5.0 10.2, 5.0 9.4).
int lanes_of(int64_t T, int E, int k, bool rounds) {
  if (E > 256 || k > 16) return 64;
  return rounds && E > 64 && T <= 2048 ? 64 : 16;
}

// CALL(lanes, experts a lane)
#define FF8_BY_SIZE(T, E, k, rounds, CALL)  \
  if (lanes_of(T, E, k, rounds) == 16) {    \
    if ((E) <= 16) return CALL(16, 1);      \
    if ((E) <= 32) return CALL(16, 2);      \
    if ((E) <= 64) return CALL(16, 4);      \
    if ((E) <= 128) return CALL(16, 8);     \
    return CALL(16, 16);                    \
  }                                         \
  if ((E) <= 64) return CALL(64, 1);        \
  if ((E) <= 128) return CALL(64, 2);       \
  if ((E) <= 256) return CALL(64, 4);       \
  if ((E) <= 512) return CALL(64, 8);       \
  return CALL(64, 16);

template <int V, typename X>
bool vector_rows(int E, const void* a, const void* b) {
  constexpr uintptr_t kBytes = V * sizeof(X) < 16 ? V * sizeof(X) : 16;
  return E % V == 0 && (reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) % kBytes == 0;
}

// (every row of a tensor in the same way; LDS that a launch needs for it)
template <int L, int V, typename X>
Rows rows_of(int E, bool ranked, const void* a, const void* b) {
  const bool aligned = (reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) % 16 == 0;
  if (experts_per_lane<L, V>(E, ranked) == V && vector_rows<V, X>(E, a, b)) return Rows::kPieces;
  return kCanStage<L, V> && aligned ? Rows::kStaged : Rows::kSingle;
}
template <int V, typename X>
unsigned stage_bytes(Rows rows) {
  return rows == Rows::kStaged ? (unsigned)(kThreads * V * sizeof(X) + 16 * V * sizeof(float)) : 0u;
}

template <int L, int V, typename X>
hipError_t topk_launch(const X* logits, const float* bias, int64_t T, int E, int k, bool sig, bool norm, float scale,
                       int32_t* idx, float* probs, hipStream_t st) {
  const unsigned grid = (unsigned)((T + kThreads / L - 1) / (kThreads / L));
  const Rows rows = rows_of<L, V, X>(E, bias || sizeof(X) != 2, logits, nullptr);
  const bool vec_bias = vector_rows<V, float>(E, bias, nullptr);
  const unsigned lds = stage_bytes<V, X>(rows);
#define FF8_GO(S, N)                                                                                               \
  if (bias)                                                                                                        \
    topk_kernel<L, V, S, N, true, X><<<grid, kThreads, lds, st>>>(logits, bias, T, E, k, scale, rows, vec_bias, idx,  \
                                                                probs);                                            \
  else                                                                                                             \
    topk_kernel<L, V, S, N, false, X><<<grid, kThreads, lds, st>>>(logits, bias, T, E, k, scale, rows, false, idx,    \
                                                                 probs);
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
  const Rows rows = rows_of<L, V, X>(E, false, logits, dlogits);
  const unsigned lds = stage_bytes<V, X>(rows);
#define FF8_GO(S, N) \
  topk_bwd_kernel<L, V, S, N, X><<<grid, kThreads, lds, st>>>(logits, idx, dprobs, T, E, k, scale, rows, dlogits)
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

template <typename X>
hipError_t topk_impl(const X* logits, const float* bias, int64_t T, int E, int k, bool sig, bool norm, float scale,
                     int32_t* idx, float* probs, hipStream_t st) {
  if (T == 0) return hipSuccess;
#define FF8_CALL(L, V) topk_launch<L, V, X>(logits, bias, T, E, k, sig, norm, scale, idx, probs, st)
  FF8_BY_SIZE(T, E, k, sizeof(X) == 2 && !bias, FF8_CALL)
#undef FF8_CALL
}

template <typename X>
hipError_t topk_bwd_impl(const X* logits, const int32_t* idx, const float* dprobs, int64_t T, int E, int k, bool sig,
                         bool norm, float scale, X* dlogits, hipStream_t st) {
  if (T == 0) return hipSuccess;
#define FF8_CALL(L, V) topk_bwd_launch<L, V, X>(logits, idx, dprobs, T, E, k, sig, norm, scale, dlogits, st)
  FF8_BY_SIZE(T, E, k, false, FF8_CALL)
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
