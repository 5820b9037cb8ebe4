// Token rows sorted by expert without a cast, and the gradient of the weighted return, for gfx950.
//
//   sort      out[row_map[t, j]] = x[t] for bf16 rows, or for rows that are e4m3 already (tokens that
//             were cast before they were dispatched; paper section 3.3.1 permutes and pads FP8 rows)
//             together with their 1x128 scales; padding rows are zeros (scale 2^-126).
//   gradient  of the return y[t] = sum_j w[t, j] y_perm[row_map[t, j]]:
//             dy_perm[row_map[t, j]] = bf16(w[t, j] dy[t]),  dw[t, j] = <dy[t], y_perm[row_map[t, j]]>.
//
// Both are bound by HBM: one wave moves one row (16-byte pieces, consecutive lanes), eight waves a workgroup, so
// that the k rows of a token are mostly written by one workgroup and its input row comes from HBM once and from
// the XCD's L2 the other times.  A lane has up to eight pieces in flight before its first store.  At 16384
// tokens x 7168 in bf16, k = 8 (2.1 GB) the sort takes 386 us, 5.5 TB/s: a workgroup per token that holds its row
// in registers took 422, loads that alternate with stores 410, a row per workgroup 516, a wave per output row in
// output order 548.  The gradient (4.0 GB) takes 757 us, 5.3 TB/s (772 with a workgroup per token).  Copying the
// same rows in order reaches 5.8 TB/s and in the sorted order 5.5, so what is left is the order that the routing
// gives.  Workgroups behind those fill the expert groups' padding rows: behind, so that they do not hold up the rows
// (512 x 7168, 64 experts, k = 8, padded to 128: gradient 38 us, 45 with the padding first).
// The routing maps are those of ff8_permute_quant.

#include "ff8_device.hpp"
#include "ff8_launch.hpp"
#include "rows_rule.hpp"

namespace ff8 {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kPadGroups = 512;
constexpr int kPieces = 8;  // 16-byte pieces that a lane has in flight

// One wave: row r becomes token t's row, or a row of zeros (scales 2^-126).  row16: 16-byte pieces of a row; n_s:
// its scales (0 for bf16 rows).
template <typename S>
__device__ __forceinline__ void move_row(const u32x4* __restrict__ x, const S* __restrict__ s, int64_t t, int64_t r,
                                         int lane, int64_t row16, int n_s, u32x4* __restrict__ out,
                                         S* __restrict__ s_out) {
  for (int64_t c0 = lane; c0 < row16; c0 += 64 * kPieces) {
    u32x4 v[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (c0 + 64 * i < row16) v[i] = ld16(x + t * row16 + c0 + 64 * i);
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (c0 + 64 * i < row16) stnt16(out + r * row16 + c0 + 64 * i, v[i]);
  }
  for (int c = lane; c < n_s; c += 64) s_out[r * n_s + c] = s[t * n_s + c];
}
// The same for kNarrowRows narrow rows at a time, so that a lane has as many pieces in flight as with long ones: row r[j]
// becomes token t[j]'s, with r[j] = -1 none.  Loads are not behind conditions (t[j] is a token in any case; missing lanes
// take the first piece): with branches between them every row waits for the one before.
template <typename S>
__device__ __forceinline__ void move_narrow(const u32x4* __restrict__ x, const S* __restrict__ s,
                                            const int (&t)[kNarrowRows], const int (&r)[kNarrowRows], int lane,
                                            int64_t row16, int n_s, u32x4* __restrict__ out, S* __restrict__ s_out) {
  u32x4 v[kNarrowRows];
  S sv[kNarrowRows];
  const int piece = lane < row16 ? lane : 0;
#pragma unroll
  for (int j = 0; j < kNarrowRows; ++j) v[j] = ld16(x + t[j] * row16 + piece);
  if (n_s) {
#pragma unroll
    for (int j = 0; j < kNarrowRows; ++j) sv[j] = s[(int64_t)t[j] * n_s + (lane < n_s ? lane : 0)];
  }
#pragma unroll
  for (int j = 0; j < kNarrowRows; ++j)
    if (r[j] >= 0 && lane < row16) stnt16(out + r[j] * row16 + lane, v[j]);
#pragma unroll
  for (int j = 0; j < kNarrowRows; ++j)
    if (r[j] >= 0 && lane < n_s) s_out[(int64_t)r[j] * n_s + lane] = sv[j];
}
// Rows and tokens of the kNarrowRows pairs from p on (p < n_pairs); r = -1 for dropped pairs and behind the last.
__device__ __forceinline__ void narrow_pairs(int p, int n_pairs, int k, int64_t M_cap, const int32_t* __restrict__ row_map,
                                             int lane, int (&t)[kNarrowRows], int (&r)[kNarrowRows]) {
  const int mine = p + lane % kNarrowRows, q = mine < n_pairs ? mine : n_pairs - 1;
  int rq = row_map[q];
  if (rq >= M_cap || mine >= n_pairs) rq = -1;
  const int tq = q / k;
#pragma unroll
  for (int j = 0; j < kNarrowRows; ++j) {
    r[j] = __builtin_amdgcn_readlane(rq, j);
    t[j] = __builtin_amdgcn_readlane(tq, j);
  }
}
template <typename S>
__device__ __forceinline__ void clear_row(int64_t r, int lane, int64_t row16, int n_s, u32x4* __restrict__ out,
                                          S* __restrict__ s_out) {
  const u32x4 z = {0u, 0u, 0u, 0u};
  for (int64_t c = lane; c < row16; c += 64) stnt16(out + r * row16 + c, z);
  for (int c = lane; c < n_s; c += 64) put_scale(&s_out[r * n_s + c], kTMin);
}

// Zeros in the padding rows (src_row < 0) of expert e's group: fewer than 128, all among the group's last 128.
// Their numbers are collected in LDS first (two loads a lane instead of one before every row), then each wave
// takes every eighth.
template <typename S>
__device__ __forceinline__ void pad_rows(int e, int part, int parts, const int32_t* __restrict__ offsets, const int32_t* __restrict__ src_row,
                                         int64_t M_cap, int64_t row16, int n_s, u32x4* __restrict__ out,
                                         S* __restrict__ s_out) {
  __shared__ int rows[kTile];
  __shared__ int n_rows;
  const int64_t g0 = offsets[e], g1 = offsets[e + 1] < M_cap ? offsets[e + 1] : M_cap;
  const int64_t r0 = g1 - g0 > kTile ? g1 - kTile : g0;
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {
    int n = 0;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int64_t r = r0 + 64 * half + lane;
      const bool pad = r < g1 && src_row[r] < 0;
      const unsigned long long m = __ballot(pad);
      if (pad) rows[n + __popcll(m & ((1ull << lane) - 1))] = 64 * half + lane;
      n += __popcll(m);
    }
    if (lane == 0) n_rows = n;
  }
  __syncthreads();
  for (int i = part * kWaves + (int)(threadIdx.x >> 6); i < n_rows; i += parts * kWaves)
    clear_row<S>(r0 + rows[i], lane, row16, n_s, out, s_out);
}

// The (token, slot) pair of a wave; the same for all its lanes.
__device__ __forceinline__ int pair_of_wave() {
  return __builtin_amdgcn_readfirstlane((int)blockIdx.x * kWaves + (int)(threadIdx.x >> 6));
}

template <typename S, bool kIsNarrow>
__global__ __launch_bounds__(kThreads) void sort_rows_kernel(const u32x4* __restrict__ x, const S* __restrict__ s,
                                                             int64_t row16, int n_s, int n_pairs, int k, int parts,
                                                             const int32_t* __restrict__ row_map,
                                                             const int32_t* __restrict__ offsets,
                                                             const int32_t* __restrict__ src_row, int64_t M_cap,
                                                             u32x4* __restrict__ out, S* __restrict__ s_out) {
  constexpr int kBlock = kWaves * (kIsNarrow ? kNarrowRows : 1);
  const int pad = (int)blockIdx.x - (n_pairs + kBlock - 1) / kBlock;
  if (pad >= 0) {
    pad_rows<S>(pad / parts, pad % parts, parts, offsets, src_row, M_cap, row16, n_s, out, s_out);
    return;
  }
  const int p = pair_of_wave() * (kIsNarrow ? kNarrowRows : 1), lane = threadIdx.x & 63;
  if (p >= n_pairs) return;
  if (kIsNarrow) {
    int t[kNarrowRows], r[kNarrowRows];
    narrow_pairs(p, n_pairs, k, M_cap, row_map, lane, t, r);
    move_narrow<S>(x, s, t, r, lane, row16, n_s, out, s_out);
  } else {
    const int64_t t = p / k, r = row_map[p];
    if (r >= 0 && r < M_cap) move_row<S>(x, s, t, r, lane, row16, n_s, out, s_out);
  }
}

// Routing and rows in one launch: a workgroup takes kWaves * kPer (token, slot) pairs, finds the pairs of each
// expert and those before its own, and so knows the group offsets and its rows.  Behind those, others fill the
// expert groups' padding.  Integer LDS atomics: the counts do not depend on order.
// Up to kMaxPairs pairs every workgroup counts them all by itself (counts NULL).
// Otherwise a launch in front has counted chunks of kChunk tokens, and a workgroup adds those up and counts in its own
// chunk alone; it then takes two pairs a wave: 16384 x 2048, 64 experts, k = 16 one, two, four, eight 236 215 215 216,
// 4096 x 7168, 256 experts, k = 8 149 143 144 143 us; of narrow rows kNarrowRows.
constexpr int kMaxExperts = 1024;
constexpr int kChunk = kRouteChunk, kPerCounted = 2;
__global__ __launch_bounds__(kThreads) void chunk_count_kernel(const int32_t* __restrict__ topk_idx, int n_pairs, int k,
                                                               int E, int32_t* __restrict__ counts) {
  __shared__ int count[kMaxExperts];
  for (int e = threadIdx.x; e < E; e += kThreads) count[e] = 0;
  __syncthreads();
  const int p0 = (int)blockIdx.x * kChunk * k, p1 = p0 + kChunk * k < n_pairs ? p0 + kChunk * k : n_pairs;
  for (int i = p0 + (int)threadIdx.x; i < p1; i += kThreads) {
    const int e = topk_idx[i];
    if (e >= 0 && e < E) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kThreads) counts[(int)blockIdx.x * E + e] = count[e];
}

template <typename S, int kPer>
__global__ __launch_bounds__(kThreads) void route_sort_kernel(
    const u32x4* __restrict__ x, const S* __restrict__ s, const int32_t* __restrict__ topk_idx, int n_pairs, int k, int E,
    int align, int parts, const int32_t* __restrict__ counts, int n_chunks, int64_t row16, int n_s, int64_t M_cap,
    int32_t* __restrict__ row_map, int32_t* __restrict__ offsets, int32_t* __restrict__ src_row,
    u32x4* __restrict__ out, S* __restrict__ s_out) {
  __shared__ int total[kMaxExperts], before[kMaxExperts];  // pairs of an expert, and those before the workgroup's
  __shared__ int start[kMaxExperts + 1], wave_sum[kWaves];
  constexpr int kBlock = kWaves * kPer;
  static_assert(kBlock <= 64, "a lane holds a pair");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_sort = (n_pairs + kBlock - 1) / kBlock, pad = (int)blockIdx.x - n_sort;  // below 0: rows
  const int p0 = pad < 0 ? (int)blockIdx.x * kBlock : 0;
  const int mine = lane < kBlock && p0 + lane < n_pairs ? topk_idx[p0 + lane] : -1;
  for (int e = tid; e < E; e += kThreads) {
    total[e] = 0;
    before[e] = 0;
  }
  __syncthreads();
  int from = 0;  // the first pair that is not counted in `before` yet
  if (counts) {
    const int chunk = p0 / (kChunk * k);
    from = chunk * kChunk * k;
    // a thread adds up one expert's counts, of every stride-th chunk
    const int stride = E < kThreads ? kThreads / E : 1;
    for (int e0 = 0; e0 < E; e0 += kThreads) {
      const int e = e0 + (E < kThreads ? tid % E : tid);
      int all = 0, front = 0;
      if (e < E)
        for (int c = E < kThreads ? tid / E : 0; c < (tid / E < stride ? n_chunks : 0); c += stride) {
          const int n = counts[c * E + e];
          all += n;
          front += c < chunk ? n : 0;
        }
      if (all) atomicAdd(&total[e], all);
      if (front) atomicAdd(&before[e], front);
    }
  }
  for (int i = from + tid; i < (counts ? p0 : n_pairs); i += kThreads) {
    const int e = topk_idx[i];
    if (e >= 0 && e < E) {
      if (!counts) atomicAdd(&total[e], 1);
      if (i < p0) atomicAdd(&before[e], 1);
    }
  }
  __syncthreads();
  // group offsets: two experts a thread, scanned over the wave and the waves
  static_assert(2 * kThreads >= kMaxExperts, "two experts a thread");
  int rows[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int e = 2 * tid + h, n = e < E ? total[e] : 0;
    rows[h] = (n + align - 1) / align * align;
  }
  int end = rows[0] + rows[1];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(end, d);
    if (lane >= d) end += u;
  }
  if (lane == 63) wave_sum[wave] = end;
  __syncthreads();
  for (int w = 0; w < wave; ++w) end += wave_sum[w];
  if (tid == 0) start[0] = 0;
  if (2 * tid < E) start[2 * tid + 1] = end - rows[1];
  if (2 * tid + 1 < E) start[2 * tid + 2] = end;
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = tid; e <= E; e += kThreads) offsets[e] = start[e];
  if (pad < 0) {
    // pair `slot` of the workgroup, the same for all lanes: its row, -1 if there is none
    auto row_of = [&](int slot) {
      const int p = p0 + slot, e = __builtin_amdgcn_readlane(mine, slot);
      if (e < 0 || e >= E) {
        if (lane == 0) row_map[p] = -1;
        return -1;
      }
      const int r = start[e] + before[e] + __popcll(__ballot(mine == e && lane < slot));
      if (r >= M_cap) return -1;
      if (lane == 0) {
        row_map[p] = r;
        src_row[r] = p;
      }
      return r;
    };
    const int w = __builtin_amdgcn_readfirstlane(wave);
    if constexpr (kPer == kNarrowRows) {
      if (p0 + w * kPer >= n_pairs) return;
      int t[kPer], r[kPer];
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int slot = w * kPer + j;
        r[j] = p0 + slot < n_pairs ? row_of(slot) : -1;
        t[j] = (p0 + slot < n_pairs ? p0 + slot : n_pairs - 1) / k;
      }
      move_narrow<S>(x, s, t, r, lane, row16, n_s, out, s_out);
    } else {
      for (int i = 0; i < kPer; ++i) {
        const int slot = w + i * kWaves;
        if (p0 + slot >= n_pairs) return;
        const int r = row_of(slot);
        if (r >= 0) move_row<S>(x, s, (p0 + slot) / k, r, lane, row16, n_s, out, s_out);
      }
    }
  } else {
    const int e = pad / parts, part = pad - e * parts;
    const int64_t r1 = start[e + 1] < M_cap ? start[e + 1] : M_cap;
    for (int64_t r = start[e] + total[e] + part * kWaves + wave; r < r1; r += parts * kWaves) {
      if (lane == 0) src_row[r] = -1;
      clear_row<S>(r, lane, row16, n_s, out, s_out);
    }
  }
}

// Sum of a dot product, fixed order: a lane's products in column order, then a butterfly over the wave.
template <bool kDprobs, bool kIsNarrow>
__global__ __launch_bounds__(kThreads) void return_bwd_kernel(
    const u32x4* __restrict__ dy, const float* __restrict__ row_w, int64_t row16, int n_pairs, int k, int parts,
    const int32_t* __restrict__ row_map, const int32_t* __restrict__ offsets, const int32_t* __restrict__ src_row,
    int64_t M_cap, u32x4* __restrict__ dy_perm, const u32x4* __restrict__ y_perm, float* __restrict__ dprobs) {
  constexpr int kBlock = kWaves * (kIsNarrow ? kNarrowRows : 1);
  const int pad = (int)blockIdx.x - (n_pairs + kBlock - 1) / kBlock;
  if (pad >= 0) {
    pad_rows<e8m0_t>(pad / parts, pad % parts, parts, offsets, src_row, M_cap, row16, 0, dy_perm, nullptr);
    return;
  }
  const int p = pair_of_wave() * (kIsNarrow ? kNarrowRows : 1), lane = threadIdx.x & 63;
  if (p >= n_pairs) return;
  // a piece of a token's gradient: weighted, and its part of the dot product
  auto weigh = [](const u32x4& d, const u32x4& y, float w, float& acc) {
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float lo = bf16_lo(d[i]), hi = bf16_hi(d[i]);
      o[i] = pack_bf16x2(w * lo, w * hi);
      if (kDprobs) {
        acc = fmaf(lo, bf16_lo(y[i]), acc);
        acc = fmaf(hi, bf16_hi(y[i]), acc);
      }
    }
    return o;
  };
  if constexpr (kIsNarrow) {
    int t[kNarrowRows], r[kNarrowRows];
    narrow_pairs(p, n_pairs, k, M_cap, row_map, lane, t, r);
    const int q = p + lane % kNarrowRows < n_pairs ? p + lane % kNarrowRows : n_pairs - 1;
    const float wq = row_w[q];
    int any = r[0];
#pragma unroll
    for (int j = 1; j < kNarrowRows; ++j) any = r[j] > any ? r[j] : any;
    if (any < 0) {  // every pair of the wave is dropped
      if (kDprobs && lane < kNarrowRows && p + lane < n_pairs) dprobs[p + lane] = 0.0f;
      return;
    }
    const int piece = lane < row16 ? lane : 0;
    u32x4 y[kNarrowRows], d[kNarrowRows];
#pragma unroll
    for (int j = 0; j < kNarrowRows; ++j) {
      if (kDprobs) y[j] = ldnt16(y_perm + (r[j] >= 0 ? r[j] : any) * row16 + piece);  // dropped: one that is read anyway
      d[j] = ld16(dy + t[j] * row16 + piece);
    }
    float mine = 0.0f;
#pragma unroll
    for (int j = 0; j < kNarrowRows; ++j) {
      const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wq), j));
      float acc = 0.0f;
      const u32x4 o = weigh(d[j], y[j], w, acc);
      if (r[j] >= 0 && lane < row16) stnt16(dy_perm + r[j] * row16 + lane, o);
      if (kDprobs) {
        acc = r[j] >= 0 && lane < row16 ? acc : 0.0f;
#pragma unroll
        for (int b = 1; b < 64; b <<= 1) acc += __shfl_xor(acc, b);
        mine = lane == j ? acc : mine;
      }
    }
    if (kDprobs && lane < kNarrowRows && p + lane < n_pairs) dprobs[p + lane] = mine;
    return;
  }
  const int64_t t = p / k, r = row_map[p];
  float acc = 0.0f;
  if (r >= 0 && r < M_cap) {
    const float w = row_w[p];
    for (int64_t c0 = lane; c0 < row16; c0 += 64 * kPieces) {
      u32x4 y[kPieces], d[kPieces];
#pragma unroll
      for (int u = 0; u < kPieces; ++u)
        if (c0 + 64 * u < row16) {
          if (kDprobs) y[u] = ldnt16(y_perm + r * row16 + c0 + 64 * u);
          d[u] = ld16(dy + t * row16 + c0 + 64 * u);
        }
#pragma unroll
      for (int u = 0; u < kPieces; ++u)
        if (c0 + 64 * u < row16) {
          const u32x4 o = weigh(d[u], y[u], w, acc);
          stnt16(dy_perm + r * row16 + c0 + 64 * u, o);
        }
    }
  }
  if (kDprobs) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) acc += __shfl_xor(acc, d);
    if (lane == 0) dprobs[p] = acc;
  }
}

// Workgroups for an expert's padding (up to align - 1 rows of zeros): a wave a row, as long as there are no more than
// kPadGroups, and one for rows below 2 KiB.  us, so / one each: 34 tokens x 6144, 24 experts, k = 7, padded to 128 9.5 /
// 16.6; 199 x 4608, 27, k = 2 8.6 / 13.3; 300 x 1024, 8, k = 2 7.2 / 7.2.  With 256 at the most 9.8 and 8.7.
int pad_parts(int E, int align, int64_t row16) {
  const int most = E < kPadGroups ? kPadGroups / E : 1, need = align / kWaves;
  return row16 < 128 ? 1 : most < need ? most : need;
}

unsigned grid_of(int64_t n_pairs, int n_pad, bool narrow) {
  const int block = kWaves * (narrow ? kNarrowRows : 1);
  return (unsigned)(n_pad + (n_pairs + block - 1) / block);
}

// With topk_idx the routing maps are built too.
template <typename S>
hipError_t sort_rows(const void* x, const S* s, int64_t T, int64_t row16, int n_s, int k, int E, const int32_t* topk_idx,
                     int align, void* workspace, int32_t* row_map, int32_t* offsets, int32_t* src_row, int64_t M_cap,
                     void* out, S* s_out, hipStream_t st) {
  const u32x4* const in = static_cast<const u32x4*>(x);
  u32x4* const to = static_cast<u32x4*>(out);
  const int64_t n_pairs = T * k;
  const bool narrow = narrow_rows(row16);
  const int parts = pad_parts(E, topk_idx ? align : kTile, row16);  // (maps that are there may have any padding)
  if (topk_idx || T == 0) {
    const int64_t n_chunks = (T + kChunk - 1) / kChunk;
    int32_t* const counts = static_cast<int32_t*>(workspace);
#define FF8_GO(PER, COUNTS)                                                                                         \
  route_sort_kernel<S, PER><<<(unsigned)(E * parts + (n_pairs + kWaves * PER - 1) / (kWaves * PER)), kThreads, 0, st>>>(    \
      in, s, topk_idx, (int)n_pairs, k, E, align, parts, COUNTS, (int)n_chunks, row16, n_s, M_cap, row_map, offsets, \
      src_row, to, s_out)
    const SortForm form = sort_form(n_pairs, n_chunks * E, row16);
    if (form == SortForm::kOneLaunch) {
      FF8_GO(1, nullptr);
      return hipGetLastError();
    }
    if (form == SortForm::kCounted) {
      chunk_count_kernel<<<(unsigned)n_chunks, kThreads, 0, st>>>(topk_idx, (int)n_pairs, k, E, counts);
      if (narrow)
        FF8_GO(kNarrowRows, counts);
      else
        FF8_GO(kPerCounted, counts);
      return hipGetLastError();
    }
#undef FF8_GO
    const hipError_t e = launch_route(topk_idx, T, k, E, align, row_map, offsets, src_row, M_cap, workspace, st);
    if (e != hipSuccess) return e;
  }
  auto* const f = narrow ? sort_rows_kernel<S, true> : sort_rows_kernel<S, false>;
  f<<<grid_of(n_pairs, E * parts, narrow), kThreads, 0, st>>>(in, s, row16, n_s, (int)n_pairs, k, parts, row_map, offsets,
                                                              src_row, M_cap, to, s_out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_permute_bf16(const uint16_t* x, int64_t T, int64_t H, int k, int E, const int32_t* topk_idx, int align,
                               void* workspace, int32_t* row_map, int32_t* offsets, int32_t* src_row, int64_t M_cap,
                               uint16_t* out, hipStream_t st) {
  return sort_rows<e8m0_t>(x, nullptr, T, H / 8, 0, k, E, topk_idx, align, workspace, row_map, offsets, src_row, M_cap,
                           out, nullptr, st);
}
hipError_t launch_permute_fp8(const uint8_t* xq, const float* xs, int64_t T, int64_t H, int k, int E,
                              const int32_t* topk_idx, int align, void* workspace, int32_t* row_map, int32_t* offsets,
                              int32_t* src_row, int64_t M_cap, uint8_t* q, float* s, hipStream_t st) {
  return sort_rows(xq, xs, T, H / 16, (int)(H / kTile), k, E, topk_idx, align, workspace, row_map, offsets, src_row,
                   M_cap, q, s, st);
}
hipError_t launch_permute_fp8(const uint8_t* xq, const e8m0_t* xs, int64_t T, int64_t H, int k, int E,
                              const int32_t* topk_idx, int align, void* workspace, int32_t* row_map, int32_t* offsets,
                              int32_t* src_row, int64_t M_cap, uint8_t* q, e8m0_t* s, hipStream_t st) {
  return sort_rows(xq, xs, T, H / 16, (int)(H / kTile), k, E, topk_idx, align, workspace, row_map, offsets, src_row,
                   M_cap, q, s, st);
}

hipError_t launch_unpermute_bwd(const uint16_t* dy, const float* row_w, int64_t T, int64_t H, int k, int E,
                                const int32_t* row_map, const int32_t* offsets, const int32_t* src_row, int64_t M_cap,
                                uint16_t* dy_perm, const uint16_t* y_perm, float* dprobs, hipStream_t st) {
  const int parts = pad_parts(E, kTile, H / 8);
  const bool narrow = narrow_rows(H / 8);
  auto* const f = dprobs ? narrow ? return_bwd_kernel<true, true> : return_bwd_kernel<true, false>
                         : narrow ? return_bwd_kernel<false, true> : return_bwd_kernel<false, false>;
  f<<<grid_of(T * k, E * parts, narrow), kThreads, 0, st>>>(
      reinterpret_cast<const u32x4*>(dy), row_w, H / 8, (int)(T * k), k, parts, row_map, offsets, src_row, M_cap,
      reinterpret_cast<u32x4*>(dy_perm), reinterpret_cast<const u32x4*>(y_perm), dprobs);
  return hipGetLastError();
}

}  // namespace ff8
