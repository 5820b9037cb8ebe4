// Token rows sorted by expert without a cast, and the gradient of the weighted return, for gfx950.
//
//   sort      out[row_map[t, j]] = x[t] for bf16 rows, or for rows that are e4m3 already (tokens that
//             were cast before they were dispatched; paper section 3.3.1 permutes and pads FP8 rows)
//             together with their 1x128 scales; padding rows are zeros (scale 2^-126).
//   gradient  of the return y[t] = sum_j w[t, j] y_perm[row_map[t, j]]:
//             dy_perm[row_map[t, j]] = bf16(w[t, j] dy[t]),  dw[t, j] = <dy[t], y_perm[row_map[t, j]]>.
//
// Both are bound by HBM: a token's row is read once, by one workgroup, and written to each of its k
// rows (whole 16-byte pieces, consecutive lanes).  The first E workgroups of a launch fill the expert
// groups' padding rows.  The routing maps are those of ff8_permute_quant.

#include "ff8_device.hpp"
#include "ff8_launch.hpp"

namespace ff8 {

namespace {

constexpr int kRowThreadsMax = 512;

// Zeros in the padding rows (src_row < 0) of expert e's group: fewer than 128, all among the group's
// last 128.  row16: 16-byte pieces of a row; n_s: its scales (0 for bf16 rows).
template <typename S>
__device__ __forceinline__ void pad_rows(int e, const int32_t* __restrict__ offsets, const int32_t* __restrict__ src_row,
                                         int64_t row16, int n_s, u32x4* __restrict__ out, S* __restrict__ s_out) {
  const int64_t g1 = offsets[e + 1], g0 = offsets[e];
  const u32x4 z = {0u, 0u, 0u, 0u};
  for (int64_t r = g1 - g0 > kTile ? g1 - kTile : g0; r < g1; ++r) {
    if (src_row[r] >= 0) continue;
    for (int64_t c = threadIdx.x; c < row16; c += blockDim.x) stnt16(out + r * row16 + c, z);
    for (int c = threadIdx.x; c < n_s; c += blockDim.x) put_scale(&s_out[r * n_s + c], kTMin);
  }
}

template <typename S>
__global__ __launch_bounds__(kRowThreadsMax) void sort_rows_kernel(const u32x4* __restrict__ x,
                                                                   const S* __restrict__ s, int64_t row16, int n_s,
                                                                   int k, int E, const int32_t* __restrict__ row_map,
                                                                   const int32_t* __restrict__ offsets,
                                                                   const int32_t* __restrict__ src_row, int64_t M_cap,
                                                                   u32x4* __restrict__ out, S* __restrict__ s_out) {
  const int64_t t = (int64_t)blockIdx.x - E;
  if (t < 0) {
    pad_rows<S>((int)blockIdx.x, offsets, src_row, row16, n_s, out, s_out);
    return;
  }
  for (int64_t c = threadIdx.x; c < row16; c += blockDim.x) {
    const u32x4 v = ldnt16(x + t * row16 + c);
    for (int j = 0; j < k; ++j) {
      const int row = row_map[t * k + j];
      if (row >= 0 && row < M_cap) stnt16(out + row * row16 + c, v);
    }
  }
  for (int i = threadIdx.x; i < n_s * k; i += blockDim.x) {
    const int j = i / n_s, c = i - j * n_s, row = row_map[t * k + j];
    if (row >= 0 && row < M_cap) s_out[(int64_t)row * n_s + c] = s[t * n_s + c];
  }
}

// Sum of a dot product, fixed order: a lane's products in column order, a butterfly over the wave,
// then the waves in order.
constexpr int kMaxK = 64;
template <bool kDprobs>
__global__ __launch_bounds__(kRowThreadsMax) void return_bwd_kernel(
    const uint16_t* __restrict__ dy, const float* __restrict__ row_w, int64_t H, int k, int E,
    const int32_t* __restrict__ row_map, const int32_t* __restrict__ offsets, const int32_t* __restrict__ src_row,
    int64_t M_cap, uint16_t* __restrict__ dy_perm, const uint16_t* __restrict__ y_perm, float* __restrict__ dprobs) {
  __shared__ float part[kMaxK * (kRowThreadsMax / 64)];
  const int64_t t = (int64_t)blockIdx.x - E, row8 = H / 8;
  if (t < 0) {
    pad_rows<e8m0_t>((int)blockIdx.x, offsets, src_row, row8, 0, reinterpret_cast<u32x4*>(dy_perm), nullptr);
    return;
  }
  const int wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
  for (int j = 0; j < k; ++j) {
    const int row = row_map[t * k + j];
    const bool ok = row >= 0 && row < M_cap;  // uniform
    float acc = 0.0f;
    if (ok) {
      const float w = row_w[t * k + j];
      for (int64_t c = threadIdx.x; c < row8; c += blockDim.x) {
        float v[8], y[8];
        unpack_bf16x8(ld16(dy + t * H + c * 8), v);
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = pack_bf16x2(w * v[2 * i], w * v[2 * i + 1]);
        stnt16(dy_perm + row * H + c * 8, o);
        if (kDprobs) {
          unpack_bf16x8(ldnt16(y_perm + row * H + c * 8), y);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc = fmaf(v[i], y[i], acc);
        }
      }
    }
    if (kDprobs) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) acc += __shfl_xor(acc, d);
      if ((threadIdx.x & 63) == 0) part[j * (kRowThreadsMax / 64) + wave] = acc;
    }
  }
  if (!kDprobs) return;
  __syncthreads();
  for (int j = threadIdx.x; j < k; j += blockDim.x) {
    float sum = 0.0f;
    for (int w = 0; w < n_waves; ++w) sum += part[j * (kRowThreadsMax / 64) + w];
    dprobs[t * k + j] = sum;
  }
}

// Threads of a one-token workgroup: one lane per 16-byte piece, whole waves, at most 512.
unsigned row_threads(int64_t pieces) {
  const int64_t n = (pieces + 63) / 64 * 64;
  return (unsigned)(n < kRowThreadsMax ? n : kRowThreadsMax);
}

template <typename S>
hipError_t sort_rows(const void* x, const S* s, int64_t T, int64_t row16, int n_s, int k, int E, const int32_t* row_map,
                     const int32_t* offsets, const int32_t* src_row, int64_t M_cap, void* out, S* s_out,
                     hipStream_t st) {
  sort_rows_kernel<S><<<(unsigned)(T + E), row_threads(row16), 0, st>>>(
      static_cast<const u32x4*>(x), s, row16, n_s, k, E, row_map, offsets, src_row, M_cap, static_cast<u32x4*>(out),
      s_out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_permute_bf16(const uint16_t* x, int64_t T, int64_t H, int k, int E, const int32_t* row_map,
                               const int32_t* offsets, const int32_t* src_row, int64_t M_cap, uint16_t* out,
                               hipStream_t st) {
  return sort_rows<e8m0_t>(x, nullptr, T, H / 8, 0, k, E, row_map, offsets, src_row, M_cap, out, nullptr, st);
}
hipError_t launch_permute_fp8(const uint8_t* xq, const float* xs, int64_t T, int64_t H, int k, int E,
                              const int32_t* row_map, const int32_t* offsets, const int32_t* src_row, int64_t M_cap,
                              uint8_t* q, float* s, hipStream_t st) {
  return sort_rows(xq, xs, T, H / 16, (int)(H / kTile), k, E, row_map, offsets, src_row, M_cap, q, s, st);
}
hipError_t launch_permute_fp8(const uint8_t* xq, const e8m0_t* xs, int64_t T, int64_t H, int k, int E,
                              const int32_t* row_map, const int32_t* offsets, const int32_t* src_row, int64_t M_cap,
                              uint8_t* q, e8m0_t* s, hipStream_t st) {
  return sort_rows(xq, xs, T, H / 16, (int)(H / kTile), k, E, row_map, offsets, src_row, M_cap, q, s, st);
}

hipError_t launch_unpermute_bwd(const uint16_t* dy, const float* row_w, int64_t T, int64_t H, int k, int E,
                                const int32_t* row_map, const int32_t* offsets, const int32_t* src_row, int64_t M_cap,
                                uint16_t* dy_perm, const uint16_t* y_perm, float* dprobs, hipStream_t st) {
  const unsigned grid = (unsigned)(T + E), threads = row_threads(H / 8);
  if (dprobs)
    return_bwd_kernel<true><<<grid, threads, 0, st>>>(dy, row_w, H, k, E, row_map, offsets, src_row, M_cap, dy_perm,
                                                      y_perm, dprobs);
  else
    return_bwd_kernel<false><<<grid, threads, 0, st>>>(dy, row_w, H, k, E, row_map, offsets, src_row, M_cap, dy_perm,
                                                       nullptr, nullptr);
  return hipGetLastError();
}

}  // namespace ff8
