// Expert products with 4-bit weights for a few rows per expert (serving), and the weights' formats,
// for gfx950.
//
// Weights are MXFP4: e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with one UE8M0 scale
// 2^T for 32 columns.  The products keep activations in bf16: every weight code * 2^T is exact in bf16
// (v_cvt_scalef32_pk_bf16_fp4 decodes two), every bf16 x bf16 product is exact in float32, and the sums
// are float32.  With few rows the weights are the traffic, so they are stored in the order in which
// the matrix instruction takes them (ff8_pack_mxfp4): a tile of 16 rows x 128 columns is 1 KiB in
// which lane l's 16 bytes are row l % 16, columns 32 (l / 16) .. + 31 -- one scale group -- and a
// wave's load is contiguous.  From row-major weights the same kernel reached 3.4 TB/s, from tiles 6.1
// (8 experts, 4096 x 7168, one row each): a wave's 16-byte loads then fall in 16 rows.

#include <math.h>

#include "ff8_device.hpp"
#include "ff8_launch.hpp"

namespace ff8 {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kGroup = 32;  // columns of one scale
constexpr int kThreads = 256;

// Scale exponent of a group: the smallest T >= -126 with amax <= 6 * 2^T (6 = 1.5 * 2^2), so that no
// value saturates; -126 for an all-zero group.
__device__ __forceinline__ int fp4_scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax), eb = u >> 23;
  if (eb == 0) return kTMin;
  const int t = (int)eb - 127 - 2 + ((u & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return t < kTMin ? kTMin : t;
}

// e2m1 code of v, |v| <= 6: round to nearest, ties to the even code, sign kept.
__device__ __forceinline__ uint32_t fp4_code(float v) {
  const float a = fabsf(v);
  const uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f);
  return c | (__float_as_uint(v) >> 31) << 3;
}

// Four lanes a group, 8 columns a lane: one dword of codes each.
__global__ __launch_bounds__(kThreads) void quant_mxfp4_kernel(const uint16_t* __restrict__ w, int64_t n8,
                                                               uint32_t* __restrict__ q, uint8_t* __restrict__ s) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n8) return;  // whole groups (n8 is a multiple of 16)
  float v[8];
  unpack_bf16x8(ldnt16(w + i * 8), v);
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[j]));
  m = max(m, (uint32_t)__shfl_xor((int)m, 1));
  m = max(m, (uint32_t)__shfl_xor((int)m, 2));
  const int t = fp4_scale_exponent(__uint_as_float(m));
  const float inv = exp2i(-t);
  uint32_t r = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) r |= fp4_code(v[j] * inv) << (4 * j);
  q[i] = r;
  if ((i & 3) == 0) s[i >> 2] = (uint8_t)(t + 127);
}

// One lane a 16-byte piece: tiles in (row block, column block) order, 64 pieces each.
__global__ __launch_bounds__(kThreads) void pack_mxfp4_kernel(const uint8_t* __restrict__ q,
                                                              const uint8_t* __restrict__ s, int64_t n, int64_t k_tiles,
                                                              uint8_t* __restrict__ tq, uint8_t* __restrict__ ts) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const int64_t tile = i >> 6, rb = tile / k_tiles, kt = tile - rb * k_tiles;
  const int l = (int)(i & 63);
  const int64_t row = rb * 16 + (l & 15), piece = kt * 4 + (l >> 4);  // of k_tiles * 4 pieces in a row
  st16(tq + i * 16, ld16(q + (row * k_tiles * 4 + piece) * 16));
  ts[i] = s[row * k_tiles * 4 + piece];
}

// 8 codes (one dword) times 2^T as bf16.
__device__ __forceinline__ bf16x8_t decode8(uint32_t w, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Which 16 rows of which expert block number mb is; e < 0 behind the last.  Every wave finds it by
// itself: 64 experts at a time, a scan of their counts of blocks.
struct RowBlock {
  int e, row, n;
};
__device__ __forceinline__ RowBlock find_block(int64_t mb, const int32_t* __restrict__ offsets, int E) {
  const int lane = threadIdx.x & 63;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int e = e0 + lane;
    const int g0 = e < E ? offsets[e] : 0, g1 = e < E ? offsets[e + 1] : 0;
    const int nb = (g1 - g0 + 15) / 16;
    int end = nb;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int u = __shfl_up(end, d);
      if (lane >= d) end += u;
    }
    const int total = __shfl(end, 63);
    if (mb < total) {
      const int at = __ffsll(__ballot((int64_t)end > mb)) - 1;
      const int row = __shfl(g0, at) + 16 * ((int)mb - __shfl(end - nb, at));
      const int left = __shfl(g1, at) - row;
      return {e0 + at, row, left < 16 ? left : 16};
    }
    mb -= total;
  }
  return {-1, 0, 0};
}

// A workgroup computes 64 weight rows (with kSwiglu 32 gate rows and the 32 up rows beside them) for 16
// token rows of one expert: four tiles of 16 weight rows, which its eight waves share by column blocks
// (wave w takes blocks w, w + 8, ...), so that nothing but the end needs the other waves: their float32
// sums meet in LDS and are added in wave order.  D = weights (16 x 32) times tokens^T (32 x 16): lane l
// holds token l % 16, weight rows 4 (l / 16) .. + 3 of a tile.
constexpr int kWaves = 8, kTiles = 4, kDepth = 2;
template <bool kSwiglu>
__global__ __launch_bounds__(kWaves * 64) void gemv_mxfp4_kernel(
    const uint16_t* __restrict__ x, int64_t x_rows, const uint8_t* __restrict__ tq, const uint8_t* __restrict__ ts,
    const int32_t* __restrict__ offsets, int E, const int32_t* __restrict__ src_row, int top_k, int64_t M_cap,
    int64_t N, int64_t K, uint16_t* __restrict__ out) {
  __shared__ float part[kWaves][kTiles * 256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n_cols = kSwiglu ? kTiles * 8 : kTiles * 16;  // columns of out that a workgroup writes
  const int64_t n_out = kSwiglu ? N / 2 : N;
  const int64_t nt = n_out / n_cols, kt = K / kTile;
  for (int64_t item = blockIdx.x;; item += gridDim.x) {
    const int64_t mb = item / nt, n0 = (item - mb * nt) * n_cols;
    const RowBlock b = find_block(mb, offsets, E);
    if (b.e < 0 || b.row + b.n > M_cap) return;  // uniform
    // the rows' inputs; padding rows (and source rows out of range) give zeros and read nothing of x
    const int c = lane & 15;
    int64_t xr = b.row + c;
    bool real = c < b.n;
    if (real && src_row) {
      const int src = src_row[b.row + c];
      real = src >= 0;
      if (top_k) {
        xr = src / top_k;
        real = real && xr < x_rows;
      }
    }
    const unsigned mask = (unsigned)__ballot(real) & 0xFFFFu;
    if (mask) {
      xr = __shfl((int)xr, real ? lane : __ffs(mask) - 1);  // others read a row that is read anyway
      const uint16_t* const xp = x + xr * K + (lane >> 4) * 32;
      int64_t tile[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        const int64_t n = kSwiglu ? (i < kTiles / 2 ? n0 + 16 * i : n_out + n0 + 16 * (i - kTiles / 2)) : n0 + 16 * i;
        tile[i] = (((int64_t)b.e * N + n) / 16) * kt;
      }
      f32x4 acc[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      u32x4 wb[kDepth][kTiles], xb[kDepth][4];
      uint32_t sb[kDepth][kTiles];
      auto fetch = [&](int64_t s, int d) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          wb[d][i] = ldnt16(tq + (tile[i] + s) * 1024 + lane * 16);
          sb[d][i] = ts[(tile[i] + s) * 64 + lane];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) xb[d][j] = ld16(xp + s * kTile + 8 * j);
      };
#pragma unroll
      for (int d = 0; d < kDepth; ++d)
        if (wave + d * kWaves < kt) fetch(wave + d * kWaves, d);
      for (int64_t s = wave; s < kt; s += kDepth * kWaves) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
          const int64_t now = s + d * kWaves;
          if (now >= kt) break;
#pragma unroll
          for (int i = 0; i < kTiles; ++i) {
            const float scale = __uint_as_float(sb[d][i] << 23);  // the hardware reads the exponent byte alone
#pragma unroll
            for (int j = 0; j < 4; ++j)
              acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8(wb[d][i][j], scale),
                                                               __builtin_bit_cast(bf16x8_t, xb[d][j]), acc[i], 0, 0, 0);
          }
          if (now + kDepth * kWaves < kt) fetch(now + kDepth * kWaves, d);
        }
      }
#pragma unroll
      for (int i = 0; i < kTiles; ++i) *reinterpret_cast<f32x4*>(&part[wave][i * 256 + lane * 4]) = acc[i];
    }
    __syncthreads();
    // element q: tile q / 256, token (q / 4) % 16, weight row 4 ((q / 64) % 4) + q % 4 of the tile
    for (int q = threadIdx.x; q < (kSwiglu ? kTiles / 2 : kTiles) * 256; q += kWaves * 64) {
      const int token = (q >> 2) & 15, n = (q >> 8) * 16 + ((q >> 6) & 3) * 4 + (q & 3);
      if (token >= b.n) continue;
      float v = 0.0f;
      if (mask >> token & 1) {
        v = part[0][q];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += part[w][q];
        if (kSwiglu) {
          float u = part[0][q + kTiles * 128];
#pragma unroll
          for (int w = 1; w < kWaves; ++w) u += part[w][q + kTiles * 128];
          v = v / (1.0f + expf(-v)) * u;
        }
      }
      out[(b.row + token) * n_out + n0 + n] = (uint16_t)f32_to_bf16(v);
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_quant_mxfp4(const uint16_t* w, int64_t rows, int64_t cols, uint8_t* q, uint8_t* s, hipStream_t st) {
  const int64_t n8 = rows * cols / 8;
  quant_mxfp4_kernel<<<(unsigned)((n8 + kThreads - 1) / kThreads), kThreads, 0, st>>>(
      w, n8, reinterpret_cast<uint32_t*>(q), s);
  return hipGetLastError();
}

hipError_t launch_pack_mxfp4(const uint8_t* q, const uint8_t* s, int64_t rows, int64_t cols, uint8_t* tq, uint8_t* ts,
                             hipStream_t st) {
  const int64_t n = rows * cols / kGroup;
  pack_mxfp4_kernel<<<(unsigned)((n + kThreads - 1) / kThreads), kThreads, 0, st>>>(q, s, n, cols / kTile, tq, ts);
  return hipGetLastError();
}

hipError_t launch_grouped_gemv_mxfp4(const uint16_t* x, int64_t x_rows, const uint8_t* tq, const uint8_t* ts,
                                     const int32_t* offsets, int E, const int32_t* src_row, int top_k, int64_t M_cap,
                                     int64_t N, int64_t K, bool swiglu, uint16_t* out, hipStream_t st) {
  // at most this many blocks of 16 rows; the workgroups walk those there are
  const int64_t items = M_cap / 16 * (N / (kTiles * 16)), fill = 2 * (int64_t)device_cu_count();
  const unsigned grid = (unsigned)(items < fill ? items : fill);
  if (swiglu)
    gemv_mxfp4_kernel<true><<<grid, kWaves * 64, 0, st>>>(x, x_rows, tq, ts, offsets, E, src_row, top_k, M_cap, N, K, out);
  else
    gemv_mxfp4_kernel<false><<<grid, kWaves * 64, 0, st>>>(x, x_rows, tq, ts, offsets, E, src_row, top_k, M_cap, N, K, out);
  return hipGetLastError();
}

}  // namespace ff8
