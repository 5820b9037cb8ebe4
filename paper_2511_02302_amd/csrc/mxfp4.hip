// Expert products with 4-bit weights for a few rows per expert (serving), and the weights' formats,
// for gfx950.
//
// Weights are MXFP4: e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with one UE8M0 scale
// 2^T for 32 columns.  The products keep activations in bf16: every weight code * 2^T is exact in bf16
// (v_cvt_scalef32_pk_bf16_fp4 decodes two), every bf16 x bf16 product is exact in float32, and the sums
// are float32.  With few rows the weights are the traffic, so they are stored in the order in which
// the matrix instruction takes them (ff8_pack_mxfp4): a tile of 16 rows x 128 columns is 1 KiB in
// which lane l's 16 bytes are row l % 16, columns 32 (l / 16) .. + 31 -- one scale group -- and a
// wave's load is contiguous; a lane's scales of the two tiles of 32 rows stand side by side.  From row-major weights
// the same kernel reached 3.4 TB/s, from tiles 6.1 (8 experts, 4096 x 7168, one row each): a wave's 16-byte loads
// of row-major weights fall in 16 rows.

#include <math.h>

#include "ff8_device.hpp"
#include "ff8_launch.hpp"
#include "mxfp4_rule.hpp"

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
  ts[(((rb >> 1) * k_tiles + kt) * 64 + l) * 2 + (rb & 1)] = s[row * k_tiles * 4 + piece];
}

__device__ __forceinline__ float swiglu(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// 8 codes (one dword) times 2^T as bf16.
__device__ __forceinline__ bf16x8_t decode8(uint32_t w, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// What a wave computes at a time: kTiles tiles of 16 weight rows (with kSwiglu half of them gate rows and half the
// up rows beside them).  D = weights (16 x 32) times tokens^T (32 x 16): lane l holds token l % 16, weight rows
// 4 (l / 16) .. + 3 of a tile.  The addresses are the same for all lanes but for the lane's own offset, so that they
// stay in scalar registers.
constexpr int kTiles = kMxTiles;
template <bool kSwiglu>
struct Weights {
  const uint8_t *q[kTiles], *s[kTiles / 2];  // at the first column block of the rows
  struct Block {
    u32x4 q[kTiles];
    uint32_t s[kTiles / 2];
    // tile i's scale in the lane's row and group, as a float
    __device__ __forceinline__ float scale(int i) const {
      return __uint_as_float(i & 1 ? s[i / 2] << 15 & 0x7F800000u : s[i / 2] << 23 & 0x7F800000u);
    }
  };
  __device__ __forceinline__ Weights(const uint8_t* __restrict__ tq, const uint8_t* __restrict__ ts, int e, int64_t n0,
                                     int64_t N, int64_t kt) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int64_t n = kSwiglu ? (i < kTiles / 2 ? n0 + 16 * i : N / 2 + n0 + 16 * (i - kTiles / 2)) : n0 + 16 * i;
      const int64_t tile = ((int64_t)e * N + n) / 16;
      q[i] = tq + tile * kt * 1024;
      if (i % 2 == 0) s[i / 2] = ts + tile * kt * 64;
    }
  }
  // kKeep: other workgroups will read the same, so that they are loaded as lines that stay in the L2.
  template <bool kKeep>
  __device__ __forceinline__ void fetch(int64_t block, Block& b) const {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
      b.q[i] = kKeep ? ld16(q[i] + block * 1024 + lane * 16) : ldnt16(q[i] + block * 1024 + lane * 16);
#pragma unroll
    for (int i = 0; i < kTiles / 2; ++i)
      b.s[i] = __builtin_nontemporal_load(reinterpret_cast<const uint16_t*>(s[i] + block * 128 + lane * 2));
  }
};
// The wave's number, as a value that the compiler knows to be the same in all lanes: what depends on it alone is
// computed once, in scalar registers.
__device__ __forceinline__ int wave_number() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }
// Loads before this point are issued before it and later ones after it: waits count loads in their order.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }

// The source row of a grouped row, -1 for padding (and for source rows out of range).
__device__ __forceinline__ int source_of(int64_t row, const int32_t* __restrict__ src_row, int top_k, int64_t x_rows) {
  if (!src_row) return (int)row;
  const int src = src_row[row];
  if (src < 0) return -1;
  if (top_k == 0) return (int)row;
  return src / top_k < x_rows ? src / top_k : -1;
}

// Where a 128-column block of x holds 16-byte piece p of row r in LDS.  Rows are 256 bytes, all 64 banks, so pieces
// are exchanged within a row by a number of the row's own; with row + 4 (instead of the row, which measured one
// conflict for every read) the 16 lanes that the hardware serves together -- 0-3, 12-15, 20-27 of a half wave, and
// the others -- meet 16 different places, as rows of one piece (reads) and as pieces of two rows (writes).
__device__ __forceinline__ int x_place(int r, int p) { return r * 16 + (p ^ ((r + 4) & 15)); }

// ---- few rows per expert ----
// A workgroup computes 64 weight rows for 16 token rows of one expert.  Its waves share the column blocks (wave w
// takes blocks w, w + kWaves, ...), so that nothing but the end needs the other waves: their float32 sums meet in
// LDS and are added in wave order.  Groups are multiples of 16 rows, so block b is rows 16 b .. + 15 and only its
// expert has to be looked up.  A wave brings its own piece of x through LDS into the order of the matrix
// instruction; in registers it has two blocks of weights and x in flight.
//
// Bound by the weights' bytes.  One token of 7168 columns, 8 experts of 2 x 2048 rows with SwiGLU (125 MB): 21 to 22.5
// us from card to card, 5.6 to 5.9 TB/s, where a read of that size out of HBM takes 18.1; 7 tokens of 6 among 64 experts,
// 2048 x 1408 (49 MB): 11 to 12.6 us, 7.1 at the same rate, the rest being the launch and the first block of each wave.
// Of the two blocks ahead: three or more spill, and loads repeated behind a wave's last block, for a loop without its
// tail, cost 5 to 15%.
//
// The products of a wave's blocks, into its part of LDS.  kX: 16-byte pieces of x that a lane brings for a block,
// four rows each; with one only the first four rows are there (the other columns of the products are not stored).
// One where the block has no row of data behind its fourth, four otherwise.  us, one / always four, each pair in one
// session: 1 token, 32 experts, k = 8, 7168 x 2048 up 22.4 / 23.0, down 14.6 / 15.1; 4 tokens 50.5 / 50.4 and 30.1 / 31.7;
// 7 tokens, 64 experts, k = 6, 2048 x 1408 down 11.0 / 11.6.
template <bool kSwiglu, int kWaves, bool kKeep, int kX>
__device__ __forceinline__ void few_rows(const uint16_t* __restrict__ x, int src, unsigned mask,
                                         const Weights<kSwiglu>& w, int wave, int64_t K, float* part) {
  const int lane = threadIdx.x & 63;
  const int64_t kt = K / kTile;
  // row 4 i + lane / 16, piece lane % 16 of a block; padding rows read one that is read anyway
  const int first = __ffs(mask) - 1;
  const u32x4* xp[kX];
#pragma unroll
  for (int i = 0; i < kX; ++i) {
    const int q = 4 * i + (lane >> 4);
    xp[i] = reinterpret_cast<const u32x4*>(x + (int64_t)__shfl(src, mask >> q & 1 ? q : first) * K) + (lane & 15);
  }
  u32x4* const xs = reinterpret_cast<u32x4*>(part);
  f32x4 acc[kTiles];
#pragma unroll
  for (int i = 0; i < kTiles; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  typename Weights<kSwiglu>::Block wb[2];
  u32x4 xb[2][kX];
  auto fetch = [&](int64_t i, int d) {
    const int64_t s = wave + i * kWaves;
    keep_order();
    w.template fetch<kKeep>(s, wb[d]);
#pragma unroll
    for (int r = 0; r < kX; ++r) xb[d][r] = xp[r][s * 16];
    keep_order();
  };
  auto step = [&](int d) {
#pragma unroll
    for (int i = 0; i < kX; ++i) xs[x_place(4 * i + (lane >> 4), lane & 15)] = xb[d][i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bf16x8_t b = __builtin_bit_cast(bf16x8_t, xs[x_place(lane & 15, (lane >> 4) * 4 + j)]);
      bf16x8_t a[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) a[i] = decode8(wb[d].q[i][j], wb[d].scale(i));
#pragma unroll
      for (int i = 0; i < kTiles; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b, acc[i], 0, 0, 0);
      keep_order();  // decoding all of the block first would take 64 more registers
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  // Two blocks in flight.  Inside a path no load is behind a condition, so that the waits in front of a step count
  // the loads behind it and leave them in flight.
  const int64_t n = (kt - wave + kWaves - 1) / kWaves;
  if (n == 1) {
    fetch(0, 0);
    step(0);
  } else if (n > 1) {
    fetch(0, 0);
    fetch(1, 1);
    int64_t i = 0;
    for (; i + 3 < n; i += 2) {
      step(0);
      fetch(i + 2, 0);
      step(1);
      fetch(i + 3, 1);
    }
    step(0);
    if (i + 2 < n) {
      fetch(i + 2, 0);
      step(1);
      step(0);
    } else {
      step(1);
    }
  }
#pragma unroll
  for (int i = 0; i < kTiles; ++i) *reinterpret_cast<f32x4*>(&part[i * 256 + lane * 4]) = acc[i];
}

template <bool kSwiglu, int kWaves, bool kKeep>
__global__ __launch_bounds__(kWaves * 64, 3) void gemv_mxfp4_kernel(
    const uint16_t* __restrict__ x, int64_t x_rows, const uint8_t* __restrict__ tq, const uint8_t* __restrict__ ts,
    const int32_t* __restrict__ offsets, int E, const int32_t* __restrict__ src_row, int top_k, int64_t N, int64_t K,
    uint16_t* __restrict__ out) {
  __shared__ float part[kWaves][kTiles * 256];  // also x, a block a wave
  const int lane = threadIdx.x & 63, wave = wave_number();
  constexpr int kCols = kSwiglu ? kTiles * 8 : kTiles * 16;  // columns of out that a workgroup writes
  const int64_t n_out = kSwiglu ? N / 2 : N;
  const unsigned nt = (unsigned)(n_out / kCols), mb = blockIdx.x / nt;
  const int64_t n0 = (int64_t)(blockIdx.x - mb * nt) * kCols, row0 = (int64_t)mb * 16;
  const int src = source_of(row0 + (lane & 15), src_row, top_k, x_rows);  // rows below M_cap; used below offsets[E]
  int e = -1;
  for (int e0 = 0; e0 < E && e < 0; e0 += 64) {
    const int i = e0 + lane;
    const bool here = i < E && offsets[i] <= row0 && row0 < offsets[i + 1];
    const unsigned long long m = __ballot(here);
    if (m) e = e0 + __ffsll(m) - 1;
  }
  if (e < 0) return;  // behind the last group; the same for the whole workgroup
  const unsigned mask = (unsigned)__ballot(src >= 0) & 0xFFFFu;
  const Weights<kSwiglu> w(tq, ts, e, n0, N, K / kTile);
  if (mask & 0xFFF0u)
    few_rows<kSwiglu, kWaves, kKeep, 4>(x, src, mask, w, wave, K, part[wave]);
  else if (mask)
    few_rows<kSwiglu, kWaves, kKeep, 1>(x, src, mask, w, wave, K, part[wave]);
  __syncthreads();
  // elements q, q + 1: tile q / 256, token (q / 4) % 16, weight rows 4 ((q / 64) % 4) + q % 4 .. + 1 of the tile
  for (int q = 2 * threadIdx.x; q < kCols * 16; q += kWaves * 128) {
    const int token = (q >> 2) & 15, n = (q >> 8) * 16 + ((q >> 6) & 3) * 4 + (q & 3);
    f32x2 v = {0.0f, 0.0f};
    if (mask >> token & 1) {
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const f32x2 p = *reinterpret_cast<const f32x2*>(&part[i][q]);
        v[0] += p[0];
        v[1] += p[1];
      }
      if (kSwiglu) {
        f32x2 u = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          const f32x2 p = *reinterpret_cast<const f32x2*>(&part[i][q + kTiles * 128]);
          u[0] += p[0];
          u[1] += p[1];
        }
        v[0] = swiglu(v[0], u[0]);
        v[1] = swiglu(v[1], u[1]);
      }
    }
    *reinterpret_cast<uint32_t*>(out + (row0 + token) * n_out + n0 + n) = pack_bf16x2(v[0], v[1]);
  }
}

// ---- many rows per expert ----
// A workgroup of four waves computes 256 weight rows (64 a wave) for up to 96 token rows of one expert: every
// wave goes through all column blocks and shares the block of x, which the workgroup brings into one of two LDS
// buffers while it computes from the other.
//
// Bound by the matrix cores and the loads together: 256 tokens of 8 among 32 experts (64 rows on average), 7168 columns, 2
// x 2048 rows (511 MB): 131 to 142 us by routing, 3.6 to 3.9 TB/s.  The loads alone take 94 us (74 at the rate of a large
// read), the matrix instructions alone 101 (88 at that of a large product, 1370 TFLOP/s).  An expert's block of 45 to
// 84 rows is computed in 16s: 2304 to 2320 rows for 2048.  With 64 rows on every expert the launch takes 117 us where that
// session's random routing took 142: of the 25 us between them some 15 are the 13% more rows, the others that CUs get
// unequal blocks.  The matrix cores are busy for 47% of the cycles and vector instructions (decoding) for 32%, at
// 2.1 GHz (2.4 where less is busy).  Blocks of 48 or 64 rows and weights three blocks ahead were slower.
constexpr int kManyThreads = 64 * kManyWaves;

// Workgroup b of a launch runs on XCD b % 8.  Each XCD takes an eighth of the (row block, weight rows) items, in
// order: the workgroups that read the same rows of x, and those that read the same weights for two row blocks of
// one expert, then share an L2.
//
// An item's row block: its expert (-1 where there is none), first row, number of rows (a multiple of 16), and which
// weight rows.  An expert's rows are split evenly over the fewest blocks of at most 96.
struct RowBlock {
  int e, row, n;
  unsigned col;
};
__device__ __forceinline__ RowBlock find_block(unsigned nt, const int32_t* __restrict__ offsets, int E) {
  const int lane = threadIdx.x & 63;
  unsigned blocks = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int i = e0 + lane;
    unsigned nb = i < E ? (unsigned)(offsets[i + 1] - offsets[i] + kManyRows - 1) / kManyRows : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) nb += __shfl_xor(nb, d);
    blocks += __builtin_amdgcn_readfirstlane(nb);
  }
  const unsigned per = (blocks * nt + 7) / 8, item = blockIdx.x % 8 * per + blockIdx.x / 8;
  if (blockIdx.x / 8 >= per || item >= blocks * nt) return {-1, 0, 0, 0};
  int mb = (int)(item / nt);
  const unsigned col = item - mb * nt;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int i = e0 + lane;
    const int g0 = i < E ? offsets[i] : 0, g = i < E ? offsets[i + 1] - g0 : 0;
    const int nb = (g + kManyRows - 1) / kManyRows;
    int end = nb;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int u = __shfl_up(end, d);
      if (lane >= d) end += u;
    }
    const int total = __builtin_amdgcn_readlane(end, 63);
    if (mb < total) {
      const int at = __ffsll(__ballot(end > mb)) - 1;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
      const int b = mb - of(end - nb), n = of(g), n_b = of(nb);
      const int rows = ((n / 16 + n_b - 1) / n_b) * 16, left = n - b * rows;
      return {e0 + at, of(g0) + b * rows, left < rows ? left : rows, col};
    }
    mb -= total;
  }
  return {-1, 0, 0, 0};
}

// The products of one workgroup with kM x 16 token rows: as many 16s as the block has rows of data.  us, so / always
// six: 128 tokens of 2 among 8 experts, 4096 x 7168 up 57 / 88; 128 of 8 among 64, 2048 x 1408 down 25 / 43; the case
// above 138 / 160.
template <bool kSwiglu, int kM>
__device__ __forceinline__ void many_rows(const uint16_t* __restrict__ x, const int* __restrict__ rows,
                                          const uint8_t* __restrict__ tq, const uint8_t* __restrict__ ts, int e,
                                          int64_t n0, int64_t N, int64_t K, bool active,
                                          const RowBlock& blk,
                                          const unsigned long long (&real)[2], u32x4* xs,
                                          uint16_t* __restrict__ out) {
  const int lane = threadIdx.x & 63, t16 = threadIdx.x >> 4, piece = threadIdx.x & 15;
  const int64_t kt = K / kTile, n_out = kSwiglu ? N / 2 : N;
  const u32x4* xp[kM];
#pragma unroll
  for (int m = 0; m < kM; ++m) xp[m] = reinterpret_cast<const u32x4*>(x + (int64_t)rows[16 * m + t16] * K) + piece;
  const Weights<kSwiglu> w(tq, ts, e, n0, N, kt);
  f32x4 acc[kTiles][kM];
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int m = 0; m < kM; ++m) acc[i][m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  typename Weights<kSwiglu>::Block wb[2];
  u32x4 xb[kM];
#pragma unroll
  for (int m = 0; m < kM; ++m) xb[m] = xp[m][0];
  keep_order();
  w.template fetch<false>(0, wb[0]);
  keep_order();
  w.template fetch<false>(kt > 1 ? 1 : 0, wb[1]);
  keep_order();
#pragma unroll
  for (int m = 0; m < kM; ++m) xs[x_place(16 * m + t16, piece)] = xb[m];
  // the weights of 32 columns are decoded while the matrix instructions work on the 32 before
  bf16x8_t a[2][kTiles];
  auto decode = [&](int d, int j, bf16x8_t (&to)[kTiles]) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) to[i] = decode8(wb[d].q[i][j], wb[d].scale(i));  // (the hardware reads a scale's exponent alone)
  };
  decode(0, 0, a[0]);
  __syncthreads();
  for (int64_t s = 0; s < kt; s += 2) {
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const int64_t now = s + d;
      if (now >= kt) break;  // uniform
      // no load is behind a condition, so that the waits count the loads behind them; the last blocks load again
      const int64_t x_next = now + 1 < kt ? now + 1 : now, w_next = now + 2 < kt ? now + 2 : kt - 1;
#pragma unroll
      for (int m = 0; m < kM; ++m) xb[m] = xp[m][x_next * 16];
      keep_order();
      const u32x4* const xd = xs + d * kManyRows * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j == 3) {
          w.template fetch<false>(w_next, wb[d]);
          keep_order();
        }
        decode(j < 3 ? d : 1 - d, (j + 1) & 3, a[(j + 1) & 1]);
#pragma unroll
        for (int m = 0; m < kM; ++m) {
          const bf16x8_t b = __builtin_bit_cast(bf16x8_t, xd[x_place(16 * m + (lane & 15), (lane >> 4) * 4 + j)]);
#pragma unroll
          for (int i = 0; i < kTiles; ++i)
            acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[j & 1][i], b, acc[i][m], 0, 0, 0);
        }
        // issue order: two LDS reads ahead, then matrix instructions with decoding between them
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
        for (int m = 0; m < kM; ++m) {
          __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        keep_order();
      }
#pragma unroll
      for (int m = 0; m < kM; ++m) xs[(1 - d) * kManyRows * 16 + x_place(16 * m + t16, piece)] = xb[m];
      __syncthreads();
    }
  }
  if (!active) return;
#pragma unroll
  for (int m = 0; m < kM; ++m) {
    const int token = 16 * m + (lane & 15);
    if (token >= blk.n) continue;
    const bool ok = real[token >> 6] >> (token & 63) & 1;
    uint16_t* const o = out + (int64_t)(blk.row + token) * n_out + n0 + (lane >> 4) * 4;
#pragma unroll
    for (int i = 0; i < (kSwiglu ? kTiles / 2 : kTiles); ++i) {
      f32x4 v = acc[i][m];
      if (kSwiglu) {
#pragma unroll
        for (int z = 0; z < 4; ++z) v[z] = swiglu(v[z], acc[i + kTiles / 2][m][z]);
      }
      const u32x2 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      st8(o + 16 * i, ok ? w : u32x2{0u, 0u});
    }
  }
}

template <bool kSwiglu>
__global__ __launch_bounds__(kManyThreads, 2) void gemm_mxfp4_kernel(
    const uint16_t* __restrict__ x, int64_t x_rows, const uint8_t* __restrict__ tq, const uint8_t* __restrict__ ts,
    const int32_t* __restrict__ offsets, int E, const int32_t* __restrict__ src_row, int top_k, int64_t M_cap,
    int64_t N, int64_t K, uint16_t* __restrict__ out) {
  __shared__ u32x4 xs[2 * kManyRows * 16];
  __shared__ int rows[128];  // two a lane of the first wave; the first kManyRows are used
  constexpr int kCols = kSwiglu ? kTiles * 8 : kTiles * 16;  // of out, a wave
  const int64_t n_out = kSwiglu ? N / 2 : N;
  const unsigned nt = (unsigned)((n_out + kManyWaves * kCols - 1) / (kManyWaves * kCols));
  const RowBlock blk = find_block(nt, offsets, E);
  if (blk.e < 0 || blk.row + blk.n > M_cap) return;  // uniform
  const int lane = threadIdx.x & 63;
  int64_t n0 = ((int64_t)blk.col * kManyWaves + wave_number()) * kCols;
  const bool active = n0 < n_out;  // not so for waves of the last workgroup where n_out is no multiple of its columns:
  if (!active) n0 = 0;             // they go along and store nothing
  unsigned long long real[2];
  int src[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = 64 * h + lane;
    src[h] = r < blk.n ? source_of(blk.row + r, src_row, top_k, x_rows) : -1;
    real[h] = __ballot(src[h] >= 0);
  }
  const int count = real[1] ? 128 - __clzll(real[1]) : real[0] ? 64 - __clzll(real[0]) : 0;
  if (threadIdx.x < 64) {
    const int first = real[0] ? __ffsll(real[0]) - 1 : real[1] ? 64 + __ffsll(real[1]) - 1 : 0;
    const int any = first < 64 ? __shfl(src[0], first & 63) : __shfl(src[1], first & 63);
#pragma unroll
    for (int h = 0; h < 2; ++h) rows[64 * h + lane] = src[h] >= 0 ? src[h] : any;  // a row that is read anyway
  }
  __syncthreads();
  const int m = (count + 15) / 16;
#define FF8_GO(M) many_rows<kSwiglu, M>(x, rows, tq, ts, blk.e, n0, N, K, active, blk, real, xs, out)
  if (m == 1)
    FF8_GO(1);
  else if (m == 2)
    FF8_GO(2);
  else if (m == 3)
    FF8_GO(3);
  else if (m == 4)
    FF8_GO(4);
  else if (m == 5)
    FF8_GO(5);
  else if (m == 6)
    FF8_GO(6);
#undef FF8_GO
  const int done = 16 * m;  // the padding rows behind
  if (active)
    for (int i = lane; i < (blk.n - done) * (kCols / 8); i += 64)
      st16(out + (int64_t)(blk.row + done + i / (kCols / 8)) * n_out + n0 + i % (kCols / 8) * 8, u32x4{0u, 0u, 0u, 0u});
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
  const int64_t n_out = swiglu ? N / 2 : N;
  const int64_t cols = kManyWaves * kTiles * (swiglu ? 8 : 16), nt = (n_out + cols - 1) / cols;
  const Mxfp4Form form = mxfp4_form(x_rows, top_k, M_cap, E, N, K, swiglu, device_cu_count());
  if (form.many) {
    const int64_t blocks = M_cap / kManyRows + (E < M_cap / 16 ? E : M_cap / 16);
    auto* const f = swiglu ? gemm_mxfp4_kernel<true> : gemm_mxfp4_kernel<false>;
    f<<<(unsigned)((blocks * nt + 7) / 8 * 8), kManyThreads, 0, st>>>(x, x_rows, tq, ts, offsets, E, src_row, top_k, M_cap, N, K, out);
  } else {
    const bool two = form.waves == 2, keep = form.keep;
    auto* const f = swiglu ? two ? keep ? gemv_mxfp4_kernel<true, 2, true> : gemv_mxfp4_kernel<true, 2, false>
                                 : keep ? gemv_mxfp4_kernel<true, 4, true> : gemv_mxfp4_kernel<true, 4, false>
                           : two ? keep ? gemv_mxfp4_kernel<false, 2, true> : gemv_mxfp4_kernel<false, 2, false>
                                 : keep ? gemv_mxfp4_kernel<false, 4, true> : gemv_mxfp4_kernel<false, 4, false>;
    f<<<(unsigned)(M_cap / 16 * (N / (16 * kTiles))), two ? 128 : 256, 0, st>>>(x, x_rows, tq, ts, offsets, E, src_row,
                                                                                top_k, N, K, out);
  }
  return hipGetLastError();
}

}  // namespace ff8
