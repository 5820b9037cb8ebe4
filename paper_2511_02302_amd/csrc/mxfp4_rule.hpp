// Which form a 4-bit product takes, by its sizes: host code only.
#pragma once

#include <cstdint>

namespace ff8 {

// A wave's weight tiles (16 rows each), waves and token rows of a workgroup of the form for many rows.
constexpr int kMxTiles = 4, kManyWaves = 4, kManyRows = 96;

struct Mxfp4Form {
  bool many;  // blocks of up to 96 rows instead of 16
  int waves;  // of a 16-row workgroup
  bool keep;  // its weights are loaded as lines that stay in the L2
};

// N: weight rows.  The offsets are on the device, so rows are estimated from the buffers: T * top_k where the tokens are
// gathered (slots of other ranks count), otherwise what 16-row padding of every expert leaves of M_cap (wider padding
// counts as rows).  The forms' results differ by the order of their float32 sums alone.
//
// Blocks of 96 rows instead of 16 (times in us, 16 / 96):
//  * from 12 rows an expert on.  7168 wide, 32 experts, up projection: 8 rows 81 / 83, 12 92 / 84, 24 158 / 89;
//    2048 wide, 64 experts, down: 4 rows 24 / 23, 12 26 / 22; with skewed routing 8 rows 25 / 30, 12 33 / 28.
//    Few rows in wide padding count as many, and are faster so, as the 16-row form has a workgroup for every 16 rows of
//    padding: 32 experts, k = 8, 2048 -> 7168, one token with 16-, 32-, 64- and 128-row padding 15.1 / 17.4, 18.6 / 17.5,
//    26.9 / 18.1, 43.8 / 19.7; 8 tokens 39.8 / 46.4, 48.9 / 48.6, 59.3 / 51.3, 81.9 / 56.0.  What the rule takes there is
//    slower than the other for 4 tokens with 32-row padding alone (38.5 / 44.3).
//  * and from 5/8 of an item per CU on: a workgroup of the 96-row form goes through all of K by itself.  4096 wide, 8
//    experts: 72 items 13 / 30, 144 7.6 / 11.5 and 44 / 46, 208 19 / 17, 232 80 / 54; 1024 wide: 116 18 / 19, 200 31 / 21.
//
// Two waves an item where K gives them at most six blocks of 128 columns each, otherwise four.  us, two waves / four: K =
// 1024, 32 experts, 8 and 32 tokens 8.4 / 9.8 and 9.8 / 11.3, 1408, 64 experts 13.2 / 14.1; 2048, one token 7.4 / 6.6, 32
// tokens 27.8 / 27.5; 7168, 16 tokens 80 / 76.  (With few blocks a wave has little to hide its start behind, and more
// workgroups fit beside one another; with many, two waves have too few loads in flight.)
//
// From 16 rows an expert on its weights are read by more than one row block.  us, kept in the L2 / not: 204 rows each on 4
// experts, 6528 x 2 x 512 25.6 / 29.6, 38 on 7, 2304 x 2 x 640 9.4 / 9.8, 32 on 8, 4096 x 2 x 512 11.3 / 11.9; not so
// with fewer: 8 on 32, 7168 x 2 x 2048 87 / 82, one token of k = 8 25.2 / 22.4.  (One token of k = 2 on 4 experts, whose
// buffer is rounded up to 128 rows and so counts as 68: 6.4 / 6.6, 2048 -> 7168.)
inline Mxfp4Form mxfp4_form(int64_t x_rows, int top_k, int64_t M_cap, int E, int64_t N, int64_t K, bool swiglu, int64_t cus) {
  const int64_t rows = top_k ? x_rows * top_k : M_cap - 15 * (int64_t)E;
  const int64_t cols = kManyWaves * kMxTiles * (swiglu ? 8 : 16), nt = ((swiglu ? N / 2 : N) + cols - 1) / cols;
  return {rows >= 12 * (int64_t)E && (E + rows / kManyRows) * nt >= cus * 5 / 8, K <= 12 * 128 ? 2 : 4,
          rows >= 16 * (int64_t)E};
}

}  // namespace ff8
