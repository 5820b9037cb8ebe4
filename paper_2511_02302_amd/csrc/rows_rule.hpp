// Which form a row sort takes, by its sizes: host code only.
#pragma once

#include "ff8_launch.hpp"

namespace ff8 {

// Rows of at most kNarrow 16-byte pieces are moved kNarrowRows at a time by a wave.  us, so / one a wave, maps there and
// maps to be built: 16000 tokens x 128 columns, 8 experts, k = 8 10.1 / 27.1 and 21 / 38, gradient 26.5 / 46; x 512, 32
// experts 25.6 / 29.7, 39 / 42, 53 / 58.  (Wider ones four or two at a time: 1024 columns 49 / 44, 2048 98 / 97.)
constexpr int kNarrow = 64, kNarrowRows = 8;
inline bool narrow_rows(int64_t row16) { return row16 <= kNarrow; }

enum class SortForm {
  kOneLaunch,    // every workgroup counts all pairs by itself
  kCounted,      // a launch in front counts chunks of tokens
  kRoutedFirst,  // the routing has its own launches
};

// Up to kMaxPairs pairs one launch.  us, so / with the routing in launches of its own: 1024 tokens x 256 columns, 8
// experts, k = 2 6.9 / 11.4; 512 x 7168, 64 experts, k = 8 17 / 26, with 128-row padding 29 / 38; 4096 x 256, 1024
// experts, k = 1 10.4 / 12.7.  (8192 x 256, 8 experts, k = 1 14.8 / 12.6.)
//
// Beyond, routing and rows share a launch behind chunk counts while that pays.  Every workgroup of 16 pairs (64 of narrow
// rows) reads the counts and half a chunk, which pays while the workgroups are few and their rows long.  us, with /
// without:
//  * rows of 4 KiB and more, up to 48K pairs: 1024 tokens x 2048 columns, 64 experts, k = 8 12.5 / 18.5; 4096 x 7168, 256,
//    k = 8 143 / 153; 5001 x 7168 bytes, 32, k = 8 60 / 64; beyond 8192 x 7168, 32, k = 8 211 / 207, 16384 tokens 427 / 409.
//  * rows between, up to 32K: 640 columns, 8 experts, k = 2 at 16K, 24K, 32K and 40K pairs 12.4 / 13.5, 16.0 / 16.0, 19.1 /
//    18.1, 22.3 / 20.5; 64 experts, k = 8 at 32K and 40K 20.7 / 21.7, 24.9 / 24.0.  The wider of them would gain beyond
//    too (1920 columns, 64 experts, k = 8 at 64K 56.6 / 62.0; 1024 columns there 37.4 / 37.4).
//  * narrow rows, up to 64K: 700 x 256, 512, k = 8 10.6 / 17.2; 4000 x 128, 8, k = 8 12.1 / 15.3; 8000 x 256, 64 17.9 /
//    20.2; 32000 x 256, 8, k = 2 16.1 / 17.1; beyond 12000 x 128, 8, k = 8 22.6 / 19.6, 16000 27 / 21.
//  * pairs times counts up to 2^27, for many experts with few pairs each: 256 columns, 1024 experts, k = 2, 4096 tokens
//    (2^27) 21.3 / 23.3, 6000 28.2 / 25.2, 8192 (2^29) 34.5 / 28.9; 1024 columns 25.5 / 27.3, 33.7 / 30.0, 42.5 / 36.1.
//    With k = 8 (2^29: 26.4 / 29.1) or rows of 7168 columns (2^29: 118.6 / 113.9, k = 8 129 / 138) the two stay close.
constexpr int kMaxPairs = 4096;
inline SortForm sort_form(int64_t n_pairs, int64_t n_counts, int64_t row16) {
  if (n_pairs <= kMaxPairs) return SortForm::kOneLaunch;
  const bool counted = n_pairs <= (narrow_rows(row16) ? 64 << 10 : row16 >= 256 ? 48 << 10 : 32 << 10) &&
                       n_pairs * n_counts <= (int64_t)1 << 27;
  return counted ? SortForm::kCounted : SortForm::kRoutedFirst;
}

}  // namespace ff8
