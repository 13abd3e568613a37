// How a product with codes is cut into workgroups.  Host code only.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "squant_few_rows.h"
#include "squant_product.h"

namespace squant {
namespace lin {

// A side of a layer, and the distance of rows that are read in place: 255 rows of two planes are less than 2^32 bytes
// apart.
constexpr int32_t kMaxSide = 1 << 22;
constexpr int64_t kMaxRows = 1 << 26;
constexpr int kCus = 256;

struct Split {
  bool few;
  int mt;              // rows of a workgroup of `product`
  int row_frags;       // few_rows: fragments of 16 rows
  int col_frags_each;  // few_rows: fragments of 16 columns a workgroup
  int tiles_m, tiles_n;
  int blocks, slices;
  int64_t workgroups;  // of a slice
  int threads;
  size_t lds;          // few_rows
  int64_t row_frags_all, col_frags_all;  // of the partial sums
  int64_t partial_vectors() const { return (int64_t)slices * row_frags_all * col_frags_all * kLanes; }
};

inline int shape_threads(int mt) {
  return mt == 256 ? Shape<256>::kThreads : mt == 128 ? Shape<128>::kThreads : Shape<64>::kThreads;
}

// `product` over rows x cols with a contraction of `depth`: the rows of a workgroup and the slices of the
// contraction by an estimate of the time.  It is there to rank them: the coefficients come from bare products of 44 shapes, of
// which its choice was within 8 % of the best tile and slices.  It knows neither the codes' format nor the epilogue nor the laying
// out of rows: bfloat16 and int8 codes, 1024 x 2048 x 4096 20.6 us for 26.3 measured, 4096 x 4096 x 8192 211 for 235 (with gelu and
// residual 250), 2048 x 2048 x 32768 217 for 262; binary32 1024 x 2048 x 4096 34 for 48, 7 to 10 of them the rows' split.
inline Split split_product(int64_t rows, int64_t cols, int64_t depth, int planes, bool may_split) {
  Split best{};
  double best_time = 1e30;
  const int blocks = (int)((depth + kBlock - 1) / kBlock);
  for (int mt = 64; mt <= 256; mt *= 2) {
    const int64_t tm = (rows + mt - 1) / mt, tn = (cols + kWide - 1) / kWide;
    // us of 64 contraction elements; two planes share the codes' conversion
    const double step = planes == 1 ? (mt == 256 ? 1.6 : mt == 128 ? 0.87 : 0.55) : (mt == 256 ? 2.9 : mt == 128 ? 1.6 : 0.97);
    for (int s = 1; s <= 64 && s <= blocks; s = s < 4 ? s + 1 : s * 2) {
      if (s > 1 && !may_split) break;
      const int64_t rounds = (tm * tn * s + kCus - 1) / kCus;
      const double join = s > 1 ? 4.5 + (double)tm * mt * tn * kWide * 4.0 * s / 3.0e6 : 0.0;
      const double time = rounds * (step * ((blocks + s - 1) / s) + 3.0) + join;
      if (time < best_time) {
        best_time = time;
        best.mt = mt; best.tiles_m = (int)tm; best.tiles_n = (int)tn; best.slices = s;
      }
    }
  }
  best.few = false;
  best.blocks = blocks;
  best.workgroups = (int64_t)best.tiles_m * best.tiles_n;
  best.threads = shape_threads(best.mt);
  best.row_frags_all = (int64_t)best.tiles_m * (best.mt / 16);
  best.col_frags_all = (int64_t)best.tiles_n * (kWide / 16);
  return best;
}

// A layer's product.  `tiled`: columns have to come in whole tiles of 64 (kept pre-activation, loss).
inline Split split_layer(int64_t rows, int64_t cols, int64_t depth, int planes, int format, bool tiled, bool may_split) {
  if (rows > few_rows_limit(planes)) return split_product(rows, cols, depth, planes, may_split);
  Split p{};
  p.few = true;
  const int frags = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  // Wide workgroups read their rows fewer times, narrow ones fill the chip: the narrowest of which one for each 16 rows
  // has a compute unit to itself.  16-bit rows with 8-bit codes stay at 32 columns while those alone fill between half of
  // the compute units and all.  us with 16, 32, 64 columns a workgroup, rows of 4096, int8 codes:
  //   13 bfloat16 rows  4096 columns 7.2 8.8 13.3, 6000 12.5 9.2 13.4, 8192 12.8 9.3 14.3, 16384 23.4 18.4 15.6
  //   64 bfloat16 rows  2048 13.6 9.8 13.7, 4096 18.8 18.2 13.8, 6000 34.9 20.8 27.2, 8192 35.3 21.0 25.2, 16384 68.6 38.5 27.2
  //   32 binary32 rows  2048 13.4 14.6 19.5, 4096 22.0 15.1 19.7, 6000 38.7 23.3 20.7, 8192 39.1 23.6 20.3, 16384 75.4 45.1 28.2
  const int64_t row_groups = (rows + 15) / 16;
  auto groups = [&](int each) { return (cols + 16 * each - 1) / (16 * each); };
  const bool rows_together = planes == 1 && format == SQUANT_OUT_INT8 && groups(2) <= kCus && groups(2) * 2 > kCus;
  if (tiled) p.col_frags_each = 4;
  else if (groups(1) * row_groups <= kCus) p.col_frags_each = 1;
  else p.col_frags_each = groups(2) * row_groups <= kCus || rows_together ? 2 : 4;
  p.blocks = (int)((depth + kBlock - 1) / kBlock);
  p.slices = 1;
  p.tiles_n = (int)((cols + 16 * p.col_frags_each - 1) / (16 * p.col_frags_each));
  // where the columns leave half of the chip without work, rows go to workgroups of their own
  p.row_frags = p.tiles_n * 2 <= kCus ? 1 : frags;
  p.tiles_m = (int)((rows + 16 * p.row_frags - 1) / (16 * p.row_frags));
  p.workgroups = p.tiles_n;
  p.threads = few_waves(p.row_frags, p.col_frags_each) * kLanes;
  p.lds = few_lds(p.row_frags, p.col_frags_each);
  return p;
}

inline Split split_gradient(int64_t rows, int64_t cols, int64_t depth, int planes) {
  return split_product(rows, cols, depth, planes, true);
}

// Columns of the vocabulary whose probabilities are held at a time: about 256 MB, at least 4096 entries.
inline int64_t vocabulary_piece(int64_t rows, int64_t cols, int planes) {
  const int64_t whole = (cols + kTile - 1) / kTile * kTile;
  const int64_t fit = (int64_t)(128 << 20) / (rows * planes) / kWide * kWide;
  return std::min(whole, std::max<int64_t>(4096, fit));
}

}  // namespace lin
}  // namespace squant
