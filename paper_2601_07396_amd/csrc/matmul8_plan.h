// How a product in 8 bits is made: host arithmetic only, apart from the launcher so that it can be checked without a GPU.
#pragma once
#include <stdint.h>

#include <algorithm>

#include "../../include/svdcache.h"
#include "eight_bit_sizes.h"

namespace svdc {

// blocks of each of `splits` parts of the columns of A and W: a multiple of four, as scales are read four at a time; the last part may have fewer
constexpr int blocks_of_part(int blocks, int splits) { return splits == 1 ? blocks : ((blocks + splits - 1) / splits + 3) / 4 * 4; }

// How a product is made.  rows 16 or 32: workgroups of that many rows by `columns` (16, 32, 64; 16 by 128 for results in 8 bits) whose waves share the blocks;
// rows 64, 128 or 256: tiles of that size through LDS, in `splits` parts of the columns of A and W (of 128 only), with `stages` of them there (2 or 4).
struct MatmulPlan {
  int rows, columns, splits, stages;
};

// The tiles of `rows` by 64 tile_width() rows of W.  Gated rows come in pairs of 32, and results in 8 bits need a whole block of columns: wider tiles of W where
// there are few rows.
constexpr int tile_width(int rows, bool gated, bool eight) { return eight && gated ? 4 : (eight || gated) && rows < 128 ? 2 : rows / 64; }

constexpr int kMaxTiles = 1 << 22;         // workgroups of a launch, far below what its 32-bit counts hold

// Rows of A that one launch of tiles takes: all of them, but for results of very many rows.
inline int64_t rows_of_launch(const MatmulPlan& plan, int N, bool gated, bool eight) {
  const int columns = 64 * tile_width(plan.rows, gated, eight) / (gated ? 2 : 1);
  return (int64_t)plan.rows * (kMaxTiles / ((N + columns - 1) / columns));
}

inline int wide_of(const svdc_matmul8& p) { return p.act == SVDC_ACT_SWIGLU ? 2 * p.N : p.N; }

// parts of the columns of A and W of which none is empty
inline int parts_of(int blocks, int splits) { return (blocks + blocks_of_part(blocks, splits) - 1) / blocks_of_part(blocks, splits); }

// Whether tiles of 64 TM by 64 TN with sums of `blocks` blocks have four stages in LDS instead of two: where all of them are at work at once all the same and the sums
// are long enough.  256 x 3072 x 3072 into bfloat16, 192 tiles of 64: 8.9 us with four, 11.7 with two; 512 x 12288 x 3072, 1536 tiles: 35 and 27; 448 x 4096 x 1024:
// 6.1 and 5.9.  With float32 sums a block takes its time from widening the operands (256 x 3072 x 3072 12.5 us with either): two.
constexpr int kUnitLds = 160 << 10, kDeepLds = 128 << 10;
constexpr int tile_lds(int TM, int TN, int stages) { return stages * 64 * (TM + TN) * 128; }
constexpr bool can_be_deep(int TM, int TN, bool exact) { return !exact && tile_lds(TM, TN, 4) <= kDeepLds; }
inline bool deep(double tiles, int blocks, int TM, int TN, bool exact, int units) {
  return can_be_deep(TM, TN, exact) && blocks > 8 && tiles <= (double)units * (kUnitLds / tile_lds(TM, TN, 4));
}

// The least of estimated times, in us: for each way what its rounds of workgroups (one on each compute unit; where several fit, they share it and
// take as long) cost for a block of columns and for their ends.  Measured over 174 products (29 sizes of 1 to 18432 rows, 64 to 18432 columns, K of 100 to 12288; three types, with and
// without gates): the estimate is within a quarter of the time for 163, the way taken within a twentieth of the fastest way's for 160 and within a sixth for 170.  The others are
// 18432 x 12288 x 100 gated into 8 bits (1.27 times) and 200 x 300 x 8192 in 8 and 16 parts (1.28 to 2.9 times): where N is no multiple of 8, matmul8_finish_kernel
// takes 0.55 us more for each part and sum (16 parts, gated, float32: N = 304 28 us, N = 300 47 us), which the estimate does not know.
inline MatmulPlan matmul8_plan(const svdc_matmul8& p, int cus) {
  const bool gated = p.act == SVDC_ACT_SWIGLU, exact = p.dtype == SVDC_F32, eight = p.dtype == SVDC_E4M3;
  const double units = cus;
  const int blocks = q8_blocks(p.K);
  const auto up = [](double x, double y) { return (double)(int64_t)((x + y - 1) / y); };
  MatmulPlan best{};
  double least = 1e300;
  // one launch, but of the largest tiles of a type, which go on with the next rows in another
  const auto consider = [&](MatmulPlan plan, double tiles, double us) {
    const bool largest = plan.rows == (exact ? 128 : 256) && plan.splits == 1;
    if (us < least && (tiles <= kMaxTiles || largest)) least = us, best = plan;
  };
  // Few rows: the time of loads of 16 rows by 64 bytes.  1 x 3072 x 3072 in 16 columns 4.4 us (32: 5.9, 64: 8.7, tiles of 64: 7.0), 1 x 8192 x 3072 gated in 32 columns 10.4 us
  // (tiles of 64: 11.8), 8 x 12288 x 4096 in 64 columns 13.5 us (16: 15.0, tiles of 64: 11.4)
  for (int rows = 16; rows <= 32; rows *= 2)
    for (int columns = eight ? 128 : 16; columns <= (eight ? 128 : gated ? 32 : 64); columns *= 2) {
      if ((rows == 32 && (eight || p.M <= 16)) || (eight && gated)) continue;
      const double tiles = up((double)p.M, rows) * up(p.N, columns);
      const double loads = columns / 16 * (gated ? 2 : 1) + std::min<int64_t>(p.M, rows) / 16.0;
      consider({rows, columns, 1, 0}, tiles, 2.5 + up(tiles, units) * up(blocks, 8) * (0.15 + 0.46 * loads) * (exact ? 1.3 : 1.0));
    }
  // Tiles of 64: 0.37 us a block of latency, 0.24 with four stages, until the rounds of tiles take longer.  256 x 3072 x 3072 into float32 12.5 us (tiles of 128 in two
  // parts: 20), into bfloat16 8.9 us (13.7); 2000 x 1024 x 1024 6.0 us (128: 7.7)
  const double tiles64 = up((double)p.M, 64) * up(p.N, eight ? 128 : 64), rounds64 = up(tiles64, units);
  const bool deep64 = deep(tiles64, blocks, 1, tile_width(64, gated, eight), exact, cus);
  const double rate64 = (exact ? 0.28 : eight ? 0.31 : 0.175) * (gated ? 1.7 : 1.0);
  const double latency64 = deep64 ? 0.24 : exact || eight || gated ? 0.42 : 0.37;
  consider({64, 64, 1, deep64 ? 4 : 2}, tiles64, 2.5 + blocks * std::max(latency64, rate64 * rounds64) + rounds64);
  // Tiles of 128: 2000 x 3072 x 3072 23.7 us (64: 32, 256: 32.6), 1000 x 3072 x 3072 15.3 us (64: 17.4).  In parts: 1160 x 320 x 11072 in eight 20.4 us (whole: 35)
  for (int splits = 1; splits <= 16; splits *= 2) {
    if (parts_of(blocks, splits) != splits) continue;
    const int part = blocks_of_part(blocks, splits);
    const double tiles = up((double)p.M, 128) * (splits > 1 ? up(wide_of(p), 128) : up(p.N, gated && !eight ? 64 : 128)) * splits;
    const bool deep128 = deep(tiles, part, 2, splits > 1 ? 2 : tile_width(128, gated, eight), exact, cus);
    const double rate128 = exact ? 0.75 : deep128 ? 0.38 : 0.42;
    const int stages = deep128 ? 4 : 2;
    if (splits == 1) {
      consider({128, 128, 1, stages}, tiles, 3 + up(tiles, units) * (blocks * rate128 * (gated && eight ? 2 : 1) + 2));
    } else {
      const double sums = (double)splits * p.M * wide_of(p);
      consider({128, 128, splits, stages}, tiles, 8 + up(tiles, units) * (part * rate128 + 3) + sums * 8 / 4e6);
    }
  }
  // Tiles of 256: 4608 x 3072 x 3072 40.4 us (128: 50)
  if (!exact) {
    const double tiles = up((double)p.M, 256) * up(p.N, gated ? 128 : 256);
    consider({256, 256, 1, 2}, tiles, 4 + up(tiles, units) * (blocks * 1.25 + 9));
  }
  return best;
}

}  // namespace svdc
