// How an attention is made: host arithmetic only, apart from the launcher so that it can be checked without a GPU.
#pragma once
#include <stdint.h>

#include <algorithm>

#include "../../include/svdcache.h"

namespace svdc {

// Columns of a head as the kernels hold them, zeros behind the last one.
constexpr int attention_width(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : head_dim <= 128 ? 128 : 256; }

// Keys that a workgroup takes at a time: 32 rows of S a matrix instruction, two of them where the registers allow it.
constexpr int attention_tile_keys(int width, bool f32) { return !f32 && width <= 128 ? 64 : 32; }

constexpr int kTileQueries = 128;      // that a workgroup has, 32 a wave
constexpr int kLeastTiles = 2;         // of a part

// Units of work are tiles of the queries of all heads that share a head of keys: batch * kv_heads * q_tiles.  The first `whole` of them are a workgroup's each, with all keys; each of the others is cut into `parts` parts of
// tiles_of_part tiles of keys, a workgroup's each, which a second launch joins.  Without others parts is 1.
struct AttentionPlan {
  int q_tiles, units, whole, parts, tiles_of_part;
};

constexpr int kMostParts = 64;         // a lane each when they are joined

inline AttentionPlan attention_plan(const svdc_attention& p, int cus) {
  const int width = attention_width(p.head_dim), keys = attention_tile_keys(width, p.dtype == SVDC_F32);
  AttentionPlan plan{};
  plan.q_tiles = (int)((p.heads / p.kv_heads * p.q_rows + kTileQueries - 1) / kTileQueries);
  plan.units = (int)(p.batch * p.kv_heads * plan.q_tiles);
  plan.whole = plan.units;
  plan.parts = 1;
  const int64_t tiles = std::max<int64_t>(1, (p.k_rows + keys - 1) / keys);
  const auto cut = [&](int whole, int64_t parts) {
    plan.tiles_of_part = (int)((tiles + parts - 1) / parts);
    plan.parts = (int)((tiles + plan.tiles_of_part - 1) / plan.tiles_of_part);
    plan.whole = plan.parts > 1 ? whole : plan.units;
  };
  plan.tiles_of_part = (int)tiles;
  const int rest = plan.units % cus;
  if (plan.units > 0 && plan.units < cus) {
    // Fewer units than compute units: parts of all, until each of these has two workgroups.  64 x 119056, 24 heads: 21 parts 270 us.  1 x 512, 24 heads: 4 parts 8.7 us,
    // whole 10.5.  One to three units stay below that, as the join has a lane for each part: 1 x 119056, one head of keys, 63 workgroups 43 us, 1.4 TB/s; three heads 51 us, 3.6 TB/s.
    cut(0, std::min<int64_t>(std::min<int64_t>(std::max(1, 2 * cus / plan.units), kMostParts), (tiles + kLeastTiles - 1) / kLeastTiles));
  } else if (rest) {
    // The last round has work for some of the compute units only: its units in parts, if that takes less than what the parts' sums cost on their way through memory.
    // 4608 x 4608, 24 heads, 864 units: the last 96 in 2 parts 234 us, whole 250; 4 sequences of it 911 and 919; 29764 x 29764, 3 heads, 4 parts 1.15 ms, whole 1.21; float32, 24 heads,
    // 8 parts 1.83, whole 2.16 ms
    // The constants are us, read off such calls of 128 columns: a round of 4608 keys takes 62 us in bfloat16 and 530 in float32, a part's sums are written and read at 4 TB/s, a launch
    // takes 5.  Narrower heads take longer than their share of a round says (4608 keys of 64 columns 43 us, not 31), but there, too, the 2 parts that this gives were the fastest of 1 to 8
    // (64 columns 144 us, whole 154; 72 columns 186 and 200).
    const double round = tiles * keys * (width / 128.0) * (p.dtype == SVDC_F32 ? 0.115 : 0.0135), sums = 2.0 * kTileQueries * width * 4 / 4e6;
    double least = round;
    int64_t best = 1;
    for (int64_t parts = 2; parts <= 8 && parts * kLeastTiles <= tiles; ++parts) {
      const double us = round * (double)((rest * parts + cus - 1) / cus) / parts + rest * parts * sums + 5;
      if (us < least) least = us, best = parts;
    }
    if (best > 1) cut(plan.units - rest, best);
  }
  return plan;
}

}  // namespace svdc
