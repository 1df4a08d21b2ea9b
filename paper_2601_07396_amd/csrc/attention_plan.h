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
    // whole 10.5
    cut(0, std::min<int64_t>(std::min<int64_t>(std::max(1, 2 * cus / plan.units), kMostParts), (tiles + kLeastTiles - 1) / kLeastTiles));
  } else if (rest) {
    // The last round has work for some of the compute units only: its units in parts, if that takes less than what the parts' sums cost on their way through memory.
    // 4608 x 4608, 24 heads, 864 units: the last 96 in 5 parts 246 us, whole 259; 4 sequences of it 949 and 965; 29764 x 29764, 3 heads 1.20 and 1.25 ms
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
