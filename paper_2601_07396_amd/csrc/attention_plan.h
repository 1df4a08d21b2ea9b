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

// parts of the keys, each a workgroup's, and the tiles of keys of a part
struct AttentionPlan {
  int parts, tiles_of_part;
};

inline AttentionPlan attention_plan(const svdc_attention& p, int cus) {
  const bool f32 = p.dtype == SVDC_F32;
  const int width = attention_width(p.head_dim), keys = attention_tile_keys(width, f32);
  AttentionPlan plan{};
  const int64_t tiles = std::max<int64_t>(1, (p.k_rows + keys - 1) / keys);
  const int64_t groups = p.batch * p.heads * ((p.q_rows + kTileQueries - 1) / kTileQueries);
  int64_t parts = 1;
  // parts of at least four tiles, until every compute unit has a workgroup or two
  if (groups > 0 && groups < cus) parts = std::min<int64_t>(std::min<int64_t>(2 * cus / groups, 64), (tiles + 3) / 4);
  plan.tiles_of_part = (int)((tiles + parts - 1) / parts);
  plan.parts = (int)((tiles + plan.tiles_of_part - 1) / plan.tiles_of_part);
  return plan;
}

}  // namespace svdc
