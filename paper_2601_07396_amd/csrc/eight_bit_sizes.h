// Sizes of a matrix in 8 bits.
#pragma once
#include <stdint.h>

namespace svdc {

constexpr int kScaleBlock = 128;   // columns (and, for weights, rows) that share a scale

constexpr int q8_blocks(int D) { return (D + kScaleBlock - 1) / kScaleBlock; }
constexpr int64_t q8_row_bytes(int D) { return (int64_t)q8_blocks(D) * kScaleBlock; }
// a reader takes the scales of four blocks as one word
constexpr int q8_scale_row_bytes(int D) { return (q8_blocks(D) + 3) / 4 * 4; }

}  // namespace svdc
