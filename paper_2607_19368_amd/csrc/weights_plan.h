// Plans of the attention weights (k_weights.hip): which kernel takes a call, over how many blocks.
#pragma once
#include "attend_plan.h"

namespace slh {

constexpr int WT_ROWS = 128, WT_BLOCK_KEYS = 256;      // of a tile

// Which kernel, and over how many blocks a head's tiles are spread: all that run at once.
struct WeightPlan {
  bool tiles;
  int runs;
  int64_t bytes;
};
// By rows of a sequence.  Few rows and tiles, 4 key/value heads of 7 and 8 of 4: 56 and 64 rows of 8 sequences of 32768 keys
// 65 and 89, 134 and 177 us; 112 and 128 rows 93 and 89, 201 and 174; 448 and 256 rows 272 and 191, 334 and 233; of 4096
// keys, 56 and 448 rows: 13 and 21, 49 and 35 us.  Where the sequences' numbers differ, one may have nearly all rows (4000 of 64
// sequences' 4063 are 63 a sequence), which are far slower by few: tiles from the smaller number on, that loses at most 2.1 times.
inline WeightPlan weights_plan(int64_t Tq, int B, int Hkv, int g, bool even) {
  WeightPlan p = {};
  p.tiles = Tq * g > (even ? 96 : 32) * (int64_t)B;
  if (!p.tiles) return p;
  p.runs = std::max(1, 2 * attend_cus() / Hkv);
  p.bytes = p.runs > 1 ? 8 * (int64_t)p.runs * Hkv * WT_BLOCK_KEYS : 0;
  return p;
}

// Whether the tiles of all sequences may be 2^31 or more.  Any entries of cu_q, not ascending ones among them, give a sequence at most all
// queries: a count that wrapped round would lead out of the rows, or past the last sequence.
inline bool weights_wide(int64_t Tq, int B, int g, int max_rows, bool even, int runs) {
  const int64_t row_tiles = ((even ? Tq / B : Tq) * g + WT_ROWS - 1) / WT_ROWS;
  return (int64_t)B * ((max_rows + WT_BLOCK_KEYS - 1) / WT_BLOCK_KEYS) * row_tiles + runs > INT32_MAX;
}

}  // namespace slh
