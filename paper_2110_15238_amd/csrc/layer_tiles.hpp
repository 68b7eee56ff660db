// Which tile runs a linear layer of E4M3 or FP16 operands, by an estimate of the time.
#pragma once
#include <algorithm>

#include "few_rows_instances.hpp"
#include "llm_checks.hpp"

namespace bolt {

struct LayerTile {
  RowsTile tile;
  int rows, cols, sets;  // sets: of waves that split the reduction
  double first_us, turn_us;
};
// Rounds of one workgroup on each of 256 compute units.
inline int64_t layer_rounds(const LayerTile& t, int64_t M, int64_t N) { return blocks_of(blocks_of(M, t.rows) * blocks_of(N, t.cols), 256); }
// Estimated time in us: the turns of a tile's sets of waves, 128 bytes of every row each, a turn as long as its own chain of loads, reads and matrix
// instructions or as its operands take from the L2s (15 TB/s for all); and no less than the weights take from memory.  row_bytes: of a row of W.
inline double layer_us(const LayerTile& t, int64_t M, int64_t N, int64_t row_bytes) {
  const int64_t blocks = blocks_of(M, t.rows) * blocks_of(N, t.cols), rounds = blocks / 256, rest = blocks % 256;
  const double bytes = (t.rows + t.cols) * 128.0 * t.sets, turns = (double)blocks_of(blocks_of(row_bytes, 128), t.sets);
  const auto turn = [&](int64_t workgroups) { return std::max(t.turn_us, workgroups * bytes / 15e6); };
  const double us = t.first_us + turns * (rounds * turn(256) + (rest > 0 ? turn(rest) : 0.0));
  return std::max(us, 2.5 + N * row_bytes / 4.5e6);
}
// Whether the tile's launch can be made; the 256 x 256 ones run on one workgroup per compute unit and address W with 31-bit offsets.
inline bool layer_launches(const LayerTile& t, int64_t M, int64_t N, int64_t row_bytes) {
  const int64_t blocks = blocks_of(M, t.rows) * blocks_of(N, t.cols);
  return t.tile == RowsTile::ROWS256_COLS256 ? blocks <= INT32_MAX && N * row_bytes <= INT32_MAX : launches(blocks);
}
// The tile of the smallest estimate, null if no launch can be made.  bias_in_sum: the layer can start its sums at beta / alpha times the bias, as FP16
// ones on 256 x 256 tiles do.
template <size_t COUNT>
const LayerTile* layer_tile(const LayerTile (&tiles)[COUNT], int64_t M, int64_t N, int64_t row_bytes, bool bias_in_sum) {
  const LayerTile* best = nullptr;
  for (const LayerTile& t : tiles)
    if ((bias_in_sum || t.tile != RowsTile::ROWS256_COLS256) && layer_launches(t, M, N, row_bytes) &&
        (!best || layer_us(t, M, N, row_bytes) < layer_us(*best, M, N, row_bytes)))
      best = &t;
  return best;
}

}  // namespace bolt
