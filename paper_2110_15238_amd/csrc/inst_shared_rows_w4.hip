// Products of some to some hundred rows, weights in 4 bits: linear layers, and the experts of routed lists.
#include "few_rows_instances.hpp"
#include "shared_rows_kernel.hpp"

namespace bolt {
template <int MODE, bool GATED, int NG>
static hipError_t launch(const RowsParams& p, SharedTile tile, hipStream_t stream) {
  // MB, R, WN, KG, S
  if constexpr (MODE == ROWS_DENSE) {
    if (tile == SharedTile::ROWS32_COLS32) return launch_shared_rows<WEIGHTS_W4, MODE, GATED, NG, 2, 1, 2, 4, 3>(p, stream);
    if (tile == SharedTile::ROWS32_COLS64) return launch_shared_rows<WEIGHTS_W4, MODE, GATED, NG, 2, 1, 4, 2, 3>(p, stream);
    if (tile == SharedTile::ROWS64_COLS128) return launch_shared_rows<WEIGHTS_W4, MODE, GATED, NG, 4, 1, 8, 1, 3>(p, stream);
  } else {
    if (tile == SharedTile::ROWS16_COLS64) return launch_shared_rows<WEIGHTS_W4, MODE, GATED, NG, 1, 2, 2, 2, 3>(p, stream);
    if (tile == SharedTile::ROWS16_COLS128) return launch_shared_rows<WEIGHTS_W4, MODE, GATED, NG, 1, 2, 4, 1, 3>(p, stream);
    if (tile == SharedTile::ROWS32_COLS128) return launch_shared_rows<WEIGHTS_W4, MODE, GATED, NG, 2, 2, 4, 1, 3>(p, stream);
    if (tile == SharedTile::ROWS64_COLS128) return launch_shared_rows<WEIGHTS_W4, MODE, GATED, NG, 4, 2, 4, 1, 3>(p, stream);
  }
  return launch_shared_rows<WEIGHTS_W4, MODE, GATED, NG, 8, 2, 8, 1, 3>(p, stream);
}
template <int MODE, bool GATED>
static hipError_t launch_group(const RowsParams& p, int group, SharedTile tile, hipStream_t stream) {
  if (group == 128) return launch<MODE, GATED, 1>(p, tile, stream);
  if (group == 64) return launch<MODE, GATED, 2>(p, tile, stream);
  return launch<MODE, GATED, 4>(p, tile, stream);
}
hipError_t launch_shared_rows_w4_marked(const LayerParams& p, int group, hipStream_t stream) {
  if (group == 128) return launch_shared_rows_marked<1, 8, 2, 8, 3>(p, stream);
  if (group == 64) return launch_shared_rows_marked<2, 8, 2, 8, 3>(p, stream);
  return launch_shared_rows_marked<4, 8, 2, 8, 3>(p, stream);
}
hipError_t launch_shared_rows_w4(const RowsParams& p, int mode, bool gated, int group, SharedTile tile, hipStream_t stream) {
  if (mode == ROWS_DENSE) return launch_group<ROWS_DENSE, false>(p, group, tile, stream);
  if (mode == ROWS_DOWN) return launch_group<ROWS_DOWN, false>(p, group, tile, stream);
  return gated ? launch_group<ROWS_UP, true>(p, group, tile, stream) : launch_group<ROWS_UP, false>(p, group, tile, stream);
}
}  // namespace bolt
