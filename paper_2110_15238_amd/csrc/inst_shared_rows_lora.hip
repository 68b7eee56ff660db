// Products of some to some hundred rows, weights in 4 bits: linear layers whose rows have adapters.
#include "few_rows_instances.hpp"
#include "shared_rows_kernel.hpp"

namespace bolt {
template <int NG>
static hipError_t launch(const LayerParams& p, SharedTile tile, hipStream_t stream) {
  // MB, R, WN, KG, S
  if (tile == SharedTile::ROWS32_COLS32) return launch_shared_rows<WEIGHTS_W4, ROWS_DENSE, false, NG, 2, 1, 2, 4, 3, true>(p, stream);
  if (tile == SharedTile::ROWS32_COLS64) return launch_shared_rows<WEIGHTS_W4, ROWS_DENSE, false, NG, 2, 1, 4, 2, 3, true>(p, stream);
  if (tile == SharedTile::ROWS64_COLS128) return launch_shared_rows<WEIGHTS_W4, ROWS_DENSE, false, NG, 4, 1, 8, 1, 3, true>(p, stream);
  return launch_shared_rows<WEIGHTS_W4, ROWS_DENSE, false, NG, 8, 2, 8, 1, 3, true>(p, stream);
}
hipError_t launch_shared_rows_w4_lora(const LayerParams& p, int group, SharedTile tile, hipStream_t stream) {
  if (group == 128) return launch<1>(p, tile, stream);
  if (group == 64) return launch<2>(p, tile, stream);
  return launch<4>(p, tile, stream);
}
}  // namespace bolt
