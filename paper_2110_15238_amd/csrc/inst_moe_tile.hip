// Products over many rows, FP16 weights: the experts of a routed list, and linear layers whose 4-bit weights were unpacked.
#include "few_rows_instances.hpp"
#include "moe_pp_kernel.hpp"
#include "moe_tile_kernel.hpp"

namespace bolt {
template <int MODE, bool GATED>
static hipError_t launch(const RowsParams& p, ManyTile tile, hipStream_t stream) {
  if (tile == ManyTile::ROWS64) return launch_moe_tiles<64, 128, 2, 2, 3, MODE, GATED>(p, stream);
  if (tile == ManyTile::ROWS128) return launch_moe_tiles<128, 128, 4, 2, 2, MODE, GATED>(p, stream);
  return launch_moe_pp<MODE, GATED>(p, stream);
}
hipError_t launch_many_rows_f16(const RowsParams& p, int mode, bool gated, ManyTile tile, hipStream_t stream) {
  if (mode == ROWS_DENSE) return launch_moe_pp<ROWS_DENSE, false>(p, stream);
  if (mode == ROWS_DOWN) return launch<ROWS_DOWN, false>(p, tile, stream);
  return gated ? launch<ROWS_UP, true>(p, tile, stream) : launch<ROWS_UP, false>(p, tile, stream);
}
}  // namespace bolt
